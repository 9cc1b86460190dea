// The norms after a block and before the next one, with gate, scale and residual sum between them:
//   s = residual[ids] + scale * act(gate) * post(y),   n = pre(s)
// One pass: a row's inputs are read once, stay in registers through both norms, and s and n are written once.
// Statistics are two passes over registers (mean, then squared distances from it), so rows with a large mean lose
// nothing; all arithmetic is fp32 and each output is rounded once.
//
// What bounds it: the bytes.  150 003 gathered fp32 rows of 256 beside bf16 ones, 461 MB: 85 us, 5.4 TB/s (83 % of the measured copy
// rate); 32 768 rows of 4096 bf16 with a full gate, 1.34 GB: 244 us, 5.5 TB/s.  What it took: rows ahead in shared memory by asynchronous copies, since a
// row's two norms are four dependent sums during which nothing would be on its way (rows held in registers: 524 us); two elements per
// instruction and one decision per call instead of per element, since at 16 to 32 elements per thread the instructions around a row
// weigh as much as its elements (62 instructions per element: 482 us; 39: 330); as many warps as fit, and only then more rows ahead
// (three rows of 24 KB per block 330 us, two 269; 16 elements per thread instead of 32: 244).  Rows that 16 bytes do not divide cost
// twice the instructions: 10 001 fp32 rows of 602, 96 MB: 32 us, 3.0 TB/s.  A few rows: 2.5 to 3.3 us.
#include "requests.cuh"

#include <algorithm>
#include <type_traits>
#include <utility>

namespace rp {

struct NormParams {
    int rows, width;
    const void* y;
    const void* gate;
    const void* residual;
    const int32_t* ids;
    const float* scale_vector;
    void* stream;
    void* normed;
    int64_t ld_y, ld_gate, ld_residual, ld_stream, ld_normed, residual_rows;
    ripple_norm post, pre;
    float scale;
    int gate_act, gate_width, clear_padding;
    int warps_per_row;
    int y_bytes, residual_bytes, stage_bytes, stages;   // of a row in the ring; rows in it
};

// ---- V neighbouring elements of a row, in fp32: pairs, which one instruction takes at a time (fma.rn.f32x2 and the like) ----
template <int V> struct Vec {
    uint64_t p[V / 2];
};
template <> struct Vec<1> {
    float x;
};
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float2 unpack2(uint64_t d) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(d));
    return v;
}
template <int V> __device__ __forceinline__ Vec<V> all_of(float x) {
    Vec<V> v;
    if constexpr (V == 1) {
        v.x = x;
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) v.p[i] = pack2(x, x);
    }
    return v;
}
template <int V> __device__ __forceinline__ void times(Vec<V>& x, const Vec<V>& w) {
    if constexpr (V == 1) {
        x.x *= w.x;
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(x.p[i]) : "l"(w.p[i]));
    }
}
template <int V> __device__ __forceinline__ void plus(Vec<V>& x, const Vec<V>& w) {
    if constexpr (V == 1) {
        x.x += w.x;
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) asm("add.rn.f32x2 %0, %0, %1;" : "+l"(x.p[i]) : "l"(w.p[i]));
    }
}
// sum += x x
template <int V> __device__ __forceinline__ void add_squares(Vec<V>& sum, const Vec<V>& x) {
    if constexpr (V == 1) {
        sum.x = fmaf(x.x, x.x, sum.x);
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) asm("fma.rn.f32x2 %0, %1, %1, %0;" : "+l"(sum.p[i]) : "l"(x.p[i]));
    }
}
template <int V> __device__ __forceinline__ float folded(const Vec<V>& v) {
    if constexpr (V == 1) {
        return v.x;
    } else {
        Vec<2> s{{v.p[0]}};
#pragma unroll
        for (int i = 1; i < V / 2; ++i) plus<2>(s, Vec<2>{{v.p[i]}});
        const float2 f = unpack2(s.p[0]);
        return f.x + f.y;
    }
}

// two 16-bit elements, and back
template <typename T> __device__ __forceinline__ uint64_t widen2(uint32_t x);
template <> __device__ __forceinline__ uint64_t widen2<__nv_bfloat16>(uint32_t x) { return pack2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
template <> __device__ __forceinline__ uint64_t widen2<__half>(uint32_t x) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x));
    return pack2(f.x, f.y);
}
template <typename T> __device__ __forceinline__ uint32_t narrow2(uint64_t x) {
    const float2 f = unpack2(x);
    uint32_t d;
    if constexpr (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(f.y), "f"(f.x));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(f.y), "f"(f.x));
    return d;
}
template <typename T, int V> __device__ __forceinline__ Vec<V> load(const void* from) {
    Vec<V> v;
    constexpr int BYTES = V * sizeof(T);
    if constexpr (V == 1) {
        v.x = to_f32(*static_cast<const T*>(from));
    } else if constexpr (sizeof(T) == 4) {
        if constexpr (BYTES == 8) {
            v.p[0] = *static_cast<const uint64_t*>(from);
        } else {
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const ulonglong2 u = static_cast<const ulonglong2*>(from)[i];
                v.p[2 * i] = u.x, v.p[2 * i + 1] = u.y;
            }
        }
    } else if constexpr (BYTES == 4) {
        v.p[0] = widen2<T>(*static_cast<const uint32_t*>(from));
    } else {
        const uint4 u = *static_cast<const uint4*>(from);
        v.p[0] = widen2<T>(u.x), v.p[1] = widen2<T>(u.y), v.p[2] = widen2<T>(u.z), v.p[3] = widen2<T>(u.w);
    }
    return v;
}
template <typename T, int V> __device__ __forceinline__ void store(void* to, const Vec<V>& v) {
    constexpr int BYTES = V * sizeof(T);
    if constexpr (V == 1) {
        *static_cast<T*>(to) = from_f32<T>(v.x);
    } else if constexpr (sizeof(T) == 4) {
        if constexpr (BYTES == 8) {
            *static_cast<uint64_t*>(to) = v.p[0];
        } else {
#pragma unroll
            for (int i = 0; i < V / 4; ++i) static_cast<ulonglong2*>(to)[i] = make_ulonglong2(v.p[2 * i], v.p[2 * i + 1]);
        }
    } else if constexpr (BYTES == 4) {
        *static_cast<uint32_t*>(to) = narrow2<T>(v.p[0]);
    } else {
        *static_cast<uint4*>(to) = make_uint4(narrow2<T>(v.p[0]), narrow2<T>(v.p[1]), narrow2<T>(v.p[2]), narrow2<T>(v.p[3]));
    }
}

// How exact a sigmoid is.  Rows of 16 bits: the hardware's exponential and reciprocal, with the rounding of the exponent off by at most
// (10 + |g|) 2^-24, where the outputs round at 2^-12 or more.  Beside an fp32 stream, which would show that: expf, off by 4 2^-24 however large
// |g|, and the hardware's reciprocal, 2 2^-24.  (150 003 rows of 256 with full gates, 537 MB: 92 us the former, 96 the latter, 108 with a division.)
enum { GATE_16, GATE_16_BESIDE_32, GATE_32 };
template <int EXACT>
__device__ __forceinline__ float sigmoid_of(float g) {
    if constexpr (EXACT == GATE_32) return 1.0f / (1.0f + expf(-g));
    float e, s;
    if constexpr (EXACT == GATE_16) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    else e = expf(-g);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
    return s;
}
// (one decision per access and not per element)
template <int EXACT, int V>
__device__ __forceinline__ void gates_of(Vec<V>& g, int act) {
    if (act == RIPPLE_GATE_IDENTITY) return;
    Vec<V> s = g;
    auto each = [&](auto f) {
        if constexpr (V == 1) {
            s.x = f(s.x);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float2 x = unpack2(s.p[i]);
                s.p[i] = pack2(f(x.x), f(x.y));
            }
        }
    };
    if (act == RIPPLE_GATE_TANH) each([](float x) { return tanhf(x); });
    else each([](float x) { return sigmoid_of<EXACT>(x); });
    if (act == RIPPLE_GATE_SILU) times<V>(g, s);
    else g = s;
}

// bytes (4, 8, 16, or 32 in two copies) to shared memory
template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    if constexpr (BYTES >= 16) {
#pragma unroll
        for (int at = 0; at < BYTES; at += 16)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + at), "l"(static_cast<const uint8_t*>(from) + at) : "memory");
    } else {
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
    }
}

// sum over the threads of a row; MULTI: scratch has two halves, used in turn
template <bool MULTI>
__device__ __forceinline__ float row_sum(float x, float* scratch, int warps, int& turn) {
    x = warp_sum(x);
    if constexpr (MULTI) {
        float* const mine = scratch + 16 * (turn ^= 1);
        if (lane_id() == 0) mine[threadIdx.x >> 5] = x;
        __syncthreads();
        x = lane_id() < warps ? mine[lane_id()] : 0.f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
        x = __shfl_sync(FULL, x, 0);
    }
    return x;
}

constexpr int RN_STAGES = 3;     // rows on their way at most

// V: neighbouring elements per access, NP: accesses per thread.  A row takes a warp, or (MULTI) the whole block.
// RING: a thread's part of the rows ahead travels as asynchronous copies into places of shared memory that it alone reads,
// so no barrier belongs to it.  Else (16-bit rows that not even pairs of elements divide) a row is read into registers when its
// turn comes.
template <typename T, typename TR, int V, int NP, bool MULTI, bool RING>
__global__ void __launch_bounds__(MULTI ? (NP * V > 16 ? 512 : 256) : 128) k_norm_rows(const __grid_constant__ NormParams p) {
    pdl_enter();
    constexpr int EXACT = sizeof(T) == 4 ? GATE_32 : sizeof(TR) == 4 ? GATE_16_BESIDE_32 : GATE_16;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float scratch[MULTI ? 32 : 1];
    const int W = MULTI ? p.warps_per_row : 1, threads = 32 * W, t = MULTI ? threadIdx.x : lane_id();
    const int first = MULTI ? blockIdx.x : blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int64_t step = MULTI ? gridDim.x : gridDim.x * (blockDim.x >> 5);
    const int D = p.width;
    const bool wide_gate = p.gate && p.gate_width != 1;
    const float inv_d = 1.0f / (float)D;
    int turn = 0;
    // the ring's rows: y, then the residual, then the gate
    const int at_r = p.y ? p.y_bytes : 0, at_g = at_r + (p.residual ? p.residual_bytes : 0), per_row = p.stage_bytes;
    const int ahead = RING ? p.stages - 1 : 0;
    uint8_t* const mine = RING ? ring + (MULTI ? 0 : (threadIdx.x >> 5) * p.stages * per_row) + t * V * (int)sizeof(T) : nullptr;
    const int at_r_mine = at_r + t * V * (int)(sizeof(TR) - sizeof(T));
    const int c0 = t * V, hop = threads * V;      // this thread's columns: c0 + j hop + (0 .. V - 1)
    const T* const y0 = static_cast<const T*>(p.y) + c0;
    const TR* const r0 = static_cast<const TR*>(p.residual) + c0;
    const T* const gate0 = static_cast<const T*>(p.gate) + c0;
    // the residual row that a row reads; negative: a padding row, or none
    auto source = [&](int64_t row) -> int64_t {
        if (row >= p.rows) return -1;
        if (!p.ids) return row;
        const int64_t from = p.ids[row];
        return from < p.residual_rows ? from : -1;
    };
    auto request = [&](int stage, int64_t row, int64_t from) {
        if constexpr (RING) {
            if (from >= 0) {
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine + stage * per_row);
                const T* const y = y0 + row * p.ld_y;
                const TR* const r = r0 + from * p.ld_residual;
                const T* const g = gate0 + row * p.ld_gate;
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const int c = j * hop;
                    if (c0 + c >= D) break;
                    if (p.y) copy_async<V * sizeof(T)>(to + c * sizeof(T), y + c);
                    if (p.residual) copy_async<V * sizeof(TR)>(to + at_r_mine + c * sizeof(TR), r + c);
                    if (wide_gate) copy_async<V * sizeof(T)>(to + at_g + c * sizeof(T), g + c);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    auto gate_row = [&](int64_t row) { return p.gate && !wide_gate && row < p.rows ? to_f32(static_cast<const T*>(p.gate)[row * p.ld_gate]) : 1.0f; };
    // where this row and the next two come from
    int64_t from = source(first), from1 = source(first + step), from2 = source(first + 2 * step);
    float g1 = gate_row(first);
    if (ahead > 0) request(0, first, from);
    if (ahead > 1) request(1, first + step, from1);
    int stage = 0;
    for (int64_t row = first; row < p.rows; row += step) {
        request(stage == 0 ? ahead : stage - 1, row + ahead * step, ahead == 2 ? from2 : ahead == 1 ? from1 : from);
        const uint8_t* const in = mine + stage * per_row;
        const int64_t source_row = from;
        from = from1, from1 = from2, from2 = source(row + 3 * step);
        const float g_now = g1;
        g1 = gate_row(row + step);
        if (++stage > ahead) stage = 0;
        if constexpr (RING) {
            if (ahead == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
            else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        if (source_row < 0) continue;
        // (branches for what a call leaves out stand outside the loops over the row's pieces; a thread's pieces beyond the row
        // are zeros, which only the subtraction of the mean has to leave alone)
        Vec<V> s[NP];
        Piece<TR, V> r_reg[RING ? 1 : NP];
        Piece<T, V> g_reg[RING ? 1 : NP];
        auto each = [&](auto f) {
#pragma unroll
            for (int j = 0; j < NP; ++j) if (c0 + j * hop < D) f(j, j * hop);
        };
#pragma unroll
        for (int j = 0; j < NP; ++j) s[j] = all_of<V>(0.f);
        if constexpr (RING) {
            if (p.y) each([&](int j, int c) { s[j] = load<T, V>(in + c * (int)sizeof(T)); });
        } else {
            Piece<T, V> y_reg[NP];
            if (p.y) each([&](int j, int c) { y_reg[j] = *reinterpret_cast<const Piece<T, V>*>(y0 + row * p.ld_y + c); });
            if (p.residual) each([&](int j, int c) { r_reg[j] = *reinterpret_cast<const Piece<TR, V>*>(r0 + source_row * p.ld_residual + c); });
            if (wide_gate) each([&](int j, int c) { g_reg[j] = *reinterpret_cast<const Piece<T, V>*>(gate0 + row * p.ld_gate + c); });
            if (p.y) each([&](int j, int) { s[j] = load<T, V>(&y_reg[j]); });
        }
        // in place: s = norm(s)
        auto norm = [&](const ripple_norm& n) {
            if (n.kind == RIPPLE_NORM_NONE) return;
            Vec<V> sum = all_of<V>(0.f);
            if (n.kind == RIPPLE_NORM_LAYER) {      // s = s - mean
#pragma unroll
                for (int j = 0; j < NP; ++j) plus<V>(sum, s[j]);
                const Vec<V> back = all_of<V>(-row_sum<MULTI>(folded<V>(sum), scratch, W, turn) * inv_d);
                each([&](int j, int) { plus<V>(s[j], back); });
                sum = all_of<V>(0.f);
            }
#pragma unroll
            for (int j = 0; j < NP; ++j) add_squares<V>(sum, s[j]);
            const Vec<V> inv = all_of<V>(rsqrtf(row_sum<MULTI>(folded<V>(sum), scratch, W, turn) * inv_d + n.eps));
#pragma unroll
            for (int j = 0; j < NP; ++j) times<V>(s[j], inv);
            if (n.weight) each([&](int j, int c) { times<V>(s[j], load<float, V>(n.weight + c0 + c)); });
            if (n.bias) each([&](int j, int c) { plus<V>(s[j], load<float, V>(n.bias + c0 + c)); });
        };
        if (p.y) {
            norm(p.post);
            if (wide_gate) {
                each([&](int j, int c) {
                    Vec<V> k = RING ? load<T, V>(in + at_g + c * (int)sizeof(T)) : load<T, V>(&g_reg[RING ? 0 : j]);
                    gates_of<EXACT, V>(k, p.gate_act);
                    times<V>(s[j], k);
                });
            }
            Vec<1> row_gate = {g_now};
            if (p.gate && !wide_gate) gates_of<EXACT, 1>(row_gate, p.gate_act);
            const Vec<V> k = all_of<V>(row_gate.x * (p.scale_vector ? 1.0f : p.scale));
#pragma unroll
            for (int j = 0; j < NP; ++j) times<V>(s[j], k);
            if (p.scale_vector) each([&](int j, int c) { times<V>(s[j], load<float, V>(p.scale_vector + c0 + c)); });
        }
        if (p.residual) each([&](int j, int c) { plus<V>(s[j], RING ? load<TR, V>(in + at_r_mine + c * (int)sizeof(TR)) : load<TR, V>(&r_reg[RING ? 0 : j])); });
        if (p.stream) {
            TR* const to = static_cast<TR*>(p.stream) + row * p.ld_stream + c0;
            each([&](int j, int c) { store<TR, V>(to + c, s[j]); });
        }
        if (!p.normed) continue;
        norm(p.pre);
        T* const to = static_cast<T*>(p.normed) + row * p.ld_normed + c0;
        each([&](int j, int c) { store<T, V>(to + c, s[j]); });
    }
    if constexpr (RING) asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Zeros in the padding rows, for calls that ask for them: a warp looks at 32 ids and clears what they leave out.  (A kernel of its own: in
// k_norm_rows, in or behind its loop, these stores cost all calls 2 to 5 %, by the registers they change.)
template <typename T, typename TR>
__global__ void __launch_bounds__(256) k_clear_padding(const __grid_constant__ NormParams p) {
    pdl_enter();
    const int64_t first = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * 32;
    const int64_t from = first + lane_id() < p.rows ? p.ids[first + lane_id()] : 0;
    for (uint32_t left = __ballot_sync(FULL, first + lane_id() < p.rows && (from < 0 || from >= p.residual_rows)); left; left &= left - 1) {
        const int64_t row = first + __ffs(left) - 1;
        for (int c = lane_id(); c < p.width; c += 32) {
            if (p.clear_padding & 1) static_cast<TR*>(p.stream)[row * p.ld_stream + c] = from_f32<TR>(0.f);
            if (p.clear_padding & 2) static_cast<T*>(p.normed)[row * p.ld_normed + c] = from_f32<T>(0.f);
        }
    }
}

template <typename T, typename TR, int V, int E, bool MULTI, bool RING>
static cudaError_t launch_norm(NormParams p, int warps, void* stream) {
    auto* const kernel = k_norm_rows<T, TR, V, E / V, MULTI, RING>;
    p.warps_per_row = warps;
    const int block = MULTI ? 32 * warps : 128, rows_per_block = MULTI ? 1 : 4;
    const int64_t blocks = ((int64_t)p.rows + rows_per_block - 1) / rows_per_block;
    int bytes = 0, per_sm = 1;
    if (RING) {
        // (three rows per warp or block where they are small, and one where not even two fit)
        const int one = p.stage_bytes * rows_per_block;
        p.stages = blocks <= sm_count() ? 1 : RN_STAGES * one <= 48 * 1024 ? RN_STAGES : 2 * one <= 200 * 1024 ? 2 : 1;
        bytes = p.stages * one;
    }
    // (the most that any call takes, once: a limit set call by call would be another thread's between its setting and its launch)
    static bool ready[64];       // by device
    const cudaError_t e = allow_shared(kernel, 200 * 1024, ready);
    if (e != cudaSuccess) return e;
    if (blocks > sm_count() && (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, block, bytes) != cudaSuccess || per_sm < 1)) per_sm = 1;
    return launch(kernel, dim3((unsigned)std::min<int64_t>(blocks, (int64_t)per_sm * sm_count())), block, bytes, stream, p);
}

template <typename T, typename TR, int V, bool RING>
static cudaError_t launch_norm(const NormParams& p, void* stream) {
    const int D = p.width;
    // Elements per thread: no more than the row needs (602 columns: 32 per thread 38 us, 24 32 us; two warps per row 59).
    if (D <= 256) return launch_norm<T, TR, V, 8, false, RING>(p, 1, stream);
    if (D <= 512) return launch_norm<T, TR, V, 16, false, RING>(p, 1, stream);
    if (D <= 768) return launch_norm<T, TR, V, 24, false, RING>(p, 1, stream);
    if (D <= 1024) return launch_norm<T, TR, V, 32, false, RING>(p, 1, stream);
    if (D <= 4096) return launch_norm<T, TR, V, 16, true, RING>(p, (D + 511) / 512, stream);
    return launch_norm<T, TR, V, 32, true, RING>(p, (D + 1023) / 1024, stream);
}

template <typename T, typename TR>
static cudaError_t launch_norm(NormParams p, int v, void* stream) {
    constexpr int WIDE = 16 / sizeof(T);
    if (p.clear_padding && p.ids) {
        const cudaError_t e = launch(k_clear_padding<T, TR>, dim3((unsigned)((p.rows + 255LL) / 256)), 256, 0, stream, p);
        if (e != cudaSuccess) return e;
    }
    auto up16 = [](int64_t x) { return (int)((x + 15) / 16 * 16); };
    p.y_bytes = up16(p.width * (int64_t)sizeof(T)), p.residual_bytes = up16(p.width * (int64_t)sizeof(TR));
    p.stage_bytes = (p.y ? p.y_bytes : 0) + (p.residual ? p.residual_bytes : 0) + (p.gate && p.gate_width != 1 ? p.y_bytes : 0);
    if (v >= WIDE) return launch_norm<T, TR, WIDE, true>(p, stream);
    if (v >= 2) return launch_norm<T, TR, 2, true>(p, stream);
    return launch_norm<T, TR, 1, sizeof(T) == 4>(p, stream);
}

}  // namespace rp

using namespace rp;

#define REFUSE(...)                        \
    do {                                   \
        note_error("norm_rows: " __VA_ARGS__); \
        return RIPPLE_ERR_INVALID_ARG;     \
    } while (0)

extern "C" ripple_status ripple_norm_rows(const ripple_norm_rows_args* a) {
    if (!a) REFUSE("null arguments");
    if (a->rows < 0 || a->rows > INT32_MAX) REFUSE("rows out of range");
    if (a->width < 1 || a->width > 16384) REFUSE("width must be 1 to 16384");
    if (!type_ok(a->type) || !type_ok(a->stream_type) || (a->stream_type != a->type && a->stream_type != RIPPLE_TYPE_F32))
        REFUSE("unknown type, or a stream type that is neither the type nor fp32");
    for (const ripple_norm* n : {&a->post, &a->pre}) {
        if (n->kind < RIPPLE_NORM_NONE || n->kind > RIPPLE_NORM_RMS) REFUSE("unknown norm");
        if (n->kind != RIPPLE_NORM_NONE && !(n->eps >= 0.f)) REFUSE("eps must not be negative");
        if ((reinterpret_cast<uintptr_t>(n->weight) | reinterpret_cast<uintptr_t>(n->bias)) & 3) REFUSE("misaligned norm vector");
    }
    if (a->gate_act < RIPPLE_GATE_IDENTITY || a->gate_act > RIPPLE_GATE_TANH) REFUSE("unknown gate activation");
    if (!a->y && !a->residual) REFUSE("neither y nor residual");
    if (!a->y && (a->gate || a->post.kind != RIPPLE_NORM_NONE)) REFUSE("gate or post norm without y");
    if (a->gate && a->gate_width != 1 && a->gate_width != a->width) REFUSE("gate width must be 1 or the width");
    if (a->ids && !a->residual) REFUSE("ids without residual");
    if (a->residual && (a->residual_rows < 0 || (!a->ids && a->residual_rows < a->rows))) REFUSE("fewer residual rows than rows");
    if (!a->stream && !a->normed) REFUSE("no output");
    if (a->clear_padding < 0 || a->clear_padding > 1) REFUSE("clear_padding must be 0 or 1");
    if ((a->normed != nullptr) != (a->pre.kind != RIPPLE_NORM_NONE)) REFUSE("normed and pre go together");
    if (a->ld_y < 0 || a->ld_gate < 0 || a->ld_residual < 0) REFUSE("negative leading dimension");
    if ((a->stream && a->ld_stream < a->width) || (a->normed && a->ld_normed < a->width)) REFUSE("leading dimension of an output below its width");
    const int ts = type_size(a->type), rs = type_size(a->stream_type);
    for (auto [ptr, size] : {std::pair<const void*, int>{a->y, ts}, {a->gate, ts}, {a->normed, ts}, {a->residual, rs}, {a->stream, rs}, {a->scale_vector, 4}, {a->ids, 4}})
        if (reinterpret_cast<uintptr_t>(ptr) % size) REFUSE("misaligned pointer");
    const Extent y{a->y, a->rows, a->ld_y, a->width, ts}, gate{a->gate, a->rows, a->ld_gate, a->gate_width, ts},
        residual{a->residual, a->residual_rows, a->ld_residual, a->width, rs}, stream{a->stream, a->rows, a->ld_stream, a->width, rs},
        normed{a->normed, a->rows, a->ld_normed, a->width, ts};
    const Extent ids{a->ids, a->rows, 1, 1, 4}, scale{a->scale_vector, 1, 1, a->width, 4}, pw{a->post.weight, 1, 1, a->width, 4},
        pb{a->post.bias, 1, 1, a->width, 4}, nw{a->pre.weight, 1, 1, a->width, 4}, nb{a->pre.bias, 1, 1, a->width, 4};
    if (extents_meet(stream, normed)) REFUSE("stream and normed overlap");
    for (const Extent& out : {stream, normed}) {
        // (a row of y, the gate or the residual is read by the threads that write it; gathered rows are read by others)
        for (const Extent* in : {&y, &gate, &residual})
            if (extents_meet(out, *in) && (!extents_same(out, *in) || (in == &residual && a->ids))) REFUSE("an output overlaps an input");
        for (const Extent& in : {ids, scale, pw, pb, nw, nb})
            if (extents_meet(out, in)) REFUSE("an output overlaps an input");
    }
    if (a->rows == 0) return RIPPLE_OK;

    // The widest access that every matrix and vector of the call allows.
    int v = 16 / ts;
    auto fits = [&](const void* ptr, int64_t ld, int size) {
        while (v > 1 && (ld % v || reinterpret_cast<uintptr_t>(ptr) % (v * size < 16 ? v * size : 16))) v >>= 1;
    };
    while (a->width % v) v >>= 1;
    if (a->y) fits(a->y, a->ld_y, ts);
    if (a->gate && a->gate_width != 1) fits(a->gate, a->ld_gate, ts);
    if (a->residual) fits(a->residual, a->ld_residual, rs);
    if (a->stream) fits(a->stream, a->ld_stream, rs);
    if (a->normed) fits(a->normed, a->ld_normed, ts);
    for (const void* ptr : {(const void*)a->scale_vector, (const void*)a->post.weight, (const void*)a->post.bias, (const void*)a->pre.weight, (const void*)a->pre.bias})
        if (ptr) fits(ptr, 0, 4);

    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    NormParams p = {};
    p.rows = (int)a->rows, p.width = a->width;
    p.y = a->y, p.gate = a->gate, p.residual = a->residual, p.ids = a->ids, p.scale_vector = a->scale_vector;
    p.stream = a->stream, p.normed = a->normed;
    p.ld_y = a->ld_y, p.ld_gate = a->ld_gate, p.ld_residual = a->ld_residual, p.ld_stream = a->ld_stream, p.ld_normed = a->ld_normed;
    p.residual_rows = a->residual_rows;
    p.post = a->post, p.pre = a->pre;
    p.scale = a->scale, p.gate_act = a->gate_act, p.gate_width = a->gate_width;
    p.clear_padding = a->clear_padding ? (a->stream ? 1 : 0) | (a->normed ? 2 : 0) : 0;
    cudaError_t e;
    const bool mixed = a->stream_type != a->type;
    switch (a->type) {
        case RIPPLE_TYPE_F32: e = launch_norm<float, float>(p, v, a->cuda_stream); break;
        case RIPPLE_TYPE_BF16: e = mixed ? launch_norm<__nv_bfloat16, float>(p, v, a->cuda_stream) : launch_norm<__nv_bfloat16, __nv_bfloat16>(p, v, a->cuda_stream); break;
        default: e = mixed ? launch_norm<__half, float>(p, v, a->cuda_stream) : launch_norm<__half, __half>(p, v, a->cuda_stream); break;
    }
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("norm_rows launch", e);
}
