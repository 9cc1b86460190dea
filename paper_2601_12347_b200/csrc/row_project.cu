// A projection with the low-rank adapters of many requests beside it:
//   y_i = act(x_i W + bias + scale_a (x_i A_a) B_a),  a = slots_i
#include "requests.cuh"
#include "tensor_core.cuh"

#include <algorithm>
#include <cstdlib>

namespace rp {

// ---- what a layout and a bank hold ---------------------------------------------------------------------------------
// Layout of W: its transpose (output columns are rows, K runs along a row), cut into groups of PJ_COLS columns and chunks
// of PJ_KC entries of K.  A chunk is PJ_COLS rows of 128 bytes in the swizzle that the tensor core reads, zeros beyond K and n;
// fp32 weights are three chunks, one per bf16 part.  Behind the chunks W itself, k x n, for calls of few rows.
constexpr int PJ_COLS = 128, PJ_KC = 64;
constexpr int PJ_CHUNK = PJ_COLS * 128;
// Bank: scale and rank of every slot; A transposed (rank x K, zeros beyond both; fp32 as three planes of bf16 parts); B transposed
// (n x rank, zeros beyond the rank) in planes of bf16: one for bf16, two for fp16 (its 11 bits), three for fp32; and the same in fp32.
struct SlotInfo { float scale; int32_t rank; };

__host__ __device__ inline int pj_parts(int type) { return type == RIPPLE_TYPE_F32 ? 3 : 1; }
__host__ __device__ constexpr int pj_b_planes(int type) { return type == RIPPLE_TYPE_F32 ? 3 : type == RIPPLE_TYPE_F16 ? 2 : 1; }
__host__ __device__ inline int pj_up(int x, int to) { return (x + to - 1) / to * to; }
__host__ __device__ inline int64_t up128(int64_t x) { return (x + 127) / 128 * 128; }

__host__ __device__ inline int64_t layout_plain_at(int type, int k, int n) {
    return (int64_t)(pj_up(n, PJ_COLS) / PJ_COLS) * (pj_up(k, PJ_KC) / PJ_KC) * pj_parts(type) * PJ_CHUNK;
}

struct BankView {
    const SlotInfo* info;
    const uint16_t* a;   // slot x plane x r_pad x k_pad
    const uint16_t* b;   // slot x plane x n x r_pad
    const float* b32;    // slot x n x r_pad
    int r_pad, k_pad;
};
__host__ __device__ inline int64_t bank_a_at(int slots) { return up128((int64_t)slots * (int64_t)sizeof(SlotInfo) + 128); }
__host__ __device__ inline int64_t bank_b_at(int type, int k, int slots, int max_rank) {
    return bank_a_at(slots) + up128((int64_t)slots * pj_up(max_rank, 16) * pj_up(k, PJ_KC) * pj_parts(type) * 2);
}
__host__ __device__ inline int64_t bank_b32_at(int type, int k, int n, int slots, int max_rank) {
    return bank_b_at(type, k, slots, max_rank) + up128((int64_t)slots * n * pj_up(max_rank, 16) * pj_b_planes(type) * 2);
}
__host__ __device__ inline BankView bank_view(const void* bank, int type, int k, int n, int slots, int max_rank) {
    const uint8_t* p = static_cast<const uint8_t*>(bank);
    return {reinterpret_cast<const SlotInfo*>(p), reinterpret_cast<const uint16_t*>(p + bank_a_at(slots)),
            reinterpret_cast<const uint16_t*>(p + bank_b_at(type, k, slots, max_rank)),
            reinterpret_cast<const float*>(p + bank_b32_at(type, k, n, slots, max_rank)), pj_up(max_rank, 16), pj_up(k, PJ_KC)};
}

// An fp32 weight as three bf16 parts, 8 bits each, rounded; both remainders are exact.  The second part has either sign and
// at most 2^-8 of the value: with the rows' parts, which are cut (pj_parts_of2: third part below 2^-15), the products that are left out stay below
// 2^-23 of the whole and have no sign of their own.  (With a first part that is cut as well x3 w2 reached 2^-22, always towards zero.)  Only
// a value that would round to infinity is cut, and an infinite value has no remainders.
__device__ __forceinline__ void pj_parts_of(float x, __nv_bfloat16 (&h)[3]) {
    h[0] = __float2bfloat16_rn(x);
    if (__hisinf(h[0]) && isfinite(x)) h[0] = __float2bfloat16_rz(x);
    float left = isfinite(x) ? x - __bfloat162float(h[0]) : 0.f;
    h[1] = __float2bfloat16_rn(left);
    h[2] = __float2bfloat16_rn(left - __bfloat162float(h[1]));
}

// Two values, every part cut: 8 + 8 + 8 bits, nothing left.  (The remainders of an infinite value are NaN: the epilogue drops the
// small products where the large one is not finite.)
__device__ __forceinline__ void pj_parts_of2(float x0, float x1, uint32_t& a, uint32_t& b, uint32_t& c) {
    auto cut = [](float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); };
    auto upper = [](float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); };
    const float h0 = cut(x0), h1 = cut(x1);
    a = upper(x0, x1);
    x0 -= h0, x1 -= h1;
    const float m0 = cut(x0), m1 = cut(x1);
    b = upper(x0, x1);
    c = upper(x0 - m0, x1 - m1);
}

// one thread per 16-byte piece of a 16-bit chunk: eight entries of K of one output column
template <typename T>
__global__ void k_layout_weights(const T* W, int64_t ld, int k, int n, uint8_t* out, int chunks, int groups, T* plain) {
    pdl_enter();
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < (int64_t)k * n; i += (int64_t)gridDim.x * blockDim.x)
        plain[i] = W[i / n * ld + i % n];
    const int parts = sizeof(T) == 4 ? 3 : 1;
    const int64_t pieces = (int64_t)groups * chunks * PJ_COLS * 8;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * blockDim.x) {
        const int col = (int)(i % PJ_COLS), c = (int)(i / PJ_COLS % 8);
        const int64_t chunk = i / (PJ_COLS * 8);
        const int kc = (int)(chunk % chunks), group = (int)(chunk / chunks), j = group * PJ_COLS + col;
        uint8_t* to = out + chunk * parts * PJ_CHUNK + tc_swz(col, c);
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int kk = kc * PJ_KC + c * 8 + e;
            v[e] = kk < k && j < n ? W[kk * ld + j] : from_f32<T>(0.f);
        }
        if constexpr (sizeof(T) == 4) {
            Piece<__nv_bfloat16, 8> part[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __nv_bfloat16 h[3];
                pj_parts_of(v[e], h);
                part[0].v[e] = h[0], part[1].v[e] = h[1], part[2].v[e] = h[2];
            }
            for (int q = 0; q < 3; ++q) *reinterpret_cast<Piece<__nv_bfloat16, 8>*>(to + q * PJ_CHUNK) = part[q];
        } else {
            Piece<T, 8> part;
#pragma unroll
            for (int e = 0; e < 8; ++e) part.v[e] = v[e];
            *reinterpret_cast<Piece<T, 8>*>(to) = part;
        }
    }
}

// count adapters into the slots from `first`; bad: set where an entry is not finite
template <int TYPE>
__global__ void k_set_adapters(uint16_t* a_out, uint16_t* b_out, float* b32_out, const typename Elem<TYPE>::T* A, const typename Elem<TYPE>::T* B, int first,
                               int count, int rank, int k, int n, int r_pad, int k_pad, int* bad) {
    pdl_enter();
    using T = typename Elem<TYPE>::T;
    constexpr int PA = TYPE == RIPPLE_TYPE_F32 ? 3 : 1, PB = pj_b_planes(TYPE);
    const int64_t per_a = (int64_t)r_pad * k_pad, per_b = (int64_t)n * r_pad, total = (per_a + per_b) * count;
    bool fine = true;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t s = i / (per_a + per_b);
        int64_t e = i % (per_a + per_b);
        T v = from_f32<T>(0.f);
        if (e < per_a) {
            const int r = (int)(e / k_pad), kk = (int)(e % k_pad);
            if (r < rank && kk < k) v = A[(s * k + kk) * rank + r];
            uint16_t* const to = a_out + (first + s) * PA * per_a + e;
            if constexpr (PA == 3) {
                __nv_bfloat16 h[3];
                pj_parts_of(v, h);
                for (int q = 0; q < 3; ++q) to[q * per_a] = __bfloat16_as_ushort(h[q]);
            } else {
                to[0] = *reinterpret_cast<const uint16_t*>(&v);
            }
        } else {
            e -= per_a;
            const int j = (int)(e / r_pad), r = (int)(e % r_pad);
            if (r < rank) v = B[(s * rank + r) * n + j];
            uint16_t* const to = b_out + (first + s) * PB * per_b + e;
            float left = to_f32(v);
            b32_out[(first + s) * per_b + e] = left;
            if constexpr (PB == 3) {
                __nv_bfloat16 h[3];
                pj_parts_of(left, h);
                for (int q = 0; q < 3; ++q) to[q * per_b] = __bfloat16_as_ushort(h[q]);
            } else {
                for (int q = 0; q < PB; ++q) {
                    const __nv_bfloat16 h = __float2bfloat16_rn(left);
                    to[q * per_b] = __bfloat16_as_ushort(h);
                    left -= __bfloat162float(h);
                }
            }
        }
        fine = fine && isfinite(to_f32(v));
    }
    if (!fine) *bad = 1;
}

// ---- the product ---------------------------------------------------------------------------------------------------
// The adapters that the rows of a tile use, in ascending order, and each row's place among them.
struct alignas(128) TilePlan {
    int32_t count;
    uint16_t slot[128];
    uint8_t row[128];      // 255: none
};
constexpr int PJ_NONE = 255;

struct ProjectParams {
    int rows, k, n, act, chunks;
    const void* x;
    int64_t ld_x, x_rows;
    const int32_t* ids;
    const uint8_t* layout;
    const void* plain;     // W, k x n
    const float* bias;
    BankView bank;         // info null: no adapters
    int n_slots;
    const int32_t* slots;
    TilePlan* plan;        // one per 128 rows
    float* base;           // JOINED: x_i W, rows x n up to a multiple of 16
    void* t;               // t_i = scale_a x_i A_a: fp32, rows x r_pad; 16-bit rows: bf16 parts, rows x t_parts x r_pad
    int t_parts;           // 16-bit results: two, 16 bits of t beside outputs of at most 11; fp32 results: three, all 24
    int batches;           // tensor-core form of t: batches of adapters that are multiplied side by side
    void* y;
    int64_t ld_y;
    int out_f32;
    int withhold;          // diagnostic: no CTA's first accumulator counts as filled
};

__device__ __forceinline__ int64_t row_of(const ProjectParams& p, int i) {
    if (!p.ids) return i;
    const int64_t r = p.ids[i];
    return r >= 0 && r < p.x_rows ? r : -1;
}
// the row's adapter, or -1
__device__ __forceinline__ int slot_of(const ProjectParams& p, int i) {
    const int a = p.slots[i];
    return a >= 0 && a < p.n_slots && p.bank.info[a].rank > 0 ? a : -1;
}

__device__ __forceinline__ void plan_tile(const ProjectParams& p, int tile) {
    constexpr int WORDS = RIPPLE_MAX_SLOTS / 32;
    __shared__ uint32_t used[WORDS], before[WORDS];
    const int t = threadIdx.x, i = tile * 128 + t;      // blocks of 128 threads
    used[t] = 0;
    __syncthreads();
    const int a = i < p.rows && row_of(p, i) >= 0 ? slot_of(p, i) : -1;
    if (a >= 0) atomicOr(&used[a >> 5], 1u << (a & 31));
    __syncthreads();
    TilePlan& plan = p.plan[tile];
    if (t < 32) {
        int n = 0;
        for (int w = 0; w < 4; ++w) n += __popc(used[4 * t + w]);
        int at = warp_inclusive_scan(n) - n;
        if (t == 31) plan.count = at + n;
        for (int w = 0; w < 4; ++w) {
            before[4 * t + w] = at;
            for (uint32_t left = used[4 * t + w]; left; left &= left - 1) plan.slot[at++] = (uint16_t)(32 * (4 * t + w) + __ffs(left) - 1);
        }
    }
    __syncthreads();
    plan.row[t] = a < 0 ? PJ_NONE : (uint8_t)(before[a >> 5] + __popc(used[a >> 5] & ((1u << (a & 31)) - 1)));
}
static_assert(RIPPLE_MAX_SLOTS == 128 * 32, "a thread of plan_tile clears one word");

__global__ void k_plan_tiles(const __grid_constant__ ProjectParams p) {
    pdl_enter();
    plan_tile(p, blockIdx.x);
}

template <int TYPE>
__device__ __forceinline__ void store_t(const ProjectParams& p, int64_t i, int r, float t, int parts) {
    const int rp = p.bank.r_pad;
    if (TYPE == RIPPLE_TYPE_F32 || !parts) {
        static_cast<float*>(p.t)[i * rp + r] = t;
    } else {
        __nv_bfloat16* const to = static_cast<__nv_bfloat16*>(p.t) + i * parts * rp + r;
        for (int q = 0; q < parts; ++q) {
            const __nv_bfloat16 h = __float2bfloat16_rn(t);
            to[q * rp] = h;
            t = __hisinf(h) ? 0.f : t - __bfloat162float(h);
        }
    }
}

// Memory that no kernel in flight writes may be read past the rules of coherence, and is: the bank alone, which is complete before a call that
// reads it is made.  Everything else may be the output of the kernel just before (t and the plan always are; rows, ids, slots, W and
// bias where the caller made them on the same stream), which this kernel's blocks may have been resident beside.
__device__ __forceinline__ float4 bank_word(const float4* from) { return __ldg(from); }
// eight neighbouring entries of the bank as fp32
__device__ __forceinline__ void bank8(float (&v)[8], const float* from) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 e = bank_word(reinterpret_cast<const float4*>(from) + i);
        v[4 * i] = e.x, v[4 * i + 1] = e.y, v[4 * i + 2] = e.z, v[4 * i + 3] = e.w;
    }
}
__device__ __forceinline__ float2 two_of(uint32_t x, __nv_bfloat16) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
__device__ __forceinline__ float2 two_of(uint32_t x, __half) {
    return make_float2(__half2float(__ushort_as_half((unsigned short)(x & 0xffff))), __half2float(__ushort_as_half((unsigned short)(x >> 16))));
}
template <typename T> __device__ __forceinline__ void bank8(float (&v)[8], const T* from) {
    const float4 w = bank_word(reinterpret_cast<const float4*>(from));
    const uint4 e = make_uint4(__float_as_uint(w.x), __float_as_uint(w.y), __float_as_uint(w.z), __float_as_uint(w.w));
    const float2 a = two_of(e.x, T()), b = two_of(e.y, T()), c = two_of(e.z, T()), d = two_of(e.w, T());
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}

// Few rows: t_i by a block per ROWS rows, a warp per four ranks, eight entries of K per lane; rows of one adapter share its loads.
// The rows lie in shared memory as fp32, SF_K entries at a time.  The blocks in front plan the tiles (of the tensor-core form; for
// k_project_few there are none, and t is fp32).
constexpr int SF_K = 1024;
template <int TYPE, int ROWS>
__global__ void __launch_bounds__(128) k_shrink_few(const __grid_constant__ ProjectParams p, int planned) {
    using T = typename Elem<TYPE>::T;
    constexpr int PA = TYPE == RIPPLE_TYPE_F32 ? 3 : 1, RANKS = 4;
    pdl_enter();
    if ((int)blockIdx.x < planned) return plan_tile(p, blockIdx.x);
    __shared__ __align__(16) float xs[ROWS][SF_K];
    const int i0 = (blockIdx.x - planned) * ROWS, lane = lane_id();
    const T* x[ROWS];
    int slot[ROWS];
    bool any = false;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {         // (an id and a slot at once: every load that waits for another costs half a microsecond)
        const int i = min(i0 + q, p.rows - 1);
        const int64_t from = row_of(p, i);
        slot[q] = p.slots[i];
        if (from < 0 || slot[q] < 0 || slot[q] >= p.n_slots || i0 + q >= p.rows) slot[q] = -1;
        x[q] = static_cast<const T*>(p.x) + max(from, (int64_t)0) * p.ld_x;
        any = any || slot[q] >= 0;
    }
    if (!any) return;
    auto stage = [&](int k0) {           // entries k0 .. k0 + SF_K - 1, zeros beyond K
        __syncthreads();
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            T v[SF_K / 128];
#pragma unroll
            for (int e = 0; e < SF_K / 128; ++e) {
                const int kk = k0 + 128 * e + (int)threadIdx.x;
                v[e] = kk < p.k ? x[q][kk] : from_f32<T>(0.f);
            }
#pragma unroll
            for (int e = 0; e < SF_K / 128; ++e) xs[q][128 * e + threadIdx.x] = to_f32(v[e]);
        }
        __syncthreads();
    };
    const bool once = p.k <= SF_K;
    if (once) stage(0);
    const int64_t plane = (int64_t)p.bank.r_pad * p.bank.k_pad;
    for (;;) {
        int a = -1;                          // the first adapter that is left, and its rows
#pragma unroll
        for (int q = ROWS - 1; q >= 0; --q) a = slot[q] >= 0 ? slot[q] : a;
        if (a < 0) break;
        bool mine[ROWS];
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            mine[q] = slot[q] == a;
            if (mine[q]) slot[q] = -1;
        }
        const SlotInfo info = p.bank.info[a];
        for (int r1 = 0; r1 < p.bank.r_pad; r1 += 4 * RANKS) {
            const int r0 = r1 + (threadIdx.x >> 5) * RANKS;
            const uint16_t* const w = p.bank.a + (int64_t)a * PA * plane + (int64_t)r0 * p.bank.k_pad;
            float sum[ROWS][RANKS] = {};
            for (int k0 = 0; k0 < p.k; k0 += SF_K) {
                if (!once) stage(k0);
                if (r0 >= info.rank) continue;
                const int end = min(SF_K, p.k - k0);
                for (int kk = lane * 8; kk < end; kk += 256) {      // (A has zeros up to a multiple of 64 entries)
                    float wv[RANKS][8];
#pragma unroll
                    for (int r = 0; r < RANKS; ++r) {
                        if constexpr (PA == 3) {
                            float part[2][8];
                            const __nv_bfloat16* const from = reinterpret_cast<const __nv_bfloat16*>(w) + r * p.bank.k_pad + k0 + kk;
                            bank8(wv[r], from), bank8(part[0], from + plane), bank8(part[1], from + 2 * plane);
#pragma unroll
                            for (int e = 0; e < 8; ++e) wv[r][e] += part[0][e] + part[1][e];
                        } else {
                            bank8(wv[r], reinterpret_cast<const T*>(w) + r * p.bank.k_pad + k0 + kk);
                        }
                    }
#pragma unroll
                    for (int q = 0; q < ROWS; ++q) {
                        const float4 x0 = *reinterpret_cast<const float4*>(&xs[q][kk]), x1 = *reinterpret_cast<const float4*>(&xs[q][kk + 4]);
#pragma unroll
                        for (int r = 0; r < RANKS; ++r) {
                            float& t = sum[q][r];
                            t = fmaf(x0.x, wv[r][0], t), t = fmaf(x0.y, wv[r][1], t), t = fmaf(x0.z, wv[r][2], t), t = fmaf(x0.w, wv[r][3], t);
                            t = fmaf(x1.x, wv[r][4], t), t = fmaf(x1.y, wv[r][5], t), t = fmaf(x1.z, wv[r][6], t), t = fmaf(x1.w, wv[r][7], t);
                        }
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < ROWS; ++q) {
                if (!mine[q]) continue;
#pragma unroll
                for (int r = 0; r < RANKS; ++r) sum[q][r] = warp_sum(sum[q][r]);
                // (entries beyond the rank are zeros whatever the row holds)
                if (lane < RANKS) {
                    float t = sum[q][0];
#pragma unroll
                    for (int r = 1; r < RANKS; ++r) t = lane == r ? sum[q][r] : t;
                    store_t<TYPE>(p, i0 + q, r0 + lane, r0 + lane < info.rank ? t * info.scale : 0.f, planned > 0 ? p.t_parts : 0);
                }
            }
        }
    }
}

// Few rows: 16 rows x 32 columns of y per block.  A lane is a column, a warp an eighth of every 256 entries of K; what the warps
// have summed meets in shared memory, where each finishes two rows: t_i B_a, bias, activation.  Sums in fp32 throughout.
// Latency is all that counts here (which calls take this form: few_form): 32 entries of W per lane and 16 of the rows per thread are always on
// their way, those of the next 256 entries while these are multiplied.  64 rows, 256 -> 256: 4.3 us alone, 6.4 with 64 adapters of rank 16; 1000
// rows, 602 -> 41: 8.8 and 13.7.  (The tensor-core form: 5.8 and 25, 21 and 37.)
constexpr int PF_ROWS = 16, PF_COLS = 32, PF_K = 256, PF_LD = 20;
template <int TYPE>
__global__ void __launch_bounds__(256) k_project_few(const __grid_constant__ ProjectParams p) {
    using T = typename Elem<TYPE>::T;
    constexpr int OWN = PF_K / 8;
    const bool adapted = p.bank.info != nullptr;
    // With adapters the kernel before computes t, which is waited for below.  It began once all before it was over, so what those kernels
    // wrote is there; up to the wait it is read out of L2, where it is, and not out of an L1 that nothing has brought up to date.
    if (!adapted) pdl_enter();
    __shared__ __align__(16) float xs[2][PF_K * PF_LD];
    const int warp = threadIdx.x >> 5, lane = lane_id(), i0 = blockIdx.x * PF_ROWS;
    const int col = blockIdx.y * PF_COLS + lane, col_in = min(col, p.n - 1);
    const T* const w = static_cast<const T*>(p.plain) + (int64_t)warp * OWN * p.n + col_in;
    T wv[OWN];
    auto fetch_w = [&](int k0) {
        const int left = p.k - k0 - warp * OWN;
#pragma unroll
        for (int j = 0; j < OWN; ++j) wv[j] = j < left ? __ldcg(w + (int64_t)(k0 + j) * p.n) : from_f32<T>(0.f);
    };
    fetch_w(0);
    // thread: a row and every 16th entry of it
    const int xr = threadIdx.x >> 4, xk = threadIdx.x & 15;
    // the row that this thread fetches and the two that its warp finishes; all is asked for before any of it is looked at, since a load that
    // waits for another costs half a microsecond
    const int row[3] = {i0 + xr, i0 + 2 * warp, i0 + 2 * warp + 1};
    int id[3], slot[2] = {-1, -1}, rank[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 3; ++h) id[h] = p.ids ? __ldcg(p.ids + min(row[h], p.rows - 1)) : row[h];
#pragma unroll
    for (int h = 0; h < 2; ++h) if (adapted) slot[h] = __ldcg(p.slots + min(row[1 + h], p.rows - 1));
#pragma unroll
    for (int h = 0; h < 3; ++h) if (row[h] >= p.rows || id[h] >= p.x_rows) id[h] = -1;
    const int64_t x_from = id[0];
    const T* const x = static_cast<const T*>(p.x) + max(x_from, (int64_t)0) * p.ld_x + xk;
    T xv[PF_K / 16];
    auto fetch_x = [&](int k0) {
        const int left = x_from >= 0 ? p.k - k0 - xk : 0;
#pragma unroll
        for (int e = 0; e < PF_K / 16; ++e) xv[e] = 16 * e < left ? __ldcg(x + k0 + 16 * e) : from_f32<T>(0.f);
    };
    auto keep_x = [&](int b) {
#pragma unroll
        for (int e = 0; e < PF_K / 16; ++e) xs[b][(xk + 16 * e) * PF_LD + xr] = to_f32(xv[e]);
    };
    fetch_x(0);
    const int rp = p.bank.r_pad;
    const float* b_at[2] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (id[1 + h] < 0 || slot[h] < 0 || slot[h] >= p.n_slots) slot[h] = -1;
        b_at[h] = p.bank.b32 + ((int64_t)max(slot[h], 0) * p.n + col_in) * rp;
        if (slot[h] >= 0) rank[h] = p.bank.info[slot[h]].rank;
    }
    const float bias = p.bias ? __ldcg(p.bias + col_in) : 0.f;
    float sum[PF_ROWS] = {};
    keep_x(0);
    __syncthreads();
    int b = 0;
    for (int k0 = 0; k0 < p.k; k0 += PF_K, b ^= 1) {
        const bool more = k0 + PF_K < p.k;
        float now[OWN];
#pragma unroll
        for (int j = 0; j < OWN; ++j) now[j] = to_f32(wv[j]);
        if (more) fetch_x(k0 + PF_K), fetch_w(k0 + PF_K);
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
#pragma unroll
            for (int r = 0; r < PF_ROWS; r += 4) {
                const float4 v = *reinterpret_cast<const float4*>(&xs[b][(warp * OWN + j) * PF_LD + r]);
                sum[r] = fmaf(v.x, now[j], sum[r]), sum[r + 1] = fmaf(v.y, now[j], sum[r + 1]);
                sum[r + 2] = fmaf(v.z, now[j], sum[r + 2]), sum[r + 3] = fmaf(v.w, now[j], sum[r + 3]);
            }
        }
        if (more) keep_x(b ^ 1);
        __syncthreads();
    }
    float* const part = xs[0];           // warp x row x column
#pragma unroll
    for (int r = 0; r < PF_ROWS; ++r) part[(warp * PF_ROWS + r) * PF_COLS + lane] = sum[r];
    if (adapted) pdl_enter();
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = 2 * warp + h, i = i0 + r;
        float y = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) y += part[(q * PF_ROWS + r) * PF_COLS + lane];
        y += bias;
        float d = 0.f;
        for (int k = 0; k < rank[h]; k += 8) {
            float t[8], bv[8];
            const float4* const t_at = reinterpret_cast<const float4*>(static_cast<const float*>(p.t) + (int64_t)i * rp + k);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float4 f = __ldcg(t_at + e);
                t[4 * e] = f.x, t[4 * e + 1] = f.y, t[4 * e + 2] = f.z, t[4 * e + 3] = f.w;
            }
            bank8(bv, b_at[h] + k);
#pragma unroll
            for (int e = 0; e < 8; ++e) d = fmaf(t[e], bv[e], d);
        }
        if (rank[h] > 0) y += d;
        if (p.act == RIPPLE_ACT_RELU && y < 0.f) y = 0.f;
        if (col < p.n && id[1 + h] >= 0) {
            if (p.out_f32) static_cast<float*>(p.y)[(int64_t)i * p.ld_y + col] = y;
            else static_cast<T*>(p.y)[(int64_t)i * p.ld_y + col] = from_f32<T>(y);
        }
    }
}

// ---- the product on the tensor cores -------------------------------------------------------------------------------
// Set where a bounded wait gave up; read and cleared by ripple_request_status.
__device__ int g_request_timeout;

constexpr int PJ_ROWS = 128;             // rows per tile: the lanes of the accumulator
constexpr int PJ_EPI_WARPS = 8;          // two per quarter of the lanes
// Rows up to which t is computed by k_shrink_few.  Both sides, us of a whole call with 32 adapters of rank 16 and 20 rows each, row by row /
// on the tensor cores: bf16 602 -> 41, 2000 rows 23 / 32, 4000 rows 27 / 35; 1024 -> 512, 3000 rows 21 / 24, 4000 rows 27 / 25;
// fp32 256 -> 256, 3000 rows 24 / 27, 4000 rows 26 / 27; 128 -> 1024, 4000 rows 30 / 29.
constexpr int PJ_FEW = 3000;
constexpr int PJ_SMS = 148;              // of a B200 (for rules that are asked where no device is current, too)
// Blocks (16 rows x 32 columns) up to which y is computed by k_project_few: few_form.
constexpr int PF_MOST = 160, PF_MOST_F32 = 320;
constexpr int PJ_T_COLS = 64;            // ranks of adapters side by side, where t is computed on the tensor cores
constexpr int PJ_UNIT = 4;               // fp32: chunks (256 entries of K) whose large products share an accumulator
// Polls after which a wait gives up: about a second.  (A limit out of the arguments, shorter for the diagnostic: project-short-runs 83 -> 86 us.)
constexpr uint32_t PJ_SPIN_LIMIT = 1u << 18;
constexpr int PJ_STAGING = PJ_EPI_WARPS * (32 * 17 + 128) * 4;    // the epilogue's turned blocks, and its bias

// MANY: fp32 rows of more than one unit, whose sums the epilogue carries in registers that twice the loader warps would need
template <int TYPE, int BN, bool MANY> struct PjShape {
    static constexpr int PARTS = TYPE == RIPPLE_TYPE_F32 ? 3 : 1;
    static constexpr int LOADERS = PARTS == 3 && !MANY ? 512 : 256;            // threads that fetch rows
    static constexpr int THREADS = LOADERS + 32 * PJ_EPI_WARPS + 64;          // and the warps that issue and that fetch weights
    // columns of tensor memory: two accumulators and, fp32, two for the small products, or room for three of them each
    static constexpr int BUFFER = PARTS == 1 ? BN : BN == 128 ? 256 : BN == 64 ? 256 : 128;
    static constexpr uint32_t TMEM = PARTS == 3 && MANY ? 4 * BN : 2 * BUFFER;
    static constexpr int X_PART = PJ_ROWS * 128, X_STAGE = PARTS * X_PART;
    static constexpr int W_PART = BN * 128, W_STAGE = PARTS * W_PART;
    static constexpr int STAGE = X_STAGE + W_STAGE;
    static constexpr int STAGES = 200 * 1024 / STAGE < 8 ? 200 * 1024 / STAGE : 8;
    static constexpr size_t BYTES = (size_t)STAGES * STAGE + PJ_STAGING + 1024;
};

// instruction descriptor: fp32 accumulators, both operands K-major, 128 rows, n columns
__device__ __forceinline__ uint32_t pj_idesc(int type, int n) {
    const uint32_t t = type == RIPPLE_TYPE_F16 ? 0u : 1u;
    return (1u << 4) | (t << 7) | (t << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(PJ_ROWS >> 4) << 24);
}

__device__ __forceinline__ uint16_t bits_of(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }
__device__ __forceinline__ uint16_t bits_of(__half x) { return __half_as_ushort(x); }

__device__ __forceinline__ void pj_store8(void* to, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

template <typename T> __device__ __forceinline__ uint32_t pj_pair(float a, float b) {
    return (uint32_t)bits_of(from_f32<T>(a)) | (uint32_t)bits_of(from_f32<T>(b)) << 16;
}

__device__ __forceinline__ void pj_sts(uint32_t to, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// 16 bytes of eight entries
__device__ __forceinline__ uint4 word_of(const Piece<float, 8>& v, int h) {
    return make_uint4(__float_as_uint(v.v[4 * h]), __float_as_uint(v.v[4 * h + 1]), __float_as_uint(v.v[4 * h + 2]), __float_as_uint(v.v[4 * h + 3]));
}
template <typename T> __device__ __forceinline__ uint4 word_of(const Piece<T, 8>& v, int) {
    auto two = [&](int e) { return (uint32_t)bits_of(v.v[e]) | (uint32_t)bits_of(v.v[e + 1]) << 16; };
    return make_uint4(two(0), two(2), two(4), two(6));
}

// What a launch of k_project_rows computes: t; y, with steps over ranks; or x W with t beside it.
// _3: t of 16-bit rows in three parts, for fp32 results, half as many ranks per step (30 011 rows, fp16, 512 -> 768, 7 adapters of rank 32 per
// tile: 139 us, in two parts 92; 65 536 bf16 rows of 1024, one adapter of rank 16 per tile: 207 and 205).
enum { PJ_SHRINK, PJ_RANKS, PJ_JOINED, PJ_SHRINK_3, PJ_RANKS_3 };

// A persistent CTA takes tiles of 128 rows x BN columns: lanes of the accumulator are rows, its columns output columns.
// SHRINK: the columns are the ranks of adapters that the tile's rows use, side by side, and each row keeps those of its own: t.
// JOINED: columns of W, and behind them such ranks: one pass over the rows for both; k_finish_rows makes y of them.
// RANKS: columns of y; behind the steps over K come steps over ranks, the adapters of the tile one behind the other, where a
// row's operand is its t at its adapter's ranks and zero at all others.
//   loaders    fetch the rows by id, chunk by chunk of 64 entries, into the swizzled layout that the tensor core reads: 16-bit
//              rows as asynchronous copies, fp32 rows (and rows that are not 16-byte aligned) through registers,
//              fp32 entries as three bf16 parts; and what comes out of the bank
//   one thread copies the weights' chunks, one issues the products
//   epilogue   takes a finished accumulator while the next is being filled: bias, activation, and out
// fp32: six products of parts (all but those below 2^-23, see pj_parts_of); the large one of the first parts is handed over every 256 entries
// and summed in registers, because the tensor core cuts what its additions lose; the small ones gather over the whole tile.
// Barriers, all waits bounded: full[s] (one arrival per loader warp, 16-bit rows: per thread; one with the bytes of the weights),
// empty[s] (the products that read stage s), acc_full[b], acc_empty[b] (one arrival per epilogue warp).
//
// What bounds it.  16-bit rows: at 65 536 x 1024 x 1024 (no adapters) 125 us, 1.1 PFLOP/s, 68 % of the measured cuBLAS rate; a step (128 rows x 256
// columns x 64 entries) takes 800 cycles, of which its products are 512, and brings 48 KB out of L2 (27 % of what L2 can): hand-overs
// between the roles, and power.  Tiles of 128 columns, half the products per hand-over: 200 us.  Asking ahead for the next step's operands,
// or for two steps' at once: 185 and 176 with adapters, against 171.  fp32: the loaders' chain per step -- loads out of L2, parts, stores -- of 1500 cycles beside
// 1000 (narrow) to 1550 (128 columns) of products, which read 192 KB of shared memory; 200 000 gathered rows of 256 to 47 columns in
// 72 us, 205 MB at 2.8 TB/s.  Two stages of 96 KB are all that fits; a third (narrow tiles, 72 KB) gained nothing.
template <int TYPE, int BN, int MODE, bool MANY>
__global__ void __launch_bounds__(PjShape<TYPE, BN, MANY>::THREADS, 1) k_project_rows(const __grid_constant__ ProjectParams p) {
    using T = typename Elem<TYPE>::T;
    using S = PjShape<TYPE, BN, MANY>;
    constexpr bool SHRINK = MODE == PJ_SHRINK || MODE == PJ_SHRINK_3, JOINED = MODE == PJ_JOINED, BATCHED = SHRINK || JOINED;
    constexpr int PJ_LOADERS = S::LOADERS, A_COLS = SHRINK ? BN : PJ_T_COLS, W_COLS = JOINED ? BN - PJ_T_COLS : BN;
    // fp32, narrow tiles: the parts of W lie one behind the other and are multiplied at once, x1 [w1 w2 w3], x2 [w1 w2], x3 w1: half the
    // instructions, and two thirds of what they read of shared memory.  Accumulators: large, small, small.
    // (Whether a tile is narrow is a matter of the projection alone, not of the adapters that its rows happen to use: a row's result does not
    // depend on its neighbours.)
    constexpr int SIDE = S::PARTS == 3 && !MANY ? (BN < S::BUFFER / 3 ? BN : S::BUFFER / 3 / 16 * 16) : 0;      // up to so many columns
    constexpr int PARTS = S::PARTS, STAGES = S::STAGES, NB = BN / 32, B_PLANES = pj_b_planes(TYPE);
    constexpr int T_PARTS = MODE == PJ_SHRINK_3 || MODE == PJ_RANKS_3 ? 3 : 2;
    constexpr int RANKS = PARTS == 3 ? 64 : T_PARTS == 3 ? 16 : 32;            // ranks that a step of t_i B_a takes
    constexpr uint32_t TMEM = S::TMEM;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int s_fail;

    const int tid = threadIdx.x, warp = __shfl_sync(FULL, tid >> 5, 0), lane = tid & 31;
    const int across = SHRINK ? p.batches : (p.n + W_COLS - 1) / W_COLS, row_tiles = (p.rows + PJ_ROWS - 1) / PJ_ROWS;
    const int64_t tiles = (int64_t)across * row_tiles;
    const int my_tiles = (int)((tiles - blockIdx.x + gridDim.x - 1) / gridDim.x), chunks = p.chunks;
    const int r_pad = p.bank.r_pad, joined_w = (p.n + 15) & ~15;
    const bool joined_side = JOINED && SIDE > 0 && joined_w + r_pad <= SIDE;
    const int at_once = BATCHED && r_pad ? (joined_side ? min(A_COLS, SIDE - joined_w) : A_COLS) / r_pad : 0;
    uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    // A tile: 128 rows, a tile of columns, and (SHRINK, JOINED) a batch of adapters: SHRINK takes every `across`-th batch that the
    // adapters of the rows fill, JOINED all of them (one where there are none).  The next row tile's count of adapters is asked for early.
    struct Tile { int lt, rows, part, batch, count, count_next; };
    // (Positions are stepped from tile to tile: two 64-bit divisions per tile and warp were 3000 cycles.)
    const int rows_on = gridDim.x / across, parts_on = gridDim.x % across;
    auto on = [&](int& rows, int& part) {
        rows += rows_on, part += parts_on;
        if (part >= across) part -= across, ++rows;
    };
    auto adapters = [&](int lt, int rows) { return p.plan && lt < my_tiles ? p.plan[rows].count : 0; };
    auto after = [&](const Tile& t) {
        Tile n = t;
        if constexpr (BATCHED) n.batch += SHRINK ? across : 1;
        while (!BATCHED || n.batch * at_once >= n.count) {
            if (++n.lt >= my_tiles) break;
            on(n.rows, n.part);
            n.batch = SHRINK ? n.part : 0, n.count = n.count_next;
            int rows = n.rows, part = n.part;
            on(rows, part);
            n.count_next = adapters(n.lt + 1, rows);
            if (!SHRINK) break;
        }
        return n;
    };
    auto first_tile = [&]() {
        const int rows = blockIdx.x / across, part = blockIdx.x % across;
        Tile before{-1, rows - rows_on, part - parts_on, 0, 0, adapters(0, rows)};
        if (before.part < 0) before.part += across, --before.rows;
        return after(before);
    };
    // columns that are multiplied: of W, and ranks of the batch behind them
    auto tile_w = [&](const Tile& t) { return SHRINK ? 0 : min(W_COLS, (p.n - t.part * W_COLS + 15) & ~15); };
    auto tile_n = [&](const Tile& t) { return tile_w(t) + (BATCHED ? min(at_once, t.count - t.batch * at_once) * r_pad : 0); };
    auto side_by_side = [&](const Tile& t) { return SIDE > 0 && (SHRINK || (JOINED ? joined_side : tile_w(t) <= SIDE)); };
    // bytes between the parts of a tile's W (and A) in a stage
    auto w_part = [&](const Tile& t) { return side_by_side(t) ? tile_n(t) * 128 : S::W_PART; };
    // Tensor memory: fp32 tiles of one unit have their large and small accumulators in one of two buffers; with MANY two of the former
    // for units, two of the latter for tiles.
    auto large_at = [&](int b) { return (uint32_t)(PARTS == 3 && !MANY ? S::BUFFER * b : BN * b); };
    auto small_at = [&](int b, int worked, bool side, int nt) { return side ? large_at(b) + (uint32_t)nt : !MANY ? large_at(b) + BN : (uint32_t)(2 * BN + (worked & 1) * BN); };
    auto rank_steps = [&](int count) { return BATCHED ? 0 : (count * r_pad + RANKS - 1) / RANKS; };

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], (PARTS == 3 ? PJ_LOADERS / 32 : PJ_LOADERS) + (SHRINK ? 0 : 1)); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], p.withhold ? 2 : 1 /* one arrives */); mbar_init(&acc_empty[b], PJ_EPI_WARPS); }
        mbar_init(&drained, 1);
        s_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_enter();

    if (warp < PJ_LOADERS / 32) {
        // ---------------- rows, and what comes out of the bank ----------------
        constexpr int RSTEP = PJ_LOADERS / 8, ITS = PJ_ROWS / RSTEP, W_ITS = ((BATCHED ? A_COLS : BN) + RSTEP - 1) / RSTEP;
        const int c = tid & 7, rb = tid >> 3;       // thread: piece c (8 entries) of the rows rb + RSTEP it
        const uint32_t mine = smem_u32(ring) + tc_swz(rb, c);
        const bool vec = (reinterpret_cast<uintptr_t>(p.x) & 15) == 0 && p.ld_x % (16 / (int)sizeof(T)) == 0;
        const bool regs = PARTS == 3 || !vec;
        const int tail = p.k - (chunks - 1) * PJ_KC - c * 8;      // entries of this thread's piece of the last chunk
        // rank steps: this thread's piece of a step is a plane's ranks from c_rank
        const int c_plane = c / (RANKS / 8), c_rank = c % (RANKS / 8) * 8;
        // This thread's pieces of the rows of the tile being fetched, at its next chunk (rows that do not exist read row 0 of x, and
        // their results are dropped); of the rows of A; the rows' places among the adapters, a byte each; and all of it for the next tile.
        const T* const x0 = static_cast<const T*>(p.x) + c * 8;
        const T* at[ITS];
        const uint16_t* a_at[BATCHED ? W_ITS : 1] = {};
        // (aim() only asks for what the next tile's addresses come from; turn(), a tile later, looks at it: what is looked at right away
        // is waited for, 4500 cycles at the start of every tile)
        int id_next[ITS], row_next[BATCHED ? 1 : ITS], slot_next[BATCHED ? W_ITS : 1], slot0 = -1;
        uint32_t which = 0;
        int place[BATCHED ? W_ITS : 1], a_row[BATCHED ? W_ITS : 1];      // rows of A that this thread fetches: adapter within the batch, offset
        if (BATCHED && r_pad) {
#pragma unroll
            for (int it = 0; it < W_ITS; ++it) place[it] = (rb + RSTEP * it) / r_pad, a_row[it] = (rb + RSTEP * it) % r_pad * p.bank.k_pad + c * 8;
        }
        const int first_place = !BATCHED && r_pad ? c_rank / r_pad : 0;
        auto aim = [&](const Tile& t) {
            if (t.lt >= my_tiles) return;
            const int r0 = t.rows * PJ_ROWS + rb;
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                const int i = min(r0 + RSTEP * it, p.rows - 1);
                id_next[it] = p.ids ? p.ids[i] : i;
            }
            if (!p.plan) return;
            const TilePlan& plan = p.plan[t.rows];
            if constexpr (BATCHED) {                // slots of the rows of A that this thread fetches
#pragma unroll
                for (int it = 0; it < W_ITS; ++it) slot_next[it] = plan.slot[min(t.batch * at_once + place[it], PJ_ROWS - 1)];
            } else {
#pragma unroll
                for (int it = 0; it < ITS; ++it) row_next[it] = plan.row[rb + RSTEP * it];
                slot_next[0] = plan.slot[min(first_place, PJ_ROWS - 1)];
            }
        };
        auto row_next_at = [&](int it) { return x0 + (id_next[it] >= 0 && id_next[it] < p.x_rows ? id_next[it] : 0) * p.ld_x; };
        auto turn = [&](const Tile& t) {            // to the tile that was aimed at
#pragma unroll
            for (int it = 0; it < ITS; ++it) at[it] = row_next_at(it);
            if (!p.plan) return;
            if constexpr (BATCHED) {
                const int64_t plane = (int64_t)r_pad * p.bank.k_pad;
#pragma unroll
                for (int it = 0; it < W_ITS; ++it) {
                    const bool real = place[it] < at_once && t.batch * at_once + place[it] < t.count;
                    a_at[it] = !real ? nullptr : p.bank.a + (int64_t)slot_next[it] * PARTS * plane + a_row[it];
                }
            } else {
                which = 0;
#pragma unroll
                for (int it = 0; it < ITS; ++it) which |= (uint32_t)row_next[it] << (8 * it);
                slot0 = first_place < t.count ? slot_next[0] : -1;
            }
        };
        constexpr int WORDS = sizeof(T) / 2;        // 16-byte words of eight entries
        uint4 raw[ITS][WORDS];
        auto fetch = [&](bool last) {               // the next chunk of the rows, through registers
            const int left = last ? tail : 8;
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                if (vec && left >= 8) {
#pragma unroll
                    for (int h = 0; h < WORDS; ++h) raw[it][h] = reinterpret_cast<const uint4*>(at[it])[h];
                } else {
                    Piece<T, 8> v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v.v[e] = e < left ? at[it][e] : from_f32<T>(0.f);
#pragma unroll
                    for (int h = 0; h < WORDS; ++h) raw[it][h] = word_of(v, h);
                }
                at[it] += PJ_KC;
            }
        };
        // a row's t, where the step's ranks are its adapter's
        auto fetch_t = [&](const Tile& t, int step) {
            if constexpr (PARTS == 3) {
                const int q = step * RANKS + c_rank, j = q / r_pad, r = q % r_pad;
                const int64_t i0 = (int64_t)t.rows * PJ_ROWS + rb;
#pragma unroll
                for (int it = 0; it < ITS; ++it) {
                    const bool own = (int)(which >> (8 * it) & 255) == j;
                    const uint4* const from = reinterpret_cast<const uint4*>(static_cast<const float*>(p.t) + (i0 + RSTEP * it) * r_pad + r);
#pragma unroll
                    for (int h = 0; h < WORDS; ++h) raw[it][h] = own ? __ldcg(from + h) : make_uint4(0, 0, 0, 0);
                }
            }
        };
        auto keep = [&](int s) {                    // what was fetched, into a stage
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                const uint32_t to = mine + (uint32_t)(s * S::STAGE + it * (RSTEP * 128));
                if constexpr (PARTS == 3) {
                    uint4 a, b, d;
                    auto f = [](uint32_t x) { return __uint_as_float(x); };
                    pj_parts_of2(f(raw[it][0].x), f(raw[it][0].y), a.x, b.x, d.x);
                    pj_parts_of2(f(raw[it][0].z), f(raw[it][0].w), a.y, b.y, d.y);
                    pj_parts_of2(f(raw[it][WORDS - 1].x), f(raw[it][WORDS - 1].y), a.z, b.z, d.z);
                    pj_parts_of2(f(raw[it][WORDS - 1].z), f(raw[it][WORDS - 1].w), a.w, b.w, d.w);
                    pj_sts(to, a), pj_sts(to + S::X_PART, b), pj_sts(to + 2 * S::X_PART, d);
                } else {
                    pj_sts(to, raw[it][0]);
                }
            }
        };
        auto copy = [&](uint32_t to, const void* from) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
        };
        auto copy_some = [&](uint32_t to, const void* from, uint32_t bytes) {    // zeros behind the first `bytes`
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
        };
        bool ok = true, fetched = false;
        int s = 0;
        uint32_t ph = 1;                            // (a fresh barrier counts as completed)
        Tile tile = first_tile();
        aim(tile);
        while (tile.lt < my_tiles && ok) {
            if (!fetched || !regs) turn(tile);
            if (regs && !fetched) fetch(chunks == 1);
            fetched = true;
            const int steps = chunks + rank_steps(tile.count);
            Tile following = tile;
            for (int st = 0; st < steps; ++st) {
                ok = mbar_wait_warp(&empty[s], ph, PJ_SPIN_LIMIT);
                if (!ok) break;
                const uint32_t x_to = mine + (uint32_t)(s * S::STAGE), w_to = x_to + S::X_STAGE + (JOINED ? 128 * tile_w(tile) : 0);
                const int between = PARTS == 3 ? w_part(tile) : 0;
                bool copied = false;
                if (st < chunks) {
                    if constexpr (BATCHED) {
                        const int64_t plane = (int64_t)r_pad * p.bank.k_pad;
#pragma unroll
                        for (int it = 0; it < W_ITS; ++it) {
                            if (!a_at[it]) continue;
                            copied = true;
#pragma unroll
                            for (int q = 0; q < PARTS; ++q) copy(w_to + q * between + it * (RSTEP * 128), a_at[it] + q * plane);
                            a_at[it] += PJ_KC;
                        }
                    }
                    if (regs) {
                        keep(s);
                    } else if (st < chunks - 1 || tail >= 8) {
#pragma unroll
                        for (int it = 0; it < ITS; ++it) {
                            copy(x_to + it * (RSTEP * 128), at[it]);
                            at[it] += PJ_KC;
                        }
                    } else {
#pragma unroll
                        for (int it = 0; it < ITS; ++it) copy_some(x_to + it * (RSTEP * 128), tail > 0 ? at[it] : at[it] - c * 8, tail > 0 ? 2 * tail : 0);
                    }
                } else if constexpr (!BATCHED) {
                    const int step = st - chunks, q = step * RANKS + c_rank, j = q / r_pad, r = q % r_pad;
                    const int slot = step == 0 ? slot0 : j < tile.count ? p.plan[tile.rows].slot[j] : -1;
                    const int64_t plane = (int64_t)p.n * r_pad;
#pragma unroll
                    for (int it = 0; it < W_ITS; ++it) {
                        const int in_tile = rb + RSTEP * it, col = tile.part * BN + in_tile;
                        if (in_tile >= (PARTS == 3 ? tile_n(tile) : BN)) continue;      // (behind them lies the next part)
                        copied = true;
                        const bool real = slot >= 0 && col < p.n;
                        const uint16_t* const from = p.bank.b + (real ? (int64_t)slot * B_PLANES * plane + (int64_t)col * r_pad + r : 0);
                        if constexpr (PARTS == 3) {
#pragma unroll
                            for (int k = 0; k < B_PLANES; ++k) copy_some(w_to + k * between + it * (RSTEP * 128), from + (real ? k * plane : 0), real ? 16 : 0);
                        } else if (c_plane < B_PLANES) {
                            copy_some(w_to + it * (RSTEP * 128), from + (real ? c_plane * plane : 0), real ? 16 : 0);
                        }
                    }
                    if constexpr (PARTS == 3) {
                        keep(s);
                    } else {
                        const int64_t i0 = (int64_t)tile.rows * PJ_ROWS + rb;
#pragma unroll
                        for (int it = 0; it < ITS; ++it) {
                            const bool own = (int)(which >> (8 * it) & 255) == j;
                            const __nv_bfloat16* const t = static_cast<const __nv_bfloat16*>(p.t);
                            if (c_plane >= T_PARTS) continue;                            // (a fourth place that no product reads)
                            copy_some(x_to + it * (RSTEP * 128), own ? t + ((i0 + RSTEP * it) * T_PARTS + c_plane) * r_pad + r : t, own ? 16 : 0);
                        }
                    }
                }
                // 16-bit rows: the barrier counts threads, and the copies of a thread arrive for it when they have landed.  fp32: it counts
                // warps, and the copies of a thread that has some are counted on top.
                if (PARTS == 1 && vec) {
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[s])) : "memory");
                } else if (PARTS == 1) {
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    mbar_arrive(&full[s]);
                } else {
                    if (copied) asm volatile("cp.async.mbarrier.arrive.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[s])) : "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&full[s]);
                }
                if (st == 0) {                      // (between two steps and not before the first: the stages ahead hide it)
                    following = after(tile);
                    aim(following);
                }
                if (PARTS == 3 && st == min(1, steps - 1) && p.ids && following.lt < my_tiles) {
                    // the next tile's rows, on their way to L2 a tile ahead: gathered rows come from far (project-cached-rows 136 -> 128 us; rows in
                    // order, and 16-bit rows, whose copies run further ahead, lose by it)
#pragma unroll
                    for (int it = 0; it < ITS; ++it) {
                        const uint8_t* const line = reinterpret_cast<const uint8_t*>(row_next_at(it) - c * 8);
                        for (int at = c * 128; at < p.k * (int)sizeof(T); at += 1024) asm volatile("prefetch.global.L2 [%0];" ::"l"(line + at));
                    }
                }
                if (regs) {                         // what the next step keeps is requested now: of this tile, or of the one after it
                    if (st + 1 < chunks) fetch(st + 2 == chunks);
                    else if (st + 1 < steps) fetch_t(tile, st + 1 - chunks);
                    else if (following.lt < my_tiles) turn(following), fetch(chunks == 1);
                }
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
            tile = following;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (!ok) s_fail = 1;
    } else if (warp < PJ_LOADERS / 32 + PJ_EPI_WARPS) {
        // ---------------- epilogue ----------------
        const int q = warp & 3, half = (warp - PJ_LOADERS / 32) >> 2;
        const uint32_t lanes = tmem + ((uint32_t)(32 * q) << 16);
        float* const staging = reinterpret_cast<float*>(ring + STAGES * S::STAGE) + (warp - PJ_LOADERS / 32) * (32 * 17);
        float* const bias = reinterpret_cast<float*>(ring + STAGES * S::STAGE) + PJ_EPI_WARPS * 32 * 17 + (warp - PJ_LOADERS / 32) * 16 * NB;
        const int out_size = p.out_f32 ? 4 : (int)sizeof(T);
        const bool vec = (reinterpret_cast<uintptr_t>(p.y) & 31) == 0 && p.ld_y * out_size % 32 == 0;
        const int units = PARTS == 3 ? (chunks + PJ_UNIT - 1) / PJ_UNIT : 1;
        bool ok = true;
        int sg = 0, worked = 0;                 // accumulators and tiles taken so far
        for (Tile tile = first_tile(); tile.lt < my_tiles && ok; tile = after(tile)) {
            // thread: a row, and the 16-column blocks half, half + 2, ... of the tile
            const int nt = tile_n(tile), nw = tile_w(tile);
            const int i = tile.rows * PJ_ROWS + 32 * q + lane, c0 = SHRINK ? 0 : tile.part * W_COLS;
            int own = -1, rank = 0;            // SHRINK, JOINED: the row's adapter within the batch
            float scale = 0.f;
            bool live = i < p.rows;
            if (!SHRINK) live = live && row_of(p, i) >= 0;
            if (BATCHED && p.plan) {
                const TilePlan& plan = p.plan[tile.rows];
                const int at = plan.row[32 * q + lane];
                if (at != PJ_NONE) {
                    const SlotInfo info = p.bank.info[plan.slot[at]];
                    rank = info.rank, scale = info.scale;
                    own = at - tile.batch * at_once;
                }
                live = live && tile.batch == 0;       // (JOINED: W's columns are multiplied with every batch, and kept with the first)
            }
            const uint32_t rows_live = __ballot_sync(FULL, live);
            if constexpr (!BATCHED) {               // the bias of this warp's columns, while the products are still on their way
                __syncwarp();
                for (int e = lane; e < 16 * NB; e += 32) {
                    const int col = c0 + 16 * (2 * (e >> 4) + half) + (e & 15);
                    bias[e] = p.bias && col < p.n ? p.bias[col] : 0.f;
                }
                __syncwarp();
            }
            // 16 finished sums of this row, from column `at` of the tile
            auto finish = [&](float (&y)[16], int at) {
                if (JOINED && at < nw) {
                    if (live) {
                        float* const to = p.base + (int64_t)i * pj_up(p.n, 16) + c0 + at;
                        uint32_t v[8], w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = __float_as_uint(y[e]), w[e] = __float_as_uint(y[8 + e]);
                        pj_store8(to, v), pj_store8(to + 8, w);
                    }
                    return;
                }
                if constexpr (BATCHED) {
                    at -= nw;
                    if (own < 0 || own != at / r_pad) return;
                    const int r = at % r_pad;
                    uint32_t v[8], w[8];
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = r + e < rank ? y[e] * scale : 0.f;
                    if constexpr (PARTS == 3) {
                        float* const to = static_cast<float*>(p.t) + (int64_t)i * r_pad + r;
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = __float_as_uint(y[e]), w[e] = __float_as_uint(y[8 + e]);
                        pj_store8(to, v), pj_store8(to + 8, w);
                    } else {
                        __nv_bfloat16* const to = static_cast<__nv_bfloat16*>(p.t) + (int64_t)i * T_PARTS * r_pad + r;
#pragma unroll
                        for (int q = 0; q < T_PARTS; ++q) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                v[e] = pj_pair<__nv_bfloat16>(y[2 * e], y[2 * e + 1]);
                                const float h0 = __uint_as_float(v[e] << 16), h1 = __uint_as_float(v[e] & 0xffff0000u);
                                y[2 * e] = fabsf(h0) < INFINITY ? y[2 * e] - h0 : 0.f, y[2 * e + 1] = fabsf(h1) < INFINITY ? y[2 * e + 1] - h1 : 0.f;
                            }
                            pj_store8(to + q * r_pad, v);
                        }
                    }
                    return;
                }
                at += c0;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    y[e] += bias[(at - c0) / 32 * 16 + e];
                    if (p.act == RIPPLE_ACT_RELU && y[e] < 0.f) y[e] = 0.f;
                }
                if (vec && at + 16 <= p.n) {
                    if (live) {
                        uint32_t v[8];
                        if (p.out_f32) {
                            float* const to = static_cast<float*>(p.y) + (int64_t)i * p.ld_y + at;
#pragma unroll
                            for (int e = 0; e < 16; e += 8) {
#pragma unroll
                                for (int k = 0; k < 8; ++k) v[k] = __float_as_uint(y[e + k]);
                                pj_store8(to + e, v);
                            }
                        } else if constexpr (PARTS == 1) {
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] = pj_pair<T>(y[2 * k], y[2 * k + 1]);
                            pj_store8(static_cast<T*>(p.y) + (int64_t)i * p.ld_y + at, v);
                        }
                    }
                } else {
                    // through shared memory: two rows of 16 columns per store
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 16; ++e) staging[lane * 17 + e] = y[e];
                    __syncwarp();
                    const int e = lane & 15;
                    if (at + e < p.n) {
#pragma unroll 4
                        for (int r = lane >> 4; r < 32; r += 2) {
                            if (!(rows_live >> r & 1)) continue;
                            const int64_t to = (int64_t)(i - lane + r) * p.ld_y + at + e;
                            const float v = staging[r * 17 + e];
                            if (p.out_f32) static_cast<float*>(p.y)[to] = v;
                            else static_cast<T*>(p.y)[to] = from_f32<T>(v);
                        }
                    }
                }
            };
            constexpr int CARRY = PARTS == 3 && MANY ? NB : 1;
            float sum[CARRY][16];              // fp32: of the units before the last
            for (int u = 0; u < units && ok; ++u, ++sg) {
                const int b = sg & 1;
                const bool side = side_by_side(tile);
                const uint32_t large = lanes + large_at(b), small = lanes + small_at(b, worked, side, nt);
                ok = mbar_wait_warp(&acc_full[b], (sg >> 1) & 1, PJ_SPIN_LIMIT);
                if (!ok) break;
                tc_fence_after();
                if (PARTS == 3 && MANY && u < units - 1) {
#pragma unroll
                    for (int j = 0; j < CARRY; ++j) {
                        const int at = 16 * (2 * j + half);
                        if (at >= nt) continue;
                        uint32_t x[16];
                        tc_load16(x, large + (uint32_t)at);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                        for (int e = 0; e < 16; ++e) sum[j][e] = u ? sum[j][e] + __uint_as_float(x[e]) : __uint_as_float(x[e]);
                    }
                } else {
#pragma unroll 1
                    for (int j = 0; j < NB; ++j) {
                        const int at = 16 * (2 * j + half);
                        if (at >= nt) break;
                        uint32_t x[16];
                        float y[16];
                        tc_load16(x, large + (uint32_t)at);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                        for (int e = 0; e < 16; ++e) y[e] = __uint_as_float(x[e]);
                        if constexpr (PARTS == 3) {
                            if (MANY && u > 0) {
#pragma unroll
                                for (int e = 0; e < 16; ++e) {
                                    float before = sum[0][e];
#pragma unroll
                                    for (int k = 1; k < CARRY; ++k) before = k == j ? sum[k][e] : before;
                                    y[e] += before;
                                }
                            }
                            tc_load16(x, small + (uint32_t)at);
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                            // (an infinite entry has no parts: its small products may be NaN)
#pragma unroll
                            for (int e = 0; e < 16; ++e) if (fabsf(y[e]) < INFINITY) y[e] += __uint_as_float(x[e]);
                            if (SIDE > 0 && side) {
                                tc_load16(x, small + (uint32_t)(nt + at));
                                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                                for (int e = 0; e < 16; ++e) if (fabsf(y[e]) < INFINITY) y[e] += __uint_as_float(x[e]);
                            }
                        }
                        finish(y, at);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[b]);
            }
            ++worked;
        }
        if (!ok) s_fail = 1;
    } else if (warp == PJ_LOADERS / 32 + PJ_EPI_WARPS) {
        // ---------------- products ----------------
        const bool lead = tc_elect();
        const uint64_t d0 = tc_smem_desc(__shfl_sync(FULL, smem_u32(ring), 0));
        int s = 0, sg = 0, worked = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (Tile tile = first_tile(); tile.lt < my_tiles && ok; tile = after(tile)) {
            const int count = __shfl_sync(FULL, tile.count, 0), nt = __shfl_sync(FULL, tile_n(tile), 0), steps = chunks + rank_steps(count);
            const bool side = __shfl_sync(FULL, side_by_side(tile), 0);
            const uint32_t idesc2 = pj_idesc(TYPE, 2 * nt), idesc3 = pj_idesc(TYPE, 3 * nt);
            const uint32_t idesc = pj_idesc(TYPE, nt), idesc_t = pj_idesc(RIPPLE_TYPE_BF16, nt);
            uint32_t acc = 0, small = 0;
            int left = p.k, left_t = count * r_pad, b = 0;
            for (int st = 0; st < steps; ++st) {
                const bool first = PARTS == 3 ? st < chunks && st % PJ_UNIT == 0 : st == 0;
                if (first) {
                    b = sg & 1;
                    const int before = sg >> 1;
                    ++sg;
                    // the epilogue must have read this accumulator (and with it the small products of the tile before the last)
                    if (before > 0) ok = mbar_wait_warp(&acc_empty[b], (before - 1) & 1, PJ_SPIN_LIMIT);
                    if (!ok) break;
                    tc_fence_after();
                    acc = __shfl_sync(FULL, tmem + large_at(b), 0), small = __shfl_sync(FULL, tmem + small_at(b, worked, side, nt), 0);
                }
                ok = mbar_wait_warp(&full[s], ph, PJ_SPIN_LIMIT);
                if (!ok) break;
                fence_async_smem();      // the loaders' stores, for the tensor core (on the reader's side: loads in flight are not waited for)
                tc_fence_after();
                // (broadcast: operands that the compiler cannot see to be the warp's take ten times as long to issue)
                const uint64_t x = d0 + (uint64_t)((uint32_t)__shfl_sync(FULL, s, 0) * (S::STAGE >> 4)), w = x + (S::X_STAGE >> 4);
                const bool last = st == steps - 1 || (PARTS == 3 && st < chunks - 1 && st % PJ_UNIT == PJ_UNIT - 1);
                constexpr uint64_t XP = S::X_PART >> 4, WP = S::W_PART >> 4;
                if (lead) {
                    if (PARTS == 3 || st < chunks) {
                        const int here = st < chunks ? left : left_t;
                        const uint32_t kind = st < chunks ? idesc : idesc_t;
#pragma unroll
                        for (int j = 0; j < PJ_KC / 16; ++j) {        // 16 entries = 32 bytes per instruction
                            if (16 * j < here) {
                                const uint64_t x1 = x + 2 * j, w1 = w + 2 * j;
                                if (SIDE > 0 && side) {
                                    tc_mma_bf16(acc, x1, w1, idesc3, (st | j) != 0);
                                    tc_mma_bf16(small, x1 + XP, w1, idesc2, 1u);
                                    tc_mma_bf16(small, x1 + 2 * XP, w1, kind, 1u);
                                    continue;
                                }
                                tc_mma_bf16(acc, x1, w1, kind, !first || j != 0);
                                if constexpr (PARTS == 3) {
                                    tc_mma_bf16(small, x1, w1 + WP, kind, (st | j) != 0);
                                    tc_mma_bf16(small, x1 + XP, w1, kind, 1u);
                                    tc_mma_bf16(small, x1 + XP, w1 + WP, kind, 1u);
                                    tc_mma_bf16(small, x1, w1 + 2 * WP, kind, 1u);
                                    tc_mma_bf16(small, x1 + 2 * XP, w1, kind, 1u);
                                }
                            }
                        }
                    } else {
                        // t in two parts (64 bytes of a row each) or three (32 bytes each), B in one or two.  Left out: with two the product
                        // of the second parts (2^-18 of t B), with three that of the third and the second (2^-27).
                        constexpr int NEXT = RANKS / 8;
#pragma unroll
                        for (int j = 0; j < RANKS / 16; ++j) {
                            if (16 * j < left_t) {
                                const uint64_t x1 = x + 2 * j, w1 = w + 2 * j;
                                tc_mma_bf16(acc, x1, w1, idesc_t, 1u);
                                tc_mma_bf16(acc, x1 + NEXT, w1, idesc_t, 1u);
                                if (B_PLANES == 2) tc_mma_bf16(acc, x1, w1 + NEXT, idesc_t, 1u);
                                if (T_PARTS == 3) tc_mma_bf16(acc, x1 + 2 * NEXT, w1, idesc_t, 1u);
                                if (T_PARTS == 3 && B_PLANES == 2) tc_mma_bf16(acc, x1 + NEXT, w1 + NEXT, idesc_t, 1u);
                            }
                        }
                    }
                    tc_commit(&empty[s]);
                    if (last) tc_commit(&acc_full[b]);
                }
                if (st < chunks) left -= PJ_KC;
                else left_t -= RANKS;
                __syncwarp();
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
            ++worked;
        }
        // no product of this CTA may be in flight when it frees its tensor memory, however the other roles end
        if (lead) {
            if (!ok) s_fail = 1;
            tc_commit(&drained);
            mbar_wait_bounded(&drained, 0, PJ_SPIN_LIMIT);
        }
    } else if (lane == 0 && !SHRINK) {
        // ---------------- weights ----------------
        int s = 0, g = 0;
        uint32_t ph = 1;
        bool ok = true;
        for (Tile tile = first_tile(); tile.lt < my_tiles && ok; tile = after(tile)) {
            const int steps = chunks + rank_steps(tile.count), c0 = tile.part * W_COLS, bytes = tile_w(tile) * 128;
            // (a tile's columns may lie in two groups of the layout, and one behind the other in shared memory)
            const int between = w_part(tile);
            const int skip = c0 % PJ_COLS * 128, bytes1 = min(bytes, PJ_CHUNK - skip), bytes2 = bytes - bytes1;
            const uint8_t* from = p.layout + (int64_t)(c0 / PJ_COLS) * chunks * PARTS * PJ_CHUNK;
            for (int st = 0; st < steps; ++st, ++g, from += PARTS * PJ_CHUNK) {
                ok = mbar_wait_bounded(&empty[s], ph, PJ_SPIN_LIMIT);
                if (!ok) break;
                if (st < chunks) {
                    mbar_expect(&full[s], PARTS * bytes);
                    for (int part = 0; part < PARTS; ++part) {
                        uint8_t* const to = ring + s * S::STAGE + S::X_STAGE + part * between;
                        tc_copy_bulk(to, from + part * PJ_CHUNK + skip, bytes1, &full[s]);
                        if (bytes2 > 0) tc_copy_bulk(to + bytes1, from + ((int64_t)chunks * PARTS + part) * PJ_CHUNK, bytes2, &full[s]);
                    }
                } else {
                    mbar_arrive(&full[s]);       // (the loaders bring what a step over ranks reads)
                }
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
        }
        if (!ok) s_fail = 1;
        // no copy of this CTA may be in flight when it leaves: the latest into each stage (usually long there)
        for (int k = 0; k < min(g, STAGES); ++k) {
            const int latest = g - 1 - k;
            mbar_wait_bounded(&full[latest % STAGES], (uint32_t)(latest / STAGES) & 1, PJ_SPIN_LIMIT);
        }
    }

    __syncwarp();
    if (s_fail && lane == 0) g_request_timeout = 1;
    tc_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM) : "memory");
}

// y = act(x W + bias + t B), x W and t from memory: a thread is a column and takes 16 rows one after the other, keeping its row of B
// (RB x 16 ranks) in registers while they are those of one adapter.  A block's t, slots and sums are all requested at once.
// Bound by the bytes of x W, t and y and by how few of them are on their way: 200 000 rows of 47 columns 40 us, 89 MB at 2.2 TB/s.
constexpr int FR_COLS = 64, FR_ROWS = 16, FR_BLOCK = 256 / FR_COLS * FR_ROWS;
template <typename T, int RB>
__global__ void __launch_bounds__(256) k_finish_rows(const __grid_constant__ ProjectParams p) {
    pdl_enter();
    __shared__ float4 ts[FR_BLOCK][RB * 4];
    __shared__ int slots[FR_BLOCK];           // -1: no adapter, -2: a padding row
    const int col = threadIdx.x % FR_COLS, first = blockIdx.x * FR_BLOCK, r0 = threadIdx.x / FR_COLS * FR_ROWS, rp = p.bank.r_pad, ld = pj_up(p.n, 16);
    float4 b[RB][4];
    int have = p.slots[min(first + r0, p.rows - 1)];      // (the adapter of the first row, whose B is asked for with the rest)
    if (have < 0 || have >= p.n_slots) have = -1;
    auto take_b = [&]() {
        const float4* const from = reinterpret_cast<const float4*>(p.bank.b32 + ((int64_t)have * p.n + col) * rp);
#pragma unroll
        for (int k = 0; k < RB; ++k)
#pragma unroll
            for (int h = 0; h < 4; ++h) b[k][h] = bank_word(from + 4 * k + h);
    };
    float x[FR_ROWS];
#pragma unroll
    for (int q = 0; q < FR_ROWS; ++q) x[q] = col < p.n ? p.base[(int64_t)min(first + r0 + q, p.rows - 1) * ld + col] : 0.f;
#pragma unroll
    for (int k = 0; k < RB; ++k) {
        const int e = k * 256 + threadIdx.x, r = e / (RB * 4);
        ts[r][e % (RB * 4)] = __ldcg(reinterpret_cast<const float4*>(static_cast<const float*>(p.t) + (int64_t)min(first + r, p.rows - 1) * rp) + e % (RB * 4));
    }
    if (threadIdx.x < FR_BLOCK) {
        const int i = first + threadIdx.x, a = i < p.rows ? p.slots[i] : -1;
        const bool live = i < p.rows && row_of(p, i) >= 0;
        slots[threadIdx.x] = !live ? -2 : a >= 0 && a < p.n_slots && p.bank.info[a].rank > 0 ? a : -1;
    }
    const float bias = p.bias && col < p.n ? p.bias[col] : 0.f;
    if (have >= 0 && col < p.n) take_b();
    __syncthreads();
    if (col >= p.n) return;
#pragma unroll
    for (int q = 0; q < FR_ROWS; ++q) {
        const int a = slots[r0 + q];
        if (a == -2) continue;
        float y = x[q] + bias;
        if (a >= 0) {
            if (a != have) {
                have = a;
                take_b();
            }
            float d[4] = {};
#pragma unroll
            for (int k = 0; k < RB; ++k)
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const float4 v = ts[r0 + q][4 * k + h], w = b[k][h];
                    d[0] = fmaf(v.x, w.x, d[0]), d[1] = fmaf(v.y, w.y, d[1]), d[2] = fmaf(v.z, w.z, d[2]), d[3] = fmaf(v.w, w.w, d[3]);
                }
            y += (d[0] + d[1]) + (d[2] + d[3]);
        }
        if (p.act == RIPPLE_ACT_RELU && y < 0.f) y = 0.f;
        static_cast<T*>(p.y)[(int64_t)(first + r0 + q) * p.ld_y + col] = from_f32<T>(y);
    }
}

static cudaError_t finish_rows(const ProjectParams& p, void* stream) {
    const dim3 grid((p.rows + FR_BLOCK - 1) / FR_BLOCK);
    switch (p.bank.r_pad / 16) {
        case 1: return launch(k_finish_rows<float, 1>, grid, 256, 0, stream, p);
        case 2: return launch(k_finish_rows<float, 2>, grid, 256, 0, stream, p);
        case 3: return launch(k_finish_rows<float, 3>, grid, 256, 0, stream, p);
        default: return launch(k_finish_rows<float, 4>, grid, 256, 0, stream, p);
    }
}

template <int TYPE, int BN, int MODE, bool MANY>
static cudaError_t project_tiles(const ProjectParams& p, void* stream) {
    using S = PjShape<TYPE, BN, MANY>;
    static bool ready[64];       // by device
    const cudaError_t e = allow_shared(k_project_rows<TYPE, BN, MODE, MANY>, (int)S::BYTES, ready);
    if (e != cudaSuccess) return e;
    const int columns = MODE == PJ_JOINED ? BN - PJ_T_COLS : BN;
    const int64_t across = MODE == PJ_SHRINK || MODE == PJ_SHRINK_3 ? p.batches : (p.n + columns - 1) / columns, tiles = across * ((p.rows + PJ_ROWS - 1) / PJ_ROWS);
    return launch(k_project_rows<TYPE, BN, MODE, MANY>, dim3((unsigned)std::min<int64_t>(tiles, sm_count())), S::THREADS, S::BYTES, stream, p);
}
template <int TYPE, int BN, int MODE>
static cudaError_t project_tiles(const ProjectParams& p, void* stream) {
    if constexpr (TYPE == RIPPLE_TYPE_F32) {
        if (p.chunks > PJ_UNIT) return project_tiles<TYPE, BN, MODE, true>(p, stream);
    }
    return project_tiles<TYPE, BN, MODE, false>(p, stream);
}

// Whether y is computed by k_project_few.  A block takes one round over K per 256 entries and blocks come in waves, so what decides is the
// number of blocks and, beyond three rounds, K.  Both sides, few / tensor cores, us:
//   16 bits:  256 -> 256 104 blocks 6.2 / 8.7, 200 blocks 10.5 / 8.9;  602 -> 41, 126 blocks 14 / 21;  rows that 16 bytes divide, one wave: K = 768
//             9.5 / 7.0, with adapters 11.5 / 11.6;  1024 12.5 / 8.0, with 14.5 / 12.2;  8192 87 / 39, with 91 / 52;  rows that they do not: 1001
//             12.3 / 16.6, with 14.4 / 22.4;  8191 88 / 98, with 93 / 114
//   fp32:     602 -> 41, 188 blocks 22 / 42, 314 blocks 32 / 42, 500 blocks 45 / 43;  256 -> 256, 200 blocks 10.8 / 12.4, 504 blocks 20 / 14;  one wave:
//             1024 10.9 / 18.4;  8192 72 / 122;  two waves: 1024 20.5 / 18.6, with adapters 25.8 / 27.4;  8192 140 / 123, with 156 / 162;  1001 20.9 / 25.5;
//             three waves: 2048 55 / 34, with 64 / 48
static bool few_form(int type, int64_t rows, int k, int n, bool adapters, bool aligned) {
    const int64_t blocks = (rows + PF_ROWS - 1) / PF_ROWS * ((n + PF_COLS - 1) / PF_COLS);
    const bool deep = k > 3 * PF_K;
    if (type != RIPPLE_TYPE_F32) return blocks <= PF_MOST && !(deep && aligned);
    return blocks <= (!deep ? PF_MOST_F32 : adapters || !aligned ? 2 * PJ_SMS : PJ_SMS);
}

// Tiles of 32 columns where that makes no more than one per SM: less to wait for in each.  A second one costs as much again, and then
// tiles of 128 do.  Both sides, 32 / 128 columns, us: bf16 1024 -> 512, 128 tiles of 32 8.3 / 9.3, 192 13.1 / 9.4; 8192 -> 130, 120 tiles 41 / 46, 160
// 76 / 47; 256 -> 256, 128 tiles 4.7 / 5.5, 192 6.2 / 5.6; fp32 1024 -> 512, 128 tiles 20 / 24, 192 36 / 24; with 32 adapters of rank 16 bf16 256 -> 256,
// 128 tiles 12.1 / 13.0, 192 18.9 / 15.8; fp32 2048 -> 300, 120 tiles 57 / 61, 160 90 / 64.
// Of 256 (16-bit rows) where those leave no SM without one (65 536 x 1024 x 1024: 128 columns 200 us, 256 columns 125).
template <int TYPE, int MODE>
static cudaError_t project_columns(const ProjectParams& p, void* stream) {
    const int row_tiles = (p.rows + PJ_ROWS - 1) / PJ_ROWS;
    if constexpr (TYPE != RIPPLE_TYPE_F32) {
        if (p.n > 128 && (int64_t)((p.n + 255) / 256) * row_tiles >= sm_count()) return project_tiles<TYPE, 256, MODE>(p, stream);
    }
    return (int64_t)((p.n + 31) / 32) * row_tiles <= PJ_SMS ? project_tiles<TYPE, 32, MODE>(p, stream) : project_tiles<TYPE, 128, MODE>(p, stream);
}

template <int TYPE>
static cudaError_t project(ProjectParams p, void* stream) {
    constexpr bool F32 = TYPE == RIPPLE_TYPE_F32;
    const int row_tiles = (p.rows + PJ_ROWS - 1) / PJ_ROWS;
    const bool aligned = (reinterpret_cast<uintptr_t>(p.x) & 15) == 0 && p.ld_x * type_size(TYPE) % 16 == 0;
    const bool few = few_form(TYPE, p.rows, p.k, p.n, p.bank.info != nullptr, aligned);
    cudaError_t e = cudaSuccess;
    if (p.bank.info) {
        // fp32, narrow: x W and t in one pass over the rows, whose parts are what takes the time (200 000 rows, 256 -> 47, rank 16: 173 us in
        // two passes, 122 in one)
        if constexpr (F32) {
            if (p.base) {
                e = launch(k_plan_tiles, dim3(row_tiles), 128, 0, stream, p);
                if (e == cudaSuccess) e = project_tiles<TYPE, 128, PJ_JOINED>(p, stream);
                return e == cudaSuccess ? finish_rows(p, stream) : e;
            }
        }
        if (few || p.rows <= PJ_FEW) {
            const int planned = few ? 0 : row_tiles;
            // (four rows per block once there are several blocks for every SM)
            if (p.rows <= 4 * sm_count()) e = launch(k_shrink_few<TYPE, 1>, dim3(planned + p.rows), 128, 0, stream, p, planned);
            else e = launch(k_shrink_few<TYPE, 4>, dim3(planned + (p.rows + 3) / 4), 128, 0, stream, p, planned);
        } else {
            // (16-bit rows, 7 adapters of rank 32 per tile: 64 side by side 91 us, 128 84, 256 86, which costs a tile with one adapter its stages)
            constexpr int T_COLS = F32 ? PJ_T_COLS : 2 * PJ_T_COLS;
            const int at_once = T_COLS / p.bank.r_pad;
            // batches of adapters side by side while there are SMs for them, one behind the other beyond
            const int batches = (std::min(p.n_slots, PJ_ROWS) + at_once - 1) / at_once;
            p.batches = std::max(1, std::min(batches, sm_count() / row_tiles));
            e = launch(k_plan_tiles, dim3(row_tiles), 128, 0, stream, p);
            if constexpr (!F32) {
                if (e == cudaSuccess && p.t_parts == 3) e = project_tiles<TYPE, T_COLS, PJ_SHRINK_3>(p, stream);
            }
            if (e == cudaSuccess && p.t_parts == 2) e = project_tiles<TYPE, T_COLS, PJ_SHRINK>(p, stream);
        }
        if (e != cudaSuccess) return e;
    }
    if (few) return launch(k_project_few<TYPE>, dim3((p.rows + PF_ROWS - 1) / PF_ROWS, (p.n + PF_COLS - 1) / PF_COLS), 256, 0, stream, p);
    if constexpr (!F32) {
        if (p.bank.info && p.t_parts == 3) return project_columns<TYPE, PJ_RANKS_3>(p, stream);
    }
    return project_columns<TYPE, PJ_RANKS>(p, stream);
}

}  // namespace rp

using namespace rp;

#define REFUSE(...)                    \
    do {                               \
        note_error(__VA_ARGS__);       \
        return RIPPLE_ERR_INVALID_ARG; \
    } while (0)

static bool shape_ok(int32_t type, int32_t k, int32_t n) {
    return type_ok(type) && k >= 1 && k <= RIPPLE_MAX_PROJECT_K && n >= 1 && n <= RIPPLE_MAX_PROJECT_N;
}
static bool bank_ok(int32_t slots, int32_t max_rank) {
    return slots >= 1 && slots <= RIPPLE_MAX_SLOTS && max_rank >= 1 && max_rank <= RIPPLE_MAX_RANK;
}
static bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

extern "C" int64_t ripple_project_layout_bytes(int32_t type, int32_t k, int32_t n) {
    if (!shape_ok(type, k, n)) return -1;
    return layout_plain_at(type, k, n) + up128((int64_t)k * n * type_size(type));
}

extern "C" int64_t ripple_adapter_bytes(int32_t type, int32_t k, int32_t n, int32_t slots, int32_t max_rank) {
    if (!shape_ok(type, k, n) || !bank_ok(slots, max_rank)) return -1;
    return bank_b32_at(type, k, n, slots, max_rank) + up128((int64_t)slots * n * pj_up(max_rank, 16) * 4);
}

extern "C" ripple_status ripple_project_layout(int32_t type, int32_t k, int32_t n, const void* W, int64_t ld_w, void* layout,
                                               int32_t device, void* cuda_stream) {
    if (!shape_ok(type, k, n)) REFUSE("project_layout: type, k or n out of range");
    if (!W || !layout || !aligned(W, type_size(type)) || !aligned(layout, 128)) REFUSE("project_layout: null or misaligned pointer");
    if (ld_w < n) REFUSE("project_layout: leading dimension below n");
    OnDevice on(device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    const int chunks = pj_up(k, PJ_KC) / PJ_KC, groups = pj_up(n, PJ_COLS) / PJ_COLS;
    const dim3 grid((unsigned)std::min<int64_t>((int64_t)groups * chunks * PJ_COLS * 8 / 256, 1184));
    uint8_t* const plain = static_cast<uint8_t*>(layout) + layout_plain_at(type, k, n);
    cudaError_t e;
    if (type == RIPPLE_TYPE_F32) e = launch(k_layout_weights<float>, grid, 256, 0, cuda_stream, (const float*)W, ld_w, k, n, (uint8_t*)layout, chunks, groups, (float*)plain);
    else if (type == RIPPLE_TYPE_BF16) e = launch(k_layout_weights<__nv_bfloat16>, grid, 256, 0, cuda_stream, (const __nv_bfloat16*)W, ld_w, k, n, (uint8_t*)layout, chunks, groups, (__nv_bfloat16*)plain);
    else e = launch(k_layout_weights<__half>, grid, 256, 0, cuda_stream, (const __half*)W, ld_w, k, n, (uint8_t*)layout, chunks, groups, (__half*)plain);
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("project_layout launch", e);
}

extern "C" ripple_status ripple_adapter_set(void* bank, int32_t type, int32_t k, int32_t n, int32_t slots, int32_t max_rank,
                                            int32_t first, int32_t count, int32_t rank, const void* A, const void* B,
                                            const float* scale, int32_t device, void* cuda_stream) {
    if (!shape_ok(type, k, n) || !bank_ok(slots, max_rank)) REFUSE("adapter_set: type, k, n, slots or max_rank out of range");
    if (!bank || !aligned(bank, 128)) REFUSE("adapter_set: null or misaligned bank");
    if (first < 0 || count < 0 || count > slots || first > slots - count) REFUSE("adapter_set: slots out of range");
    if (rank < 0 || rank > max_rank) REFUSE("adapter_set: rank out of range");
    const int size = type_size(type);
    if (rank > 0 && (!A || !B || !scale || !aligned(A, size) || !aligned(B, size))) REFUSE("adapter_set: null or misaligned pointer");
    if (count == 0) return RIPPLE_OK;
    bool bad_scale = false;
    for (int i = 0; rank > 0 && i < count; ++i) bad_scale = bad_scale || !(scale[i] - scale[i] == 0.f);
    OnDevice on(device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const BankView v = bank_view(bank, type, k, n, slots, max_rank);
    SlotInfo* info = const_cast<SlotInfo*>(v.info);
    // (the 128 bytes behind the slots' table: the flag)
    int* bad = reinterpret_cast<int*>(static_cast<uint8_t*>(bank) + bank_a_at(slots) - 128);
    int host_bad = 0;
    SlotInfo host_info[256];
    const bool holds = rank > 0 && !bad_scale;
    cudaError_t e = cudaMemsetAsync(bad, 0, sizeof(int), st);
    if (e == cudaSuccess && holds) {
        const dim3 grid(592);
        uint16_t *a = const_cast<uint16_t*>(v.a), *b = const_cast<uint16_t*>(v.b);
        float* const b32 = const_cast<float*>(v.b32);
        if (type == RIPPLE_TYPE_F32) e = launch(k_set_adapters<RIPPLE_TYPE_F32>, grid, 256, 0, cuda_stream, a, b, b32, (const float*)A, (const float*)B, first, count, rank, k, n, v.r_pad, v.k_pad, bad);
        else if (type == RIPPLE_TYPE_BF16) e = launch(k_set_adapters<RIPPLE_TYPE_BF16>, grid, 256, 0, cuda_stream, a, b, b32, (const __nv_bfloat16*)A, (const __nv_bfloat16*)B, first, count, rank, k, n, v.r_pad, v.k_pad, bad);
        else e = launch(k_set_adapters<RIPPLE_TYPE_F16>, grid, 256, 0, cuda_stream, a, b, b32, (const __half*)A, (const __half*)B, first, count, rank, k, n, v.r_pad, v.k_pad, bad);
        if (e == cudaSuccess) e = cudaMemcpyAsync(&host_bad, bad, sizeof(int), cudaMemcpyDeviceToHost, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    for (int at = 0; at < count && e == cudaSuccess; at += 256) {
        const int m = std::min(256, count - at);
        for (int i = 0; i < m; ++i) host_info[i] = holds && !host_bad ? SlotInfo{scale[at + i], rank} : SlotInfo{0.f, 0};
        e = cudaMemcpyAsync(info + first + at, host_info, m * sizeof(SlotInfo), cudaMemcpyHostToDevice, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    // (wrong whether or not there was a device to empty the slots on)
    if (bad_scale) REFUSE("adapter_set: a scale is not finite%s%s", e == cudaSuccess ? "" : ", and the slots could not be emptied: ", e == cudaSuccess ? "" : cudaGetErrorString(e));
    if (e != cudaSuccess) return launch_failed("adapter_set", e);
    if (host_bad) REFUSE("adapter_set: an entry is not finite");
    return RIPPLE_OK;
}

static bool pj_joined(const ripple_project_rows_args* a) {
    return a->bank && a->type == RIPPLE_TYPE_F32 && a->rows > PJ_FEW && !few_form(a->type, a->rows, a->k, a->n, true, true) && a->n <= 128 - PJ_T_COLS;
}

// t: fp32, or up to three bf16 parts (what of it a call needs depends on the result's type, its size does not)
static int64_t t_bytes(const ripple_project_rows_args* a) { return up128(a->rows * pj_up(a->max_rank, 16) * (a->type == RIPPLE_TYPE_F32 ? 4 : 6)); }

extern "C" int64_t ripple_project_workspace_bytes(const ripple_project_rows_args* a) {
    if (!a || a->rows < 0 || !shape_ok(a->type, a->k, a->n)) return -1;
    if (!a->bank) return 0;
    if (!bank_ok(a->n_slots, a->max_rank)) return -1;
    return (a->rows + 127) / 128 * (int64_t)sizeof(TilePlan) + t_bytes(a) + (pj_joined(a) ? up128(a->rows * pj_up(a->n, 16) * 4) : 0);
}

extern "C" ripple_status ripple_project_rows(const ripple_project_rows_args* a) {
    if (!a) REFUSE("project_rows: null arguments");
    if (a->rows < 0 || a->rows > INT32_MAX - 128) REFUSE("project_rows: rows out of range");
    if (!shape_ok(a->type, a->k, a->n)) REFUSE("project_rows: type, k or n out of range");
    if (a->out_type != a->type && a->out_type != RIPPLE_TYPE_F32) REFUSE("project_rows: an output type that is neither the type nor fp32");
    if (a->act != RIPPLE_ACT_IDENTITY && a->act != RIPPLE_ACT_RELU) REFUSE("project_rows: unknown activation");
    const int size = type_size(a->type), out_size = type_size(a->out_type);
    if (a->rows == 0) return RIPPLE_OK;
    if ((!a->x && a->x_rows != 0) || !a->layout || !a->y) REFUSE("project_rows: null pointer");
    if (!aligned(a->x, size) || !aligned(a->y, out_size) || !aligned(a->layout, 128) || !aligned(a->bias, 4) || !aligned(a->ids, 4) || !aligned(a->slots, 4) || !aligned(a->bank, 128))
        REFUSE("project_rows: misaligned pointer");
    if (a->ld_x < 0 || a->ld_y < a->n) REFUSE("project_rows: leading dimension out of range");
    if (a->x_rows < 0 || (!a->ids && a->x_rows < a->rows)) REFUSE("project_rows: fewer rows of x than rows");
    if ((a->bank != nullptr) != (a->slots != nullptr)) REFUSE("project_rows: bank and slots go together");
    if (a->bank && !bank_ok(a->n_slots, a->max_rank)) REFUSE("project_rows: n_slots or max_rank out of range");
    const int64_t need = ripple_project_workspace_bytes(a);
    if (need > 0 && (!a->workspace || a->workspace_bytes < need || !aligned(a->workspace, 128))) REFUSE("project_rows: workspace missing, too small or misaligned");
    const Extent y{a->y, a->rows, a->ld_y, a->n, out_size};
    const Extent x{a->x, a->x_rows, a->ld_x, a->k, size}, ids{a->ids, a->rows, 1, 1, 4}, slots{a->slots, a->rows, 1, 1, 4}, bias{a->bias, 1, 1, a->n, 4},
        layout{a->layout, 1, 1, ripple_project_layout_bytes(a->type, a->k, a->n), 1},
        bank{a->bank, 1, 1, a->bank ? ripple_adapter_bytes(a->type, a->k, a->n, a->n_slots, a->max_rank) : 0, 1}, work{need > 0 ? a->workspace : nullptr, 1, 1, need, 1};
    for (const Extent& e : {x, ids, slots, bias, layout, bank}) {
        if (extents_meet(y, e)) REFUSE("project_rows: y overlaps an input");
        if (extents_meet(work, e)) REFUSE("project_rows: the workspace overlaps an input");
    }
    if (extents_meet(y, work)) REFUSE("project_rows: y overlaps the workspace");

    if (a->x_rows == 0) return RIPPLE_OK;     // every row is a padding row
    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    ProjectParams p = {};
    p.rows = (int)a->rows, p.k = a->k, p.n = a->n, p.act = a->act, p.chunks = pj_up(a->k, PJ_KC) / PJ_KC;
    p.x = a->x, p.ld_x = a->ld_x, p.x_rows = a->x_rows, p.ids = a->ids;
    p.layout = static_cast<const uint8_t*>(a->layout), p.bias = a->bias;
    p.plain = p.layout + layout_plain_at(a->type, a->k, a->n);
    if (a->bank) p.bank = bank_view(a->bank, a->type, a->k, a->n, a->n_slots, a->max_rank);
    p.n_slots = a->n_slots, p.slots = a->slots, p.plan = static_cast<TilePlan*>(a->workspace);
    if (a->bank) p.t = static_cast<uint8_t*>(a->workspace) + (a->rows + 127) / 128 * (int64_t)sizeof(TilePlan);
    else p.plan = nullptr;
    if (pj_joined(a)) p.base = reinterpret_cast<float*>(static_cast<uint8_t*>(p.t) + t_bytes(a));
    p.y = a->y, p.ld_y = a->ld_y, p.out_f32 = a->out_type == RIPPLE_TYPE_F32, p.t_parts = a->type != RIPPLE_TYPE_F32 && p.out_f32 ? 3 : 2;
    const char* const withhold = getenv("RIPPLE_DEBUG_TC_WITHHOLD");
    p.withhold = withhold && withhold[0] == '1';
    cudaError_t e;
    if (a->type == RIPPLE_TYPE_F32) e = project<RIPPLE_TYPE_F32>(p, a->cuda_stream);
    else if (a->type == RIPPLE_TYPE_BF16) e = project<RIPPLE_TYPE_BF16>(p, a->cuda_stream);
    else e = project<RIPPLE_TYPE_F16>(p, a->cuda_stream);
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("project_rows launch", e);
}

extern "C" ripple_status ripple_request_status(int32_t device) {
    OnDevice on(device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    int gave_up = 0;
    const int zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&gave_up, g_request_timeout, sizeof(int));
    if (e == cudaSuccess && gave_up) e = cudaMemcpyToSymbol(g_request_timeout, &zero, sizeof(int));
    if (e != cudaSuccess) return launch_failed("request_status", e);
    if (!gave_up) return RIPPLE_OK;
    note_error("project_rows: a bounded device-side wait gave up; the results of calls since the last query are not to be used");
    return RIPPLE_ERR_TIMEOUT;
}
