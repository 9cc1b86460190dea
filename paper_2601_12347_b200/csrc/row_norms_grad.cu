// The way back through n = norm(x[ids]): dx, and the gradients of the norm's vectors.  With x^ the normalised row and d = dn * weight,
//   dx = (d - mean(d) - x^ mean(d x^)) inv + add,   inv = 1 / sqrt(var + eps)      (RMS: without mean(d))
//   dweight = sum over the rows of dn x^,   dbias = sum of dn.
// One pass: a row's inputs are read once and stay in registers; the mean comes first, then the squared distances and both sums of d in one
// reduction.  A thread has the same columns of every row, so that dweight and dbias gather in its registers (rows too wide for that: in
// places of shared memory that are its own); blocks write what they have gathered, and a second kernel adds it up in the order of the blocks.
//
// What bounds it: issue slots, then bytes.  150 003 gathered fp32 rows of 256 beside bf16 ones, 385 MB: 71 us, 5.4 TB/s (84 % of the measured copy rate);
// 32 768 rows of 4096 bf16 with a further gradient, 1.07 GB: 236 us, 4.5 TB/s.  What it took: weights in registers instead of two loads of them for every row (84 and
// 270 us); rows of 513 to 1024 columns on two warps, whose sixteen columns a thread leave them room for that (10 001 fp32 rows of 602, 72 MB: 24 us; on one warp 38).
#include "row_vectors.cuh"

#include <algorithm>
#include <utility>

namespace rp {

struct NormGradParams {
    int rows, width;
    const void* dn;
    const void* x;
    const int32_t* ids;
    const void* add;
    void* dx;
    float* dweight;
    float* dbias;
    float* gathered;       // blocks x 2 x width (not read: one block)
    const float* weight;
    int64_t ld_dn, ld_x, ld_add, ld_dx, x_rows;
    float eps;
    int layer;
    int warps_per_row;
    int dn_bytes, x_bytes, stage_bytes, stages;   // of a row in the ring; rows in it
};

// sums over the threads of a row, several at once; MULTI: scratch has two halves, used in turn
template <bool MULTI, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float* scratch, int warps, int& turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
    }
    if constexpr (MULTI) {
        float* const mine = scratch + 48 * (turn ^= 1);
        if (lane_id() == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) mine[16 * i + (threadIdx.x >> 5)] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = lane_id() < warps ? mine[16 * i + lane_id()] : 0.f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __shfl_sync(FULL, x[i], 0);
    }
}

constexpr int NG_STAGES = 3;     // rows on their way at most
// Columns from which the vectors' gradients gather in shared memory: a thread's 32 columns would need 64 registers more.
constexpr int NG_WIDE = 8192;

// V: neighbouring elements per access, NP: accesses per thread.  A row takes a warp, or (MULTI) the whole block, of up to THREADS.
// RING: a thread's part of the rows ahead travels as asynchronous copies into places of shared memory that it alone reads, so no
// barrier belongs to it.  Else a row is read when its turn comes.  SHARED: dweight and dbias gather in shared memory.
// KEEP: the weights of a thread's columns stay in registers (else they are read twice for every row: two fifths of what the kernel asks of L1).
template <typename T, typename TR, int V, int NP, bool MULTI, bool RING, bool SHARED, bool KEEP, int THREADS>
__global__ void __launch_bounds__(THREADS) k_norm_rows_grad(const __grid_constant__ NormGradParams p) {
    pdl_enter();
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float scratch[MULTI ? 96 : 1];
    const int W = MULTI ? p.warps_per_row : 1, threads = 32 * W, t = MULTI ? threadIdx.x : lane_id();
    const int first = MULTI ? blockIdx.x : blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int64_t step = MULTI ? gridDim.x : gridDim.x * (blockDim.x >> 5);
    const int D = p.width;
    const float inv_d = 1.0f / (float)D;
    const bool vectors = p.dweight || p.dbias;
    int turn = 0;
    // the ring's rows: dn, then x, then add
    const int at_x = p.dn_bytes, at_a = at_x + p.x_bytes, per_row = p.stage_bytes;
    const int ahead = RING ? p.stages - 1 : 0;
    uint8_t* const mine = RING ? ring + (MULTI ? 0 : (threadIdx.x >> 5) * p.stages * per_row) + t * V * (int)sizeof(T) : nullptr;
    const int more = t * V * (int)(sizeof(TR) - sizeof(T)), at_x_mine = at_x + more, at_a_mine = at_a + more;
    const int c0 = t * V, hop = threads * V;      // this thread's columns: c0 + j hop + (0 .. V - 1)
    const T* const dn0 = static_cast<const T*>(p.dn) + c0;
    const TR* const x0 = static_cast<const TR*>(p.x) + c0;
    const TR* const add0 = static_cast<const TR*>(p.add) + c0;
    TR* const dx0 = static_cast<TR*>(p.dx) + c0;
    // the row of x that a row reads; negative: a padding row, or none
    auto source = [&](int64_t row) -> int64_t {
        if (row >= p.rows) return -1;
        if (!p.ids) return row;
        const int64_t from = p.ids[row];
        return from < p.x_rows ? from : -1;
    };
    auto request = [&](int stage, int64_t row, int64_t from) {
        if constexpr (RING) {
            if (from >= 0) {
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine + stage * per_row);
                const T* const dn = dn0 + row * p.ld_dn;
                const TR* const x = x0 + from * p.ld_x;
                const TR* const add = add0 + row * p.ld_add;
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const int c = j * hop;
                    if (c0 + c >= D) break;
                    copy_async<V * sizeof(T)>(to + c * sizeof(T), dn + c);
                    copy_async<V * sizeof(TR)>(to + at_x_mine + c * sizeof(TR), x + c);
                    if (p.add) copy_async<V * sizeof(TR)>(to + at_a_mine + c * sizeof(TR), add + c);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < NP; ++j) if (c0 + j * hop < D) f(j, j * hop);
    };
    // gathered so far: registers, or this thread's places of shared memory
    Vec<V> dw[SHARED ? 1 : NP], db[SHARED ? 1 : NP];
    float* const gather = reinterpret_cast<float*>(ring) + c0;      // SHARED (there is no ring then): dweight, dbias behind it
#pragma unroll
    for (int j = 0; j < (SHARED ? 1 : NP); ++j) dw[j] = db[j] = all_of<V>(0.f);
    if constexpr (SHARED) each([&](int, int c) { store<float, V>(gather + c, all_of<V>(0.f)), store<float, V>(gather + D + c, all_of<V>(0.f)); });

    Vec<V> weights[KEEP ? NP : 1];
#pragma unroll
    for (int j = 0; j < (KEEP ? NP : 1); ++j) weights[j] = all_of<V>(1.f);
    if constexpr (KEEP) if (p.weight) each([&](int j, int c) { weights[j] = load<float, V>(p.weight + c0 + c); });
    // where this row and the next two come from
    int64_t from = source(first), from1 = source(first + step), from2 = source(first + 2 * step);
    if (ahead > 0) request(0, first, from);
    if (ahead > 1) request(1, first + step, from1);
    int stage = 0;
    for (int64_t row = first; row < p.rows; row += step) {
        request(stage == 0 ? ahead : stage - 1, row + ahead * step, ahead == 2 ? from2 : ahead == 1 ? from1 : from);
        const uint8_t* const in = mine + stage * per_row;
        const int64_t source_row = from;
        from = from1, from1 = from2, from2 = source(row + 3 * step);
        if (++stage > ahead) stage = 0;
        if constexpr (RING) {
            if (ahead == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
            else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        TR* const to = dx0 + row * p.ld_dx;
        if (source_row < 0) {                     // a padding row
            if (p.dx) each([&](int, int c) { store<TR, V>(to + c, all_of<V>(0.f)); });
            continue;
        }
        // (pieces beyond the row are zeros, which only the subtraction of the mean has to leave alone)
        Vec<V> x[NP], d[NP];
#pragma unroll
        for (int j = 0; j < NP; ++j) x[j] = d[j] = all_of<V>(0.f);
        if constexpr (RING) {
            each([&](int j, int c) { x[j] = load<TR, V>(in + at_x_mine + c * (int)sizeof(TR)); });
            each([&](int j, int c) { d[j] = load<T, V>(in + c * (int)sizeof(T)); });
        } else {
            each([&](int j, int c) { x[j] = load<TR, V>(x0 + source_row * p.ld_x + c); });
            each([&](int j, int c) { d[j] = load<T, V>(dn0 + row * p.ld_dn + c); });
        }
        if (p.layer) {
            Vec<V> sum = all_of<V>(0.f);
#pragma unroll
            for (int j = 0; j < NP; ++j) plus<V>(sum, x[j]);
            float mean[1] = {folded<V>(sum)};
            row_sums<MULTI, 1>(mean, scratch, W, turn);
            const Vec<V> back = all_of<V>(-mean[0] * inv_d);
            each([&](int j, int) { plus<V>(x[j], back); });
        }
        auto weighted = [&](int j, int c) {
            Vec<V> u = d[j];
            if constexpr (KEEP) times<V>(u, weights[j]);
            else if (p.weight) times<V>(u, load<float, V>(p.weight + c0 + c));
            return u;
        };
        Vec<V> squares = all_of<V>(0.f), of_d = squares, of_dx = squares;
        each([&](int j, int c) {
            const Vec<V> u = weighted(j, c);
            add_squares<V>(squares, x[j]);
            plus<V>(of_d, u);
            add_product<V>(of_dx, u, x[j]);
        });
        float sums[3] = {folded<V>(squares), folded<V>(of_dx), 0.f};
        if (p.layer) {
            sums[2] = folded<V>(of_d);
            row_sums<MULTI, 3>(sums, scratch, W, turn);
        } else {
            float two[2] = {sums[0], sums[1]};
            row_sums<MULTI, 2>(two, scratch, W, turn);
            sums[0] = two[0], sums[1] = two[1];
        }
        const float inv = rsqrtf(sums[0] * inv_d + p.eps);
        const Vec<V> inv_v = all_of<V>(inv), off = all_of<V>(-sums[2] * inv_d), along = all_of<V>(-sums[1] * inv * inv_d);
        each([&](int j, int) { times<V>(x[j], inv_v); });
        if (vectors) {
            if constexpr (SHARED) {
                each([&](int j, int c) {
                    Vec<V> w = load<float, V>(gather + c), b = load<float, V>(gather + D + c);
                    add_product<V>(w, d[j], x[j]), plus<V>(b, d[j]);
                    store<float, V>(gather + c, w), store<float, V>(gather + D + c, b);
                });
            } else {
#pragma unroll
                for (int j = 0; j < NP; ++j) add_product<V>(dw[j], d[j], x[j]), plus<V>(db[j], d[j]);
            }
        }
        if (!p.dx) continue;
        each([&](int j, int c) {
            Vec<V> u = weighted(j, c);
            plus<V>(u, off);
            add_product<V>(u, along, x[j]);
            times<V>(u, inv_v);
            if (p.add) plus<V>(u, RING ? load<TR, V>(in + at_a_mine + c * (int)sizeof(TR)) : load<TR, V>(add0 + row * p.ld_add + c));
            store<TR, V>(to + c, u);
        });
    }
    if constexpr (RING) asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!vectors) return;
    // one block writes the results, several what each has gathered
    float* const out_w = gridDim.x == 1 ? p.dweight : p.gathered + (int64_t)blockIdx.x * 2 * D;
    float* const out_b = gridDim.x == 1 ? p.dbias : p.gathered + ((int64_t)blockIdx.x * 2 + 1) * D;
    if constexpr (MULTI) {
        each([&](int j, int c) {
            const Vec<V> w = SHARED ? load<float, V>(gather + c) : dw[SHARED ? 0 : j], b = SHARED ? load<float, V>(gather + D + c) : db[SHARED ? 0 : j];
            if (out_w) store<float, V>(out_w + c0 + c, w);
            if (out_b) store<float, V>(out_b + c0 + c, b);
        });
    } else {
        // warps of the block one after the other; the last one writes
        const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
        float* const sum_w = reinterpret_cast<float*>(ring) + c0;
        float* const sum_b = sum_w + (D + 7) / 8 * 8;
        __syncthreads();
        for (int w = 0; w < warps; ++w) {
            if (w == warp) {
                each([&](int j, int c) {
                    if (w > 0) plus<V>(dw[SHARED ? 0 : j], load<float, V>(sum_w + c)), plus<V>(db[SHARED ? 0 : j], load<float, V>(sum_b + c));
                    if (w < warps - 1) {
                        store<float, V>(sum_w + c, dw[SHARED ? 0 : j]), store<float, V>(sum_b + c, db[SHARED ? 0 : j]);
                    } else {
                        if (out_w) store<float, V>(out_w + c0 + c, dw[SHARED ? 0 : j]);
                        if (out_b) store<float, V>(out_b + c0 + c, db[SHARED ? 0 : j]);
                    }
                });
            }
            __syncthreads();
        }
    }
}

// dweight and dbias from what the blocks have gathered.  A block has 32 columns, its warps take turns over the blocks' parts; in the end the
// warps' sums are added in order.
__global__ void __launch_bounds__(512) k_join_vectors(const float* gathered, int parts, int width, float* dweight, float* dbias) {
    pdl_enter();
    __shared__ float sums[16][33];
    const int warp = threadIdx.x >> 5, lane = lane_id(), c = blockIdx.x * 32 + lane;
    float* const out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    float s = 0.f;
    if (c < width) {
        const float* const from = gathered + blockIdx.y * (int64_t)width + c;
#pragma unroll 8
        for (int i = warp; i < parts; i += 16) s += from[(int64_t)i * 2 * width];
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < width) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) total += sums[w][lane];
        out[c] = total;
    }
}

// Blocks that a call may launch, so that what they gather has a place: more than fit at once at no width, and no more than have rows.
static int grad_blocks_most(int64_t rows, int width) {
    const int64_t per_block = width <= 512 ? 4 : 1;
    return (int)std::min<int64_t>((rows + per_block - 1) / per_block, 148 * 8);
}

template <typename T, typename TR, int V, int E, bool MULTI, bool RING, bool SHARED, bool KEEP, int THREADS>
static cudaError_t launch_grad(NormGradParams p, int warps, void* stream) {
    auto* const kernel = k_norm_rows_grad<T, TR, V, E / V, MULTI, RING, SHARED, KEEP, THREADS>;
    p.warps_per_row = warps;
    const int block = MULTI ? 32 * warps : 128, rows_per_block = MULTI ? 1 : 4;
    const int64_t blocks = ((int64_t)p.rows + rows_per_block - 1) / rows_per_block;
    int bytes = 0, per_sm = 1;
    if (RING) {
        const int one = p.stage_bytes * rows_per_block;
        p.stages = blocks <= sm_count() ? 1 : NG_STAGES * one <= 64 * 1024 ? NG_STAGES : 2 * one <= 200 * 1024 ? 2 : 1;
        bytes = p.stages * one;
    }
    bytes = std::max(bytes, SHARED || !MULTI ? (p.width + 7) / 8 * 8 * 8 : 0);
    static bool ready[64];       // by device
    cudaError_t e = allow_shared(kernel, 200 * 1024, ready);
    if (e != cudaSuccess) return e;
    if (blocks > sm_count() && (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, block, bytes) != cudaSuccess || per_sm < 1)) per_sm = 1;
    const int grid = (int)std::min<int64_t>({blocks, (int64_t)per_sm * sm_count(), (int64_t)grad_blocks_most(p.rows, p.width)});
    e = launch(kernel, dim3((unsigned)grid), block, bytes, stream, p);
    if (e != cudaSuccess || grid == 1 || !(p.dweight || p.dbias)) return e;
    return launch(k_join_vectors, dim3((unsigned)(p.width + 31) / 32, 2), 512, 0, stream, (const float*)p.gathered, grid, p.width, p.dweight, p.dbias);
}

template <typename T, typename TR, int V, bool RING>
static cudaError_t launch_grad(const NormGradParams& p, void* stream) {
    const int D = p.width;
    if (D <= 256) return launch_grad<T, TR, V, 8, false, RING, false, true, 128>(p, 1, stream);
    if (D <= 512) return launch_grad<T, TR, V, 16, false, RING, false, true, 128>(p, 1, stream);
    if (D <= 1024) return launch_grad<T, TR, V, 16, true, RING, false, true, 64>(p, 2, stream);
    if (D <= 4096) return launch_grad<T, TR, V, 16, true, RING, false, true, 256>(p, (D + 511) / 512, stream);
    if (D <= NG_WIDE) return launch_grad<T, TR, V, 16, true, RING, false, false, 512>(p, (D + 511) / 512, stream);
    return launch_grad<T, TR, V, 32, true, false, true, false, 512>(p, (D + 1023) / 1024, stream);
}

template <typename T, typename TR>
static cudaError_t launch_grad(NormGradParams p, int v, void* stream) {
    constexpr int WIDE = 16 / sizeof(T);
    auto up16 = [](int64_t x) { return (int)((x + 15) / 16 * 16); };
    p.dn_bytes = up16(p.width * (int64_t)sizeof(T)), p.x_bytes = up16(p.width * (int64_t)sizeof(TR));
    p.stage_bytes = p.dn_bytes + (p.add ? 2 : 1) * p.x_bytes;
    if (v >= WIDE) return launch_grad<T, TR, WIDE, true>(p, stream);
    if (v >= 2) return launch_grad<T, TR, 2, true>(p, stream);
    return launch_grad<T, TR, 1, sizeof(T) == 4>(p, stream);
}

}  // namespace rp

using namespace rp;

#define REFUSE(...)                             \
    do {                                        \
        note_error("norm_rows_grad: " __VA_ARGS__); \
        return RIPPLE_ERR_INVALID_ARG;          \
    } while (0)

static int64_t grad_workspace(int64_t rows, int width) {
    const int64_t blocks = grad_blocks_most(rows, width);
    return blocks > 1 ? blocks * 2 * width * 4 : 0;       // (one block writes the results)
}

extern "C" int64_t ripple_norm_rows_grad_workspace_bytes(const ripple_norm_rows_grad_args* a) {
    if (!a || a->rows < 0 || a->rows > INT32_MAX || a->width < 1 || a->width > 16384) return -1;
    return a->dweight || a->dbias ? grad_workspace(a->rows, a->width) : 0;
}

extern "C" ripple_status ripple_norm_rows_grad(const ripple_norm_rows_grad_args* a) {
    if (!a) REFUSE("null arguments");
    if (a->rows < 0 || a->rows > INT32_MAX) REFUSE("rows out of range");
    if (a->width < 1 || a->width > 16384) REFUSE("width must be 1 to 16384");
    if (!type_ok(a->type) || !type_ok(a->x_type) || (a->x_type != a->type && a->x_type != RIPPLE_TYPE_F32))
        REFUSE("unknown type, or a type of x that is neither dn's nor fp32");
    if (a->norm.kind != RIPPLE_NORM_LAYER && a->norm.kind != RIPPLE_NORM_RMS) REFUSE("unknown norm");
    if (!(a->norm.eps >= 0.f)) REFUSE("eps must not be negative");
    if (!a->dx && !a->dweight && !a->dbias) REFUSE("no output");
    if (a->add && !a->dx) REFUSE("add without dx");
    if (a->x_rows < 0 || (!a->ids && a->x_rows < a->rows)) REFUSE("fewer rows of x than rows");
    if ((!a->dn && a->rows > 0) || (!a->x && a->x_rows > 0 && a->rows > 0)) REFUSE("null dn or x");
    if (a->ld_dn < 0 || a->ld_x < 0 || a->ld_add < 0) REFUSE("negative leading dimension");
    if (a->dx && a->ld_dx < a->width) REFUSE("leading dimension of dx below its width");
    const int ts = type_size(a->type), xs = type_size(a->x_type);
    for (auto [ptr, size] : {std::pair<const void*, int>{a->dn, ts}, {a->x, xs}, {a->add, xs}, {a->dx, xs}, {a->dweight, 4}, {a->dbias, 4}, {a->norm.weight, 4}, {a->ids, 4}})
        if (reinterpret_cast<uintptr_t>(ptr) % size) REFUSE("misaligned pointer");
    const int64_t need = a->dweight || a->dbias ? grad_workspace(a->rows, a->width) : 0;
    if (a->workspace_bytes < need || (need > 0 && !a->workspace)) REFUSE("workspace too small");
    if (reinterpret_cast<uintptr_t>(a->workspace) & 127) REFUSE("misaligned workspace");
    const Extent dn{a->dn, a->rows, a->ld_dn, a->width, ts}, x{a->x, a->x_rows, a->ld_x, a->width, xs}, add{a->add, a->rows, a->ld_add, a->width, xs},
        dx{a->dx, a->rows, a->ld_dx, a->width, xs}, ids{a->ids, a->rows, 1, 1, 4}, weight{a->norm.weight, 1, 1, a->width, 4},
        dw{a->dweight, 1, 1, a->width, 4}, db{a->dbias, 1, 1, a->width, 4}, work{need > 0 ? a->workspace : nullptr, 1, 1, need, 1};
    // (a row of dn, add and, without ids, x is read by the threads that write its dx)
    for (const Extent* in : {&dn, &x, &add})
        if (extents_meet(dx, *in) && (!extents_same(dx, *in) || (in == &x && a->ids))) REFUSE("dx overlaps an input");
    for (const Extent& out : {dw, db, work})
        for (const Extent& other : {dn, x, add, dx, ids, weight})
            if (extents_meet(out, other)) REFUSE("an output or the workspace overlaps another argument");
    if (extents_meet(dx, ids) || extents_meet(dx, weight)) REFUSE("dx overlaps an input");
    if (extents_meet(dw, db) || extents_meet(dw, work) || extents_meet(db, work)) REFUSE("outputs or workspace overlap");

    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    cudaError_t e;
    if (a->rows == 0) {          // sums of nothing
        for (float* v : {a->dweight, a->dbias})
            if (v && (e = cudaMemsetAsync(v, 0, (size_t)a->width * 4, static_cast<cudaStream_t>(a->cuda_stream))) != cudaSuccess)
                return launch_failed("norm_rows_grad", e);
        return RIPPLE_OK;
    }
    // The widest access that every matrix and vector of the call allows (of the workspace's, too, whose rows are `width` apart).
    int v = 16 / ts;
    auto fits = [&](const void* ptr, int64_t ld, int size) {
        while (v > 1 && (ld % v || reinterpret_cast<uintptr_t>(ptr) % (v * size < 16 ? v * size : 16))) v >>= 1;
    };
    while (a->width % v) v >>= 1;
    fits(a->dn, a->ld_dn, ts), fits(a->x, a->ld_x, xs);
    if (a->add) fits(a->add, a->ld_add, xs);
    if (a->dx) fits(a->dx, a->ld_dx, xs);
    for (const void* ptr : {(const void*)a->norm.weight, (const void*)a->dweight, (const void*)a->dbias})
        if (ptr) fits(ptr, 0, 4);

    NormGradParams p = {};
    p.rows = (int)a->rows, p.width = a->width;
    p.dn = a->dn, p.x = a->x, p.ids = a->ids, p.add = a->add, p.dx = a->dx, p.dweight = a->dweight, p.dbias = a->dbias;
    p.gathered = static_cast<float*>(a->workspace);
    p.weight = a->norm.weight, p.eps = a->norm.eps, p.layer = a->norm.kind == RIPPLE_NORM_LAYER;
    p.ld_dn = a->ld_dn, p.ld_x = a->ld_x, p.ld_add = a->ld_add, p.ld_dx = a->ld_dx, p.x_rows = a->x_rows;
    const bool mixed = a->x_type != a->type;
    switch (a->type) {
        case RIPPLE_TYPE_F32: e = launch_grad<float, float>(p, v, a->cuda_stream); break;
        case RIPPLE_TYPE_BF16: e = mixed ? launch_grad<__nv_bfloat16, float>(p, v, a->cuda_stream) : launch_grad<__nv_bfloat16, __nv_bfloat16>(p, v, a->cuda_stream); break;
        default: e = mixed ? launch_grad<__half, float>(p, v, a->cuda_stream) : launch_grad<__half, __half>(p, v, a->cuda_stream); break;
    }
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("norm_rows_grad launch", e);
}
