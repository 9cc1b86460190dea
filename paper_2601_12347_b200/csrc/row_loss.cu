// Softmax cross entropy of a linear layer over many classes, and its gradient, without the logits ever being in memory:
//   z = x W + b,  lse_i = log sum_c exp z_ic,  loss_i = lse_i - z_i,label;
//   g = dloss_i (softmax(z)_ic - [c = label_i]),  dx = g W^T,  dW = x^T g,  db = sum over the rows of g.
// Four products of one kernel (k_product) with three ends: maxima and sums of exponentials of a tile (the loss); g of a tile, as an operand of
// the products that follow (the gradient, in pieces of the classes); and plain results.
#include "requests.cuh"
#include "tensor_core.cuh"

#include <cuda.h>

#include <algorithm>
#include <cstdlib>
#include <type_traits>
#include <utility>

namespace rp {

// Set where a bounded wait gave up; read and cleared by ripple_request_status.
__device__ int g_loss_timeout;

cudaError_t take_loss_timeout(int* gave_up) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(gave_up, g_loss_timeout, sizeof(int));
    if (e == cudaSuccess && *gave_up) e = cudaMemcpyToSymbol(g_loss_timeout, &zero, sizeof(int));
    return e;
}

// ---- a product on pairs of tensor cores ----------------------------------------------------------------------------
// C [m, n] = A B over k, operands of 16 bits, fp32 as three planes of bf16 parts.  A pair of CTAs takes 256 rows x COLS columns of C: each
// brings its 128 rows of A and its half of the tile's columns of B, the pair's tensor cores read both halves, and each has its 128 rows
// of C: 32 KB per 64 entries of k and CTA, where a CTA by itself would bring 48 for the same products.  Operands come by TMA in either order, k along the rows of memory or across them; what lies outside a matrix arrives as zeros.
constexpr int LS_ROWS = 256, LS_KC = 64;
constexpr int LS_PAIRS = 74;             // of a B200 (for plans that are asked where no device is current, too)
enum { END_LSE, END_GRAD, END_OUT };
// Chunks of k whose products share an accumulator, which then is handed over and summed in registers: the tensor core cuts what its additions lose, so sums of
// terms of one sign come out too small, in proportion to their length (fp16, 100 000 entries: 6.5e-4 of it, more than half a step of the result, bf16 2e-3).  fp32: of the
// large products.  Results in 16 bits: an eighth of half a step of theirs.  (The epilogue has half the warps then, for the registers: 6001 x 512 x 32 003 in fp16, dx and dW 144 us
// and 151 in one accumulator, 155 and 161 in pieces of 4096.)
__host__ __device__ constexpr int unit_of(int type, int end) { return type == RIPPLE_TYPE_F32 ? 4 : end != END_OUT ? 32 : type == RIPPLE_TYPE_F16 ? 128 : 512; }
constexpr int LS_GROUP = 8;              // tiles of rows that are worked on side by side, so that B's tiles are read out of L2
constexpr uint32_t LS_SPIN_LIMIT = 1u << 18;       // polls after which a wait gives up: about a second
constexpr float LOG2E = 1.4426950408889634f;

// MANY: more than one unit of k, whose sums the epilogue carries in registers.  RAW: A is fp32 as the caller has it; warps fetch it and make its parts.
template <int TYPE, bool MANY, bool RAW = false> struct LossShape {
    static constexpr int PARTS = TYPE == RIPPLE_TYPE_F32 ? 3 : 1;
    static constexpr int COLS = PARTS == 3 ? 128 : 256;
    static constexpr int A_PART = 128 * 128, B_PART = COLS / 2 * 128;       // bytes of a CTA's operands of 64 entries of k
    static constexpr int STAGE = PARTS * (A_PART + B_PART);
    static constexpr int STAGES = PARTS == 3 ? 3 : 6;
    // Warps that take accumulators: sixteen, four to a scheduler, so that one's exponentials are on their way while others add (loss-wide, g
    // of a piece: 281 us with eight, 215 with sixteen); eight where the sums carried need the registers.
    static constexpr int EPI_WARPS = MANY || RAW ? 8 : 16, GROUPS = EPI_WARPS / 4;
    static constexpr int FIRST = RAW ? 4 : 2;            // of them; RAW: whole warpgroups, which share out registers
    static constexpr int LOADERS = RAW ? 16 : 0;
    static constexpr int THREADS = 32 * (FIRST + EPI_WARPS + LOADERS);
    static constexpr int BIAS = EPI_WARPS * (COLS / GROUPS) * 4;
    static constexpr size_t BYTES = (size_t)STAGES * STAGE + BIAS + 1024;
};

constexpr int LS_CONTROL = 512;          // blocks of k_look_at_rows (where few rows have labels, it reads most of x)

// What k_look_at_rows found, block by block.
struct RowControl {
    float most[LS_CONTROL], least[LS_CONTROL];      // largest and smallest |dloss| that is finite and not zero (0, infinity: none)
    int32_t odd[LS_CONTROL];             // a row without a label holds something that is not finite
    int32_t differ;                      // fp16: weights_differ (written by the first product that forms g)
};

struct alignas(64) ProductParams {
    CUtensorMap a, a_clean, b;           // a_clean: read in place of a where rows without labels hold something that is not finite
    const RowControl* control;           // null: a as it is
    const float* raw;                    // RAW: A, raw_rows x raw_cols
    int64_t ld_raw;
    int raw_rows, raw_cols;
    const int32_t* raw_labels;           // rows of it without a label are zeros; or null
    int m, n, k;
    int row_tiles, col_tiles, splits, split_chunks;
    int b_col0, b_k0;                    // where this piece begins in B
    // logits
    const float* bias;                   // of the piece
    const int32_t* labels;
    int class0, classes;                 // first class of the piece, number of all
    float2* sums;                        // LSE: GROUPS x col_tiles x m: largest logit, sum of exp(logit - largest)
    float* at_label;
    const float* lse;                    // GRAD
    const float* dloss;
    float scale;
    uint16_t* g;                         // planes x m x ld_g; null: not wanted
    int64_t ld_g, g_plane;
    float* g_sums;                       // row groups of 32 x ld_g; null: not wanted
    // OUT
    void* out;
    int64_t ld_out, split_stride;        // fp32: elements between the splits' results
    int out_f32, add_to_out;
    int unscale;                         // g was scaled: see grad_scale
    int by_row;                          // fp16, GRAD: runs only where weights differ, and scales every row by itself; OUT: g was formed so, there
    int32_t* differ;                     // fp16, GRAD: where to write whether they do; else null
    const int32_t* dead_rows;            // labels, where rows without one are zeros; else null
    int withhold;                        // diagnostic: no first accumulator counts as filled
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of a shared variable in the pair's first CTA
__device__ __forceinline__ uint32_t in_leader(const void* p) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(p)));
    return a;
}
// (relaxed: what is handed over is tensor memory, ordered by the fences of tcgen05; a release would wait for the warp's stores to global memory)
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// a box of a tensor, completing on a barrier of either CTA of the pair
__device__ __forceinline__ void load_box(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives at the barrier of both CTAs once the products issued so far have finished
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// Descriptor of an operand whose rows of memory run across k, 128-byte swizzle: 64 entries of its rows or columns side by side, 8 entries of k
// 1024 bytes apart, the next 64 rows or columns 8192.
__device__ __forceinline__ uint64_t across_desc(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(8192 >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void store8(void* to, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
template <typename T> __device__ __forceinline__ uint32_t pair_of(float a, float b) {
    uint32_t d;
    if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}
// An fp32 value as three bf16 parts, rounded; both remainders are exact.  An infinite value has no remainders.
__device__ __forceinline__ void three_parts(float x, __nv_bfloat16 (&h)[3]) {
    h[0] = __float2bfloat16_rn(x);
    if (__hisinf(h[0]) && isfinite(x)) h[0] = __float2bfloat16_rz(x);
    const float left = isfinite(x) ? x - __bfloat162float(h[0]) : 0.f;
    h[1] = __float2bfloat16_rn(left);
    h[2] = __float2bfloat16_rn(left - __bfloat162float(h[1]));
}

// The power of two that brings a weight to 2^14 .. 2^15.
__device__ __forceinline__ float scale_of(float weight) {
    weight = fabsf(weight);
    if (!(weight > 0.f) || !isfinite(weight)) return 1.f;
    int e;
    frexpf(weight, &e);          // weight <= 2^e
    return ldexpf(1.f, max(-126, min(126, 15 - e)));
}
// fp16: g is scaled by the power of two of the largest |dloss|, so that probabilities down to 2^-29 of it keep all bits, and the results are scaled back.  (bf16
// and its parts have fp32's range.)
__device__ __forceinline__ float grad_scale(const RowControl* control, float scale) {
    float most = 0.f;
    for (int i = lane_id(); i < LS_CONTROL; i += 32) most = fmaxf(most, control->most[i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(FULL, most, o));
    return scale_of(most * scale);
}
// Rows whose weight is far below the largest would have few bits left of their small probabilities (2^-24 of it: none of 2^-16), which dW does not notice and their own rows
// of dx do.  Where weights lie more than 2^8 apart, g is formed a second time for dx, every row scaled by itself.
__device__ __forceinline__ bool weights_differ(const RowControl* control) {
    float most = 0.f, least = INFINITY;
    for (int i = lane_id(); i < LS_CONTROL; i += 32) most = fmaxf(most, control->most[i]), least = fminf(least, control->least[i]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(FULL, most, o)), least = fminf(least, __shfl_xor_sync(FULL, least, o));
    return least < most * (1.f / 256);
}

// Two fp32 operations in one instruction: (a, b) += (c, d), (a, b) *= (c, d).  (A warp's block of 32 columns of g took 564 instructions,
// a tile 4500 cycles of issue slots beside 4096 of products at k = 512.)
__device__ __forceinline__ void add2(float& a, float& b, float c, float d) {
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
__device__ __forceinline__ void mul2(float& a, float& b, float c, float d) {
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}

// Sums over the warp's rows of 32 columns: lane c has the sum of v[c].
__device__ __forceinline__ float column_sums(float (&v)[32]) {
#pragma unroll
    for (int half = 16; half > 0; half >>= 1) {
        const bool upper = lane_id() & half;
        if (half == 1) return (upper ? v[1] : v[0]) + __shfl_xor_sync(FULL, upper ? v[0] : v[1], 1);
#pragma unroll
        for (int i = 0; i < half; i += 2) {
            float mine[2], other[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mine[e] = upper ? v[i + e + half] : v[i + e];
                other[e] = __shfl_xor_sync(FULL, upper ? v[i + e] : v[i + e + half], half);
            }
            add2(mine[0], mine[1], other[0], other[1]);
            v[i] = mine[0], v[i + 1] = mine[1];
        }
    }
    return 0.f;
}

// Warp 0 of each CTA brings operands, warp 1 of the pair's first CTA issues the products, the others take finished accumulators while the next
// are being filled.  Barriers, all waits bounded: full[s] in the first CTA (its one arrival announces the bytes of both), empty[s] in both
// (the products that read stage s), acc_full[b] in both, acc_empty[b] in the first CTA (one arrival per epilogue warp of the pair).
// RAW: sixteen more warps bring A, fetched through registers and split into parts on its way (a pass that writes the parts and one that reads them move 16
// bytes an entry in place of 4: loss-cached-rows, 78 us for the former alone); a warp in each CTA passes on to full[s] that a stage is made.
//
// What bounds it.  16-bit operands: the tensor cores, 85 to 89 % of the time active with plain results and maxima, 77 where sums are handed over (16 384 x 1024 x 65 536: 1.40 ms, 1.57
// PFLOP/s; dx and dW of it 1.4 to 1.5), over seconds the 1000 W of the card; g of a tile takes its warps longer than products over less than a thousand entries of k
// (6001 x 512 x 32 003: 222 us, 0.89 PFLOP/s; exponentials, column sums by shuffles).  fp32 x: hand-overs between the roles, 3500 cycles for 64 entries of k whose products are
// 1000 and whose operands take 1600 cycles of shared memory (200 000 rows of 256 to 47 classes: 78 us, 2.6 TB/s).  Tried there: 8 warps (79 us), two chunks on their way in
// registers (93, spills), asynchronous copies into shared memory and two stages (104).
// fp32: six products of parts.  What they leave out is below 1.5 2^-23 of a term where A's parts are cut on their way (RAW: the third of x by the second of W 2^-23, the second
// by the third 2^-24; cut parts have x's sign, so that it does not average out), 2^-24 where both have rounded parts.  The large product, of the first parts, is handed over every 256 entries of k and
// summed in registers, because the tensor core cuts what its additions lose (see unit_of); the small ones gather over the whole tile.
template <int TYPE, bool A_ACROSS, bool B_ACROSS, int END, bool MANY, bool RAW>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LossShape<TYPE, MANY, RAW>::THREADS, 1) k_product(const __grid_constant__ ProductParams p) {
    using S = LossShape<TYPE, MANY, RAW>;
    // What a thread of each role holds in registers, out of what the block is launched with: 896 threads of 72.
    constexpr bool SHARE = RAW;
    static_assert(!SHARE || (S::THREADS == 896 && 128 * 48 + 256 * 144 + 512 * 40 <= 896 * 72), "no more registers are shared out than there are");
    using T = typename Elem<TYPE == RIPPLE_TYPE_F16 ? RIPPLE_TYPE_F16 : RIPPLE_TYPE_BF16>::T;      // of the operands
    constexpr int PARTS = S::PARTS, STAGES = S::STAGES, COLS = S::COLS, GROUPS = S::GROUPS, NB = COLS / (32 * GROUPS), UNIT = unit_of(TYPE, END);      // NB: 32-column blocks of an epilogue warp
    if constexpr (TYPE == RIPPLE_TYPE_F16 && END == END_GRAD) {
        if (p.by_row) {
            pdl_enter();
            if (!p.control->differ) return;
        }
    }
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[STAGES], empty[STAGES], made[RAW ? STAGES : 1], acc_full[2], acc_empty[2], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int s_fail;

    const int tid = threadIdx.x, warp = __shfl_sync(FULL, tid >> 5, 0), lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int64_t tiles = (int64_t)p.row_tiles * p.col_tiles, all = tiles * p.splits;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1, chunks = (p.k + LS_KC - 1) / LS_KC;
    uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    // A tile of C, and the chunks of k of its split.  nt: columns that are multiplied, a multiple of 32; each CTA brings half of them.
    struct Tile { int row, col, split, first, last, nt; };
    auto tile_at = [&](int64_t i) {
        Tile t;
        auto place = [&](auto in, auto in_split) {       // (64-bit divisions take hundreds of cycles: only where there are so many tiles)
            t.split = (int)(in / in_split), in -= (decltype(in))t.split * in_split;
            const decltype(in) per_group = (decltype(in))LS_GROUP * p.col_tiles;
            const int group = (int)(in / per_group), rows = min(LS_GROUP, p.row_tiles - group * LS_GROUP);
            const uint32_t rest = (uint32_t)(in - group * per_group);
            t.col = (int)(rest / (uint32_t)rows), t.row = group * LS_GROUP + (int)(rest - (uint32_t)t.col * (uint32_t)rows);
        };
        if (all < (1ll << 31)) place((uint32_t)i, (uint32_t)tiles);
        else place((uint64_t)i, (uint64_t)tiles);
        t.first = t.split * p.split_chunks, t.last = min(chunks, t.first + p.split_chunks);
        t.nt = min(COLS, (p.n - t.col * COLS + 31) & ~31);
        return t;
    };

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], RAW ? 3 : 1); mbar_init(&empty[s], 1); if (RAW) mbar_init(&made[s], S::LOADERS); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], p.withhold ? 2 : 1 /* one arrives */); mbar_init(&acc_empty[b], 2 * S::EPI_WARPS); }
        mbar_init(&drained, 1);
        s_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_enter();
    // Tensor memory: two accumulators and, fp32, two for the small products
    auto large_at = [&](int b) { return (uint32_t)(COLS * b); };
    auto small_at = [&](int worked) { return (uint32_t)(2 * COLS + COLS * (worked & 1)); };

    if (warp < S::FIRST) {
        if constexpr (SHARE) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 0) {
        // ---------------- operands ----------------
        bool odd = false;
        if (p.control) {
            for (int i = lane; i < LS_CONTROL; i += 32) odd = odd || p.control->odd[i];
            odd = __any_sync(FULL, odd);
        }
        asm volatile("fence.proxy.async;" ::: "memory");      // (what kernels before wrote, for the copies)
        const bool lead = tc_elect();
        if (lead) {
            const CUtensorMap* const a = odd ? &p.a_clean : &p.a;
            const uint32_t to0 = smem_u32(ring);
            bool ok = true;
            int s = 0, issued = 0;
            uint32_t ph = 1;                    // (a fresh barrier counts as completed)
            for (int64_t i = pair; i < all && ok; i += pairs) {
                const Tile t = tile_at(i);
                const int row0 = t.row * LS_ROWS + (int)rank * 128, col0 = p.b_col0 + t.col * COLS + (int)rank * (t.nt / 2);
                for (int c = t.first; c < t.last; ++c) {
                    ok = mbar_wait_bounded(&empty[s], ph, LS_SPIN_LIMIT);
                    if (!ok) break;
                    if (rank == 0) mbar_expect(&full[s], 2 * PARTS * (RAW ? S::B_PART : S::A_PART + S::B_PART));
                    const uint32_t bar = in_leader(&full[s]), to = to0 + (uint32_t)(s * S::STAGE), to_b = to + PARTS * S::A_PART;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) {
                        if constexpr (RAW) {
                        } else if constexpr (A_ACROSS) {
                            for (int h = 0; h < 2; ++h) load_box(to + q * S::A_PART + h * 8192, a, row0 + 64 * h, c * LS_KC, q, bar);
                        } else {
                            load_box(to + q * S::A_PART, a, c * LS_KC, row0, q, bar);
                        }
                        if constexpr (B_ACROSS) {
                            for (int h = 0; h < COLS / 128; ++h) load_box(to_b + q * S::B_PART + h * 8192, &p.b, col0 + 64 * h, p.b_k0 + c * LS_KC, q, bar);
                        } else {
                            load_box(to_b + q * S::B_PART, &p.b, p.b_k0 + c * LS_KC, col0, q, bar);
                        }
                    }
                    ++issued;
                    if (++s == STAGES) { s = 0; ph ^= 1; }
                }
            }
            if (!ok) {
                s_fail = 1;
                // copies in flight: the last of every stage (they complete in the first CTA, which outlives the second's)
                if (rank == 0) {
                    for (int back = min(issued, STAGES); back > 0; --back) {
                        const int at = issued - back;
                        mbar_wait_bounded(&full[at % STAGES], (uint32_t)(at / STAGES) & 1, LS_SPIN_LIMIT);
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- products ----------------
        if (rank == 0) {
            const bool lead = tc_elect();
            const uint32_t base = __shfl_sync(FULL, smem_u32(ring), 0);
            const uint64_t a0 = A_ACROSS ? across_desc(base) : tc_smem_desc(base);
            const uint64_t b0 = B_ACROSS ? across_desc(base + PARTS * S::A_PART) : tc_smem_desc(base + PARTS * S::A_PART);
            constexpr uint64_t A_STEP = A_ACROSS ? 128 : 2, B_STEP = B_ACROSS ? 128 : 2;       // 16 entries of k
            constexpr uint64_t AP = S::A_PART >> 4, BP = S::B_PART >> 4;
            constexpr uint32_t KIND = TYPE == RIPPLE_TYPE_F16 ? 0u : 1u;
            int s = 0, sg = 0, worked = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int64_t i = pair; i < all && ok; i += pairs, ++worked) {
                const Tile t = tile_at(i);
                const int nt = __shfl_sync(FULL, t.nt, 0), first = __shfl_sync(FULL, t.first, 0), last = __shfl_sync(FULL, t.last, 0);
                const uint32_t idesc = (1u << 4) | (KIND << 7) | (KIND << 10) | ((uint32_t)A_ACROSS << 15) | ((uint32_t)B_ACROSS << 16)
                                     | ((uint32_t)(nt >> 3) << 17) | ((uint32_t)(LS_ROWS >> 4) << 24);
                uint32_t acc = 0;
                const uint32_t small = __shfl_sync(FULL, tmem + small_at(worked), 0);
                int b = 0;
                for (int c = first; c < last; ++c) {
                    const int in = c - first;
                    const bool fresh = MANY ? in % UNIT == 0 : in == 0;
                    if (fresh) {
                        b = sg & 1;
                        const int before = sg >> 1;
                        ++sg;
                        // the epilogue must have read this accumulator (and with it the small products of the tile before the last)
                        if (before > 0) ok = mbar_wait_warp(&acc_empty[b], (before - 1) & 1, LS_SPIN_LIMIT);
                        if (!ok) break;
                        tc_fence_after();
                        acc = __shfl_sync(FULL, tmem + large_at(b), 0);
                    }
                    ok = mbar_wait_warp(&full[s], ph, LS_SPIN_LIMIT);
                    if (!ok) break;
                    tc_fence_after();
                    // (broadcast: operands that the compiler cannot see to be the warp's take ten times as long to issue)
                    const uint64_t at = (uint64_t)((uint32_t)__shfl_sync(FULL, s, 0) * (S::STAGE >> 4)), a = a0 + at, w = b0 + at;
                    const bool done = c == last - 1 || (MANY && in % UNIT == UNIT - 1);
                    if (lead) {
#pragma unroll
                        for (int j = 0; j < LS_KC / 16; ++j) {
                            const uint64_t a1 = a + A_STEP * j, w1 = w + B_STEP * j;
                            pair_mma(acc, a1, w1, idesc, !fresh || j != 0);
                            if constexpr (PARTS == 3) {
                                pair_mma(small, a1, w1 + BP, idesc, (in | j) != 0);
                                pair_mma(small, a1 + AP, w1, idesc, 1u);
                                pair_mma(small, a1 + AP, w1 + BP, idesc, 1u);
                                pair_mma(small, a1, w1 + 2 * BP, idesc, 1u);
                                pair_mma(small, a1 + 2 * AP, w1, idesc, 1u);
                            }
                        }
                        pair_commit(&empty[s]);
                        if (done) pair_commit(&acc_full[b]);
                    }
                    __syncwarp();
                    if (++s == STAGES) { s = 0; ph ^= 1; }
                }
            }
            if (!ok) {
                if (lead) {
                    s_fail = 1;
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&drained)) : "memory");
                    mbar_wait_bounded(&drained, 0, LS_SPIN_LIMIT);
                }
                __syncwarp();
            }
        }
    } else if (RAW && warp == 2) {
        // ---------------- passes on that a stage of A is made ----------------
        // (what makes it visible to the other CTA waits for all that a thread has on its way: the loaders' next rows, if they did it themselves)
        const uint32_t full0 = in_leader(&full[0]);
        bool ok = true;
        int s = 0;
        uint32_t ph = 0;
        for (int64_t i = pair; i < all && ok; i += pairs) {
            const Tile t = tile_at(i);
            for (int c = t.first; c < t.last; ++c) {
                ok = mbar_wait_warp(&made[s], ph, LS_SPIN_LIMIT);
                if (!ok) break;
                if (lane == 0) {
                    asm volatile("fence.proxy.async;" ::: "memory");
                    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(full0 + 8 * (uint32_t)s) : "memory");
                }
                __syncwarp();
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
        }
        if (!ok) s_fail = 1;
    }
    } else if (RAW && warp >= S::FIRST + S::EPI_WARPS) {
        if constexpr (SHARE) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        // ---------------- A, from fp32 ----------------
        // thread: a piece of eight entries of PIECES rows of memory, `apart` rows from one another
        constexpr int PIECES = 1024 / (32 * (RAW ? S::LOADERS : 32));
        const int lt = tid - 32 * (S::FIRST + S::EPI_WARPS), across = A_ACROSS ? 16 : 8, apart = 32 * S::LOADERS / across;
        const int piece = lt % across, row_in = lt / across;
        const uint32_t to = smem_u32(ring) + (piece >> 3) * 8192 + tc_swz(row_in, piece & 7);       // (`apart` rows on: the same place, so many 1024 bytes on)
        const uintptr_t base = reinterpret_cast<uintptr_t>(p.raw);
        const int wide = base % 32 == 0 && p.ld_raw % 8 == 0 ? 8 : base % 16 == 0 && p.ld_raw % 4 == 0 ? 4 : base % 8 == 0 && p.ld_raw % 2 == 0 ? 2 : 1;
        int of_row[PIECES];               // labels of the rows fetched (looked at when they are there: the rows do not wait for them)
        auto fetch = [&](float (&v)[PIECES][8], const Tile& t, int c) {
            const int row0 = (A_ACROSS ? c * LS_KC : t.row * LS_ROWS + (int)rank * 128) + row_in;
            const int col = (A_ACROSS ? t.row * LS_ROWS + (int)rank * 128 : c * LS_KC) + piece * 8, left = p.raw_cols - col;
#pragma unroll
            for (int it = 0; it < PIECES; ++it) {
                const int row = row0 + apart * it;
                const bool there = row < p.raw_rows && left > 0;
                const float* const from = p.raw + (int64_t)row * p.ld_raw + col;
                if (A_ACROSS) of_row[it] = there && p.raw_labels ? p.raw_labels[row] : 0;
                // rows further on, on their way to L2: AHEAD chunks, one access in 128 bytes
                constexpr int AHEAD = 2;
                if (A_ACROSS && (piece & 3) == 0 && left > 0 && row + AHEAD * LS_KC < p.raw_rows) asm volatile("prefetch.global.L2 [%0];" ::"l"(from + AHEAD * LS_KC * p.ld_raw));
                if (!A_ACROSS && (piece & 3) == 0 && row < p.raw_rows && left > AHEAD * LS_KC) asm volatile("prefetch.global.L2 [%0];" ::"l"(from + AHEAD * LS_KC));
                if (there && left >= 8 && wide == 8) {
                    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                                 : "=f"(v[it][0]), "=f"(v[it][1]), "=f"(v[it][2]), "=f"(v[it][3]), "=f"(v[it][4]), "=f"(v[it][5]), "=f"(v[it][6]), "=f"(v[it][7]) : "l"(from));
                } else if (there && left >= 8 && wide == 4) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 f = reinterpret_cast<const float4*>(from)[h];
                        v[it][4 * h] = f.x, v[it][4 * h + 1] = f.y, v[it][4 * h + 2] = f.z, v[it][4 * h + 3] = f.w;
                    }
                } else if (there && left >= 8 && wide == 2) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const float2 f = reinterpret_cast<const float2*>(from)[h];
                        v[it][2 * h] = f.x, v[it][2 * h + 1] = f.y;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[it][e] = there && e < left ? from[e] : 0.f;
                }
            }
        };
        bool ok = true;
        int s = 0;
        uint32_t ph = 1;
        auto hand = [&](float (&v)[PIECES][8]) {
            ok = mbar_wait_warp(&empty[s], ph, LS_SPIN_LIMIT);
            if (!ok) return;
#pragma unroll
            for (int it = 0; it < PIECES; ++it) {
                if (A_ACROSS && (uint32_t)of_row[it] >= (uint32_t)p.classes) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[it][e] = 0.f;
                }
                // parts that are cut, 8 bits each, nothing left (of an infinite entry they are NaN: see the epilogue)
                uint32_t a[4], b[4], d[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x0 = v[it][2 * e], x1 = v[it][2 * e + 1];
                    const float m0 = x0 - __uint_as_float(__float_as_uint(x0) & 0xffff0000u), m1 = x1 - __uint_as_float(__float_as_uint(x1) & 0xffff0000u);
                    const float l0 = m0 - __uint_as_float(__float_as_uint(m0) & 0xffff0000u), l1 = m1 - __uint_as_float(__float_as_uint(m1) & 0xffff0000u);
                    a[e] = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
                    b[e] = __byte_perm(__float_as_uint(m0), __float_as_uint(m1), 0x7632);
                    d[e] = __byte_perm(__float_as_uint(l0), __float_as_uint(l1), 0x7632);
                }
                const uint32_t at = to + (uint32_t)(s * S::STAGE + it * (apart / 8) * 1024);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + S::A_PART), "r"(b[0]), "r"(b[1]), "r"(b[2]), "r"(b[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 2 * S::A_PART), "r"(d[0]), "r"(d[1]), "r"(d[2]), "r"(d[3]) : "memory");
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&made[s]);
            if (++s == STAGES) { s = 0; ph ^= 1; }
        };
        // (the next rows are asked for as soon as these are in shared memory)
        float v[PIECES][8];
        int64_t i = pair;
        Tile t = {};
        int c = 0;
        if (i < all) t = tile_at(i), c = t.first, fetch(v, t, c);
        while (i < all) {
            hand(v);
            if (!ok) break;
            if (++c >= t.last) {
                i += pairs;
                if (i >= all) break;
                t = tile_at(i), c = t.first;
            }
            fetch(v, t, c);
            if (!A_ACROSS && c == t.first && i + pairs < all) {
                // and the first chunks of the tile after this one
                const Tile n = tile_at(i + pairs);
                const int row = n.row * LS_ROWS + (int)rank * 128 + (lt & 127), col = n.first * LS_KC + (lt >> 7) * 32;
                const float* const from = p.raw + (int64_t)row * p.ld_raw + col;
                if (row < p.raw_rows && col < p.raw_cols) asm volatile("prefetch.global.L2 [%0];" ::"l"(from));
            }
        }
        if (!ok) s_fail = 1;
    } else {
        if constexpr (SHARE) asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
        // ---------------- epilogue ----------------
        // thread: a row, and the 32-column blocks part, part + GROUPS, ... of the tile
        const int q = warp & 3, part = (warp - S::FIRST) >> 2;
        const uint32_t lanes = tmem + ((uint32_t)(32 * q) << 16);
        float* const bias = reinterpret_cast<float*>(ring + STAGES * S::STAGE) + (warp - S::FIRST) * 32 * NB;
        float factor = 1.f, unfactor = 1.f;      // GRAD: of g, and of its sums; OUT: of the result
        bool by_row = false;
        if (TYPE == RIPPLE_TYPE_F16 && p.control) {
            if (END == END_GRAD) factor = grad_scale(p.control, p.scale), unfactor = 1.f / factor, by_row = p.by_row;
            if (END == END_GRAD && p.differ && blockIdx.x == 0 && warp == S::FIRST) {
                const bool differ = weights_differ(p.control);
                if (lane == 0) *p.differ = differ;
            }
            if (END == END_OUT && p.unscale) factor = 1.f / grad_scale(p.control, p.scale), by_row = p.by_row && p.control->differ;
        }
        const uint32_t release = in_leader(&acc_empty[0]);
        bool ok = true;
        int sg = 0, worked = 0;
        // What a tile's rows and columns have to do with: asked for a tile ahead.
        struct Ahead { int label; float lse, dloss, bias[NB]; };
        auto row_of_tile = [&](const Tile& t) { return t.row * LS_ROWS + (int)rank * 128 + 32 * q + lane; };
        auto ask = [&](const Tile& t) {
            Ahead a = {-1, 0.f, 1.f};
            const int row = row_of_tile(t);
            const int32_t* const labels = END == END_OUT ? p.dead_rows : p.labels;
            if (row < p.m && labels) a.label = labels[row];
            if constexpr (END == END_GRAD) {
                if (row < p.m) a.lse = p.lse[row];
            }
            if (END == END_GRAD || (END == END_OUT && by_row)) if (row < p.m && p.dloss) a.dloss = p.dloss[row];
            if constexpr (END != END_OUT) {
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const int col = t.col * COLS + 32 * (GROUPS * j + part) + lane;
                    a.bias[j] = col >= p.n ? -INFINITY : p.bias ? p.bias[col] : 0.f;
                }
            }
            return a;
        };
        Tile following = tile_at(pair);
        Ahead asked = ask(following);
        for (int64_t i = pair; i < all && ok; i += pairs, ++worked) {
            const Tile t = following;
            const int row = row_of_tile(t), col0 = t.col * COLS;
            const bool in_rows = row < p.m, labelled = asked.label >= 0 && asked.label < p.classes;
            bool live = END == END_OUT ? in_rows && (!p.dead_rows || labelled) : labelled;
            if (TYPE == RIPPLE_TYPE_F16 && by_row) {
                factor = scale_of(p.scale * asked.dloss);
                if (END == END_OUT) factor = 1.f / factor;
            }
            const float lse = asked.lse, weight = p.scale * asked.dloss * (END == END_GRAD ? factor : 1.f);
            float top = -INFINITY, sum = 0.f;
            if (END == END_GRAD) live = live && lse != -INFINITY;
            const int label = live ? asked.label - p.class0 - col0 : -1;       // within the tile
            if constexpr (END != END_OUT) {
                __syncwarp();
#pragma unroll
                for (int j = 0; j < NB; ++j) bias[32 * j + lane] = asked.bias[j];
                __syncwarp();
            }
            if (i + pairs < all) following = tile_at(i + pairs), asked = ask(following);
            // 32 finished sums of this row, from column `at` of the tile
            auto finish = [&](float (&y)[32], int j) {
                const int at = 32 * (GROUPS * j + part);
                if constexpr (END == END_LSE) {
                    const float4* const b4 = reinterpret_cast<const float4*>(bias + 32 * j);
                    float high[4] = {top, top, top, top};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 b = b4[e];
                        add2(y[4 * e], y[4 * e + 1], b.x, b.y), add2(y[4 * e + 2], y[4 * e + 3], b.z, b.w);
                    }
                    if (__any_sync(FULL, (unsigned)(label - at) < 32u)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) if (label == at + e) p.at_label[row] = y[e];
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) high[e & 3] = fmaxf(high[e & 3], y[e]);
                    const float most = fmaxf(fmaxf(high[0], high[1]), fmaxf(high[2], high[3]));
                    // (subtracted first: the largest logit adds exactly one, so that lse is no smaller than any logit and no loss negative)
                    const float base = most == -INFINITY ? 0.f : most;
                    sum *= exp2_of((top - base) * LOG2E);
                    float more[4] = {};
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        add2(y[e], y[e + 1], -base, -base);
                        mul2(y[e], y[e + 1], LOG2E, LOG2E);
                        add2(more[e & 2], more[(e & 2) + 1], exp2_of(y[e]), exp2_of(y[e + 1]));
                    }
                    sum += (more[0] + more[1]) + (more[2] + more[3]);
                    top = most;
                } else if constexpr (END == END_GRAD) {
                    const float4* const b4 = reinterpret_cast<const float4*>(bias + 32 * j);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 b = b4[e];
                        add2(y[4 * e], y[4 * e + 1], b.x, b.y), add2(y[4 * e + 2], y[4 * e + 3], b.z, b.w);
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        add2(y[e], y[e + 1], -lse, -lse);
                        mul2(y[e], y[e + 1], LOG2E, LOG2E);
                        y[e] = exp2_of(y[e]), y[e + 1] = exp2_of(y[e + 1]);
                    }
                    if (__any_sync(FULL, (unsigned)(label - at) < 32u)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) if (label == at + e) y[e] -= 1.f;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 2) mul2(y[e], y[e + 1], weight, weight);
                    if (!__all_sync(FULL, live)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = live ? y[e] : 0.f;
                    }
                    // (16 bits: g is rounded to its operand's type, half a step beside the half step of dx and dW; in parts the products would take three times as long)
                    if (p.g && in_rows) {
                        uint16_t* const to = p.g + (int64_t)row * p.ld_g + col0 + at;
                        if constexpr (PARTS == 1) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                uint32_t v[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[e] = pair_of<T>(y[16 * h + 2 * e], y[16 * h + 2 * e + 1]);
                                store8(to + 16 * h, v);
                            }
                        } else {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float left[16];
#pragma unroll
                                for (int e = 0; e < 16; ++e) left[e] = y[16 * h + e];
#pragma unroll
                                for (int q3 = 0; q3 < 3; ++q3) {
                                    uint32_t v[8];
#pragma unroll
                                    for (int e = 0; e < 8; ++e) {
                                        v[e] = pair_of<__nv_bfloat16>(left[2 * e], left[2 * e + 1]);
                                        const float h0 = __uint_as_float(v[e] << 16), h1 = __uint_as_float(v[e] & 0xffff0000u);
                                        left[2 * e] = fabsf(h0) < INFINITY ? left[2 * e] - h0 : 0.f, left[2 * e + 1] = fabsf(h1) < INFINITY ? left[2 * e + 1] - h1 : 0.f;
                                    }
                                    store8(to + q3 * p.g_plane + 16 * h, v);
                                }
                            }
                        }
                    }
                    if (p.g_sums) {
                        const float s = column_sums(y);
                        if (row - lane < p.m) p.g_sums[(int64_t)((row - lane) >> 5) * p.ld_g + col0 + at + lane] = s * unfactor;
                    }
                } else {
                    if (!in_rows) return;
                    const int col = col0 + at, out_size = p.out_f32 ? 4 : 2;
                    uint8_t* const to = static_cast<uint8_t*>(p.out) + ((int64_t)row * p.ld_out + col + t.split * p.split_stride) * out_size;
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[e] = live ? y[e] * factor : 0.f;
                    if (p.add_to_out) {
                        const float* const from = reinterpret_cast<const float*>(to);
#pragma unroll
                        for (int e = 0; e < 32; ++e) if (col + e < p.n) y[e] += from[e];
                    }
                    if (col + 32 <= p.n) {
                        uint32_t v[8];
                        if (p.out_f32) {
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[e] = __float_as_uint(y[8 * h + e]);
                                store8(to + 32 * h, v);
                            }
                        } else {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[e] = pair_of<T>(y[16 * h + 2 * e], y[16 * h + 2 * e + 1]);
                                store8(to + 32 * h, v);
                            }
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (col + e >= p.n) continue;
                            if (p.out_f32) reinterpret_cast<float*>(to)[e] = y[e];
                            else reinterpret_cast<T*>(to)[e] = from_f32<T>(y[e]);
                        }
                    }
                }
            };
            const int units = MANY ? (t.last - t.first + UNIT - 1) / UNIT : 1;
            float carry[MANY ? NB : 1][32];          // of the units before the last
            for (int u = 0; u < units && ok; ++u, ++sg) {
                const int b = sg & 1;
                ok = mbar_wait_warp(&acc_full[b], (sg >> 1) & 1, LS_SPIN_LIMIT);
                if (!ok) break;
                tc_fence_after();
                const uint32_t large = lanes + large_at(b), small = lanes + small_at(worked);
                // the accumulator is handed back once this warp's last block has been read
                const int blocks = t.nt > 32 * part ? min(NB, (t.nt - 32 * part + 32 * GROUPS - 1) / (32 * GROUPS)) : 0;
                auto hand_back = [&]() {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_at(release + 8 * (uint32_t)b);
                };
                if (blocks == 0) hand_back();
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const int at = 32 * (GROUPS * j + part);
                    if (j >= blocks) continue;
                    uint32_t x[32];
                    float y[32];
                    tc_load32(x, large + (uint32_t)at);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(x[e]);
                    if constexpr (MANY) {
                        if (u > 0) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) y[e] += carry[j][e];
                        }
                        if (u < units - 1) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) carry[j][e] = y[e];
                            if (j == blocks - 1) hand_back();
                            continue;
                        }
                    }
                    if constexpr (PARTS == 3) {
                        // (an infinite entry has no parts: its small products may be NaN)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t w[16];
                            tc_load16(w, small + (uint32_t)(at + 16 * h));
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                            for (int e = 0; e < 16; ++e) if (fabsf(y[16 * h + e]) < INFINITY) y[16 * h + e] += __uint_as_float(w[e]);
                        }
                    }
                    if (j == blocks - 1) hand_back();
                    finish(y, j);
                }
            }
            if (END == END_LSE && ok && in_rows) p.sums[(int64_t)(GROUPS * t.col + part) * p.m + row] = make_float2(top, sum);
        }
        if (!ok) s_fail = 1;
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    if (s_fail && tid == 0) g_loss_timeout = 1;
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// ---- what stands around the products -----------------------------------------------------------------------------------
__device__ __forceinline__ bool has_label(const int32_t* labels, int64_t row, int classes) { return (uint32_t)labels[row] < (uint32_t)classes; }

// A matrix as an operand: planes of 16-bit parts, rows `ld` apart, zeros beyond the columns.  labels: rows without one become zeros, because in x^T g
// whatever they hold is multiplied by zero.  control: only if such a row holds something that is not finite.
struct OperandParams {
    const void* from;
    int64_t rows, ld_from;
    int cols, lanes;
    uint16_t* to;
    int64_t ld, plane;
    const int32_t* labels;
    int classes;
    const RowControl* control;
};
template <typename T>
__global__ void __launch_bounds__(256) k_operand(const __grid_constant__ OperandParams p) {
    pdl_enter();
    if (p.control) {
        bool odd = false;
        for (int i = lane_id(); i < LS_CONTROL; i += 32) odd = odd || p.control->odd[i];
        if (!__any_sync(FULL, odd)) return;
    }
    const int t = threadIdx.x & (p.lanes - 1), per_block = 256 / p.lanes;
    const bool vec = (reinterpret_cast<uintptr_t>(p.from) & 15) == 0 && p.ld_from % (16 / (int)sizeof(T)) == 0;
    for (int64_t row = (int64_t)blockIdx.x * per_block + threadIdx.x / p.lanes; row < p.rows; row += (int64_t)gridDim.x * per_block) {
        const T* const from = static_cast<const T*>(p.from) + row * p.ld_from;
        uint16_t* const to = p.to + row * p.ld;
        const bool live = !p.labels || has_label(p.labels, row, p.classes);
        for (int c = t * 8; c < p.ld; c += p.lanes * 8) {
            Piece<T, 8> v;
            if (live && vec && c + 8 <= p.cols) {
                v = *reinterpret_cast<const Piece<T, 8>*>(from + c);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v.v[e] = live && c + e < p.cols ? from[c + e] : from_f32<T>(0.f);
            }
            if constexpr (sizeof(T) == 4) {
                Piece<__nv_bfloat16, 8> part[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    __nv_bfloat16 h[3];
                    three_parts(v.v[e], h);
                    part[0].v[e] = h[0], part[1].v[e] = h[1], part[2].v[e] = h[2];
                }
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<Piece<__nv_bfloat16, 8>*>(to + q * p.plane + c) = part[q];
            } else {
                *reinterpret_cast<Piece<T, 8>*>(to + c) = v;
            }
        }
    }
}

// What the gradient has to know of all rows: the largest and the smallest dloss (fp16), and whether a row without a label holds something that is not finite (x read in place).
template <typename T>
__global__ void __launch_bounds__(256) k_look_at_rows(const T* x, int64_t ld_x, int k, const int32_t* labels, const float* dloss, int64_t rows, int classes, RowControl* control) {
    pdl_enter();
    __shared__ float2 scratch[8];
    float most = 0.f, least = INFINITY;
    bool odd = false;
    for (int64_t r0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * 32; r0 < rows; r0 += (int64_t)LS_CONTROL * 256) {
        const int64_t row = r0 + lane_id();
        const bool live = row < rows && has_label(labels, row, classes);
        if (live) {
            const float w = dloss ? fabsf(dloss[row]) : 1.f;
            if (isfinite(w)) most = fmaxf(most, w);
            if (w > 0.f) least = fminf(least, w);
        }
        for (uint32_t left = x ? __ballot_sync(FULL, row < rows && !live) : 0; left; left &= left - 1) {
            const T* const from = x + (r0 + __ffs(left) - 1) * ld_x;
#pragma unroll 8
            for (int c = lane_id(); c < k; c += 32) odd = odd | !isfinite(to_f32(from[c]));
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(FULL, most, o)), least = fminf(least, __shfl_xor_sync(FULL, least, o));
    if (lane_id() == 0) scratch[threadIdx.x >> 5] = make_float2(most, least);
    const int any = __syncthreads_or(odd);
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) most = fmaxf(most, scratch[w].x), least = fminf(least, scratch[w].y);
        control->most[blockIdx.x] = most, control->least[blockIdx.x] = least, control->odd[blockIdx.x] = any;
    }
}

// Loss and lse from the tiles' sums; a block has 32 rows for every TURNS of its 16 warps, which take turns over the tiles.
// running: what the pieces of the classes before gave, and this one adds to; null: it is the only one.
template <int TURNS>
__global__ void __launch_bounds__(512) k_finish_loss(const float2* sums, int parts, int64_t rows, const float* at_label, const int32_t* labels, int classes, float* loss, float* lse,
                                                     float2* running, int first, int last) {
    pdl_enter();
    __shared__ float2 mine[16][33];
    const int warp = threadIdx.x >> 5, lane = lane_id(), turn = warp % TURNS;
    const int64_t row = ((int64_t)blockIdx.x * (16 / TURNS) + warp / TURNS) * 32 + lane;
    float top = -INFINITY, sum = 0.f;
    auto join = [&](float2 s) {
        const float most = fmaxf(top, s.x), base = most == -INFINITY ? 0.f : most;
        sum = sum * exp2_of((top - base) * LOG2E) + s.y * exp2_of((s.x - base) * LOG2E);
        top = most;
    };
    if (row < rows) {
#pragma unroll 8
        for (int i = turn; i < parts; i += TURNS) join(sums[i * rows + row]);
    }
    if constexpr (TURNS > 1) {
        mine[warp][lane] = make_float2(top, sum);
        __syncthreads();
        if (turn == 0) {
            top = -INFINITY, sum = 0.f;
            for (int w = 0; w < TURNS; ++w) join(mine[warp + w][lane]);
        }
    }
    if (turn > 0 || row >= rows) return;
    if (!first) join(running[row]);
    if (!last) {
        running[row] = make_float2(top, sum);
        return;
    }
    const float l = top == -INFINITY && sum == 0.f ? -INFINITY : top + logf(sum);
    lse[row] = l;
    if (loss) loss[row] = has_label(labels, row, classes) && l != -INFINITY ? l - at_label[row] : 0.f;
}

// out = the sum of the splits' results, in order.
template <typename T>
__global__ void __launch_bounds__(256) k_join_parts(const float* parts, int splits, int64_t split_stride, int64_t ld, T* out, int64_t ld_out, int64_t rows, int cols) {
    pdl_enter();
    constexpr int U = 4;
    const int c0 = blockIdx.x * (256 * U) + threadIdx.x;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        float sum[U] = {};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) {
            const float* const from = parts + s * split_stride + row * ld;
#pragma unroll
            for (int u = 0; u < U; ++u) if (c0 + 256 * u < cols) sum[u] += from[c0 + 256 * u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) if (c0 + 256 * u < cols) out[row * ld_out + c0 + 256 * u] = from_f32<T>(sum[u]);
    }
}

// The same for few columns and many parts: a block has 32 columns of a row, its eight warps take turns over the parts.
template <typename T>
__global__ void __launch_bounds__(256) k_join_many_parts(const float* parts, int splits, int64_t split_stride, int64_t ld, T* out, int64_t ld_out, int64_t rows, int cols) {
    pdl_enter();
    __shared__ float mine[8][32];
    const int warp = threadIdx.x >> 5, lane = lane_id(), c = blockIdx.x * 32 + lane;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        float sum = 0.f;
        if (c < cols) {
#pragma unroll 10
            for (int s = warp; s < splits; s += 8) sum += parts[s * split_stride + row * ld + c];
        }
        mine[warp][lane] = sum;
        __syncthreads();
        if (warp == 0 && c < cols) {
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) sum += mine[w][lane];
            out[row * ld_out + c] = from_f32<T>(sum);
        }
        __syncthreads();
    }
}

// dbias from the sums over groups of 32 rows; a block has COLS columns, its warps and the parts of a warp take turns over the groups.  Eight where that is
// what makes a block for every SM, else 32 (16 384 columns: 28 us and 11).
template <int COLS>
__global__ void __launch_bounds__(1024) k_join_columns(const float* sums, int64_t groups, int64_t ld, int cols, float* out) {
    pdl_enter();
    __shared__ float mine[32][COLS];
    constexpr int TURNS = 32 / COLS;
    const int warp = threadIdx.x >> 5, lane = lane_id(), c = blockIdx.x * COLS + lane % COLS;
    float sum = 0.f;
    if (c < cols) {
#pragma unroll 16
        for (int64_t i = warp * TURNS + lane / COLS; i < groups; i += 32 * TURNS) sum += sums[i * ld + c];
    }
#pragma unroll
    for (int o = COLS; o < 32; o *= 2) sum += __shfl_xor_sync(FULL, sum, o);
    if (lane < COLS) mine[warp][lane] = sum;
    __syncthreads();
    if (warp > 0 || lane >= COLS || c >= cols) return;
    sum = 0.f;
    for (int w = 0; w < 32; ++w) sum += mine[w][lane];
    out[c] = sum;
}

// ---- plans -----------------------------------------------------------------------------------------------------------
static int up_to(int64_t x, int to) { return (int)((x + to - 1) / to * to); }
static int64_t aligned128(int64_t x) { return (x + 127) / 128 * 128; }
static int parts_of(int type) { return type == RIPPLE_TYPE_F32 ? 3 : 1; }
// column groups of a tile whose sums the loss keeps apart
static int groups_of(int type, int k) {
    const bool many = (k + LS_KC - 1) / LS_KC > unit_of(type, END_LSE);
    return type == RIPPLE_TYPE_F32 ? LossShape<RIPPLE_TYPE_F32, true, true>::GROUPS : many ? LossShape<RIPPLE_TYPE_BF16, true>::GROUPS : LossShape<RIPPLE_TYPE_BF16, false>::GROUPS;
}
static int cols_of(int type) { return type == RIPPLE_TYPE_F32 ? 128 : 256; }

// Whether TMA can read a matrix where it lies.
static bool readable(int type, const void* p, int64_t ld, int64_t cols) {
    return type != RIPPLE_TYPE_F32 && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 && ld >= cols && ld < (1ll << 36);
}
static bool writable(int size, const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0 && ld * size % 32 == 0; }

// ---- few rows, small heads ---------------------------------------------------------------------------------------------
// W lies in shared memory as fp32, eight rows of x beside it; a lane is a class, warps share the classes and k.  Plain fp32 sums, one launch
// for the loss, two for its gradient (the second: dW and dbias from g, which is of a few rows).
constexpr int FL_ROWS = 8, FL_THREADS = 1024, FL_WARPS = FL_THREADS / 32;
constexpr int FL_BYTES = 220 * 1024;
constexpr int FL_K = 8;                  // rows of dW per block

struct FewParams {
    int rows, k, n;
    const void* x;
    const void* W;
    int64_t ld_x, ld_w;
    const float* bias;
    const int32_t* labels;
    float* loss;
    float* lse;                          // the gradient reads it
    const float* dloss;
    float scale;
    float* g;                            // rows x n; null: not wanted
    void* dx;
    int64_t ld_dx;
    void* dW;
    int64_t ld_dw;
    float* dbias;
};
__host__ __device__ inline bool few_at_once(int rows, int k, int n);
__host__ __device__ inline int few_pitch(int n) { return n | 1; }          // of W in shared memory: lanes that are rows of W meet no bank twice
static int64_t few_bytes(int k, int n) { return ((int64_t)k * few_pitch(n) + FL_ROWS * ((int64_t)k + up_to(n, 32)) + 8 + FL_WARPS * FL_ROWS * 32) * 4; }

template <typename T, bool GRAD>
__global__ void __launch_bounds__(FL_THREADS, 1) k_loss_few(const __grid_constant__ FewParams p) {
    pdl_enter();
    extern __shared__ __align__(16) float few[];
    const int pitch = GRAD ? few_pitch(p.n) : p.n, warp = threadIdx.x >> 5, lane = lane_id();       // (the loss has classes as lanes alone)
    const int cols = (p.n + 31) / 32, shares = FL_WARPS / cols, each = (p.k + shares - 1) / shares;      // 32-class blocks; parts of k
    float* const xs = few;                                // k x FL_ROWS
    float* const gs = xs + FL_ROWS * p.k;                 // classes x FL_ROWS: logits, then g
    float* const sums = gs + FL_ROWS * 32 * cols;         // part of k x class block x FL_ROWS x 32
    float* const ws = sums + FL_WARPS * FL_ROWS * 32;     // k x pitch
    const T* const x = static_cast<const T*>(p.x);
    auto copy = [](float* to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(to)), "l"(from) : "memory"); };
    const T* const W = static_cast<const T*>(p.W);
    if (pitch == p.n && p.ld_w == p.n && (reinterpret_cast<uintptr_t>(W) & 15) == 0) {
        // W lies in memory as it will here: 16 bytes at a time (1000 fp32 rows, 602 -> 41, loss and gradient: 40 us by single entries, 37 so)
        constexpr int E = 16 / sizeof(T);
        const int all = p.k * p.n;
#pragma unroll 8
        for (int i = threadIdx.x * E; i + E <= all; i += FL_THREADS * E) {
            if constexpr (sizeof(T) == 4) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(ws + i)), "l"(W + i) : "memory");
            } else {
                const Piece<T, 8> v = *reinterpret_cast<const Piece<T, 8>*>(W + i);
#pragma unroll
                for (int h = 0; h < 8; h += 4)
                    *reinterpret_cast<float4*>(ws + i + h) = make_float4(to_f32(v.v[h]), to_f32(v.v[h + 1]), to_f32(v.v[h + 2]), to_f32(v.v[h + 3]));
            }
        }
        for (int i = all / E * E + threadIdx.x; i < all; i += FL_THREADS) ws[i] = to_f32(W[i]);
    } else {
        constexpr int U = 16;            // rows that are on their way (fp32: all)
        const int c = warp % cols * 32 + lane;
        if (c < p.n) {
            for (int k0 = warp / cols; k0 < p.k && warp / cols < shares; k0 += shares * U) {
                T v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int k = k0 + u * shares;
                    if (k >= p.k) continue;
                    if constexpr (sizeof(T) == 4) copy(ws + k * pitch + c, W + (int64_t)k * p.ld_w + c);
                    else v[u] = W[(int64_t)k * p.ld_w + c];
                }
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int u = 0; u < U; ++u) if (k0 + u * shares < p.k) ws[(k0 + u * shares) * pitch + c] = to_f32(v[u]);
                }
            }
        }
    }
    for (int row0 = blockIdx.x * FL_ROWS; row0 < p.rows; row0 += gridDim.x * FL_ROWS) {
        for (int k = threadIdx.x; k < p.k; k += FL_THREADS) {
            T v[FL_ROWS];
#pragma unroll
            for (int r = 0; r < FL_ROWS; ++r) {
                if constexpr (sizeof(T) == 4) {
                    if (row0 + r < p.rows) copy(xs + k * FL_ROWS + r, x + (int64_t)(row0 + r) * p.ld_x + k);
                    else xs[k * FL_ROWS + r] = 0.f;
                } else {
                    v[r] = row0 + r < p.rows ? x[(int64_t)(row0 + r) * p.ld_x + k] : from_f32<T>(0.f);
                }
            }
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int r = 0; r < FL_ROWS; ++r) xs[k * FL_ROWS + r] = to_f32(v[r]);
            }
        }
        if constexpr (sizeof(T) == 4) asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        const int block = warp % cols, share = warp / cols;
        if (share < shares) {
            const int c = min(block * 32 + lane, p.n - 1), end = min(p.k, (share + 1) * each);
            float z[FL_ROWS] = {};
#pragma unroll 4
            for (int k = share * each; k < end; ++k) {
                const float w = ws[k * pitch + c];
                const float4 a = *reinterpret_cast<const float4*>(xs + k * FL_ROWS), b = *reinterpret_cast<const float4*>(xs + k * FL_ROWS + 4);
                z[0] = fmaf(a.x, w, z[0]), z[1] = fmaf(a.y, w, z[1]), z[2] = fmaf(a.z, w, z[2]), z[3] = fmaf(a.w, w, z[3]);
                z[4] = fmaf(b.x, w, z[4]), z[5] = fmaf(b.y, w, z[5]), z[6] = fmaf(b.z, w, z[6]), z[7] = fmaf(b.w, w, z[7]);
            }
#pragma unroll
            for (int r = 0; r < FL_ROWS; ++r) sums[(warp * FL_ROWS + r) * 32 + lane] = z[r];
        }
        __syncthreads();
        for (int e = threadIdx.x; e < FL_ROWS * 32 * cols; e += FL_THREADS) {
            const int r = e / (32 * cols), c = e - r * 32 * cols, row = row0 + r;
            float z = 0.f;
            for (int s = 0; s < shares; ++s) z += sums[((s * cols + (c >> 5)) * FL_ROWS + r) * 32 + (c & 31)];
            if (c < p.n && p.bias) z += p.bias[c];
            if constexpr (GRAD) {
                float g = 0.f;
                if (c < p.n && row < p.rows && has_label(p.labels, row, p.n)) {
                    const float lse = p.lse[row];
                    if (lse != -INFINITY) g = (exp2_of((z - lse) * LOG2E) - (p.labels[row] == c ? 1.f : 0.f)) * (p.scale * (p.dloss ? p.dloss[row] : 1.f));
                }
                if (p.g && c < p.n && row < p.rows) p.g[(int64_t)row * p.n + c] = g;
                z = g;
            }
            gs[c * FL_ROWS + r] = c < p.n || GRAD ? z : -INFINITY;
        }
        __syncthreads();
        if constexpr (!GRAD) {
            const int row = row0 + warp;
            if (warp < FL_ROWS && row < p.rows) {
                float top = -INFINITY, sum = 0.f;
                for (int c = lane; c < 32 * cols; c += 32) top = fmaxf(top, gs[c * FL_ROWS + warp]);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
                const float base = top == -INFINITY ? 0.f : top;
                for (int c = lane; c < 32 * cols; c += 32) sum += exp2_of((gs[c * FL_ROWS + warp] - base) * LOG2E);
                sum = warp_sum(sum);
                if (lane == 0) {
                    const float lse = sum == 0.f && top == -INFINITY ? -INFINITY : top + logf(sum);
                    p.lse[row] = lse;
                    if (p.loss) p.loss[row] = has_label(p.labels, row, p.n) && lse != -INFINITY ? lse - gs[p.labels[row] * FL_ROWS + warp] : 0.f;
                }
            }
        } else {
            for (int k = threadIdx.x; k < p.k && p.dx; k += FL_THREADS) {
                float d[FL_ROWS] = {};
#pragma unroll 4
                for (int c = 0; c < p.n; ++c) {
                    const float w = ws[k * pitch + c];
                    const float4 a = *reinterpret_cast<const float4*>(gs + c * FL_ROWS), b = *reinterpret_cast<const float4*>(gs + c * FL_ROWS + 4);
                    d[0] = fmaf(a.x, w, d[0]), d[1] = fmaf(a.y, w, d[1]), d[2] = fmaf(a.z, w, d[2]), d[3] = fmaf(a.w, w, d[3]);
                    d[4] = fmaf(b.x, w, d[4]), d[5] = fmaf(b.y, w, d[5]), d[6] = fmaf(b.z, w, d[6]), d[7] = fmaf(b.w, w, d[7]);
                }
#pragma unroll
                for (int r = 0; r < FL_ROWS; ++r) {
                    const int row = row0 + r;
                    if (row < p.rows) static_cast<T*>(p.dx)[(int64_t)row * p.ld_dx + k] = from_f32<T>(has_label(p.labels, row, p.n) ? d[r] : 0.f);
                }
            }
            if (few_at_once(p.rows, p.k, p.n)) {         // dW and dbias as well
                bool live[FL_ROWS];
#pragma unroll
                for (int r = 0; r < FL_ROWS; ++r) live[r] = r < p.rows && has_label(p.labels, r, p.n);
                const int c = warp % cols * 32 + lane;
                if (c < p.n && warp / cols < shares) {
                    float g[FL_ROWS], sum = 0.f;
#pragma unroll
                    for (int r = 0; r < FL_ROWS; ++r) g[r] = gs[c * FL_ROWS + r], sum += g[r];
                    if (p.dbias && warp < cols) p.dbias[c] = sum;
                    for (int k = warp / cols; k < p.k && p.dW; k += shares) {
                        float d = 0.f;
#pragma unroll
                        for (int r = 0; r < FL_ROWS; ++r) if (live[r]) d = fmaf(xs[k * FL_ROWS + r], g[r], d);
                        static_cast<T*>(p.dW)[(int64_t)k * p.ld_dw + c] = from_f32<T>(d);
                    }
                }
            }
        }
        __syncthreads();
    }
}

// dW = x^T g and dbias: a block has FL_K rows of dW and 32 columns, its warps take turns over the rows of x; those without a label are passed over.
template <typename T>
__global__ void __launch_bounds__(FL_THREADS) k_loss_few_weights(const __grid_constant__ FewParams p) {
    pdl_enter();
    constexpr int U = 16;                  // rows of a warp that are on their way
    __shared__ __align__(16) float sums[FL_WARPS][FL_K + 1][32];       // (and before the end, rows of x)
    static_assert(U <= 32 && U * FL_K <= (FL_K + 1) * 32 && 32 % FL_K == 0, "a warp's rows of x lie in its sums");
    const int warp = threadIdx.x >> 5, lane = lane_id(), k0 = blockIdx.x * FL_K, c = blockIdx.y * 32 + lane;
    const int k = min(k0 + (lane & (FL_K - 1)), p.k - 1), c_in = min(c, p.n - 1);
    const T* const x = static_cast<const T*>(p.x) + k;
    float* const xs = &sums[warp][0][0];
    float d[FL_K] = {}, of_bias = 0.f;
    for (int row0 = warp; row0 < p.rows; row0 += FL_WARPS * U) {
        // x: a lane has one of the columns of every fourth row
        constexpr int PER = 32 / FL_K, XU = U / PER;
        float v[XU], g[U];
#pragma unroll
        for (int u = 0; u < XU; ++u) v[u] = to_f32(x[(int64_t)min(row0 + (u * PER + lane / FL_K) * FL_WARPS, p.rows - 1) * p.ld_x]);
#pragma unroll
        for (int u = 0; u < U; ++u) g[u] = p.g[(int64_t)min(row0 + u * FL_WARPS, p.rows - 1) * p.n + c_in];
        const int mine = row0 + (lane % U) * FL_WARPS;
        const uint32_t live = __ballot_sync(FULL, mine < p.rows && has_label(p.labels, min(mine, p.rows - 1), p.n));
#pragma unroll
        for (int u = 0; u < XU; ++u) xs[(u * PER + lane / FL_K) * FL_K + lane % FL_K] = live >> (u * PER + lane / FL_K) & 1 ? v[u] : 0.f;
        __syncwarp();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float gu = live >> u & 1 ? g[u] : 0.f;
            of_bias += gu;
#pragma unroll
            for (int j = 0; j < FL_K; j += 4) {
                const float4 a = *reinterpret_cast<const float4*>(xs + u * FL_K + j);
                d[j] = fmaf(a.x, gu, d[j]), d[j + 1] = fmaf(a.y, gu, d[j + 1]), d[j + 2] = fmaf(a.z, gu, d[j + 2]), d[j + 3] = fmaf(a.w, gu, d[j + 3]);
            }
        }
        __syncwarp();
    }
#pragma unroll
    for (int j = 0; j < FL_K; ++j) sums[warp][j][lane] = d[j];
    sums[warp][FL_K][lane] = of_bias;
    __syncthreads();
    if (warp > FL_K || c >= p.n) return;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < FL_WARPS; ++w) total += sums[w][warp][lane];
    if (warp == FL_K) {
        if (p.dbias && k0 == 0) p.dbias[c] = total;
    } else if (p.dW && k0 + warp < p.k) {
        static_cast<T*>(p.dW)[(int64_t)(k0 + warp) * p.ld_dw + c] = from_f32<T>(total);
    }
}

// Rounds of eight rows on every SM up to which calls of small heads take this form.  Both sides, us on the device for the loss and its gradient, this form / tensor
// cores.  fp32 602 -> 41: 1184 rows (a round) 9 + 26 / 23 + 58, 3552 rows 21 + 60 / 23 + 61; 256 -> 47: 3552 rows 14 + 34 / 13 + 42; 256 -> 150: 1184 rows
// 9 + 34 / 14 + 49, 2368 rows 16 + 54 / 15 + 49.  bf16 256 -> 47: 2368 rows 10 + 24 / 9 + 34, 3552 rows 13 + 33 / 9 + 35; 602 -> 41: 1184 rows 9 + 26 / 13 + 30, 2368 rows
// 14 + 42 / 13 + 33; 64 -> 500: 1184 rows 10 + 29 / 10 + 36, 2368 rows 18 + 48 / 10 + 37.  Above 512 classes, one share of k: 64 -> 600, 300 and 1184 rows, fp32 11 + 29 / 10 + 39 and
// 11 + 40 / 10 + 48, bf16 12 + 31 / 8 + 32 and 12 + 42 / 8 + 34, fp16 12 + 31 / 8 + 39 and 12 + 42 / 8 + 43; 32 -> 1000, fp32 12 + 33 / 10 + 39 and 12 + 38 / 11 + 48, bf16 13 + 34 / 8 + 33 and
// 13 + 38 / 8 + 37, fp16 13 + 34 / 8 + 41 and 13 + 39 / 8 + 45: bf16 would be 5 to 11 us faster on the tensor cores there.
constexpr int FL_ROUND = FL_ROWS * 2 * LS_PAIRS;
static bool few_form(int type, int64_t rows, int k, int n) {
    const int rounds = n > 64 ? 1 : type == RIPPLE_TYPE_F32 ? 3 : k <= 256 ? 2 : 1;
    return rows <= rounds * FL_ROUND && n <= 32 * FL_WARPS && few_bytes(k, n) <= FL_BYTES;
}
// Whether one block forms dW too (1 row, 128 -> 40: 8.6 us for the gradient, 9.5 with a launch more; 256 -> 47: 13.4 and 11.7).
__host__ __device__ inline bool few_at_once(int rows, int k, int n) { return rows <= FL_ROWS && k * n <= 8192; }

template <int TYPE, bool GRAD>
static cudaError_t launch_few(const FewParams& p, void* stream) {
    auto* const kernel = k_loss_few<typename Elem<TYPE>::T, GRAD>;
    static bool ready[64];
    const cudaError_t e = allow_shared(kernel, FL_BYTES, ready);
    if (e != cudaSuccess) return e;
    return launch(kernel, dim3((unsigned)std::min((p.rows + FL_ROWS - 1) / FL_ROWS, sm_count())), FL_THREADS, (size_t)few_bytes(p.k, p.n), stream, p);
}

struct Slots {
    int64_t at = 0;
    int64_t take(int64_t bytes) {
        const int64_t here = at;
        at += aligned128(bytes);
        return here;
    }
};

struct Operand { int64_t at = -1, ld = 0, plane = 0; };      // at: in the workspace; -1: read where it is
// raw: read as it is in fp32, parts and all (x)
static Operand operand(Slots& s, int type, const void* p, int64_t ld, int64_t rows, int64_t cols, bool copy, bool raw) {
    Operand o;
    if (!copy && ((raw && type == RIPPLE_TYPE_F32) || readable(type, p, ld, cols))) return o;
    o.ld = up_to(cols, 8), o.plane = aligned128(rows * o.ld * 2) / 2;
    o.at = s.take(parts_of(type) * o.plane * 2);
    return o;
}

// Bytes of the tiles' sums that are in memory at once (one tile of columns of all rows at least).
constexpr int64_t LS_SUMS = 1ll << 27;

struct LossPlan {
    Operand x, w;
    int64_t sums, at_label, running, bytes;
    int piece, pieces;           // classes
};
static LossPlan plan_loss(const ripple_loss_rows_args& a) {
    LossPlan l = {};
    if (few_form(a.type, a.rows, a.k, a.n)) return l;
    Slots s;
    l.x = operand(s, a.type, a.x, a.ld_x, a.rows, a.k, false, true), l.w = operand(s, a.type, a.W, a.ld_w, a.k, a.n, false, false);
    const int cols = cols_of(a.type), tiles = (a.n + cols - 1) / cols;
    const int64_t of_tile = groups_of(a.type, a.k) * std::max<int64_t>(a.rows, 1) * 8, at_once = std::min<int64_t>(tiles, std::max<int64_t>(1, LS_SUMS / of_tile));
    l.piece = (int)at_once * cols, l.pieces = (tiles + (int)at_once - 1) / (int)at_once;
    l.sums = s.take(at_once * of_tile), l.at_label = s.take(a.rows * 4);
    if (l.pieces > 1) l.running = s.take(a.rows * 8);
    l.bytes = s.at;
    return l;
}

// 16-bit entries of g, of all its planes, that are in memory at once (whole tiles of columns of all rows, one tile at least): 512 MB.  Fewer cost loss-wide
// the rounds of dx in fp32 and tiles of dW too few for all SMs.
constexpr int64_t LS_PIECE = 1ll << 28;

// A product C [m, n] over k: how many parts k is split into where there are fewer tiles than pairs of SMs, so that as many as can be are busy; each part is
// at least eight chunks long, and their results are written in fp32 and added up.  (Also where there are more tiles, but the last round of
// them leaves pairs idle: 256 tiles of loss-wide's dx, 212 us a piece in one part, 258 in two.)
static int splits_of(int type, int64_t m, int64_t n, int64_t k) {
    const int64_t tiles = ((m + LS_ROWS - 1) / LS_ROWS) * ((n + cols_of(type) - 1) / cols_of(type)), chunks = (k + LS_KC - 1) / LS_KC;
    int best = 1;
    double least = 1e30;
    for (int s = 1; tiles < LS_PAIRS && s <= std::max<int64_t>(1, std::min<int64_t>(LS_PAIRS, chunks / 8)); ++s) {
        const int64_t each = (chunks + s - 1) / s;
        if ((chunks + each - 1) / each != s) continue;
        const double time = (double)((tiles * s + LS_PAIRS - 1) / LS_PAIRS) * each * (1 + s / 64.0);
        if (time < least) least = time, best = s;
    }
    return best;
}

struct GradPlanLoss {
    Operand x, x_clean, w;
    int piece, pieces;
    int64_t g, ld_g, g_plane, g_sums, control, dx, ld_dx, dw, ld_dw, bytes;     // dx, dw: -1: written where the caller wants them
    int dx_splits, dw_splits;
};
static GradPlanLoss plan_loss_grad(const ripple_loss_rows_grad_args& a) {
    GradPlanLoss l = {};
    Slots s;
    if (few_form(a.type, a.rows, a.k, a.n)) {
        if ((a.dW || a.dbias) && !few_at_once((int)a.rows, a.k, a.n)) s.take(a.rows * a.n * 4);        // g
        l.bytes = s.at;
        return l;
    }
    l.control = s.take(sizeof(RowControl));
    l.x = operand(s, a.type, a.x, a.ld_x, a.rows, a.k, false, true), l.w = operand(s, a.type, a.W, a.ld_w, a.k, a.n, false, false);
    if (a.dW && l.x.at < 0 && a.type != RIPPLE_TYPE_F32) l.x_clean = operand(s, a.type, a.x, a.ld_x, a.rows, a.k, true, false);
    const int cols = cols_of(a.type), parts = parts_of(a.type), all = up_to(a.n, 64);
    l.piece = (int)std::min<int64_t>(all, std::max<int64_t>(cols, LS_PIECE / parts / std::max<int64_t>(a.rows, 1) / cols * cols));
    l.pieces = (a.n + l.piece - 1) / l.piece;
    l.ld_g = l.piece, l.g_plane = aligned128(a.rows * l.ld_g * 2) / 2;
    if (a.dx || a.dW) l.g = s.take(parts * l.g_plane * 2);
    if (a.dbias) l.g_sums = s.take((a.rows + 31) / 32 * l.ld_g * 4);
    const int out_size = type_size(a.type);
    l.dx = l.dw = -1;
    if (a.dx) {
        l.dx_splits = splits_of(a.type, a.rows, a.k, l.piece);
        l.ld_dx = up_to(a.k, 8);
        if (l.pieces > 1 || l.dx_splits > 1 || !writable(out_size, a.dx, a.ld_dx)) l.dx = s.take(l.dx_splits * a.rows * l.ld_dx * 4);
    }
    if (a.dW) {
        l.dw_splits = splits_of(a.type, a.k, l.piece, a.rows);
        l.ld_dw = l.piece;
        if (l.dw_splits > 1 || !writable(out_size, a.dW, a.ld_dw) || (int64_t)l.piece * out_size % 32) l.dw = s.take(l.dw_splits * (int64_t)a.k * l.ld_dw * 4);
    }
    l.bytes = s.at;
    return l;
}

// ---- launches ----------------------------------------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) fn = nullptr;
        return reinterpret_cast<EncodeTiled>(fn);
    }();
    return f;
}

// A matrix of 16-bit planes in memory, rows `ld` apart.
struct Matrix {
    const void* p;
    int64_t rows, cols, ld, plane;
    int planes;
};
// Boxes of 64 columns x `box` rows.
static bool tensor_map(CUtensorMap* map, int type, const Matrix& x, int box) {
    const cuuint64_t dims[3] = {(cuuint64_t)x.cols, (cuuint64_t)x.rows, (cuuint64_t)x.planes};
    const cuuint64_t strides[2] = {(cuuint64_t)x.ld * 2, (cuuint64_t)(x.planes > 1 ? x.plane * 2 : x.ld * 2 * x.rows)};
    const cuuint32_t boxes[3] = {64, (cuuint32_t)box, 1}, steps[3] = {1, 1, 1};
    const EncodeTiled encode = encode_tiled();
    return encode && encode(map, type == RIPPLE_TYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(x.p), dims, strides, boxes, steps,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// a [.., k] (A_ACROSS: [k, ..]), b [.., k] (B_ACROSS: [k, ..])
template <int TYPE, bool A_ACROSS, bool B_ACROSS, int END, bool MANY, bool RAW>
static cudaError_t launch_product(ProductParams p, const Matrix& a, const Matrix* a_clean, const Matrix& b, void* stream) {
    using S = LossShape<TYPE, MANY, RAW>;
    auto* const kernel = k_product<TYPE, A_ACROSS, B_ACROSS, END, MANY, RAW>;
    static bool ready[64];
    cudaError_t e = allow_shared(kernel, (int)S::BYTES, ready);
    if (e != cudaSuccess) return e;
    if (!tensor_map(&p.b, TYPE, b, B_ACROSS ? 64 : S::COLS / 2)) return cudaErrorInvalidValue;
    if constexpr (RAW) {
        p.raw = static_cast<const float*>(a.p), p.ld_raw = a.ld, p.raw_rows = (int)a.rows, p.raw_cols = (int)a.cols;
    } else {
        if (!tensor_map(&p.a, TYPE, a, A_ACROSS ? 64 : 128) || !tensor_map(&p.a_clean, TYPE, a_clean ? *a_clean : a, A_ACROSS ? 64 : 128)) return cudaErrorInvalidValue;
    }
    p.row_tiles = (p.m + LS_ROWS - 1) / LS_ROWS, p.col_tiles = (p.n + S::COLS - 1) / S::COLS;
    const char* const withhold = std::getenv("RIPPLE_DEBUG_TC_WITHHOLD");
    p.withhold = withhold && withhold[0] == '1';
    const int64_t all = (int64_t)p.row_tiles * p.col_tiles * p.splits;
    return launch(kernel, dim3((unsigned)(2 * std::min<int64_t>(all, std::max(1, sm_count() / 2)))), S::THREADS, S::BYTES, stream, p);
}
// X: the product reads x as A, which in fp32 is taken as it is
template <int TYPE, bool A_ACROSS, bool B_ACROSS, int END, bool X>
static cudaError_t launch_product(ProductParams p, const Matrix& a, const Matrix* a_clean, const Matrix& b, int splits, void* stream) {
    const int chunks = (p.k + LS_KC - 1) / LS_KC;
    constexpr bool RAW = X && TYPE == RIPPLE_TYPE_F32;
    p.split_chunks = (chunks + splits - 1) / splits, p.splits = (chunks + p.split_chunks - 1) / p.split_chunks;      // (none empty)
    if (p.split_chunks > unit_of(TYPE, END)) return launch_product<TYPE, A_ACROSS, B_ACROSS, END, true, RAW>(p, a, a_clean, b, stream);
    return launch_product<TYPE, A_ACROSS, B_ACROSS, END, false, RAW>(p, a, a_clean, b, stream);
}

template <int TYPE>
static cudaError_t launch_operand(const void* from, int64_t ld_from, int64_t rows, int64_t cols, const Operand& o, uint8_t* work, const int32_t* labels, int classes,
                                  const RowControl* control, void* stream) {
    OperandParams p = {from, rows, ld_from, (int)cols, 1, reinterpret_cast<uint16_t*>(work + o.at), o.ld, o.plane, labels, classes, control};
    while (p.lanes < 256 && p.lanes * 8 < o.ld) p.lanes *= 2;
    const int64_t blocks = (rows * p.lanes + 255) / 256;
    return launch(k_operand<typename Elem<TYPE>::T>, dim3((unsigned)std::min<int64_t>(blocks, (int64_t)sm_count() * 16)), 256, 0, stream, p);
}

static Matrix matrix_of(const Operand& o, int type, const void* p, int64_t ld, int64_t rows, int64_t cols, const uint8_t* work) {
    if (o.at < 0) return {p, rows, cols, ld, 0, 1};
    return {work + o.at, rows, cols, o.ld, o.plane, parts_of(type)};
}

template <int TYPE>
static cudaError_t run_loss(const ripple_loss_rows_args& a) {
    if (few_form(a.type, a.rows, a.k, a.n)) {
        FewParams f = {};
        f.rows = (int)a.rows, f.k = a.k, f.n = a.n, f.x = a.x, f.W = a.W, f.ld_x = a.ld_x, f.ld_w = a.ld_w, f.bias = a.bias, f.labels = a.labels, f.loss = a.loss, f.lse = a.lse;
        return launch_few<TYPE, false>(f, a.cuda_stream);
    }
    const LossPlan l = plan_loss(a);
    uint8_t* const work = static_cast<uint8_t*>(a.workspace);
    cudaError_t e = cudaSuccess;
    if (l.x.at >= 0) e = launch_operand<TYPE>(a.x, a.ld_x, a.rows, a.k, l.x, work, nullptr, 0, nullptr, a.cuda_stream);
    if (e == cudaSuccess && l.w.at >= 0) e = launch_operand<TYPE>(a.W, a.ld_w, a.k, a.n, l.w, work, nullptr, 0, nullptr, a.cuda_stream);
    if (e != cudaSuccess) return e;
    const Matrix x = matrix_of(l.x, a.type, a.x, a.ld_x, a.rows, a.k, work), w = matrix_of(l.w, a.type, a.W, a.ld_w, a.k, a.n, work);
    ProductParams p = {};
    p.m = (int)a.rows, p.k = a.k, p.labels = a.labels, p.classes = a.n;
    p.sums = reinterpret_cast<float2*>(work + l.sums), p.at_label = reinterpret_cast<float*>(work + l.at_label);
    for (int piece = 0; piece < l.pieces && e == cudaSuccess; ++piece) {
        const int c0 = piece * l.piece;
        p.n = std::min(l.piece, a.n - c0), p.b_col0 = p.class0 = c0, p.bias = a.bias ? a.bias + c0 : nullptr;
        e = launch_product<TYPE, false, true, END_LSE, true>(p, x, nullptr, w, 1, a.cuda_stream);
        if (e != cudaSuccess) break;
        const int parts = groups_of(a.type, a.k) * ((p.n + cols_of(a.type) - 1) / cols_of(a.type));
        auto finish = [&](auto* kernel, int rows) {
            return launch(kernel, dim3((unsigned)((a.rows + rows - 1) / rows)), 512, 0, a.cuda_stream, (const float2*)p.sums, parts, a.rows, (const float*)p.at_label, a.labels, a.n, a.loss,
                          a.lse, l.pieces > 1 ? reinterpret_cast<float2*>(work + l.running) : nullptr, piece == 0 ? 1 : 0, piece == l.pieces - 1 ? 1 : 0);
        };
        e = parts <= 8 ? finish(k_finish_loss<1>, 512) : finish(k_finish_loss<16>, 32);
    }
    return e;
}

template <typename T>
static cudaError_t join_parts(const float* parts, int splits, int64_t stride, int64_t ld, void* out, int64_t ld_out, int64_t rows, int cols, void* stream) {
    if (splits >= 16 && cols <= 1024)
        return launch(k_join_many_parts<T>, dim3((unsigned)((cols + 31) / 32), (unsigned)std::min<int64_t>(rows, 16384)), 256, 0, stream, parts, splits, stride, ld, static_cast<T*>(out), ld_out, rows, cols);
    return launch(k_join_parts<T>, dim3((unsigned)((cols + 1023) / 1024), (unsigned)std::min<int64_t>(rows, 16384)), 256, 0, stream, parts, splits, stride, ld, static_cast<T*>(out), ld_out, rows, cols);
}

template <int TYPE>
static cudaError_t run_loss_grad(const ripple_loss_rows_grad_args& a) {
    using T = typename Elem<TYPE>::T;
    if (few_form(a.type, a.rows, a.k, a.n)) {
        FewParams f = {};
        f.rows = (int)a.rows, f.k = a.k, f.n = a.n, f.x = a.x, f.W = a.W, f.ld_x = a.ld_x, f.ld_w = a.ld_w, f.bias = a.bias, f.labels = a.labels;
        f.lse = const_cast<float*>(a.lse), f.dloss = a.dloss, f.scale = a.scale, f.dx = a.dx, f.ld_dx = a.ld_dx, f.dW = a.dW, f.ld_dw = a.ld_dw, f.dbias = a.dbias;
        if ((a.dW || a.dbias) && !few_at_once(f.rows, a.k, a.n)) f.g = static_cast<float*>(a.workspace);
        const cudaError_t e = launch_few<TYPE, true>(f, a.cuda_stream);
        if (e != cudaSuccess || !f.g) return e;
        return launch(k_loss_few_weights<T>, dim3((unsigned)(a.dW ? (a.k + FL_K - 1) / FL_K : 1), (unsigned)(a.n + 31) / 32), FL_THREADS, 0, a.cuda_stream, f);
    }
    const GradPlanLoss l = plan_loss_grad(a);
    uint8_t* const work = static_cast<uint8_t*>(a.workspace);
    void* const stream = a.cuda_stream;
    RowControl* const control = reinterpret_cast<RowControl*>(work + l.control);
    const bool look_in_x = l.x_clean.at >= 0;
    cudaError_t e = cudaSuccess;
    if (look_in_x || TYPE == RIPPLE_TYPE_F16)
        e = launch(k_look_at_rows<T>, dim3(LS_CONTROL), 256, 0, stream, look_in_x ? static_cast<const T*>(a.x) : nullptr, a.ld_x, a.k, a.labels, a.dloss, a.rows, a.n, control);
    if (e == cudaSuccess && l.x.at >= 0) e = launch_operand<TYPE>(a.x, a.ld_x, a.rows, a.k, l.x, work, a.labels, a.n, nullptr, stream);
    if (e == cudaSuccess && look_in_x) e = launch_operand<TYPE>(a.x, a.ld_x, a.rows, a.k, l.x_clean, work, a.labels, a.n, control, stream);
    if (e == cudaSuccess && l.w.at >= 0) e = launch_operand<TYPE>(a.W, a.ld_w, a.k, a.n, l.w, work, nullptr, 0, nullptr, stream);
    if (e != cudaSuccess) return e;
    const Matrix x = matrix_of(l.x, a.type, a.x, a.ld_x, a.rows, a.k, work), w = matrix_of(l.w, a.type, a.W, a.ld_w, a.k, a.n, work);
    const Matrix x_clean = look_in_x ? matrix_of(l.x_clean, a.type, a.x, a.ld_x, a.rows, a.k, work) : x;
    for (int c0 = 0; c0 < a.n; c0 += l.piece) {
        const int classes = std::min(l.piece, a.n - c0);
        ProductParams p = {};
        p.m = (int)a.rows, p.n = classes, p.k = a.k, p.b_col0 = c0;
        p.bias = a.bias ? a.bias + c0 : nullptr, p.labels = a.labels, p.class0 = c0, p.classes = a.n;
        p.lse = a.lse, p.dloss = a.dloss, p.scale = a.scale;
        p.ld_g = l.ld_g, p.g_plane = l.g_plane;
        if (a.dx || a.dW) p.g = reinterpret_cast<uint16_t*>(work + l.g);
        if (a.dbias) p.g_sums = reinterpret_cast<float*>(work + l.g_sums);
        p.control = TYPE == RIPPLE_TYPE_F16 ? control : nullptr, p.differ = TYPE == RIPPLE_TYPE_F16 && c0 == 0 ? &control->differ : nullptr;
        // (rows without labels are zeros in g whatever their logits: x as it is)
        const Matrix* const same = TYPE == RIPPLE_TYPE_F16 ? &x : nullptr;
        e = launch_product<TYPE, false, true, END_GRAD, true>(p, x, same, w, 1, stream);
        if (e != cudaSuccess) return e;
        if (a.dbias) {
            const int wide = classes > 8 * 2 * LS_PAIRS ? 32 : 8;
            auto* const join = wide == 32 ? k_join_columns<32> : k_join_columns<8>;
            e = launch(join, dim3((unsigned)((classes + wide - 1) / wide)), 1024, 0, stream, (const float*)p.g_sums, (a.rows + 31) / 32, l.ld_g, classes, a.dbias + c0);
            if (e != cudaSuccess) return e;
        }
        const Matrix g{work + l.g, a.rows, classes, l.ld_g, l.g_plane, parts_of(TYPE)};
        ProductParams o = {};
        o.unscale = TYPE == RIPPLE_TYPE_F16, o.scale = a.scale, o.classes = a.n;
        const bool by_row = TYPE == RIPPLE_TYPE_F16 && a.dx && a.dloss;        // dx behind dW then: its g may be another
        auto form_dx = [&]() {
            ProductParams d = o;
            d.m = (int)a.rows, d.n = a.k, d.k = classes, d.b_k0 = c0, d.control = p.control, d.dead_rows = a.labels, d.dloss = a.dloss, d.by_row = by_row;
            if (l.dx < 0) d.out = a.dx, d.ld_out = a.ld_dx, d.out_f32 = TYPE == RIPPLE_TYPE_F32;
            else d.out = work + l.dx, d.ld_out = l.ld_dx, d.split_stride = a.rows * l.ld_dx, d.out_f32 = 1, d.add_to_out = c0 > 0;
            // (the last piece may be too short for all parts: the last of them keep what they have)
            return launch_product<TYPE, false, false, END_OUT, false>(d, g, &g, w, l.dx_splits, stream);
        };
        if (a.dx && !by_row && (e = form_dx()) != cudaSuccess) return e;
        if (a.dW) {
            ProductParams d = o;
            d.m = a.k, d.n = classes, d.k = (int)a.rows, d.raw_labels = a.labels;
            d.control = look_in_x || TYPE == RIPPLE_TYPE_F16 ? control : nullptr;
            if (l.dw < 0) d.out = static_cast<T*>(a.dW) + c0, d.ld_out = a.ld_dw, d.out_f32 = TYPE == RIPPLE_TYPE_F32;
            else d.out = work + l.dw, d.ld_out = l.ld_dw, d.split_stride = a.k * l.ld_dw, d.out_f32 = 1;
            e = launch_product<TYPE, true, true, END_OUT, true>(d, x, &x_clean, g, l.dw_splits, stream);
            if (e == cudaSuccess && l.dw >= 0) e = join_parts<T>(static_cast<const float*>(d.out), l.dw_splits, d.split_stride, d.ld_out, static_cast<T*>(a.dW) + c0, a.ld_dw, a.k, classes, stream);
            if (e != cudaSuccess) return e;
        }
        if (by_row) {
            p.by_row = 1, p.g_sums = nullptr, p.differ = nullptr;
            e = launch_product<TYPE, false, true, END_GRAD, true>(p, x, same, w, 1, stream);
            if (e == cudaSuccess) e = form_dx();
            if (e != cudaSuccess) return e;
        }
    }
    if (a.dx && l.dx >= 0) e = join_parts<T>(reinterpret_cast<const float*>(work + l.dx), l.dx_splits, a.rows * l.ld_dx, l.ld_dx, a.dx, a.ld_dx, a.rows, a.k, stream);
    return e;
}

}  // namespace rp

using namespace rp;

#define REFUSE(...)                        \
    do {                                   \
        note_error(WHAT ": " __VA_ARGS__); \
        return RIPPLE_ERR_INVALID_ARG;     \
    } while (0)

template <typename A> static bool loss_sizes_ok(const A* a) {
    return a->rows >= 0 && a->rows <= INT32_MAX - LS_ROWS && type_ok(a->type) && a->k >= 1 && a->k <= RIPPLE_MAX_LOSS_K && a->n >= 1 && a->n <= RIPPLE_MAX_CLASSES;
}

extern "C" int64_t ripple_loss_rows_workspace_bytes(const ripple_loss_rows_args* a) { return a && loss_sizes_ok(a) ? plan_loss(*a).bytes : -1; }
extern "C" int64_t ripple_loss_rows_grad_workspace_bytes(const ripple_loss_rows_grad_args* a) { return a && loss_sizes_ok(a) ? plan_loss_grad(*a).bytes : -1; }

#define WHAT "loss_rows"
extern "C" ripple_status ripple_loss_rows(const ripple_loss_rows_args* a) {
    if (!a) REFUSE("null arguments");
    if (!loss_sizes_ok(a)) REFUSE("rows, type, k or n out of range");
    if (a->ld_x < 0 || a->ld_w < 0) REFUSE("negative leading dimension");
    if (a->rows > 0 && (!a->x || !a->W || !a->labels || !a->lse)) REFUSE("null x, W, labels or lse");
    const int ts = type_size(a->type);
    for (auto [ptr, size] : {std::pair<const void*, int>{a->x, ts}, {a->W, ts}, {a->bias, 4}, {a->labels, 4}, {a->loss, 4}, {a->lse, 4}})
        if (reinterpret_cast<uintptr_t>(ptr) % size) REFUSE("misaligned pointer");
    if (a->rows == 0) return RIPPLE_OK;
    const int64_t need = plan_loss(*a).bytes;
    if (a->workspace_bytes < need || (need > 0 && !a->workspace)) REFUSE("workspace too small");
    if (reinterpret_cast<uintptr_t>(a->workspace) & 127) REFUSE("misaligned workspace");
    const Extent x{a->x, a->rows, a->ld_x, a->k, ts}, W{a->W, a->k, a->ld_w, a->n, ts}, bias{a->bias, 1, 1, a->n, 4}, labels{a->labels, a->rows, 1, 1, 4},
        loss{a->loss, a->rows, 1, 1, 4}, lse{a->lse, a->rows, 1, 1, 4}, work{need > 0 ? a->workspace : nullptr, 1, 1, need, 1};
    for (const Extent* out : {&loss, &lse, &work})
        for (const Extent* in : {&x, &W, &bias, &labels})
            if (extents_meet(*out, *in)) REFUSE("an output or the workspace overlaps an input");
    if (extents_meet(loss, lse) || extents_meet(loss, work) || extents_meet(lse, work)) REFUSE("outputs or workspace overlap");
    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    const cudaError_t e = a->type == RIPPLE_TYPE_F32 ? run_loss<RIPPLE_TYPE_F32>(*a) : a->type == RIPPLE_TYPE_BF16 ? run_loss<RIPPLE_TYPE_BF16>(*a) : run_loss<RIPPLE_TYPE_F16>(*a);
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("loss_rows launch", e);
}
#undef WHAT

#define WHAT "loss_rows_grad"
extern "C" ripple_status ripple_loss_rows_grad(const ripple_loss_rows_grad_args* a) {
    if (!a) REFUSE("null arguments");
    if (!loss_sizes_ok(a)) REFUSE("rows, type, k or n out of range");
    if (!a->dx && !a->dW && !a->dbias) REFUSE("no output");
    if (a->ld_x < 0 || a->ld_w < 0 || (a->dx && a->ld_dx < a->k) || (a->dW && a->ld_dw < a->n)) REFUSE("leading dimension negative, or of an output below its width");
    if (a->rows > 0 && (!a->x || !a->W || !a->labels || !a->lse)) REFUSE("null x, W, labels or lse");
    const int ts = type_size(a->type);
    for (auto [ptr, size] : {std::pair<const void*, int>{a->x, ts}, {a->W, ts}, {a->bias, 4}, {a->labels, 4}, {a->lse, 4}, {a->dloss, 4}, {a->dx, ts}, {a->dW, ts}, {a->dbias, 4}})
        if (reinterpret_cast<uintptr_t>(ptr) % size) REFUSE("misaligned pointer");
    const int64_t need = a->rows > 0 ? plan_loss_grad(*a).bytes : 0;
    if (a->workspace_bytes < need || (need > 0 && !a->workspace)) REFUSE("workspace too small");
    if (reinterpret_cast<uintptr_t>(a->workspace) & 127) REFUSE("misaligned workspace");
    const Extent x{a->x, a->rows, a->ld_x, a->k, ts}, W{a->W, a->k, a->ld_w, a->n, ts}, bias{a->bias, 1, 1, a->n, 4}, labels{a->labels, a->rows, 1, 1, 4},
        lse{a->lse, a->rows, 1, 1, 4}, dloss{a->dloss, a->rows, 1, 1, 4}, dx{a->dx, a->rows, a->ld_dx, a->k, ts}, dW{a->dW, a->k, a->ld_dw, a->n, ts},
        db{a->dbias, 1, 1, a->n, 4}, work{need > 0 ? a->workspace : nullptr, 1, 1, need, 1};
    for (const Extent* out : {&dx, &dW, &db, &work})
        for (const Extent* in : {&x, &W, &bias, &labels, &lse, &dloss})
            if (extents_meet(*out, *in)) REFUSE("an output or the workspace overlaps an input");
    for (auto [p, q] : {std::pair<const Extent*, const Extent*>{&dx, &dW}, {&dx, &db}, {&dx, &work}, {&dW, &db}, {&dW, &work}, {&db, &work}})
        if (extents_meet(*p, *q)) REFUSE("outputs or workspace overlap");
    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    cudaError_t e = cudaSuccess;
    if (a->rows == 0) {          // sums of nothing
        cudaStream_t stream = static_cast<cudaStream_t>(a->cuda_stream);
        if (a->dW) e = cudaMemset2DAsync(a->dW, (size_t)a->ld_dw * ts, 0, (size_t)a->n * ts, (size_t)a->k, stream);
        if (e == cudaSuccess && a->dbias) e = cudaMemsetAsync(a->dbias, 0, (size_t)a->n * 4, stream);
    } else {
        e = a->type == RIPPLE_TYPE_F32 ? run_loss_grad<RIPPLE_TYPE_F32>(*a) : a->type == RIPPLE_TYPE_BF16 ? run_loss_grad<RIPPLE_TYPE_BF16>(*a) : run_loss_grad<RIPPLE_TYPE_F16>(*a);
    }
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("loss_rows_grad launch", e);
}
