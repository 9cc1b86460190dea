// A projection with the low-rank adapters of many requests beside it:
//   y_i = act(x_i W + bias + scale_a (x_i A_a) B_a),  a = slots_i
#include "requests.cuh"

#include <algorithm>

namespace rp {

// ---- what a layout and a bank hold ---------------------------------------------------------------------------------
// Layout of W: its transpose (output columns are rows, K runs along a row), cut into groups of PJ_COLS columns and chunks
// of PJ_KC entries of K.  A chunk is PJ_COLS rows of 128 bytes in the swizzle that the tensor core reads, zeros beyond K and n;
// fp32 weights are three chunks, one per bf16 part.
constexpr int PJ_COLS = 128, PJ_KC = 64;
constexpr int PJ_CHUNK = PJ_COLS * 128;
// Bank: scale and rank of every slot, then A transposed (rank x K, zeros beyond both), then B transposed (n x rank).
struct SlotInfo { float scale; int32_t rank; };

__host__ __device__ inline int pj_parts(int type) { return type == RIPPLE_TYPE_F32 ? 3 : 1; }
__host__ __device__ inline int pj_up(int x, int to) { return (x + to - 1) / to * to; }
__host__ __device__ inline int64_t up128(int64_t x) { return (x + 127) / 128 * 128; }

struct BankView {
    const SlotInfo* info;
    const uint8_t* a;   // A transposed: slot x r_pad x k_pad
    const uint8_t* b;   // B transposed: slot x n x r_pad
    int r_pad, k_pad;
};
__host__ __device__ inline int64_t bank_a_at(int slots) { return up128((int64_t)slots * (int64_t)sizeof(SlotInfo) + 128); }
__host__ __device__ inline int64_t bank_b_at(int size, int k, int slots, int max_rank) {
    return bank_a_at(slots) + up128((int64_t)slots * pj_up(max_rank, 16) * pj_up(k, PJ_KC) * size);
}
__host__ __device__ inline BankView bank_view(const void* bank, int size, int k, int slots, int max_rank) {
    const uint8_t* p = static_cast<const uint8_t*>(bank);
    return {reinterpret_cast<const SlotInfo*>(p), p + bank_a_at(slots), p + bank_b_at(size, k, slots, max_rank), pj_up(max_rank, 16), pj_up(k, PJ_KC)};
}

// byte offset of 16-byte piece c (0..7) of row r inside a K-major tile with 128-byte rows, swizzled
__host__ __device__ __forceinline__ uint32_t pj_swz(int r, int c) {
    return (uint32_t)((r >> 3) * 1024 + (r & 7) * 128 + (((c ^ r) & 7) << 4));
}

// An fp32 value as three bf16 parts, 8 bits each: the first cut (rounded, values next to the largest would become
// infinite), the others what is left, rounded; both remainders are exact.  An infinite value has no remainders.
__device__ __forceinline__ void pj_parts_of(float x, __nv_bfloat16 (&h)[3]) {
    h[0] = __float2bfloat16_rz(x);
    float left = isfinite(x) ? x - __bfloat162float(h[0]) : 0.f;
    h[1] = __float2bfloat16_rn(left);
    h[2] = __float2bfloat16_rn(left - __bfloat162float(h[1]));
}

// one thread per 16-byte piece of a 16-bit chunk: eight entries of K of one output column
template <typename T>
__global__ void k_layout_weights(const T* W, int64_t ld, int k, int n, uint8_t* out, int chunks, int groups) {
    pdl_enter();
    const int parts = sizeof(T) == 4 ? 3 : 1;
    const int64_t pieces = (int64_t)groups * chunks * PJ_COLS * 8;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * blockDim.x) {
        const int col = (int)(i % PJ_COLS), c = (int)(i / PJ_COLS % 8);
        const int64_t chunk = i / (PJ_COLS * 8);
        const int kc = (int)(chunk % chunks), group = (int)(chunk / chunks), j = group * PJ_COLS + col;
        uint8_t* to = out + chunk * parts * PJ_CHUNK + pj_swz(col, c);
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
template <typename T>
__global__ void k_set_adapters(uint8_t* a_out, uint8_t* b_out, const T* A, const T* B, int first, int count, int rank, int k, int n,
                               int r_pad, int k_pad, int* bad) {
    pdl_enter();
    T* const at = reinterpret_cast<T*>(a_out);
    T* const bt = reinterpret_cast<T*>(b_out);
    const int64_t per_a = (int64_t)r_pad * k_pad, per_b = (int64_t)n * r_pad, total = (per_a + per_b) * count;
    bool fine = true;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t s = i / (per_a + per_b);
        int64_t e = i % (per_a + per_b);
        T v = from_f32<T>(0.f);
        if (e < per_a) {
            const int r = (int)(e / k_pad), kk = (int)(e % k_pad);
            if (r < rank && kk < k) v = A[(s * k + kk) * rank + r];
            at[(first + s) * per_a + e] = v;
        } else {
            e -= per_a;
            const int j = (int)(e / r_pad), r = (int)(e % r_pad);
            if (r < rank) v = B[(s * rank + r) * n + j];
            bt[(first + s) * per_b + e] = v;
        }
        fine = fine && isfinite(to_f32(v));
    }
    if (!fine) *bad = 1;
}


// ---- the product ---------------------------------------------------------------------------------------------------
struct ProjectParams {
    int rows, k, n, act, chunks;
    const void* x;
    int64_t ld_x, x_rows;
    const int32_t* ids;
    const uint8_t* layout;
    const float* bias;
    BankView bank;         // info null: no adapters
    int n_slots;
    const int32_t* slots;
    float* t;              // rows x bank.r_pad: scale_a x_i A_a
    void* y;
    int64_t ld_y;
    int out_f32;
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

// t_i = scale_a x_i A_a: a warp per row and rank
template <typename T>
__global__ void k_shrink_rows(const __grid_constant__ ProjectParams p) {
    pdl_enter();
    const int i = blockIdx.x, lane = lane_id();
    const int64_t from = row_of(p, i);
    const int a = slot_of(p, i);
    if (from < 0 || a < 0) return;
    const T* const x = static_cast<const T*>(p.x) + from * p.ld_x;
    const SlotInfo info = p.bank.info[a];
    for (int r = threadIdx.x >> 5; r < p.bank.r_pad; r += blockDim.x >> 5) {
        float sum = 0.f;
        if (r < info.rank) {
            const T* const w = reinterpret_cast<const T*>(p.bank.a) + ((int64_t)a * p.bank.r_pad + r) * p.bank.k_pad;
            for (int kk = lane; kk < p.k; kk += 32) sum += to_f32(x[kk]) * to_f32(w[kk]);
            sum = warp_sum(sum) * info.scale;
        }
        if (lane == 0) p.t[(int64_t)i * p.bank.r_pad + r] = sum;
    }
}

// the simplest form: a thread per output
template <typename T>
__global__ void k_project_simple(const __grid_constant__ ProjectParams p) {
    pdl_enter();
    const int j = blockIdx.y * 32 + (threadIdx.x & 31), i = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (j >= p.n || i >= p.rows) return;
    const int64_t from = row_of(p, i);
    if (from < 0) return;
    const T* const x = static_cast<const T*>(p.x) + from * p.ld_x;
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    float sum = 0.f;
    for (int kk = 0; kk < p.k; ++kk) {
        const uint8_t* at = p.layout + ((int64_t)(j / PJ_COLS) * p.chunks + kk / PJ_KC) * PARTS * PJ_CHUNK + pj_swz(j % PJ_COLS, kk % PJ_KC / 8) + 2 * (kk % 8);
        float w;
        if constexpr (PARTS == 3) {
            w = 0.f;
            for (int q = 2; q >= 0; --q) w += to_f32(*reinterpret_cast<const __nv_bfloat16*>(at + q * PJ_CHUNK));
        } else {
            w = to_f32(*reinterpret_cast<const T*>(at));
        }
        sum += to_f32(x[kk]) * w;
    }
    if (p.bias) sum += p.bias[j];
    const int a = p.bank.info ? slot_of(p, i) : -1;
    if (a >= 0) {
        const T* const b = reinterpret_cast<const T*>(p.bank.b) + ((int64_t)a * p.n + j) * p.bank.r_pad;
        float d = 0.f;
        for (int r = 0; r < p.bank.info[a].rank; ++r) d += p.t[(int64_t)i * p.bank.r_pad + r] * to_f32(b[r]);
        sum += d;
    }
    if (p.act == RIPPLE_ACT_RELU && sum < 0.f) sum = 0.f;
    if (p.out_f32) static_cast<float*>(p.y)[(int64_t)i * p.ld_y + j] = sum;
    else static_cast<T*>(p.y)[(int64_t)i * p.ld_y + j] = from_f32<T>(sum);
}

template <typename T>
static cudaError_t project(const ProjectParams& p, void* stream) {
    if (p.bank.info) {
        const cudaError_t e = launch(k_shrink_rows<T>, dim3(p.rows), 128, 0, stream, p);
        if (e != cudaSuccess) return e;
    }
    return launch(k_project_simple<T>, dim3((p.rows + 7) / 8, (p.n + 31) / 32), 256, 0, stream, p);
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
    return (int64_t)(pj_up(n, PJ_COLS) / PJ_COLS) * (pj_up(k, PJ_KC) / PJ_KC) * pj_parts(type) * PJ_CHUNK;
}

extern "C" int64_t ripple_adapter_bytes(int32_t type, int32_t k, int32_t n, int32_t slots, int32_t max_rank) {
    if (!shape_ok(type, k, n) || !bank_ok(slots, max_rank)) return -1;
    const int size = type_size(type);
    return bank_b_at(size, k, slots, max_rank) + up128((int64_t)slots * n * pj_up(max_rank, 16) * size);
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
    cudaError_t e;
    if (type == RIPPLE_TYPE_F32) e = launch(k_layout_weights<float>, grid, 256, 0, cuda_stream, (const float*)W, ld_w, k, n, (uint8_t*)layout, chunks, groups);
    else if (type == RIPPLE_TYPE_BF16) e = launch(k_layout_weights<__nv_bfloat16>, grid, 256, 0, cuda_stream, (const __nv_bfloat16*)W, ld_w, k, n, (uint8_t*)layout, chunks, groups);
    else e = launch(k_layout_weights<__half>, grid, 256, 0, cuda_stream, (const __half*)W, ld_w, k, n, (uint8_t*)layout, chunks, groups);
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
    if (rank > 0)
        for (int i = 0; i < count; ++i)
            if (!(scale[i] - scale[i] == 0.f)) REFUSE("adapter_set: a scale is not finite");
    OnDevice on(device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const BankView v = bank_view(bank, size, k, slots, max_rank);
    SlotInfo* info = const_cast<SlotInfo*>(v.info);
    // (the 128 bytes behind the slots' table: the flag)
    int* bad = reinterpret_cast<int*>(static_cast<uint8_t*>(bank) + bank_a_at(slots) - 128);
    int host_bad = 0;
    SlotInfo host_info[256];
    cudaError_t e = cudaMemsetAsync(bad, 0, sizeof(int), st);
    if (e == cudaSuccess && rank > 0) {
        const dim3 grid(592);
        uint8_t *a = const_cast<uint8_t*>(v.a), *b = const_cast<uint8_t*>(v.b);
        if (type == RIPPLE_TYPE_F32) e = launch(k_set_adapters<float>, grid, 256, 0, cuda_stream, a, b, (const float*)A, (const float*)B, first, count, rank, k, n, v.r_pad, v.k_pad, bad);
        else if (type == RIPPLE_TYPE_BF16) e = launch(k_set_adapters<__nv_bfloat16>, grid, 256, 0, cuda_stream, a, b, (const __nv_bfloat16*)A, (const __nv_bfloat16*)B, first, count, rank, k, n, v.r_pad, v.k_pad, bad);
        else e = launch(k_set_adapters<__half>, grid, 256, 0, cuda_stream, a, b, (const __half*)A, (const __half*)B, first, count, rank, k, n, v.r_pad, v.k_pad, bad);
        if (e == cudaSuccess) e = cudaMemcpyAsync(&host_bad, bad, sizeof(int), cudaMemcpyDeviceToHost, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    for (int at = 0; at < count && e == cudaSuccess; at += 256) {
        const int m = std::min(256, count - at);
        for (int i = 0; i < m; ++i) host_info[i] = rank > 0 && !host_bad ? SlotInfo{scale[at + i], rank} : SlotInfo{0.f, 0};
        e = cudaMemcpyAsync(info + first + at, host_info, m * sizeof(SlotInfo), cudaMemcpyHostToDevice, st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return launch_failed("adapter_set", e);
    if (host_bad) REFUSE("adapter_set: an entry is not finite");
    return RIPPLE_OK;
}

extern "C" int64_t ripple_project_workspace_bytes(const ripple_project_rows_args* a) {
    if (!a || a->rows < 0 || !shape_ok(a->type, a->k, a->n)) return -1;
    if (!a->bank) return 0;
    if (!bank_ok(a->n_slots, a->max_rank)) return -1;
    return up128(a->rows * pj_up(a->max_rank, 16) * 4);
}

extern "C" ripple_status ripple_project_rows(const ripple_project_rows_args* a) {
    if (!a) REFUSE("project_rows: null arguments");
    if (a->rows < 0 || a->rows > INT32_MAX) REFUSE("project_rows: rows out of range");
    if (!shape_ok(a->type, a->k, a->n)) REFUSE("project_rows: type, k or n out of range");
    if (a->out_type != a->type && a->out_type != RIPPLE_TYPE_F32) REFUSE("project_rows: an output type that is neither the type nor fp32");
    if (a->act != RIPPLE_ACT_IDENTITY && a->act != RIPPLE_ACT_RELU) REFUSE("project_rows: unknown activation");
    const int size = type_size(a->type), out_size = type_size(a->out_type);
    if (a->rows == 0) return RIPPLE_OK;
    if (!a->x || !a->layout || !a->y) REFUSE("project_rows: null pointer");
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

    OnDevice on(a->device);
    if (on.err != cudaSuccess) return launch_failed("cudaSetDevice", on.err);
    ProjectParams p = {};
    p.rows = (int)a->rows, p.k = a->k, p.n = a->n, p.act = a->act, p.chunks = pj_up(a->k, PJ_KC) / PJ_KC;
    p.x = a->x, p.ld_x = a->ld_x, p.x_rows = a->x_rows, p.ids = a->ids;
    p.layout = static_cast<const uint8_t*>(a->layout), p.bias = a->bias;
    if (a->bank) p.bank = bank_view(a->bank, size, a->k, a->n_slots, a->max_rank);
    p.n_slots = a->n_slots, p.slots = a->slots, p.t = static_cast<float*>(a->workspace);
    p.y = a->y, p.ld_y = a->ld_y, p.out_f32 = a->out_type == RIPPLE_TYPE_F32;
    cudaError_t e;
    if (a->type == RIPPLE_TYPE_F32) e = project<float>(p, a->cuda_stream);
    else if (a->type == RIPPLE_TYPE_BF16) e = project<__nv_bfloat16>(p, a->cuda_stream);
    else e = project<__half>(p, a->cuda_stream);
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("project_rows launch", e);
}
