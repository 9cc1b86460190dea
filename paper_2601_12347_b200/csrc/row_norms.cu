// The norms after a block and before the next one, with gate, scale and residual sum between them:
//   s = residual[ids] + scale * act(gate) * post(y),   n = pre(s)
// One pass: a row's inputs are read once, stay in registers through both norms, and s and n are written once.
// Statistics are two passes over registers (mean, then squared distances from it), so rows with a large mean lose
// nothing; all arithmetic is fp32 and each output is rounded once.
#include "requests.cuh"

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
    int gate_act, gate_width;
    int warps_per_row;
};

__device__ __forceinline__ float gate_of(float g, int act) {
    if (act == RIPPLE_GATE_IDENTITY) return g;
    if (act == RIPPLE_GATE_TANH) return tanhf(g);
    const float s = 1.0f / (1.0f + expf(-g));
    return act == RIPPLE_GATE_SILU ? g * s : s;
}

// sum over the threads of a row
template <bool MULTI>
__device__ __forceinline__ float row_sum(float x, float* scratch, int warps) {
    x = warp_sum(x);
    if constexpr (MULTI) {
        __syncthreads();
        if (lane_id() == 0) scratch[threadIdx.x >> 5] = x;
        __syncthreads();
        x = 0.f;
        for (int w = 0; w < warps; ++w) x += scratch[w];
    }
    return x;
}

// V: neighbouring elements per access, NP: accesses per thread.  A row takes a warp, or (MULTI) the whole block.
template <typename T, typename TR, int V, int NP, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : 128) k_norm_rows(const __grid_constant__ NormParams p) {
    pdl_enter();
    __shared__ float scratch[MULTI ? 16 : 1];
    const int W = MULTI ? p.warps_per_row : 1, threads = 32 * W, t = MULTI ? threadIdx.x : lane_id();
    const int row = MULTI ? blockIdx.x : blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    int64_t from = row;
    if (p.ids) {
        from = p.ids[row];
        if (from < 0 || from >= p.residual_rows) return;
    }
    const int D = p.width;
    Piece<T, V> y[NP], g[NP];
    Piece<TR, V> r[NP];
    float g1 = 1.0f;
    const bool wide_gate = p.gate && p.gate_width != 1;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int c = (j * threads + t) * V;
        if (c >= D) continue;
        if (p.y) y[j] = *reinterpret_cast<const Piece<T, V>*>(static_cast<const T*>(p.y) + row * p.ld_y + c);
        if (p.residual) r[j] = *reinterpret_cast<const Piece<TR, V>*>(static_cast<const TR*>(p.residual) + from * p.ld_residual + c);
        if (wide_gate) g[j] = *reinterpret_cast<const Piece<T, V>*>(static_cast<const T*>(p.gate) + row * p.ld_gate + c);
    }
    if (p.gate && !wide_gate) g1 = gate_of(to_f32(static_cast<const T*>(p.gate)[row * p.ld_gate]), p.gate_act);
    float s[NP * V];
    const float inv_d = 1.0f / (float)D;
    // in place: s = norm(s)
    auto norm = [&](const ripple_norm& n) {
        if (n.kind == RIPPLE_NORM_NONE) return;
        float mean = 0.f;
        if (n.kind == RIPPLE_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < NP * V; ++e) sum += s[e];
            mean = row_sum<MULTI>(sum, scratch, W) * inv_d;
        }
        float sq = 0.f;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            if ((j * threads + t) * V >= D) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = s[j * V + e] - mean;
                sq += d * d;
            }
        }
        const float inv = 1.0f / sqrtf(row_sum<MULTI>(sq, scratch, W) * inv_d + n.eps);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int c = (j * threads + t) * V;
            if (c >= D) continue;
            Piece<float, V> w, b;
#pragma unroll
            for (int e = 0; e < V; ++e) w.v[e] = 1.0f, b.v[e] = 0.0f;
            if (n.weight) w = *reinterpret_cast<const Piece<float, V>*>(n.weight + c);
            if (n.bias) b = *reinterpret_cast<const Piece<float, V>*>(n.bias + c);
#pragma unroll
            for (int e = 0; e < V; ++e) s[j * V + e] = (s[j * V + e] - mean) * inv * w.v[e] + b.v[e];
        }
    };
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) s[j * V + e] = p.y && (j * threads + t) * V < D ? to_f32(y[j].v[e]) : 0.f;
    if (p.y) norm(p.post);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int c = (j * threads + t) * V;
        if (c >= D) continue;
        Piece<float, V> k;
#pragma unroll
        for (int e = 0; e < V; ++e) k.v[e] = p.scale;
        if (p.scale_vector) k = *reinterpret_cast<const Piece<float, V>*>(p.scale_vector + c);
        Piece<TR, V> out;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float& x = s[j * V + e];
            if (p.y) x = k.v[e] * ((wide_gate ? gate_of(to_f32(g[j].v[e]), p.gate_act) : g1) * x);
            if (p.residual) x += to_f32(r[j].v[e]);
            out.v[e] = from_f32<TR>(x);
        }
        if (p.stream) *reinterpret_cast<Piece<TR, V>*>(static_cast<TR*>(p.stream) + row * p.ld_stream + c) = out;
    }
    if (!p.normed) return;
    norm(p.pre);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int c = (j * threads + t) * V;
        if (c >= D) continue;
        Piece<T, V> out;
#pragma unroll
        for (int e = 0; e < V; ++e) out.v[e] = from_f32<T>(s[j * V + e]);
        *reinterpret_cast<Piece<T, V>*>(static_cast<T*>(p.normed) + row * p.ld_normed + c) = out;
    }
}

template <typename T, typename TR, int V>
static cudaError_t launch_norm(const NormParams& p0, void* stream) {
    NormParams p = p0;
    const int D = p.width;
    p.warps_per_row = 1;
    if (D <= 256) return launch(k_norm_rows<T, TR, V, 8 / V, false>, dim3((p.rows + 3) / 4), 128, 0, stream, p);
    if (D <= 1024) return launch(k_norm_rows<T, TR, V, 32 / V, false>, dim3((p.rows + 3) / 4), 128, 0, stream, p);
    const int per_thread = D <= 8192 ? 16 : 32;
    p.warps_per_row = (D + 32 * per_thread - 1) / (32 * per_thread);
    if (per_thread == 16) return launch(k_norm_rows<T, TR, V, 16 / V, true>, dim3(p.rows), 32 * p.warps_per_row, 0, stream, p);
    return launch(k_norm_rows<T, TR, V, 32 / V, true>, dim3(p.rows), 32 * p.warps_per_row, 0, stream, p);
}

template <typename T, typename TR>
static cudaError_t launch_norm(const NormParams& p, int v, void* stream) {
    constexpr int WIDE = 16 / sizeof(T);
    if (v >= WIDE) return launch_norm<T, TR, WIDE>(p, stream);
    if (v >= 2) return launch_norm<T, TR, 2>(p, stream);
    return launch_norm<T, TR, 1>(p, stream);
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
    cudaError_t e;
    const bool mixed = a->stream_type != a->type;
    switch (a->type) {
        case RIPPLE_TYPE_F32: e = launch_norm<float, float>(p, v, a->cuda_stream); break;
        case RIPPLE_TYPE_BF16: e = mixed ? launch_norm<__nv_bfloat16, float>(p, v, a->cuda_stream) : launch_norm<__nv_bfloat16, __nv_bfloat16>(p, v, a->cuda_stream); break;
        default: e = mixed ? launch_norm<__half, float>(p, v, a->cuda_stream) : launch_norm<__half, __half>(p, v, a->cuda_stream); break;
    }
    return e == cudaSuccess ? RIPPLE_OK : launch_failed("norm_rows launch", e);
}
