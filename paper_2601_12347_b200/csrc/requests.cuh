// What the operators that answer requests share: rows in fp32 or 16 bits, argument checks, launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ripple.h"
#include "device_utils.cuh"

namespace rp {

void note_error(const char* fmt, ...);   // text for ripple_last_error(NULL)
cudaError_t take_loss_timeout(int* gave_up);   // whether a bounded wait of row_loss.cu gave up on the current device; cleared

inline int type_size(int t) { return t == RIPPLE_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int t) { return t >= RIPPLE_TYPE_F32 && t <= RIPPLE_TYPE_F16; }

template <int TYPE> struct Elem;
template <> struct Elem<RIPPLE_TYPE_F32> { using T = float; };
template <> struct Elem<RIPPLE_TYPE_BF16> { using T = __nv_bfloat16; };
template <> struct Elem<RIPPLE_TYPE_F16> { using T = __half; };

// V neighbouring elements as they lie in memory, and as fp32
template <typename T, int V>
struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Piece { T v[V]; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// A matrix of an argument list: where its elements lie.
struct Extent {
    const void* p;
    int64_t rows, ld;
    int64_t width;
    int size;
    uintptr_t at() const { return reinterpret_cast<uintptr_t>(p); }
    uintptr_t end() const { return rows > 0 ? at() + ((rows - 1) * ld + width) * (int64_t)size : at(); }
};

// Whether two matrices share memory.  Columns of one matrix side by side do not.
inline bool extents_meet(const Extent& a, const Extent& b) {
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.end() <= b.at() || b.end() <= a.at()) return false;
    const int64_t la = a.ld * a.size, lb = b.ld * b.size;
    if (la == lb && la > 0) {
        const int64_t off = ((int64_t)(b.at() - a.at()) % la + la) % la;
        if (off >= a.width * a.size && off + b.width * b.size <= la) return false;
    }
    return true;
}
inline bool extents_same(const Extent& a, const Extent& b) { return a.p == b.p && a.ld == b.ld && a.size == b.size && a.width == b.width; }

// Makes a device current for the length of a call.
struct OnDevice {
    int before = -1;
    cudaError_t err = cudaSuccess;
    explicit OnDevice(int device) {
        if (device < 0) return;
        int now = 0;
        err = cudaGetDevice(&now);
        if (err == cudaSuccess && now != device) {
            err = cudaSetDevice(device);
            if (err == cudaSuccess) before = now;
        }
    }
    ~OnDevice() { if (before >= 0) cudaSetDevice(before); }
};

// Programmatic stream serialisation: see pdl_enter
template <typename... P, typename... A>
inline cudaError_t launch(void (*kernel)(P...), dim3 grid, int block, size_t smem, void* stream, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// multiprocessors of the current device
inline int sm_count() {
    static int per_device[64];
    int d = 0, n = 0;
    if (cudaGetDevice(&d) != cudaSuccess) return 1;
    if (d < 64 && per_device[d]) return per_device[d];
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, d) != cudaSuccess || n < 1) n = 1;
    if (d < 64) per_device[d] = n;
    return n;
}

// Lets a kernel have `bytes` of dynamic shared memory; `ready`: the devices where it has been told so
template <typename K>
inline cudaError_t allow_shared(K kernel, int bytes, bool (&ready)[64]) {
    int d = 0;
    cudaError_t e = cudaGetDevice(&d);
    if (e != cudaSuccess || (d < 64 && ready[d])) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && d < 64) ready[d] = true;
    return e;
}

inline ripple_status launch_failed(const char* what, cudaError_t e) {
    note_error("%s failed: %s", what, cudaGetErrorString(e));
    return e == cudaErrorMemoryAllocation ? RIPPLE_ERR_OOM : RIPPLE_ERR_CUDA;
}

}  // namespace rp
