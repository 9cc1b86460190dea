// Pieces of rows in registers: what the kernels that go over rows element by element share.
#pragma once

#include "requests.cuh"

#include <type_traits>

namespace rp {

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
// x += a b
template <int V> __device__ __forceinline__ void add_product(Vec<V>& x, const Vec<V>& a, const Vec<V>& b) {
    if constexpr (V == 1) {
        x.x = fmaf(a.x, b.x, x.x);
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(x.p[i]) : "l"(a.p[i]), "l"(b.p[i]));
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
    } else if constexpr (BYTES == 8) {
        const uint2 u = *static_cast<const uint2*>(from);
        v.p[0] = widen2<T>(u.x), v.p[1] = widen2<T>(u.y);
    } else {
        static_assert(BYTES == 16, "1, 2, 4 or 8 elements");
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
    } else if constexpr (BYTES == 8) {
        *static_cast<uint2*>(to) = make_uint2(narrow2<T>(v.p[0]), narrow2<T>(v.p[1]));
    } else {
        static_assert(BYTES == 16, "1, 2, 4 or 8 elements");
        *static_cast<uint4*>(to) = make_uint4(narrow2<T>(v.p[0]), narrow2<T>(v.p[1]), narrow2<T>(v.p[2]), narrow2<T>(v.p[3]));
    }
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

}  // namespace rp
