// Shared by the stand-alone operators of sequence policies: element types, vector access, argument checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "internal.h"

namespace gala {

// Message for the caller's errbuf; returns the status so that a refusal is one statement.
__attribute__((format(printf, 4, 5))) inline int refuse(int status, char* buf, int len, const char* fmt, ...) {
    if (buf && len > 0) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(buf, (size_t)len, fmt, ap);
        va_end(ap);
    }
    return status;
}
inline int launched(cudaError_t e, char* buf, int len, const char* what) {
    return e == cudaSuccess ? GALA_OK : refuse(GALA_ECUDA, buf, len, "%s: %s", what, cudaGetErrorString(e));
}
inline bool dtype_ok(int t) { return t == GALA_F32 || t == GALA_BF16 || t == GALA_F16; }
inline int dtype_size(int t) { return t == GALA_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

#ifdef __CUDACC__
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// V neighbouring elements held as they lie in memory (in 32-bit registers, so that a value that waits costs half a
// register): 16 bytes, or a single element.
template <typename T, int V> struct Vec {
    uint4 w;
    __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
    __device__ __forceinline__ float get(int j) const {
        if (sizeof(T) == 4) return __uint_as_float(word(j));
        const uint32_t u = word(j >> 1);
        if (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(j & 1 ? u & 0xffff0000u : u << 16);
        const __half2 h = *reinterpret_cast<const __half2*>(&u);
        return j & 1 ? __high2float(h) : __low2float(h);
    }
    static __device__ __forceinline__ uint32_t pair(float a, float b) {
        if (std::is_same<T, __nv_bfloat16>::value) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
            return *reinterpret_cast<const uint32_t*>(&h);
        }
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    __device__ __forceinline__ void put(const float (&f)[V]) {
        if (sizeof(T) == 4)
            w = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        else
            w = make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4 % V], f[5 % V]), pair(f[6 % V], f[7 % V]));
    }
};
template <typename T> struct Vec<T, 1> {
    T w;
    __device__ __forceinline__ float get(int) const { return to_f32<T>(w); }
    __device__ __forceinline__ void put(const float (&f)[1]) { w = from_f32<T>(f[0]); }
};
#endif

}  // namespace gala
