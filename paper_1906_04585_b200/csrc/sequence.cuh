// Shared by the stand-alone operators of sequence policies: element types, vector access, argument checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdarg>
#include <cstdio>

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

// V neighbouring elements as one register-sized object
template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };
#endif

}  // namespace gala
