// Keys of logits and the key ranges that the draw's threshold search goes through (sample.cu).  Plain arithmetic that
// compiles for the host as well, so that a test can walk through the rounds of a search and see every bin's index.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <cstdint>
#include <cstring>
#include <type_traits>

namespace gala {

// Key of a logit: unsigned order = order of the values, in as many bits as the type has.
template <typename T> using Bits = typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type;
template <typename T> constexpr int kKeyBits = 8 * (int)sizeof(T);
template <typename T> constexpr uint32_t kSign = 1u << (kKeyBits<T> - 1);
template <typename T> constexpr uint32_t kInfinite = std::is_same<T, float>::value ? 0x7f800000u : std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
template <typename T>
__host__ __device__ __forceinline__ uint32_t key_of(uint32_t u) {       // from the stored bits
    constexpr uint32_t sign = kSign<T>, rest = sign - 1u;
    if ((u & rest) > kInfinite<T>) u = sign | kInfinite<T>;    // NaN counts as -inf
    if (u == sign) u = 0;                                      // -0 and +0 tie
    return u & sign ? ~u & (sign | rest) : u | sign;
}
template <typename T>
__host__ __device__ __forceinline__ float value_of(uint32_t u) {        // of the stored bits; NaN stays NaN
    if (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)u));
    if (std::is_same<T, __nv_bfloat16>::value) u <<= 16;
    float f;
    memcpy(&f, &u, 4);
    return f;
}
template <typename T>
__host__ __device__ __forceinline__ float logit_of(uint32_t key) {
    constexpr uint32_t sign = kSign<T>, rest = sign - 1u;
    return value_of<T>(key & sign ? key & rest : ~key & (sign | rest));
}
template <typename T> __host__ __device__ __forceinline__ uint32_t key_bottom() { return key_of<T>(kSign<T> | kInfinite<T>); }   // of -inf: keys above it can be drawn

constexpr int kBins = 2048;               // of a histogram round
constexpr float kFirstBins = 128.0f;      // bins of one unit of (m - l) / T in the first round

// The keys among which a threshold lies, in bins of 2^shift() keys from the largest down.  Entries are looked up by value:
// from() <= l <= to().
template <typename T>
struct KeyRange {
    uint32_t lo, hi;
    __host__ __device__ __forceinline__ float from() const { return logit_of<T>(lo); }
    __host__ __device__ __forceinline__ float to() const { return logit_of<T>(hi); }
    __host__ __device__ __forceinline__ int shift() const {       // 2048 bins or fewer
        int s = 0;
#ifdef __CUDA_ARCH__
        s = 21 - __clz((int)(hi - lo));
#else
        s = hi == lo ? 0 : 21 - __builtin_clz(hi - lo);
#endif
        return s > 0 ? s : 0;
    }
    __host__ __device__ __forceinline__ uint32_t bin(uint32_t bits, int shift) const { return (hi - key_of<T>(bits)) >> shift; }
    // To the keys of one bin.  The largest of them may be that of -0, the value 0 to a comparison: entries equal to +0, whose
    // key is the next one and outside the range, would pass l <= to() and have a bin far outside the histogram.  No entry has
    // that key, so the range ends below it.  (As the smallest key it does no harm: +0 is then inside.)
    __host__ __device__ __forceinline__ void narrow(int bin, int shift) {
        hi -= (uint32_t)bin << shift;
        const uint32_t span = (1u << shift) - 1u;
        if (hi - lo > span) lo = hi - span;
        if (hi == kSign<T> - 1u && hi > lo) hi--;
    }
};

}  // namespace gala
