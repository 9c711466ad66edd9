// Logits before a draw: penalties of the tokens in a row's history, biases of listed tokens, a bit mask, for sm_100a.
//
// A block has a segment of a row.  Which entries of it the history or the bias list touches is a bit map in shared memory; a
// word an entry holds the count of the entry (low 20 bits) and the place of its first bias in the list (high 12 bits, counted
// from the end, so that a maximum finds the first).  Only words of touched entries are ever cleared or read, so a segment costs
// what its share of the lists costs, and entries that nothing touches stream through: two bytes (or four) in, out, and a bit.
// Counts are whole numbers and duplicates of a bias are added by the thread of the first in the order of the list, so the
// result does not depend on the order in which threads run.
#include "sequence.cuh"

namespace gala {
namespace {

constexpr int kSegment = 16384;
constexpr int kMaxBiases = 4095;
constexpr int kMaxWidth = 1 << 20;

struct Adjust {
    long long rows;
    int vocab, width, biases, segment, segments;
    const void* x;
    long long x_ld;
    void* y;
    long long y_ld;
    const int* history;
    long long history_ld;
    const int* lengths;
    const float *repetition, *frequency, *presence;
    const int* bias_ids;
    long long bias_ids_ld;
    const float* bias_values;
    long long bias_values_ld;
    const int* mask;
    long long mask_ld;
};

template <typename T, int V, bool TABLE>
__global__ void adjust_kernel(const Adjust a) {
    extern __shared__ uint32_t table[];                  // [segment]
    __shared__ uint32_t touched[TABLE ? kSegment / 32 : 1];
    float* bias = reinterpret_cast<float*>(table + (TABLE ? a.segment : 0));     // [biases], at the place of the first of its id
    const long long row = blockIdx.x / a.segments;
    const int first = (int)(blockIdx.x - row * a.segments) * a.segment, size = min(a.segment, a.vocab - first);
    pdl_wait();
    pdl_launch();
    const int* history = nullptr;
    const int* ids = nullptr;
    int length = 0;
    if (TABLE) {
        if (a.history) {
            history = a.history + row * a.history_ld;
            length = a.lengths ? min(max(a.lengths[row], 0), a.width) : a.width;
        }
        if (a.biases > 0) ids = a.bias_ids + row * a.bias_ids_ld;
        for (int i = threadIdx.x; i < (size + 31) / 32; i += blockDim.x) touched[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < length; i += blockDim.x) {
            const uint32_t e = (uint32_t)history[i] - (uint32_t)first;
            if (e < (uint32_t)size) {
                table[e] = 0;
                atomicOr(&touched[e >> 5], 1u << (e & 31));
            }
        }
        for (int i = threadIdx.x; ids && i < a.biases; i += blockDim.x) {
            const uint32_t e = (uint32_t)ids[i] - (uint32_t)first;
            if (e < (uint32_t)size) {
                table[e] = 0;
                atomicOr(&touched[e >> 5], 1u << (e & 31));
            }
        }
        __syncthreads();
        if (ids) {
            for (int i = threadIdx.x; i < a.biases; i += blockDim.x) {
                const uint32_t e = (uint32_t)ids[i] - (uint32_t)first;
                if (e < (uint32_t)size) atomicMax(&table[e], (uint32_t)(kMaxBiases - i) << 20);
            }
            __syncthreads();
            for (int i = threadIdx.x; i < a.biases; i += blockDim.x) {
                const int id = ids[i];
                const uint32_t e = (uint32_t)id - (uint32_t)first;
                if (e < (uint32_t)size && (int)(table[e] >> 20) == kMaxBiases - i) {
                    const float* values = a.bias_values + row * a.bias_values_ld;
                    float s = values[i];
                    for (int j = i + 1; j < a.biases; j++)
                        if (ids[j] == id) s += values[j];
                    bias[i] = s;
                }
            }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < length; i += blockDim.x) {
            const uint32_t e = (uint32_t)history[i] - (uint32_t)first;
            if (e < (uint32_t)size) atomicAdd(&table[e], 1u);
        }
        __syncthreads();
    }
    float rep = 1.0f, freq = 0.0f, pres = 0.0f;
    if (TABLE && a.history) {
        if (a.repetition) rep = a.repetition[row];
        if (a.frequency) freq = a.frequency[row];
        if (a.presence) pres = a.presence[row];
    }
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld + first;
    T* y = static_cast<T*>(a.y) + row * a.y_ld + first;
    const uint32_t* mask = a.mask ? reinterpret_cast<const uint32_t*>(a.mask) + row * a.mask_ld : nullptr;
    for (int e = threadIdx.x * V; e < size; e += blockDim.x * V) {
        Vec<T, V> v;
        v.w = *reinterpret_cast<const decltype(v.w)*>(x + e);
        constexpr uint32_t kAll = (1u << V) - 1;
        const uint32_t hit = TABLE ? touched[e >> 5] >> (e & 31) & kAll : 0u;
        const uint32_t open = mask ? mask[(first + e) >> 5] >> ((first + e) & 31) & kAll : kAll;
        if (hit || open != kAll) {
            float f[V];
#pragma unroll
            for (int j = 0; j < V; j++) {
                float l = v.get(j);
                if (hit >> j & 1u) {
                    const uint32_t w = table[e + j], count = w & 0xfffffu, place = w >> 20;
                    if (count) {
                        l = l > 0.0f ? l / rep : l * rep;
                        l = l - freq * (float)count - pres;
                    }
                    if (place) l += bias[kMaxBiases - place];
                }
                f[j] = open >> j & 1u ? l : -INFINITY;
            }
            v.put(f);
        }
        *reinterpret_cast<decltype(v.w)*>(y + e) = v.w;
    }
}

template <typename T, int V> cudaError_t launch_adjust(Adjust a, cudaStream_t st) {
    const bool table = a.history || a.biases > 0;
    // Segments are whole words of the mask and whole vectors.  Without lists a segment is four vectors a thread.
    a.segment = table ? kSegment : 256 * V * 4;
    if (a.segment > a.vocab) a.segment = (a.vocab + 31) / 32 * 32;
    a.segments = (a.vocab + a.segment - 1) / a.segment;
    int threads = (a.segment / V + 31) / 32 * 32;
    if (table && threads < 128 && a.width + a.biases > 64) threads = 128;
    if (threads > 256) threads = 256;
    const long long blocks = a.rows * a.segments;
    if (blocks >= 1ll << 31) return cudaErrorInvalidConfiguration;
    if (!table) return launch_pdl(adjust_kernel<T, V, false>, dim3((unsigned)blocks), dim3(threads), 0, st, a);
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(adjust_kernel<T, V, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (kSegment + kMaxBiases) * 4);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    return launch_pdl(adjust_kernel<T, V, true>, dim3((unsigned)blocks), dim3(threads), (size_t)(a.segment + a.biases) * 4, st, a);
}
template <typename T> cudaError_t adjust(const Adjust& a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    const bool wide = aligned(a.x, 16) && aligned(a.y, 16) && a.vocab % V == 0 && (a.rows <= 1 || (a.x_ld % V == 0 && a.y_ld % V == 0));
    return wide ? launch_adjust<T, V>(a, st) : launch_adjust<T, 1>(a, st);
}

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

extern "C" int gala_adjust_logits(const gala_adjust_logits_args* q, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!q) SAY("gala_adjust_logits: null arguments");
    const gala_adjust_logits_args& a = *q;
    if (!dtype_ok(a.dtype)) SAY("gala_adjust_logits: dtype %d", a.dtype);
    if (a.rows < 0 || a.rows >= (1ll << 27) || a.vocab < 1 || a.vocab > (1 << 30)) SAY("gala_adjust_logits: %lld rows of %d entries", a.rows, a.vocab);
    if (a.width < 0 || a.width >= kMaxWidth || a.biases < 0 || a.biases > kMaxBiases)
        SAY("gala_adjust_logits: histories of %d tokens, %d biases (below 2^20 and 4096)", a.width, a.biases);
    if (a.rows == 0) return GALA_OK;
    const int es = dtype_size(a.dtype);
    if (!a.logits || !a.out) SAY("gala_adjust_logits: logits and out are needed");
    if (!aligned(a.logits, es) || !aligned(a.out, es)) SAY("gala_adjust_logits: a pointer is not aligned to its elements");
    const bool history = a.history && a.width > 0;
    if (a.biases > 0 && (!a.bias_ids || !a.bias_values)) SAY("gala_adjust_logits: bias_ids and bias_values are needed");
    if (a.rows > 1 && (a.logits_ld < a.vocab || a.out_ld < a.vocab || (history && a.history_ld < a.width) ||
                       (a.biases > 0 && (a.bias_ids_ld < a.biases || a.bias_values_ld < a.biases)) || (a.mask && a.mask_ld != 0 && a.mask_ld < (a.vocab + 31) / 32)))
        SAY("gala_adjust_logits: a row stride is smaller than its row");
    if (!aligned(a.history, 4) || !aligned(a.lengths, 4) || !aligned(a.repetition, 4) || !aligned(a.frequency, 4) || !aligned(a.presence, 4) ||
        !aligned(a.bias_ids, 4) || !aligned(a.bias_values, 4) || !aligned(a.mask, 4))
        SAY("gala_adjust_logits: a pointer is not aligned to its elements");
    Adjust p = {};
    p.rows = a.rows;
    p.vocab = a.vocab;
    p.width = history ? a.width : 0;
    p.biases = a.biases;
    p.x = a.logits;
    p.x_ld = a.rows > 1 ? a.logits_ld : 0;
    p.y = a.out;
    p.y_ld = a.rows > 1 ? a.out_ld : 0;
    p.history = history ? a.history : nullptr;
    p.history_ld = a.rows > 1 ? a.history_ld : 0;
    p.lengths = a.lengths;
    p.repetition = a.repetition;
    p.frequency = a.frequency;
    p.presence = a.presence;
    p.bias_ids = a.bias_ids;
    p.bias_ids_ld = a.rows > 1 ? a.bias_ids_ld : 0;
    p.bias_values = a.bias_values;
    p.bias_values_ld = a.rows > 1 ? a.bias_values_ld : 0;
    p.mask = a.mask;
    p.mask_ld = a.rows > 1 ? a.mask_ld : 0;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = a.dtype == GALA_F32 ? adjust<float>(p, st) : a.dtype == GALA_BF16 ? adjust<__nv_bfloat16>(p, st) : adjust<__half>(p, st);
    return launched(e, errbuf, errbuf_len, "gala_adjust_logits");
}
