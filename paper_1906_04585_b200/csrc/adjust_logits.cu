// Logits before a draw: penalties of the tokens in a row's history, biases of listed tokens, a bit mask, for sm_100a.
//
// Two ways.  Either a block has a segment of a row, whose logits are on their way while it counts: a word an entry in shared
// memory holds the count of the entry (low 20 bits) and the place of its first bias in the list (high 12 bits, counted from the
// end, so that a maximum finds the first).  Segments begin where 16 bytes do, whatever the row's address.  Or, for rows of several
// segments, where every segment would read the row's lists again, the mask is applied to all entries by blocks that stream, and a
// block a row counts its lists in a hash table of the same words, beside the stream as far as there is room: it starts once every
// block of the stream has.  When the stream is done it goes over the few entries that the lists touch (out may be logits itself: an
// entry that the stream has crossed out stays so whatever it was).
// Counts are whole numbers and duplicates of a bias are added by the thread of the first in the order of the list, so the result
// does not depend on the order in which threads run.
// Measured on a B200: 256 x 32768 bfloat16 with histories of 2048, 64 biases and masks 20 us, 64 x 131072 float32 with histories of
// 8192 and 300 biases 36 us (by segments alone 21 and 50 us; counting in the shared memory of a cluster's blocks 31 and 56 us).
// Bound by latency: the stream takes 12 and 18 us cold, in two waves of blocks, and the chain of the lists (fetch, count, fetch what
// they touch), 16 and 26, begins in the second.  A mask alone: 256 x 131072 bfloat16 27 us (5.1 TB/s).
#include "sequence.cuh"

namespace gala {
namespace {

constexpr int kThreads = 256;
constexpr int kSegment = 8192;      // entries of a block with lists
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
    int hash_shift, stream_first;      // touched_kernel: 32 - log2 of its slots; whether the stream is the kernel before it
};

struct Settings {
    float rep, freq, pres;
    __device__ __forceinline__ void read(const Adjust& a, long long row) {
        rep = a.history && a.repetition ? a.repetition[row] : 1.0f;
        freq = a.history && a.frequency ? a.frequency[row] : 0.0f;
        pres = a.history && a.presence ? a.presence[row] : 0.0f;
    }
    // the entry whose word is w
    __device__ __forceinline__ float changed(uint32_t w, float l, const float* bias) const {
        const uint32_t count = w & 0xfffffu, at = w >> 20;
        if (count) {
            l = l > 0.0f ? l / rep : l * rep;      // a product with 1 / rep: one rounding more, and infinite where rep < 2^-128
            l = l - freq * (float)count - pres;
        }
        if (at) l += bias[kMaxBiases - at];
        return l;
    }
};
__device__ __forceinline__ int tokens_of(const Adjust& a, long long row) { return !a.history ? 0 : a.lengths ? min(max(a.lengths[row], 0), a.width) : a.width; }
// An id that meets another of its kind in its word (`old`, as the maximum found it) marks both places; the first of its kind is
// marked then, whichever comes last.
__device__ __forceinline__ void mark(float* bias, int i, uint32_t old) {
    if (old) bias[i] = bias[kMaxBiases - (old >> 20)] = 1.0f;
}
// the sum of the biases of the id at place i of a list, which is its first; marked: it is listed again
__device__ __forceinline__ float bias_of(const Adjust& a, const int* ids, const float* values, int i, bool marked) {
    float s = values[i];
    if (marked)
        for (int j = i + 1; j < a.biases; j++)
            if (ids[j] == ids[i]) s += values[j];
    return s;
}

// -inf where a bit is 0
template <typename T, int V> __device__ __forceinline__ void shut(Vec<T, V>& v, uint32_t open) {
    if constexpr (V == 1) {
        v.w = open & 1u ? v.w : from_f32<T>(-INFINITY);
    } else {
        uint32_t* w = reinterpret_cast<uint32_t*>(&v.w);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if (sizeof(T) == 4) {
                w[j] = open >> j & 1u ? w[j] : 0xff800000u;
            } else {
                const uint32_t keep = (open >> (2 * j) & 1u ? 0xffffu : 0u) | (open >> (2 * j + 1) & 1u ? 0xffff0000u : 0u);
                w[j] = (w[j] & keep) | ((std::is_same<T, __nv_bfloat16>::value ? 0xff80ff80u : 0xfc00fc00u) & ~keep);
            }
        }
    }
}

// V entries at once (16 bytes), N times a thread under way together
template <typename T, int V, int N, bool TABLE>
__global__ void __launch_bounds__(kThreads) adjust_kernel(const Adjust a) {
    extern __shared__ __align__(16) uint32_t table[];                            // [segment]
    float* bias = reinterpret_cast<float*>(table + (TABLE ? a.segment : 0));     // [biases], at the place of the first of its id
    const int tid = threadIdx.x, threads = blockDim.x;
    const long long row = blockIdx.x / a.segments;
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    T* y = static_cast<T*>(a.y) + row * a.y_ld;
    // entry `first` and every V-th after it lies on 16 bytes
    const int pad = V == 1 ? 0 : (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    const int first = (int)(blockIdx.x - row * a.segments) * a.segment - pad, end = min(first + a.segment, a.vocab);
    pdl_wait();
    pdl_launch();
    if (first >= a.vocab) return;
    const uint32_t* mask = a.mask ? reinterpret_cast<const uint32_t*>(a.mask) + row * a.mask_ld : nullptr;
    constexpr uint32_t kAll = (1u << V) - 1;
    Vec<T, V> v[N];
    uint32_t open[N];
    auto bring = [&](int base) {
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int e = base + (i * threads + tid) * V;
            open[i] = kAll;
            if (e < 0 || e + V > end) continue;
            v[i].w = *reinterpret_cast<const decltype(v[i].w)*>(x + e);
            if (mask) {
                open[i] = mask[e >> 5] >> (e & 31);
                if ((e & 31) + V > 32) open[i] |= mask[(e >> 5) + 1] << (32 - (e & 31));
                open[i] &= kAll;
            }
        }
    };
    bring(first);
    Settings set;
    if (TABLE) {
        const int* history = a.history ? a.history + row * a.history_ld : nullptr;
        const int* ids = a.biases > 0 ? a.bias_ids + row * a.bias_ids_ld : nullptr;
        int length = 0, id[8];
        // the first tokens are on their way before it is known how many count
        auto tokens = [&](int base) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int at = base + i * threads + tid;
                id[i] = at < a.width ? history[at] : -1;
            }
        };
        if (history) {
            tokens(0);
            length = tokens_of(a, row);
        }
        set.read(a, row);
        // where an id of a list lies in this segment, or past its end
        auto place = [&](int id) { return id >= 0 && id < a.vocab ? (uint32_t)(id - first) : 0xffffffffu; };
        const uint32_t size = (uint32_t)(end - first);
        for (int i = tid; i < a.segment / 4; i += threads) reinterpret_cast<uint4*>(table)[i] = make_uint4(0, 0, 0, 0);
        for (int i = tid; i < a.biases; i += threads) bias[i] = 0.0f;
        __syncthreads();
        if (ids) {
            for (int i = tid; i < a.biases; i += threads) {
                const uint32_t e = place(ids[i]);
                if (e < size) mark(bias, i, atomicMax(&table[e], (uint32_t)(kMaxBiases - i) << 20));
            }
            __syncthreads();
            const float* values = a.bias_values + row * a.bias_values_ld;
            for (int i = tid; i < a.biases; i += threads) {
                const uint32_t e = place(ids[i]);
                if (e < size && (int)(table[e] >> 20) == kMaxBiases - i) bias[i] = bias_of(a, ids, values, i, bias[i] != 0.0f);
            }
        }
        for (int base = 0; base < length; base += 8 * threads) {
            if (base > 0) tokens(base);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t e = place(id[i]);
                if (e < size && base + i * threads + tid < length) atomicAdd(&table[e], 1u);
            }
        }
        __syncthreads();
    }
    for (int base = first; base < end; base += N * threads * V) {
        if (base > first) bring(base);
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int e = base + (i * threads + tid) * V;
            if (e >= 0 && e + V <= end) {
                if (TABLE) {
                    uint32_t w[V], hit = 0;
                    if constexpr (V >= 4) {
#pragma unroll
                        for (int j = 0; j < V; j += 4) {
                            const uint4 t = reinterpret_cast<const uint4*>(table)[(e - first + j) / 4];
                            w[j] = t.x, w[j + 1] = t.y, w[j + 2] = t.z, w[j + 3] = t.w;
                            hit |= t.x | t.y | t.z | t.w;
                        }
                    } else {
                        hit = w[0] = table[e - first];
                    }
                    if (hit) {
                        float f[V];
#pragma unroll
                        for (int j = 0; j < V; j++) f[j] = w[j] ? set.changed(w[j], v[i].get(j), bias) : v[i].get(j);
                        v[i].put(f);
                    }
                }
                if (open[i] != kAll) shut(v[i], open[i]);
                *reinterpret_cast<decltype(v[i].w)*>(y + e) = v[i].w;
            } else if (V > 1) {      // the ends of a row
                for (int j = max(0, e); j < min(end, e + V); j++) y[j] = mask && !(mask[j >> 5] >> (j & 31) & 1u) ? from_f32<T>(-INFINITY) : TABLE && table[j - first] ? from_f32<T>(set.changed(table[j - first], to_f32<T>(x[j]), bias)) : x[j];
            }
        }
    }
}

// The entries that a row's lists touch, after the mask has been applied to all.  slots: a power of two, at least one and a half times the lists.
template <typename T>
__global__ void __launch_bounds__(1024) touched_kernel(const Adjust a, int slots) {
    extern __shared__ __align__(16) uint32_t shared[];
    uint32_t *words = shared, *keys = shared + slots;       // keys: id + 1, 0 where there is none
    float* bias = reinterpret_cast<float*>(keys + slots);
    const int tid = threadIdx.x, threads = blockDim.x;
    const long long row = blockIdx.x;
    for (int i = tid; i < slots / 2; i += threads) reinterpret_cast<uint4*>(shared)[i] = make_uint4(0, 0, 0, 0);
    for (int i = tid; i < a.biases; i += threads) bias[i] = 0.0f;
    if (!a.stream_first) pdl_wait();      // else the kernel before is the stream, and what came before it is complete
    const int* history = a.history ? a.history + row * a.history_ld : nullptr;
    const int* ids = a.biases > 0 ? a.bias_ids + row * a.bias_ids_ld : nullptr;
    int next[8];      // tokens under way
    auto tokens = [&](int base) {
#pragma unroll
        for (int i = 0; i < 8; i++) next[i] = base + i * threads + tid < a.width ? history[base + i * threads + tid] : -1;
    };
    if (history) tokens(0);
    const int length = tokens_of(a, row);
    Settings set;
    set.read(a, row);
    auto slot_of = [&](uint32_t id) {
        uint32_t s = (id * 0x9e3779b1u) >> a.hash_shift;
        for (;;) {      // a third of the table is empty at least
            uint32_t k = *static_cast<volatile uint32_t*>(&keys[s]);      // most tokens have been seen before
            if (k == 0) k = atomicCAS(&keys[s], 0u, id + 1);
            if (k == 0 || k == id + 1) return s;
            s = (s + 1) & (slots - 1);
        }
    };
    __syncthreads();
    for (int i = tid; ids && i < a.biases; i += threads) {
        const int id = ids[i];
        if (id >= 0 && id < a.vocab) mark(bias, i, atomicMax(&words[slot_of(id)], (uint32_t)(kMaxBiases - i) << 20));
    }
    __syncthreads();
    for (int base = 0; base < length; base += 8 * threads) {
        if (base > 0) tokens(base);
#pragma unroll 1
        for (int i = 0; i < 8; i++) {
            const int id = next[0];
#pragma unroll
            for (int j = 0; j < 7; j++) next[j] = next[j + 1];
            if (id >= 0 && id < a.vocab && base + i * threads + tid < length) atomicAdd(&words[slot_of(id)], 1u);
        }
    }
    for (int i = tid; ids && i < a.biases; i += threads) {
        const int id = ids[i];
        if (id >= 0 && id < a.vocab && (int)(words[slot_of(id)] >> 20) == kMaxBiases - i)
            bias[i] = bias_of(a, ids, a.bias_values + row * a.bias_values_ld, i, bias[i] != 0.0f);
    }
    __syncthreads();
    if (a.stream_first) pdl_wait();
    pdl_launch();
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    T* y = static_cast<T*>(a.y) + row * a.y_ld;
    const uint32_t* mask = a.mask ? reinterpret_cast<const uint32_t*>(a.mask) + row * a.mask_ld : nullptr;
    for (int base = tid; base < slots; base += 8 * threads) {
        uint32_t key[8], open[8];
        T l[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int at = base + i * threads;
            key[i] = at < slots ? keys[at] : 0u;
            open[i] = 1u;
            if (key[i]) {
                const int e = (int)(key[i] - 1);
                l[i] = x[e];
                if (mask) open[i] = mask[e >> 5] >> (e & 31) & 1u;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (key[i] && open[i]) y[key[i] - 1] = from_f32<T>(set.changed(words[base + i * threads], to_f32<T>(l[i]), bias));      // else crossed out
    }
}

template <typename T, int V, int N> cudaError_t launch_adjust(Adjust a, cudaStream_t st) {
    const bool table = a.history || a.biases > 0;
    // Short rows: a block as small as the row.  Without lists a segment is what a block holds at once.
    const int ends = V == 1 || (aligned(a.x, 16) && (a.rows <= 1 || a.x_ld % V == 0)) ? 0 : V - 1;      // entries before the first 16 bytes
    int threads = ((a.vocab + ends + V - 1) / V + 31) / 32 * 32;
    if (table && threads < 128 && a.width + a.biases > 64) threads = 128;
    if (threads > kThreads) threads = kThreads;
    a.segment = table ? kSegment : kThreads * V * N;
    const int whole = (a.vocab + ends + 31) / 32 * 32;
    if (a.segment > whole) a.segment = whole;
    a.segments = (a.vocab + ends + a.segment - 1) / a.segment;
    const long long blocks = a.rows * a.segments;
    if (blocks >= 1ll << 31) return cudaErrorInvalidConfiguration;
    if (!table) return launch_pdl(adjust_kernel<T, V, N, false>, dim3((unsigned)blocks), dim3(threads), 0, st, a);
    return launch_pdl(adjust_kernel<T, V, N, true>, dim3((unsigned)blocks), dim3(threads), (size_t)(a.segment + a.biases) * 4, st, a);
}
constexpr int kMostSlots = 16384, kMostTouched = kMostSlots / 3 * 2;      // of a hash table, and the longest lists that are counted in one
template <typename T> cudaError_t launch_touched(Adjust a, cudaStream_t st) {
    int slots = 256;
    a.hash_shift = 24;
    while (2 * slots < 3 * (a.width + a.biases)) slots *= 2, a.hash_shift--;
    const size_t smem = (size_t)slots * 8 + (size_t)a.biases * 4;
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(touched_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSlots * 8 + kMaxBiases * 4);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    const int threads = slots >= 8192 ? 1024 : slots >= 1024 ? 512 : 256;
    return launch_pdl(touched_kernel<T>, dim3((unsigned)a.rows), dim3(threads), smem, st, a, slots);
}
template <typename T> cudaError_t adjust(const Adjust& a, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    // vectors where logits and result lie on 16 bytes at the same entries of every row
    const bool wide = ((reinterpret_cast<uintptr_t>(a.x) ^ reinterpret_cast<uintptr_t>(a.y)) & 15) == 0 && (a.rows <= 1 || (a.x_ld - a.y_ld) % V == 0);
    auto segments = [&](const Adjust& b) { return wide ? launch_adjust<T, V, 32 / V>(b, st) : launch_adjust<T, 1, 8>(b, st); };
    const bool lists = a.history || a.biases > 0;
    // Rows of one segment are read once anyway; lists past the hash table's size go by segments.
    if (!lists || a.vocab <= kSegment || a.width + a.biases > kMostTouched) return segments(a);
    Adjust b = a;
    const bool stream = a.mask || a.x != a.y;
    if (stream) {
        b.history = nullptr;
        b.width = b.biases = 0;
        const cudaError_t e = segments(b);
        if (e != cudaSuccess) return e;
    }
    b = a;
    b.stream_first = stream;
    return launch_touched<T>(b, st);
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
