// One draw per row from temperature, top-k, top-p and min-p filtered logits, by inverse CDF, for sm_100a.
//
// Every filter keeps a prefix of the ranking (largest logit first, ties by lowest index), so nothing is sorted: a filter
// is a threshold - a key, and how many of the entries equal to it stay - and the draw is a sum in the order of the index.
// A logit becomes an unsigned key whose order is the logit's; the row stays in registers from its one read on.
//
// A row belongs to a team: a warp (up to 1024 entries; four rows a block), a block (up to 32768), or a cluster of up to
// eight blocks, whose sums go through distributed shared memory.
// A warp finds a threshold bit by bit from the top: a bit stays set when the entries at or above the key so far still
// reach the wanted count (top-k) or mass (top-p).  A block or a cluster finds it by histograms in shared memory: the first
// one over equal steps of (m - l) / T, where the entries are spread well (over the key's own leading bits most would fall
// into a dozen bins and the atomics would queue), the next ones over the keys of the bin that holds the threshold, 2048
// bins each, until a bin is one key: two rounds for 16-bit logits, two or three for 32-bit ones.  The first round leaves
// out the tail that cannot matter: what lies 16 and more below the largest, and, for top-p, weights so small that all of
// them together cannot reach the share that is cut off.
//
// Weights are summed as whole multiples of 2^-44 in 64 bits: any order, any team and any atomics give the same sum, and
// the sums of up to 2^18 weights fit.
#include <cooperative_groups.h>

#include "sequence.cuh"

namespace gala {
namespace cg = cooperative_groups;

constexpr int kMaxVocab = 262144;
constexpr float kOne = 17592186044416.0f;   // 2^44
typedef unsigned long long u64;

// Key of a logit: unsigned order = order of the values; the low bits that a 16-bit type never uses are dropped.
template <typename T> constexpr int kDrop = 0;
template <> constexpr int kDrop<__nv_bfloat16> = 16;
template <> constexpr int kDrop<__half> = 13;
template <typename T>
__device__ __forceinline__ uint32_t key_of(float l) {
    if (isnan(l)) l = -INFINITY;
    const uint32_t u = __float_as_uint(l + 0.0f);       // -0 and +0 tie
    return (u & 0x80000000u ? ~u : u | 0x80000000u) >> kDrop<T>;
}
template <typename T>
__device__ __forceinline__ float logit_of(uint32_t key) {
    constexpr uint32_t low = (1u << kDrop<T>)-1u;
    const uint32_t k = key << kDrop<T>;
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~(k | low));
}
template <typename T> __device__ __forceinline__ uint32_t key_bottom() { return key_of<T>(-INFINITY); }   // keys above it can be drawn

__device__ __forceinline__ u64 warp_sum(u64 v) {
    // 27 bits at a time: 32 of them fit the 32-bit sum
    const u64 a = __reduce_add_sync(0xffffffffu, (uint32_t)(v & 0x7ffffffu));
    const u64 b = __reduce_add_sync(0xffffffffu, (uint32_t)((v >> 27) & 0x7ffffffu));
    const u64 c = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 54));
    return a + (b << 27) + (c << 54);
}

enum { TEAM_WARP, TEAM_BLOCK, TEAM_CLUSTER };

constexpr int kBins = 2048;
constexpr float kFirstBins = 128.0f;      // bins of one unit of (m - l) / T in the first round
struct Histogram {
    uint32_t lo[kBins], hi[kBins];        // 64-bit sums as two words with a carry
    u64 sums[32];                         // of the warps
    u64 before;                           // answer: sum ahead of the bin
    int bin;
    uint32_t least[32], most[32];
};

// Sums over a team.  Every exchange uses the slots of the other parity than the one before, so that one barrier each does.
template <int TEAM>
struct Team {
    u64* warp_slots;      // [2][32] of this block
    u64* rank_slots;      // [2][8]
    int warps, ranks, rank, par;
    __device__ __forceinline__ int place() const { return TEAM == TEAM_WARP ? 0 : rank * warps + (int)(threadIdx.x >> 5); }

    __device__ __forceinline__ u64 sum(u64 v) {
        v = warp_sum(v);
        if (TEAM == TEAM_WARP) return v;
        u64 mine, ahead;
        return exchange(v, mine, ahead);
    }
    // smallest and largest of the team's values
    __device__ __forceinline__ void extremes(uint32_t& least, uint32_t& most) {
        least = __reduce_min_sync(0xffffffffu, least);
        most = __reduce_max_sync(0xffffffffu, most);
        if (TEAM == TEAM_WARP) return;
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const u64 none = 0xffffffff00000000ull;
        u64* ws = warp_slots + par * 32;
        if (lane == 0) ws[w] = ((u64)least << 32) | most;
        __syncthreads();
        u64 x = lane < warps ? ws[lane] : none;
        least = __reduce_min_sync(0xffffffffu, (uint32_t)(x >> 32));
        most = __reduce_max_sync(0xffffffffu, (uint32_t)x);
        if (TEAM == TEAM_CLUSTER) {
            cg::cluster_group cl = cg::this_cluster();
            u64* rs = rank_slots + par * 8;
            if (w == 0 && lane < ranks) *cl.map_shared_rank(rs + rank, lane) = ((u64)least << 32) | most;
            cl.sync();
            x = lane < ranks ? rs[lane] : none;
            least = __reduce_min_sync(0xffffffffu, (uint32_t)(x >> 32));
            most = __reduce_max_sync(0xffffffffu, (uint32_t)x);
        }
        par ^= 1;
    }
    // every thread of the team has come here
    __device__ __forceinline__ void barrier() {
        if (TEAM == TEAM_CLUSTER) cg::this_cluster().sync();
        else if (TEAM == TEAM_BLOCK) __syncthreads();
    }
    // v: this warp's value.  Returns the team's sum; `ahead` is the sum over the warps before this one.
    __device__ __forceinline__ u64 scan(u64 v, u64& ahead) {
        ahead = 0;
        if (TEAM == TEAM_WARP) return v;
        u64 mine;
        return exchange(v, mine, ahead);
    }

private:
    __device__ __forceinline__ u64 exchange(u64 v, u64& block, u64& ahead) {
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        u64* ws = warp_slots + par * 32;
        if (lane == 0) ws[w] = v;
        __syncthreads();
        const u64 x = lane < warps ? ws[lane] : 0;
        block = warp_sum(x);
        ahead = warp_sum(lane < w ? x : 0);
        u64 all = block;
        if (TEAM == TEAM_CLUSTER) {
            cg::cluster_group cl = cg::this_cluster();
            u64* rs = rank_slots + par * 8;
            if (w == 0 && lane < ranks) *cl.map_shared_rank(rs + rank, lane) = block;
            cl.sync();
            const u64 y = lane < ranks ? rs[lane] : 0;
            all = warp_sum(y);
            ahead += warp_sum(lane < rank ? y : 0);
        }
        par ^= 1;
        return all;
    }
};

template <typename T, int E, int TEAM>
__global__ void __launch_bounds__(TEAM == TEAM_WARP ? 128 : 1024) sample_kernel(const gala_sample_args p, const int ranks) {
    __shared__ u64 warp_slots[64];
    __shared__ u64 rank_slots[16];
    __shared__ __align__(8) uint8_t hist_memory[TEAM == TEAM_WARP ? 8 : sizeof(Histogram)];
    const int lane = threadIdx.x & 31;
    Team<TEAM> team;
    team.warp_slots = warp_slots;
    team.rank_slots = rank_slots;
    team.warps = blockDim.x >> 5;
    team.ranks = TEAM == TEAM_CLUSTER ? ranks : 1;
    team.rank = TEAM == TEAM_CLUSTER ? (int)(blockIdx.x % ranks) : 0;
    team.par = 0;
    pdl_wait();
    pdl_launch();
    long long row;
    if (TEAM == TEAM_WARP) row = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    else row = TEAM == TEAM_CLUSTER ? (long long)(blockIdx.x / ranks) : (long long)blockIdx.x;
    if (TEAM == TEAM_WARP && row >= p.rows) return;
    if (TEAM == TEAM_CLUSTER) cg::this_cluster().sync();     // every block runs before one writes to another's shared memory

    // this warp's 32 E successive entries; entry i of a lane is at base + 32 i + lane
    const int base = team.place() * 32 * E + lane;
    const T* l = static_cast<const T*>(p.logits) + row * p.logits_ld;
    uint32_t key[E];
#pragma unroll
    for (int i = 0; i < E; i++) key[i] = base + 32 * i < p.vocab ? key_of<T>(to_f32<T>(l[base + 32 * i])) : 0u;
    uint32_t top = 0, unused = 0;
#pragma unroll
    for (int i = 0; i < E; i++) top = max(top, key[i]);
    team.extremes(unused, top);
    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    const bool greedy = !(temp > 0.0f);
    const bool empty = top <= key_bottom<T>();
    const float lmax = logit_of<T>(top);
    // (l - m) / T by the row's reciprocal and one correction step with the exact remainder (Markstein), which is the
    // rounded quotient; plain division where the reciprocal leaves the normal range
    const float inv = 1.0f / temp;
    const bool plain = !(temp > 1e-30f && temp < 1e30f);
    auto weight = [&](uint32_t k) -> float {
        if (k == top) return 1.0f;
        if (k <= key_bottom<T>()) return 0.0f;
        const float d = logit_of<T>(k) - lmax;
        float z = plain ? __fdiv_rn(d, temp) : d * inv;
        if (z < -150.0f) return 0.0f;                     // and nothing infinite goes on
        if (!plain) z = fmaf(fmaf(-z, temp, d), inv, z);
        return expf(z);
    };
    // w 2^44 as a whole number, without the conversion unit: 22 bits at a time in the mantissa of 2^23
    auto quant = [&](float w) -> u64 {
        const float a = fmaf(w, 4194304.0f, 8388608.0f);                    // 2^23 + the nearest multiple of 2^-22
        const float rest = fmaf(a - 8388608.0f, -1.0f / 4194304.0f, w);     // exact, within 2^-23
        const float b = fmaf(rest, 17592186044416.0f, 12582912.0f);         // 1.5 2^23 + the rest in units of 2^-44
        return ((u64)(__float_as_uint(a) & 0x7fffffu) << 22) + (u64)(long long)((int)(__float_as_uint(b) & 0x7fffffu) - 0x400000);
    };

    // kept: key > cut, and the first `room` of those equal to it
    uint32_t cut = key_bottom<T>();
    long long room = 0;
    auto reach = [&](uint32_t at, bool mass) -> u64 {     // count or mass of the entries with key >= at
        u64 s = 0;
#pragma unroll
        for (int i = 0; i < E; i++)
            if (key[i] >= at) s += mass ? quant(weight(key[i])) : 1ull;
        return team.sum(s);
    };
    // The largest key whose entries at or above it, of those above `floor`, reach `want`, which all of them together do;
    // `ahead` is the count or mass above it.  Entries that weigh less than `least` cannot be what reaches it.
    auto search = [&](u64 want, bool mass, float least, uint32_t floor, u64& ahead) -> uint32_t {
        if (TEAM == TEAM_WARP) {
            uint32_t k = 0;
            for (int b = 31 - kDrop<T>; b >= 0; b--)
                if (reach(k | (1u << b), mass) >= want) k |= 1u << b;
            ahead = reach(k + 1, mass);
            return k;
        }
        Histogram& h = *reinterpret_cast<Histogram*>(hist_memory);
        const int w = threadIdx.x >> 5, nt = blockDim.x;
        // one round: bin_of(key) is the bin of an entry or -1; returns the bin that reaches `want` (-1: none does)
        auto round = [&](auto bin_of) -> int {
            team.barrier();        // nobody reads the last round's bins any more
            for (int i = threadIdx.x; i < kBins; i += nt) h.lo[i] = h.hi[i] = 0;
            if (threadIdx.x == 0) h.bin = -1;
            __syncthreads();
            int at = -1;           // entries of one bin after another are added up before they go to memory
            u64 run = 0;
            auto flush = [&] {
                const uint32_t low = (uint32_t)run, old = atomicAdd(&h.lo[at], low);
                const uint32_t high = (uint32_t)(run >> 32) + (old + low < old ? 1u : 0u);
                if (high) atomicAdd(&h.hi[at], high);
            };
#pragma unroll
            for (int i = 0; i < E; i++) {
                const int b = bin_of(key[i]);
                if (b >= 0) {
                    const u64 q = mass ? quant(weight(key[i])) : 1ull;
                    if (b != at) {
                        if (at >= 0) flush();
                        at = b;
                        run = 0;
                    }
                    run += q;
                }
            }
            if (at >= 0) flush();
            team.barrier();
            const int per = (kBins + nt - 1) / nt, b0 = (int)threadIdx.x * per, b1 = min(b0 + per, kBins);
            auto value = [&](int b) -> u64 {
                if (TEAM == TEAM_BLOCK) return ((u64)h.hi[b] << 32) | h.lo[b];
                cg::cluster_group cl = cg::this_cluster();
                u64 v = 0;
                for (int r = 0; r < team.ranks; r++) v += ((u64)*cl.map_shared_rank(&h.hi[b], r) << 32) + *cl.map_shared_rank(&h.lo[b], r);
                return v;
            };
            u64 mine = 0;
            for (int b = b0; b < b1; b++) mine += value(b);
            u64 upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 up = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += up;
            }
            if (lane == 31) h.sums[w] = upto;
            __syncthreads();
            const u64 x = lane < team.warps ? h.sums[lane] : 0;
            const u64 start = warp_sum(lane < w ? x : 0) + upto - mine;
            const u64 need = want - ahead;
            if (start < need && start + mine >= need) {        // one thread at most
                u64 c = start;
                for (int b = b0; b < b1; b++) {
                    const u64 v = value(b);
                    if (c + v >= need) {
                        h.bin = b;
                        h.before = c;
                        break;
                    }
                    c += v;
                }
            }
            __syncthreads();
            const int b = h.bin;
            if (b >= 0) ahead += h.before;
            return b;
        };
        ahead = 0;
        uint32_t least_key = floor + 1, most_key = top;
        auto step_of = [&](uint32_t k) -> int { return plain ? 0 : min((int)((lmax - logit_of<T>(k)) * inv * kFirstBins), kBins - 1); };
        const int first = round([&](uint32_t k) -> int {
            if (k <= floor) return -1;
            if (k == top) return 0;
            const int b = step_of(k);
            return b == kBins - 1 || (mass && weight(k) < least) ? -1 : b;
        });
        if (first >= 0) {
            uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
            for (int i = 0; i < E; i++)
                if (key[i] > floor && (key[i] == top ? 0 : step_of(key[i])) == first) {
                    lo = min(lo, key[i]);
                    hi = max(hi, key[i]);
                }
            team.extremes(lo, hi);
            least_key = lo;
            most_key = hi;
        }
        while (least_key < most_key) {
            const int shift = max(0, 21 - __clz(most_key - least_key));
            const int b = round([&](uint32_t k) -> int { return k < least_key || k > most_key ? -1 : (int)((most_key - k) >> shift); });
            if (b < 0) break;      // does not happen: the range reaches `want`
            most_key -= (uint32_t)b << shift;
            const uint32_t span = (1u << shift) - 1u;
            if (most_key - least_key > span) least_key = most_key - span;
        }
        return most_key;
    };
    if (greedy) {
        cut = top;
        room = 1;
    } else if (!empty) {
        const int k = p.top_k ? p.top_k[row] : 0;
        // with fewer than k entries that can be drawn at all, nothing is cut
        if (k > 0 && k < p.vocab && reach(cut + 1, false) > (u64)k) {
            u64 ahead;
            cut = search((u64)k, false, 0.0f, cut, ahead);
            room = k - (long long)ahead;
        }
        const float tp = p.top_p ? p.top_p[row] : 1.0f;
        if (!(tp >= 1.0f)) {
            const u64 above = reach(cut + 1, true), each = quant(weight(cut));
            const u64 sum = above + (u64)room * each;
            const double goal = ceil((double)tp * (double)sum);
            const u64 want = goal >= 1.0 ? (u64)goal : 1ull;       // NaN and what is not positive: the first alone
            u64 ahead = above;
            if (above >= want) {
                // all entries lighter than this together weigh less than half of what is cut off
                const float least = 0.5f * (1.0f - fmaxf(tp, 0.0f)) * (float)((double)above / (double)kOne) / (float)p.vocab;
                cut = search(want, true, least >= 0.0f ? least : 0.0f, cut, ahead);
                room = p.vocab;
            }
            // ties stay while what is ranked before them is less than wanted
            const u64 one = quant(weight(cut));
            const u64 fit = one ? (want - ahead + one - 1) / one : 0ull;
            if ((long long)fit < room) room = (long long)fit;
        }
    }
    const float mp = p.min_p && !greedy ? fminf(p.min_p[row], 1.0f) : 0.0f;

    // which of the ties are among the first `room`
    uint32_t keep = 0;
    {
        uint32_t mine = 0;
        int ties = 0;
#pragma unroll
        for (int i = 0; i < E; i++) {
            if (key[i] > cut) keep |= 1u << i;
            if (key[i] == cut && cut > key_bottom<T>()) mine |= 1u << i;
        }
        ties = __reduce_add_sync(0xffffffffu, (uint32_t)__popc(mine));
        u64 ahead;
        const u64 all = team.scan((u64)ties, ahead);
        if (room > 0 && all > 0) {
            if (all <= (u64)room) {
                keep |= mine;
            } else {
                long long left = room - (long long)ahead;     // for this warp's entries, in order
#pragma unroll
                for (int i = 0; i < E; i++) {
                    const uint32_t g = __ballot_sync(0xffffffffu, (mine >> i) & 1u);
                    if (((mine >> i) & 1u) && (long long)__popc(g & ((1u << lane) - 1u)) < left) keep |= 1u << i;
                    left -= __popc(g);
                }
            }
        }
    }
    u64 mass = 0;
#pragma unroll
    for (int i = 0; i < E; i++)
        if ((keep >> i) & 1u) {
            const float w = weight(key[i]);
            if (w >= mp) mass += quant(w);
            else keep &= ~(1u << i);
        }
    u64 before;
    const u64 here = warp_sum(mass);
    const u64 total = team.scan(here, before);
    if (empty) {
        if (team.place() == 0 && (TEAM == TEAM_WARP || threadIdx.x == 0) && lane == 0) {
            p.tokens[row] = -1;
            if (p.logprobs) p.logprobs[row] = -INFINITY;
        }
    } else {
        const double goal = (double)p.uniforms[row] * (double)total;
        u64 target = goal > 0.0 ? (u64)goal : 0ull;
        if (target >= total) target = total - 1;
        if (target >= before && target - before < here) {      // one warp of the team
            u64 left = target - before;
            int token = -1;
            float wt = 0.0f;
#pragma unroll
            for (int i = 0; i < E; i++) {
                const float w = (keep >> i) & 1u ? weight(key[i]) : 0.0f;
                const u64 q = quant(w);
                const u64 group = warp_sum(q);
                if (token < 0) {
                    if (left < group) {
                        u64 run = q;        // inclusive sum over the lanes
#pragma unroll
                        for (int o = 1; o < 32; o <<= 1) {
                            const u64 up = __shfl_up_sync(0xffffffffu, run, o);
                            if (lane >= o) run += up;
                        }
                        const uint32_t hit = __ballot_sync(0xffffffffu, run > left);
                        const int at = __ffs(hit) - 1;
                        token = base - lane + 32 * i + at;
                        wt = __shfl_sync(0xffffffffu, w, at);
                    } else {
                        left -= group;
                    }
                }
            }
            if (lane == 0) {
                p.tokens[row] = token;
                if (p.logprobs) p.logprobs[row] = (float)log((double)wt * (double)kOne / (double)total);
            }
        }
    }
    if (TEAM == TEAM_CLUSTER) cg::this_cluster().sync();
}

// ------------------------------------------------------------------------------------------------ host side
namespace {

template <typename T, int E, int TEAM>
cudaError_t go(const gala_sample_args& a, unsigned grid, unsigned block, int ranks, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ranks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T, E, TEAM>, a, ranks);
}

template <typename T>
cudaError_t pick(const gala_sample_args& a, cudaStream_t st) {
    const int v = a.vocab;
    if (v <= 1024) {
        const unsigned grid = (unsigned)((a.rows + 3) / 4);
        if (v <= 32) return go<T, 1, TEAM_WARP>(a, grid, 128, 1, st);
        if (v <= 256) return go<T, 8, TEAM_WARP>(a, grid, 128, 1, st);
        return go<T, 32, TEAM_WARP>(a, grid, 128, 1, st);
    }
    if (v <= 16384) return go<T, 16, TEAM_BLOCK>(a, (unsigned)a.rows, (unsigned)((v + 511) / 512 * 32), 1, st);
    int ranks = 1;
    while (ranks * 32768 < v) ranks *= 2;
    const unsigned block = (unsigned)(((v + ranks - 1) / ranks + 1023) / 1024 * 32);
    if (ranks == 1) return go<T, 32, TEAM_BLOCK>(a, (unsigned)a.rows, block, 1, st);
    return go<T, 32, TEAM_CLUSTER>(a, (unsigned)a.rows * ranks, block, ranks, st);
}

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

extern "C" int gala_sample(const gala_sample_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_sample: null arguments");
    const gala_sample_args& a = *p;
    if (!dtype_ok(a.dtype)) SAY("gala_sample: dtype %d", a.dtype);
    if (a.rows < 0 || a.rows >= (1ll << 27) || a.vocab < 1 || a.vocab > kMaxVocab)
        SAY("gala_sample: %lld rows of %d entries (1..%d)", a.rows, a.vocab, kMaxVocab);
    if (a.rows == 0) return GALA_OK;
    if (!a.logits || !a.uniforms || !a.tokens) SAY("gala_sample: logits, uniforms and tokens are needed");
    if (a.logits_ld < a.vocab) SAY("gala_sample: the row stride is smaller than the %d entries", a.vocab);
    if (!aligned(a.logits, dtype_size(a.dtype)) || !aligned(a.uniforms, 4) || !aligned(a.temperature, 4) || !aligned(a.top_k, 4) ||
        !aligned(a.top_p, 4) || !aligned(a.min_p, 4) || !aligned(a.tokens, 4) || !aligned(a.logprobs, 4))
        SAY("gala_sample: a pointer is not aligned to its element type");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = a.dtype == GALA_F32 ? pick<float>(a, st) : a.dtype == GALA_BF16 ? pick<__nv_bfloat16>(a, st) : pick<__half>(a, st);
    return launched(e, errbuf, errbuf_len, "gala_sample");
}
