// The next token of each row of logits: temperature, top-k, top-p and min-p, then the inverse of the distribution at a given random number.
//
// Every filter keeps a leading part of the tokens in the order (falling logit, rising number).  With key(x) the bits of x in an order of
// unsigned numbers that part is written as a border: all keys above `key` and the first `ties` tokens with that key.  A border is found without a sort: the
// tokens are counted, or their weights added up, in bins of 1 / 64 of an octave of the weight; the bin in which the sum passes its aim
// is found, and the few tokens in it are compared with each other.  Where they are more than kList (equal logits) the border is searched by keys instead, kRanges
// parts of their range at a time.
//
// Weights are exponentials in 64 bits, as whole multiples of 2^-44: sums of whole numbers do not depend on their order, and a token is found as in
// exact arithmetic but for those 2^-44.  In 32 bits the sums would be off by 2^-24 or so of themselves, and of 32000 tokens without a filter one row in some thousands
// would get a neighbouring one.  An exponential is a table of 64 and a polynomial, which 64 bits cost no more cycles than 32 here.
//
// One block a row, whose keys stay in registers up to 32768 tokens; a longer row is read again in every pass, and lies in L2 by then.
#include <type_traits>

#include "qail_internal.h"

namespace qail {

namespace {

constexpr int kBlock = 1024, kWaves = kBlock / kWave;
constexpr int kPiece = 8;                          // neighbouring tokens of a thread
constexpr int kChunk = kBlock * kPiece;            // tokens of a pass over the block
constexpr int kMostChunks = (1 << 18) / kChunk;
constexpr int kBins = 3 * kBlock;
constexpr int kParts = 64;                         // of an octave: a bin of weights
constexpr int kLowestPart = -45 * kParts;          // of a weight of 2^-45; below, weights are 0
static_assert(-kLowestPart < kBins, "a bin for each part");
constexpr double kOne = 17592186044416.0;          // 2^44: the weight of the largest logit
constexpr int kList = kBlock;                      // tokens of a bin that are compared with each other
constexpr int kRanges = 2 * kBlock;
constexpr int kKept = 2 * kBlock;                  // kept tokens that are listed

struct SampleArgs {
    const void* logits;
    long long stride;
    int V;
    qail_sampling s;
    const float* u;
    int32_t* token;
    float* logprob;
    uint32_t* errors;
};

__device__ __forceinline__ uint32_t key_of(float x) {   // equal values have equal keys (-0 is 0), NaN the largest
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 0xFFFFFFFFu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
constexpr uint32_t kLowest = 0x007FFFFFu, kHighest = 0xFF800000u;   // keys of minus and plus infinity

typedef unsigned long long u64;

__device__ __forceinline__ u64 shfl_up64(u64 v, int n) {
    const uint32_t lo = __shfl_up((uint32_t)v, n, kWave), hi = __shfl_up((uint32_t)(v >> 32), n, kWave);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 shfl64(u64 v, int from) {
    const uint32_t lo = __shfl((uint32_t)v, from, kWave), hi = __shfl((uint32_t)(v >> 32), from, kWave);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 wave_scan(u64 v) {   // inclusive
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const u64 t = shfl_up64(v, o);
        if (lane >= o) v += t;
    }
    return v;
}

struct Shared {
    u64 bins[kBins];
    uint32_t counts[kBins];
    u64 wave_sum[kWaves];
    u64 segment[kMostChunks * kWaves];       // weight above the border of 512 neighbouring tokens each
    uint32_t ties[kMostChunks * kWaves];     // ... and how many lie on it
    double part[kParts];                     // 2^(i / 64)
    union {
        struct {
            u64 weight[kList];
            uint32_t key[kList], number[kList];
        } in_bin;
        u64 ranges[kRanges];                 // of keys
        uint2 kept[kKept];                   // key, segment
    };
    uint32_t wave_key[kWaves];
    u64 before;                              // what the chosen bin or segment has in front of it
    int chosen, ties_before, listed, border_ties;
    uint32_t first, border_key;
};

// Inclusive sums over the block's threads in their order; `total`: of all of them.  The threads have met before.
__device__ __forceinline__ u64 block_scan(Shared& sh, u64 v, u64& total) {
    const int wave = threadIdx.x / kWave;
    const u64 in = wave_scan(v);
    if (threadIdx.x % kWave == kWave - 1) sh.wave_sum[wave] = in;
    __syncthreads();
    u64 front = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const u64 t = sh.wave_sum[w];
        front += w < wave ? t : 0;
        total += t;
    }
    __syncthreads();
    return in + front;
}

// kEach bins a thread: the first one with which the sum over the bins reaches aim(sum of all) > 0, into sh.chosen, and the sum in front of it into sh.before; returns the
// sum of all (nothing is chosen where that is below the aim).
template <int kEach, typename Get, typename Aim>
__device__ __forceinline__ u64 find(Shared& sh, Get get, Aim aim_of) {
    u64 v[kEach], sum = 0, total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += v[i] = get(kEach * threadIdx.x + i);
    const u64 upto = block_scan(sh, sum, total), aim = aim_of(total);
    u64 front = upto - sum;
    if (front < aim && aim <= upto) {   // one thread
        int i = 0;
#pragma unroll
        for (int e = 0; e + 1 < kEach; ++e)
            if (i == e && front + v[e] < aim) front += v[e], ++i;
        sh.chosen = kEach * threadIdx.x + i;
        sh.before = front;
    }
    __syncthreads();
    return total;
}

// The keys of a row, 8 neighbouring tokens of a thread in each of its chunks; kLowest behind the row.  kChunks of them stay in registers; 0: none.
template <bool kBf16, bool kAligned, int kChunks>
struct Row {
    const uint8_t* p;
    int V, chunks;
    uint32_t kept[kChunks > 0 ? kChunks : 1][kPiece];

    __device__ __forceinline__ void read(int c, uint32_t* k) const {
        const int j = (c * kBlock + threadIdx.x) * kPiece;
        float f[kPiece];
        if (kAligned && j + kPiece <= V) {
            if constexpr (kBf16) {
                unpack8(*reinterpret_cast<const uint4*>(p + 2ll * j), f);
            } else {
                const float4 a = *reinterpret_cast<const float4*>(p + 4ll * j), b = *reinterpret_cast<const float4*>(p + 4ll * j + 16);
                f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                f[i] = j + i >= V ? -__builtin_inff()
                       : kBf16    ? bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[j + i])
                                  : reinterpret_cast<const float*>(p)[j + i];
        }
#pragma unroll
        for (int i = 0; i < kPiece; ++i) k[i] = key_of(f[i]);
    }
    __device__ __forceinline__ explicit Row(const void* at, int V_) : p(static_cast<const uint8_t*>(at)), V(V_), chunks((V_ + kChunk - 1) / kChunk) {
        static_assert(kChunks <= 4, "one by one: a loop is unrolled too late for registers");
        if constexpr (kChunks > 0) read(0, kept[0]);
        if constexpr (kChunks > 1) read(1, kept[1]);
        if constexpr (kChunks > 2) read(2, kept[2]);
        if constexpr (kChunks > 3) read(3, kept[3]);
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {   // f(chunk, keys)
        if constexpr (kChunks > 0) {
const auto one = [&](auto chunk) __attribute__((always_inline)) {
                constexpr int c = decltype(chunk)::value;
                if constexpr (c < kChunks) {
                    uint32_t k[kPiece];
#pragma unroll
                    for (int i = 0; i < kPiece; ++i) {
                        k[i] = kept[c][i];
                        asm volatile("" : "+v"(k[i]));   // else what a pass computes of all keys is kept for the next one, in scratch memory
                    }
                    f(c, k);
                }
            };
            one(std::integral_constant<int, 0>{});
            one(std::integral_constant<int, 1>{});
            one(std::integral_constant<int, 2>{});
            one(std::integral_constant<int, 3>{});
        } else {
            for (int c = 0; c < chunks; ++c) {
                uint32_t k[kPiece];
                read(c, k);
                f(c, k);
            }
        }
    }
};

struct Weight {
    double most, inverse, scale;     // the largest logit, 1 / temperature, 64 log2(e) / temperature
    const double* part;
    __device__ __forceinline__ double down(uint32_t key) const { return ((double)value_of(key) - most) * inverse; }
    __device__ __forceinline__ double parts(uint32_t key) const { return ((double)value_of(key) - most) * scale; }   // of an octave, below the largest
    // Of t parts, whose nearest whole number is n >= kLowestPart: 2^(n / 64) from the table, 2^((t - n) / 64) by its series (to 2^-54).  Adding 2^52 rounds
    // to a whole number, which is then the low bits.
    __device__ __forceinline__ u64 of(double t, int n) const {
        const double x = (t - (double)n) * 0.010830424696249145;   // ln(2) / 64
        double e = fma(x, 1.0 / 120.0, 1.0 / 24.0);
        e = fma(x, e, 1.0 / 6.0);
        e = fma(x, e, 0.5);
        e = fma(x, e, 1.0);
        e = fma(x, e, 1.0);
        const double octave = __builtin_bit_cast(double, (u64)(1023 + 44 + (n >> 6)) << 52);
        return __builtin_bit_cast(u64, fma(part[n & (kParts - 1)] * e, octave, 4503599627370496.0)) & ((1ull << 52) - 1);
    }
    __device__ __forceinline__ int nearest(double t) const { return t < kLowestPart - 1 ? kLowestPart - 1 : (int)rint(t); }
    __device__ __forceinline__ u64 operator()(uint32_t key) const {
        const double t = parts(key);
        const int n = nearest(t);
        return n < kLowestPart ? 0 : of(t, n);
    }
};

struct Border {
    uint32_t key;
    int ties;     // tokens with that key that are kept
};

// The shortest leading part of the tokens inside `in` whose count (kCount) or weight is at least `aim` (> 0 and no more than all of them have), by their keys.
template <bool kCount, typename R>
__device__ __forceinline__ Border border_by_keys(Shared& sh, const R row, uint32_t top, Border in, const Weight weight, u64 aim) {
    uint32_t base = top;                              // the largest key of the range
    uint32_t width = top - in.key;                    // ... and how far it goes below
    for (;;) {
        const int shift = max(0, 21 - __builtin_clz(width | 1));   // width >> shift < kRanges = 2^11
        for (int i = threadIdx.x; i < kRanges; i += kBlock) sh.ranges[i] = 0;
        __syncthreads();
        row.each([&](int, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (k[i] > in.key && k[i] <= base && base - k[i] <= width) atomicAdd(&sh.ranges[(base - k[i]) >> shift], kCount ? 1ull : weight(k[i]));
        });
        __syncthreads();
        if (threadIdx.x == 0 && in.ties > 0 && in.key <= base && base - in.key <= width)
            sh.ranges[(base - in.key) >> shift] += (u64)in.ties * (kCount ? 1ull : weight(in.key));
        __syncthreads();
        find<2>(sh, [&](int i) { return sh.ranges[i]; }, [&](u64) { return aim; });
        const uint32_t at = sh.chosen;
        aim -= sh.before;
        __syncthreads();
        base -= at << shift;
        if (shift == 0) return {base, (int)(kCount ? aim : (aim - 1) / weight(base) + 1)};
        width = min(width - (at << shift), (1u << shift) - 1);
    }
}

// The same where it lies in a bin of weights, whose tokens are to count or weigh `aim` > 0; ahead: what those up to the border weigh.  false: the bin has
// more than about kList tokens.
template <bool kCount, typename R>
__device__ __forceinline__ bool border_in_bin(Shared& sh, const R& row, int bin, const Weight& weight, u64 aim, Border& b, u64& ahead) {
    // the bin's keys, and two more at either end for the roundings of its bounds; they are looked at one by one below
    const uint32_t hi = key_of((float)(weight.most + (0.5 - bin) / weight.scale)), lo = key_of((float)(weight.most - (0.5 + bin) / weight.scale));
    const uint32_t from = max(lo - 2, kLowest + 1), to = min(hi + 2, kHighest - 1);
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    row.each([&](int c, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (k[i] >= from && k[i] <= to) {
                const int at = atomicAdd(&sh.listed, 1);
                if (at < kList) sh.in_bin.key[at] = k[i], sh.in_bin.number[at] = (c * kBlock + threadIdx.x) * kPiece + i;
            }
    });
    __syncthreads();
    const int n = sh.listed;
    if (n > kList) {
        __syncthreads();
        return false;
    }
    uint32_t key = 0, number = 0;
    u64 mine = 0;
    if ((int)threadIdx.x < n) {
        key = sh.in_bin.key[threadIdx.x], number = sh.in_bin.number[threadIdx.x];
        const double t = weight.parts(key);
        const int part = weight.nearest(t);
        if (-part == bin) mine = weight.of(t, part);
        else sh.in_bin.key[threadIdx.x] = key = 0;
        sh.in_bin.weight[threadIdx.x] = mine;
    }
    __syncthreads();
    if (key != 0) {
        u64 front = 0, heavy = 0;
        int equal = 0;
        for (int i = 0; i < n; ++i) {
            const uint32_t other = sh.in_bin.key[i];
            const bool before = other > key || (other == key && sh.in_bin.number[i] < number);
            front += before ? 1 : 0;
            heavy += before ? sh.in_bin.weight[i] : 0;
            equal += before && other == key;
        }
        const u64 at = kCount ? front : heavy;
        if (at < aim && aim <= at + (kCount ? 1 : mine)) sh.border_key = key, sh.border_ties = equal + 1, sh.before = heavy + mine;   // one thread
    }
    __syncthreads();
    b = {sh.border_key, sh.border_ties};
    ahead = sh.before;
    __syncthreads();
    return true;
}

template <bool kBf16, bool kAligned, int kChunks>
__global__ __launch_bounds__(kBlock) void sample_kernel(const SampleArgs a) {
    __shared__ Shared sh;
    const int r = blockIdx.x, V = a.V, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const Row<kBf16, kAligned, kChunks> row(static_cast<const uint8_t*>(a.logits) + (long long)r * a.stride * (kBf16 ? 2 : 4), V);
    const Row<kBf16, kAligned, 0> again(row.p, V);   // the same from memory
    const float temperature = a.s.temperature ? a.s.temperature[r] : 1.f, top_p = a.s.top_p ? a.s.top_p[r] : 1.f, min_p = a.s.min_p ? a.s.min_p[r] : 0.f;
    const float u = a.u[r];
    const int top_k = a.s.top_k ? a.s.top_k[r] : 0;

    for (int i = threadIdx.x; i < kBins; i += kBlock) sh.bins[i] = 0, sh.counts[i] = 0;
    if (threadIdx.x < kParts) sh.part[threadIdx.x] = exp2((double)threadIdx.x / kParts);
    if (threadIdx.x == 0) sh.first = 0xFFFFFFFFu;
    uint32_t most = 0;
    row.each([&](int, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) most = max(most, k[i]);
    });
    uint32_t m = most;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
    if (lane == 0) sh.wave_key[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = max(m, sh.wave_key[w]);
    const bool numbers = m > kLowest && m < kHighest && temperature >= 0.f && temperature <= 3.4028235e38f && top_p == top_p && min_p == min_p;
    if (!numbers || (temperature > 0.f && !(u >= 0.f && u < 1.f))) {   // the same for the whole block, as all that follows
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = __builtin_nanf("");
            if (a.errors) atomicAdd(a.errors, 1u);
        }
        return;
    }
    if (temperature == 0.f || min_p > 1.f || top_k == 1) {             // the first of the order
        if (most == m) {
            uint32_t place = 0xFFFFFFFFu;
            row.each([&](int c, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < kPiece; ++i)
                    if (k[i] == m) place = min(place, (uint32_t)((c * kBlock + threadIdx.x) * kPiece + i));
            });
            atomicMin(&sh.first, place);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            a.token[r] = (int32_t)sh.first;
            if (a.logprob) a.logprob[r] = 0.f;
        }
        return;
    }

    const double inverse = 1.0 / (double)temperature;
    const Weight weight = {(double)value_of(m), inverse, inverse * 92.332482616893658, sh.part};   // 64 log2(e)
    const bool by_count = top_k > 0 && top_k < V, by_share = top_p < 1.f;
    Border b = {kLowest, 0};
    u64 kept = 0;                      // what the first top_k weigh
    if (by_count || by_share) {
        row.each([&](int, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const double t = weight.parts(k[i]);
                const int n = weight.nearest(t);
                if (n < kLowestPart) continue;
                if (by_share) atomicAdd(&sh.bins[-n], weight.of(t, n));
                if (by_count) atomicAdd(&sh.counts[-n], 1u);
            }
        });
        __syncthreads();
    }
    if (by_count) {
        const u64 counted = find<kBins / kBlock>(sh, [&](int i) { return (u64)sh.counts[i]; }, [&](u64) { return (u64)top_k; });
        if (counted >= (u64)top_k) {   // else all that has a weight is among the first top_k
            const int bin = sh.chosen;
            const u64 aim = (u64)top_k - sh.before;
            __syncthreads();
            if (border_in_bin<true>(sh, row, bin, weight, aim, b, kept)) {
                if (by_share) {
                    u64 mine = 0, front;
                    for (int i = threadIdx.x; i < bin; i += kBlock) mine += sh.bins[i];
                    block_scan(sh, mine, front);
                    kept += front;
                }
            } else {
                b = border_by_keys<true>(sh, again, m, {kLowest, 0}, weight, (u64)top_k);
                if (by_share) {
                    u64 mine = 0;
                    again.each([&](int, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
                        for (int i = 0; i < kPiece; ++i)
                            if (k[i] > b.key) mine += weight(k[i]);
                    });
                    block_scan(sh, mine, kept);
                    kept += (u64)b.ties * weight(b.key);
                }
            }
        } else {
            __syncthreads();
        }
    }
    if (by_share) {
        u64 aim = 0, ahead;
        find<kBins / kBlock>(sh, [&](int i) { return sh.bins[i]; }, [&](u64 total) {
            const double share = ceil((double)top_p * (double)(b.ties > 0 ? kept : total));
            return aim = share > 1.0 ? (u64)share : 1;
        });
        const int bin = sh.chosen;
        const u64 rest = aim - sh.before;
        __syncthreads();
        const Border in = b;
        if (!border_in_bin<false>(sh, row, bin, weight, rest, b, ahead)) b = border_by_keys<false>(sh, again, m, in, weight, aim);
    }

    // The kept weight of every 512 neighbouring tokens, then the one in which the sum passes u.  Where few are kept they are listed first, so that no
    // exponential is computed for the others beside them.
    const double least = min_p > 0.f ? log((double)min_p) : -__builtin_inf();
    const u64 on = b.ties > 0 && weight.down(b.key) >= least ? weight(b.key) : 0;
    const uint32_t low = min_p > 0.f ? key_of((float)(weight.most + least * (double)temperature)) - 2 : 0;   // no key below it is kept: two steps for its rounding
    const int segments = row.chunks * kWaves;           // at most 512: one a thread
    if (threadIdx.x == 0) sh.listed = 0;
    if ((int)threadIdx.x < segments) sh.segment[threadIdx.x] = 0, sh.ties[threadIdx.x] = 0;
    __syncthreads();
    if (by_count || by_share || min_p > 0.f) {
        row.each([&](int c, const uint32_t* k) __attribute__((always_inline)) {
            uint32_t ties = 0;
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                ties += __popcll(__ballot(k[i] == b.key));
                const bool keep = k[i] > b.key && k[i] >= low;
                const u64 all = __ballot(keep);
                if (all == 0) continue;
                int at = 0;
                if (lane == 0) at = atomicAdd(&sh.listed, __popcll(all));
                at = __shfl(at, 0, kWave) + __popcll(all & ((1ull << lane) - 1));
                if (keep && at < kKept) sh.kept[at] = make_uint2(k[i], c * kWaves + wave);
            }
            if (lane == 0 && c < row.chunks) sh.ties[c * kWaves + wave] = ties;
        });
        __syncthreads();
    }
    const int listed = sh.listed;
    if ((by_count || by_share || min_p > 0.f) && listed <= kKept) {
        for (int i = threadIdx.x; i < listed; i += kBlock) {
            const uint2 t = sh.kept[i];
            if (weight.down(t.x) >= least) atomicAdd(&sh.segment[t.y], weight(t.x));
        }
    } else {
        row.each([&](int c, const uint32_t* k) __attribute__((always_inline)) {
            u64 mine = 0;
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (k[i] > b.key && k[i] >= low && weight.down(k[i]) >= least) mine += weight(k[i]);
            mine = shfl64(wave_scan(mine), kWave - 1);
            if (lane == 0 && c < row.chunks) sh.segment[c * kWaves + wave] = mine;
        });
    }
    __syncthreads();
    const bool held = (int)threadIdx.x < segments;
    const u64 above = held ? sh.segment[threadIdx.x] : 0, equal = held ? sh.ties[threadIdx.x] : 0, room = b.ties;
    u64 all;
    const u64 ties_upto = block_scan(sh, equal, all), ties_front = ties_upto - equal;
    const u64 here = above + ((ties_upto < room ? ties_upto : room) - (ties_front < room ? ties_front : room)) * on;
    const u64 upto = block_scan(sh, here, all);
    const u64 aim = (u64)((double)u * (double)all);
    if (upto - here <= aim && aim < upto) sh.chosen = threadIdx.x, sh.before = upto - here, sh.ties_before = (int)ties_front;
    __syncthreads();
    if (wave != sh.chosen % kWaves) return;
    const int c = sh.chosen / kWaves;
    uint32_t k[kPiece];
    again.read(c, k);
    u64 equal_here = 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) equal_here += k[i] == b.key;
    u64 number = sh.ties_before + wave_scan(equal_here) - equal_here;
    u64 w[kPiece], sum = 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        w[i] = k[i] > b.key ? (weight.down(k[i]) >= least ? weight(k[i]) : 0) : k[i] == b.key && number < room ? on : 0;
        number += k[i] == b.key;
        sum += w[i];
    }
    u64 at = sh.before + wave_scan(sum) - sum;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        if (at <= aim && aim < at + w[i]) {              // one token
            a.token[r] = (c * kBlock + threadIdx.x) * kPiece + i;
            if (a.logprob) a.logprob[r] = (float)(weight.down(k[i]) - log((double)all / kOne));
        }
        at += w[i];
    }
}

}  // namespace

hipError_t launch_sample(const void* logits, int type, int64_t stride, int R, int V, const qail_sampling& s, const float* u, int32_t* token, float* logprob,
                         uint32_t* errors, hipStream_t st) {
    const SampleArgs a = {logits, stride, V, s, u, token, logprob, errors};
    const bool aligned = stride % (type == QAIL_LOGITS_BF16 ? 8 : 4) == 0 || R == 1;
    const auto of_type = [&](auto bf16) {
        constexpr bool kBf16 = decltype(bf16)::value;
        return !aligned ? sample_kernel<kBf16, false, 0> : V <= kChunk ? sample_kernel<kBf16, true, 1> : V <= 4 * kChunk ? sample_kernel<kBf16, true, 4> : sample_kernel<kBf16, true, 0>;
    };
    const auto kernel = type == QAIL_LOGITS_BF16 ? of_type(std::true_type{}) : of_type(std::false_type{});
    hipLaunchKernelGGL(kernel, dim3((unsigned)R), dim3(kBlock), 0, st, a);
    return hipGetLastError();
}

}  // namespace qail
