// The next token of each row of logits: temperature, top-k, top-p and min-p, then the inverse of the distribution at a given random number.
//
// Every filter keeps a leading part of the tokens in the order (falling logit, rising number).  That
// part is written as a border: all tokens above a value and the first `ties` of those with it.  A border is found without a sort: the
// tokens are counted, or their weights added up, in bins of 1 / 64 of an octave of the weight; the bin in which the sum passes its aim
// is found, and the few tokens in it are searched by their keys, kRanges parts of their range at a time; where they are more than kList (equal logits) the
// whole row is.
//
// Weights are exponentials in 64 bits, as whole multiples of 2^-44: sums of whole numbers do not depend on their order, and a token is found as in
// exact arithmetic but for those 2^-44.  In 32 bits the sums would be off by 2^-24 or so of themselves, and of 32000 tokens without a filter one row in some thousands
// would get a neighbouring one.  An exponential is a table of 512 and a polynomial; 64 bits cost no more cycles than 32 here.
//
// One block a row, whose values stay in registers up to 32768 tokens; a longer row is read again in every pass, and lies in L2 by then.  Several blocks a row
// would have to meet in memory, which this call has none of.  Bound by instructions and by the meetings of the 16 waves, not by memory: one row of 32000 takes
// 18 us (15.6 of 40 thousand cycles are the exponentials of top-p, thirty instructions each), 256 rows 33, 48 rows of 131072 63 to 92: as
// the slowest of them, 35 to 50 us where little is kept and 90 where top-p keeps nearly all of a flat row, whose exponentials are computed twice.
#include <type_traits>

#include "qail_internal.h"

namespace qail {

namespace {

constexpr int kBlock = 1024, kWaves = kBlock / kWave;
constexpr int kPiece = 8;                          // neighbouring tokens of a thread
constexpr int kChunk = kBlock * kPiece;            // tokens of a pass over the block
constexpr int kMostChunks = (1 << 18) / kChunk + 1;   // (a row may begin inside a piece)
constexpr int kGroup = 4;                          // chunks that are looked at together
static_assert(kGroup * kPiece == 32, "a bit for each of a thread's tokens of a group");
constexpr int kBins = 3 * kBlock;
constexpr int kParts = 512;                        // of an octave
constexpr int kBinParts = 8;                       // of a bin
constexpr int kLowestPart = -45 * kParts;          // of a weight of 2^-45; below, weights are 0
constexpr int kLowestBin = (kLowestPart - 1) / kBinParts - 1;
static_assert(-kLowestBin < kBins, "bins for all parts");
constexpr double kOne = 17592186044416.0;          // 2^44: the weight of the largest logit
constexpr int kList = kBlock;                      // tokens of a bin that are listed: one a thread
constexpr int kRanges = kBlock;
constexpr int kKept = 8 * kBlock;                  // kept tokens of a group that are listed
static_assert(kGroup * kChunk <= 1 << 16, "their numbers");

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

// v plus, in each lane, the value of the lane that kDpp names (0 where there is none, or the row is not in kRows).
template <int kDpp, int kRows>
__device__ __forceinline__ u64 add_from(u64 v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, kDpp, kRows, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), kDpp, kRows, 0xF, false);
    return v + ((u64)hi << 32 | lo);
}
__device__ __forceinline__ u64 row_scan(u64 v) {     // inclusive sums over 16 lanes
    v = add_from<0x111, 0xF>(v);                     // row_shr:1, 2, 4, 8
    v = add_from<0x112, 0xF>(v);
    v = add_from<0x114, 0xF>(v);
    return add_from<0x118, 0xF>(v);
}
__device__ __forceinline__ u64 wave_scan(u64 v) {    // ... over the wave
    v = row_scan(v);
    v = add_from<0x142, 0xA>(v);                     // row_bcast:15 into rows 1 and 3
    return add_from<0x143, 0xC>(v);                  // row_bcast:31 into rows 2 and 3
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane) {
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

struct Shared {
    u64 bins[kBins];
    uint32_t counts[kBins];
    u64 wave_sum[kWaves];
    u64 segment[kMostChunks * kWaves];       // weight above the border of 512 neighbouring tokens each
    uint32_t ties[kMostChunks * kWaves];     // ... and how many lie on it
    double part[kParts];                     // 2^(i / 512)
    union {
        u64 ranges[kRanges];                 // of keys
        uint32_t list[kList];                // numbers of tokens
        uint16_t kept[kKept];                // ... from a group's first one
    };
    float wave_most[kWaves];
    u64 before;                              // what the chosen bin or segment has in front of it
    int chosen, ties_before, listed, border_ties;
    uint32_t first, border_key, equal;
};

// Inclusive sums over the block's threads in their order; `total`: of all of them.  The threads have met before.
__device__ __forceinline__ u64 block_scan(Shared& sh, u64 v, u64& total) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const u64 in = wave_scan(v);
    if (lane == kWave - 1) sh.wave_sum[wave] = in;
    __syncthreads();
    static_assert(kWaves == 16, "a row of lanes holds the waves' sums");
    const u64 waves = row_scan(sh.wave_sum[lane % 16]);
    total = lane_of(waves, 15);
    const u64 front = wave > 0 ? lane_of(waves, wave - 1) : 0;
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

// The values of a row, 8 neighbouring tokens of a thread in each of its chunks; minus infinity behind the row.  kChunks of them stay in registers; 0: none.
// A row that begins inside 16 bytes is read from their beginning on, so that all loads but the last are wide: its tokens are numbered from there (`skip` is the first one's
// number), and the values in front of it, which are those of the row before, are minus infinity as well.
template <bool kBf16, int kChunks>
struct Row {
    const uint8_t* p;
    int end, skip, chunks;
    float kept[kChunks > 0 ? kChunks : 1][kPiece];

    __device__ __forceinline__ void values(int c, float* f) const {
        const int j = (c * kBlock + threadIdx.x) * kPiece;
        if (j + kPiece <= end) {
            if constexpr (kBf16) {
                unpack8(*reinterpret_cast<const uint4*>(p + 2ll * j), f);
            } else {
                const float4 a = *reinterpret_cast<const float4*>(p + 4ll * j), b = *reinterpret_cast<const float4*>(p + 4ll * j + 16);
                f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) f[i] = j + i >= end ? -__builtin_inff() : at(j + i);
        }
        if (j < skip) {   // (a row that is shorter than its skip has no piece but this)
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (i < skip) f[i] = -__builtin_inff();
        }
    }
    __device__ __forceinline__ Row(const uint8_t* first, int V) {
        skip = (int)(reinterpret_cast<uintptr_t>(first) & 15u) / (kBf16 ? 2 : 4);
        p = first - skip * (kBf16 ? 2 : 4);
        end = V + skip;
        chunks = (end + kChunk - 1) / kChunk;
        static_assert(kChunks <= 4, "one by one: a loop is unrolled too late for registers");
        if constexpr (kChunks > 0) values(0, kept[0]);
        if constexpr (kChunks > 1) values(1, kept[1]);
        if constexpr (kChunks > 2) values(2, kept[2]);
        if constexpr (kChunks > 3) values(3, kept[3]);
    }
    // f(chunk, values) for the kGroup chunks from `first` on, those behind the row among them (minus infinity): unrolled, the loads in front.  For passes that
    // do little with a value.
    template <typename F>
    __device__ __forceinline__ void group(int first, F f) const {
        if constexpr (kChunks > 0) {
            if constexpr (kChunks > 0) f(0, kept[0]);
            if constexpr (kChunks > 1) f(1, kept[1]);
            if constexpr (kChunks > 2) f(2, kept[2]);
            if constexpr (kChunks > 3) f(3, kept[3]);
        } else {
            float v[kGroup][kPiece];
            values(first, v[0]);
            values(first + 1, v[1]);
            values(first + 2, v[2]);
            values(first + 3, v[3]);
            f(first, v[0]);
            f(first + 1, v[1]);
            f(first + 2, v[2]);
            f(first + 3, v[3]);
        }
    }
    // The same for the whole row.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        if constexpr (kChunks > 0) {
            group(0, f);
        } else {
            for (int c = 0; c < chunks; c += kGroup) group(c, f);
        }
    }
    // One bit for each of a thread's tokens of a group, the first one's the highest.
    template <typename P>
    __device__ __forceinline__ uint32_t select(int first, P chosen) const {
        uint32_t bits = 0;
        group(first, [&](int, const float* x) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i) bits = bits << 1 | (chosen(x[i]) ? 1u : 0u);
        });
        return kChunks > 0 ? bits << (32 - kPiece * kChunks) : bits;
    }
    __device__ __forceinline__ float at(uint32_t number) const {
        if constexpr (kBf16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[number]);
        else return reinterpret_cast<const float*>(p)[number];
    }
    // f(chunk, values) for chunks first .. end - 1 from memory.  For passes with exponentials: unrolled over the kept chunks their code is long.
    template <typename F>
    __device__ __forceinline__ void each_again(int first, int end, F f) const {
#pragma unroll 1
        for (int c = first; c < end; ++c) {
            float v[kPiece];
            values(c, v);
            f(c, v);
        }
    }
};

struct Weight {
    double most, inverse, scale;     // the largest logit, 1 / temperature, 512 log2(e) / temperature
    double step;                     // 1 / scale
    float low;                       // the least value from one part below kLowestPart on: below it weights are 0
    const double* part;
    __device__ __forceinline__ Weight(float most_, float temperature, const double* part_) : most(most_), part(part_) {
        inverse = 1.0 / (double)temperature;
        scale = inverse * 738.65986093514926;
        step = (double)temperature * 0.0013538030870311431;
        const double end = most + (kLowestPart - 1) * step;
        low = fmaxf((float)end, -3.4028235e38f);
        if ((double)low < end) low = value_of(key_of(low) + 1);
    }
    __device__ __forceinline__ double down(float x) const { return ((double)x - most) * inverse; }
    // x >= low lies n + rest parts of an octave from the largest logit, n the nearest whole number (adding 1.5 * 2^52 rounds to it, in the low bits).
    __device__ __forceinline__ void parts(float x, int& n, double& rest) const {
        constexpr double kRound = 6755399441055744.0;
        const double d = (double)x - most, r = fma(d, scale, kRound);
        n = (int)(uint32_t)__builtin_bit_cast(u64, r);
        rest = fma(d, scale, kRound - r);
    }
    // The weight of n parts and a rest: 2^(n / 512) from the table, 2^(rest / 512) by its series (to 2^-46).  Adding 2^52 rounds to a whole number, which is
    // then the low bits.
    __device__ __forceinline__ u64 of(int n, double rest) const {
        constexpr double c = 0.0013538030870311431;   // ln(2) / 512
        double e = fma(rest, c * c * c / 6, c * c / 2);
        e = fma(rest, e, c);
        e = fma(rest, e, 1.0);
        const double octave = __builtin_bit_cast(double, (u64)(uint32_t)(((1023 + 44) << 20) + ((n & -kParts) << (20 - 9))) << 32);
        return __builtin_bit_cast(u64, fma(part[n & (kParts - 1)] * e, octave, 4503599627370496.0)) & ((1ull << 52) - 1);
    }
    __device__ __forceinline__ u64 operator()(float x) const {
        int n;
        double rest;
        parts(x, n, rest);
        const u64 w = of(n, rest);
        return x < low ? 0 : w;
    }
};
__device__ __forceinline__ int bin_of(int part) { return -(part >> 3); }   // 0 for the largest logits
static_assert(kBinParts == 1 << 3 && kParts == 1 << 9, "shifts");

// The numbers of the tokens that a wave's threads have chosen from a group (Row::select), counted from chunk `origin` on, into list[0 .. most), in any order; sh.listed
// counts them all.
template <typename Number>
__device__ __forceinline__ void append(Shared& sh, Number* list, int most, int first, int origin, uint32_t bits) {
    const int lane = threadIdx.x % kWave, mine = __popc(bits);
    const int upto = (int)wave_scan((u64)mine), total = __builtin_amdgcn_readlane(upto, kWave - 1);
    if (total == 0) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&sh.listed, total);
    at = __builtin_amdgcn_readfirstlane(at) + upto - mine;
    for (; bits != 0; ++at) {
        const int i = __clz(bits);
        bits &= ~(0x80000000u >> i);
        if (at < most) list[at] = (Number)(((first - origin + i / kPiece) * kBlock + threadIdx.x) * kPiece + i % kPiece);
    }
}

struct Border {
    float value;  // what lies above it is kept
    int ties;     // ... and so many tokens with that value
};

// The shortest leading part of some tokens whose sum is at least `aim` (> 0 and no more than all of them have), by ranges of their keys.  each(f): f(key, what the
// token adds to the sum) for a thread's tokens, all of which have keys from low to base; one: what a token of a key adds.
template <typename Each, typename One>
__device__ __forceinline__ Border border_by_keys(Shared& sh, Each each, uint32_t base, uint32_t low, u64 aim, One one) {
    uint32_t width = base - low;                      // base: the largest key of the range; width: how far it goes below
    for (;;) {
        const int shift = max(0, 22 - __builtin_clz(width | 1));   // width >> shift < kRanges = 2^10
        sh.ranges[threadIdx.x] = 0;
        __syncthreads();
        each([&](uint32_t key, u64 adds) __attribute__((always_inline)) {
            if (key <= base && base - key <= width) atomicAdd(&sh.ranges[(base - key) >> shift], adds);
        });
        __syncthreads();
        find<1>(sh, [&](int i) { return sh.ranges[i]; }, [&](u64) { return aim; });
        const uint32_t at = sh.chosen;
        aim -= sh.before;
        __syncthreads();
        base -= at << shift;
        if (shift == 0) return {value_of(base), (int)((aim - 1) / one(base) + 1)};
        width = min(width - (at << shift), (1u << shift) - 1);
    }
}

// The same of n <= kList listed tokens, one a thread.
template <bool kCount>
__device__ __forceinline__ Border border_of_list(Shared& sh, int n, bool held, uint32_t key, u64 mine, uint32_t base, uint32_t low, u64 aim, const Weight& weight) {
    if (n > kWave)
        return border_by_keys(
            sh,
            [&](auto f) __attribute__((always_inline)) {
                if (held) f(key, kCount ? 1 : mine);
            },
            base, low, aim, [&](uint32_t k) { return kCount ? 1 : weight(value_of(k)); });
    // few: the first wave compares them with each other, which saves the meetings of a search (one row of 32000 20.7 -> 18.3 us)
    if (threadIdx.x < kWave) {
        u64 front = 0;                                // what lies above
        uint32_t equal = 0;
        const u64 adds = !held ? 0 : kCount ? 1 : mine;
        const int whose = held ? (int)key : 0;
        for (int i = 0; i < n; ++i) {
            const uint32_t other = (uint32_t)__builtin_amdgcn_readlane(whose, i);
            const u64 w = lane_of(adds, i);
            front += other > key ? w : 0;
            equal += other == key;
        }
        if (held && front < aim && aim <= front + equal * adds) sh.border_key = key, sh.border_ties = (int)((aim - front - 1) / adds + 1);   // all of one value say the same
    }
    __syncthreads();
    const Border b = {value_of(sh.border_key), sh.border_ties};
    __syncthreads();
    return b;
}

// The border in a bin of weights, whose tokens are to count (kCount) or weigh `aim` > 0; ahead: what those up to the border weigh (with kWeigh).  false: the bin has
// more than about kList tokens.
template <bool kCount, bool kWeigh, typename R>
__device__ __forceinline__ bool border_in_bin(Shared& sh, const R& row, int bin, const Weight& weight, u64 aim, Border& b, u64& ahead) {
    // the bin's values, and two keys more at either end for the roundings of its bounds; they are looked at one by one below
    const uint32_t hi = key_of((float)(weight.most + (kBinParts - 0.5 - kBinParts * bin) * weight.step)) + 2;
    const uint32_t lo = key_of((float)(weight.most - (0.5 + kBinParts * bin) * weight.step)) - 2;
    const float from = value_of(max(lo, kLowest + 1)), to = value_of(min(hi, kHighest - 1));
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
    for (int g = 0; g < row.chunks; g += kGroup)
        append(sh, sh.list, kList, g, 0, row.select(g, [&](float x) { return __builtin_amdgcn_fmed3f(x, from, to) == x; }));
    __syncthreads();
    const int n = sh.listed;
    if (n > kList) {
        __syncthreads();
        return false;
    }
    uint32_t key = 0;
    u64 mine = 0;
    bool held = false;
    if ((int)threadIdx.x < n) {
        const float x = row.at(sh.list[threadIdx.x]);
        int part;
        double rest;
        weight.parts(x, part, rest);
        held = x >= weight.low && bin_of(part) == bin;
        key = key_of(x);
        mine = weight.of(part, rest);
    }
    __syncthreads();                                  // the list has been read: the ranges lie there as well
    b = border_of_list<kCount>(sh, n, held, key, mine, key_of(to), key_of(from), aim, weight);
    if constexpr (kWeigh) {
        block_scan(sh, held && key > key_of(b.value) ? mine : 0, ahead);
        ahead += (u64)b.ties * weight(b.value);
    }
    return true;
}

template <bool kBf16, int kChunks>
__global__ __launch_bounds__(kBlock) void sample_kernel(const SampleArgs a) {
    __shared__ Shared sh;
    const int r = blockIdx.x, V = a.V, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const Row<kBf16, kChunks> row(static_cast<const uint8_t*>(a.logits) + (long long)r * a.stride * (kBf16 ? 2 : 4), V);
    const float temperature = a.s.temperature ? a.s.temperature[r] : 1.f, top_p = a.s.top_p ? a.s.top_p[r] : 1.f, min_p = a.s.min_p ? a.s.min_p[r] : 0.f;
    const float u = a.u[r];
    const int top_k = a.s.top_k ? a.s.top_k[r] : 0;

    for (int i = threadIdx.x; i < kBins; i += kBlock) sh.bins[i] = 0, sh.counts[i] = 0;
    if (threadIdx.x < kParts) sh.part[threadIdx.x] = exp2((double)threadIdx.x / kParts);
    if (threadIdx.x == 0) sh.first = 0xFFFFFFFFu;
    float mine = -__builtin_inff();
    bool bad = false;
    row.each([&](int, const float* x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            mine = fmaxf(mine, x[i]);                                  // (passes by NaN)
            bad |= x[i] != x[i];
        }
    });
    float m = bad ? __builtin_inff() : mine;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
    if (lane == 0) sh.wave_most[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sh.wave_most[w]);
    const bool numbers = m >= -3.4028235e38f && m <= 3.4028235e38f && temperature >= 0.f && temperature <= 3.4028235e38f && top_p == top_p && min_p == min_p;
    if (!numbers || (temperature > 0.f && !(u >= 0.f && u < 1.f))) {   // the same for the whole block, as all that follows
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = __builtin_nanf("");
            if (a.errors) atomicAdd(a.errors, 1u);
        }
        return;
    }
    if (temperature == 0.f || min_p > 1.f || top_k == 1) {             // the first of the order
        for (int g = 0; g < row.chunks; g += kGroup) {
            const uint32_t bits = row.select(g, [&](float x) { return x == m; });
            const int i = bits != 0 ? __clz(bits) : 0;
            if (bits != 0) atomicMin(&sh.first, ((g + i / kPiece) * kBlock + threadIdx.x) * kPiece + i % kPiece);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            a.token[r] = (int32_t)sh.first - row.skip;
            if (a.logprob) a.logprob[r] = 0.f;
        }
        return;
    }

    const Weight weight(m, temperature, sh.part);
    const bool by_count = top_k > 0 && top_k < V, by_share = top_p < 1.f;
    Border b = {-__builtin_inff(), 0};
    u64 kept = 0;                      // what the first top_k weigh
    const auto weigh = [&]() __attribute__((always_inline)) {   // from the row itself
        u64 some = 0;
        row.each_again(0, row.chunks, [&](int, const float* x) __attribute__((always_inline)) {
#pragma unroll 1
            for (int i = 0; i < kPiece; ++i)
                if (x[i] > b.value) some += weight(x[i]);
        });
        block_scan(sh, some, kept);
        kept += (u64)b.ties * weight(b.value);
    };
    const auto all_keys = [&](bool weights) {   // of the row, for where a bin has too many tokens
        return [&, weights](auto f) __attribute__((always_inline)) {
            row.each_again(0, row.chunks, [&](int, const float* x) __attribute__((always_inline)) {
#pragma unroll 1
                for (int i = 0; i < kPiece; ++i)
                    if (x[i] >= weight.low) f(key_of(x[i]), weights ? weight(x[i]) : 1);
            });
        };
    };
    // the tokens' weights in bins
    const auto fill = [&]() __attribute__((always_inline)) {
        row.each_again(0, row.chunks, [&](int, const float* x) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (x[i] >= weight.low) {
                    int n;
                    double rest;
                    weight.parts(x[i], n, rest);
                    atomicAdd(&sh.bins[bin_of(n)], weight.of(n, rest));
                }
        });
        __syncthreads();
    };
    const bool few = by_count && top_k <= kList;       // top_p's border is then looked for among the first top_k alone
    if (by_share && !few) fill();
    if (by_count) {
        row.each([&](int, const float* x) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (x[i] >= weight.low) {
                    int n;
                    double rest;
                    weight.parts(x[i], n, rest);
                    atomicAdd(&sh.counts[bin_of(n)], 1u);
                }
        });
    }
    __syncthreads();
    if (by_count) {
        const u64 counted = find<kBins / kBlock>(sh, [&](int i) { return (u64)sh.counts[i]; }, [&](u64) { return (u64)top_k; });
        if (counted >= (u64)top_k) {   // else all that has a weight is among the first top_k
            const int bin = sh.chosen;
            const u64 aim = (u64)top_k - sh.before;
            __syncthreads();
            if (!(by_share && !few ? border_in_bin<true, true>(sh, row, bin, weight, aim, b, kept) : border_in_bin<true, false>(sh, row, bin, weight, aim, b, kept))) {
                b = border_by_keys(sh, all_keys(false), key_of(m), kLowest, (u64)top_k, [&](uint32_t) { return 1; });
                if (by_share && !few) weigh();
            } else if (by_share && !few) {
                u64 some = 0, front;
                for (int i = threadIdx.x; i < bin; i += kBlock) some += sh.bins[i];
                block_scan(sh, some, front);
                kept += front;
            }
        } else {
            __syncthreads();
        }
    }
    bool by_list = false;
    if (by_share && few) {
        if (b.ties > 0) {
            if (threadIdx.x == 0) sh.listed = 0;
            __syncthreads();
            for (int g = 0; g < row.chunks; g += kGroup) append(sh, sh.list, kList, g, 0, row.select(g, [&](float x) { return x >= b.value; }));
            __syncthreads();
            const int n = sh.listed;
            by_list = n <= kList;                       // else many are equal to the last one
            if (by_list) {
                const bool held = (int)threadIdx.x < n;
                const float x = held ? row.at(sh.list[threadIdx.x]) : 0.f;
                const u64 mine = held ? weight(x) : 0;
                block_scan(sh, x > b.value ? mine : 0, kept);   // (nobody writes the list before all have read it)
                kept += (u64)b.ties * weight(b.value);
                const double share = ceil((double)top_p * (double)kept);
                b = border_of_list<false>(sh, n, held, key_of(x), mine, key_of(m), key_of(b.value), share > 1.0 ? (u64)share : 1, weight);
            } else {
                __syncthreads();
                weigh();
            }
        }
        if (!by_list) fill();
    }
    if (by_share && !by_list) {
        u64 aim = 0, none;
        find<kBins / kBlock>(sh, [&](int i) { return sh.bins[i]; }, [&](u64 total) {
            const double share = ceil((double)top_p * (double)(b.ties > 0 ? kept : total));
            return aim = share > 1.0 ? (u64)share : 1;
        });
        const int bin = sh.chosen;
        const u64 rest = aim - sh.before;
        __syncthreads();
        // (the border of top_k, which may lie in the same bin, is not reached: the aim is less than what is in front of it weighs)
        if (!border_in_bin<false, false>(sh, row, bin, weight, rest, b, none))
            b = border_by_keys(sh, all_keys(true), key_of(m), kLowest, aim, [&](uint32_t k) { return weight(value_of(k)); });
    }

    // The kept weight of every 512 neighbouring tokens, then the one in which the sum passes u.  Where few are kept they are listed first, so that no
    // exponential is computed for the others beside them.
    const bool filtered = by_count || by_share || min_p > 0.f;
    const double least = min_p > 0.f ? log((double)min_p) : -__builtin_inf();
    const u64 on = b.ties > 0 && weight.down(b.value) >= least ? weight(b.value) : 0;
    float low = fmaxf(weight.low, b.ties > 0 ? value_of(key_of(b.value) + 1) : b.value);   // what is kept beside the ties; of min_p's border two steps below for its rounding
    if (min_p > 0.f) low = fmaxf(low, value_of(max(key_of((float)(weight.most + least * (double)temperature)), kLowest + 3) - 2));
    const float from = on > 0 ? fminf(low, b.value) : low;   // (between them there may be what min_p does not keep)
    const int segments = row.chunks * kWaves;           // at most 528
    static_assert(kMostChunks * kWaves <= kBlock, "one a thread");
    if ((int)threadIdx.x < segments) sh.segment[threadIdx.x] = 0, sh.ties[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.equal = 0;
    for (int g = 0; g < row.chunks; g += kGroup) {
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        if (filtered) append(sh, sh.kept, kKept, g, g, row.select(g, [&](float x) { return x >= from; }));
        __syncthreads();
        const int listed = sh.listed;
        if (filtered && listed <= kKept) {
            for (int i = threadIdx.x; i < listed; i += kBlock) {
                const uint32_t number = g * kChunk + sh.kept[i], at = number / (kWave * kPiece);
                const float x = row.at(number);
                if (x < low) {
                    if (x == b.value) atomicAdd(&sh.ties[at], 1u), atomicAdd(&sh.equal, 1u);
                } else if (weight.down(x) >= least) {
                    atomicAdd(&sh.segment[at], weight(x));
                }
            }
        } else {
            row.each_again(g, min(g + kGroup, row.chunks), [&](int c, const float* x) __attribute__((always_inline)) {
                u64 some = 0;
#pragma unroll
                for (int i = 0; i < kPiece; ++i) {
                    const u64 w = weight(x[i]);
                    some += x[i] >= low && weight.down(x[i]) >= least ? w : 0;
                }
                some = lane_of(wave_scan(some), kWave - 1);
                if (lane == 0) sh.segment[c * kWaves + wave] = some;
            });
            if (b.ties > 0) {
                const uint32_t bits = row.select(g, [&](float x) { return x == b.value; });
                u64 four = 0;                           // a chunk's count in 16 bits each
#pragma unroll
                for (int c = 0; c < kGroup; ++c) four |= (u64)__popc(bits >> (24 - kPiece * c) & 0xFFu) << (16 * c);
                four = lane_of(wave_scan(four), kWave - 1);
                if (lane < kGroup && g + lane < row.chunks) {
                    const uint32_t c = four >> (16 * lane) & 0xFFFF;
                    sh.ties[(g + lane) * kWaves + wave] = c;
                    if (c > 0) atomicAdd(&sh.equal, c);
                }
            }
        }
        __syncthreads();
    }
    const bool held = (int)threadIdx.x < segments;
    const u64 above = held ? sh.segment[threadIdx.x] : 0, room = b.ties;
    u64 ties_front = 0, here = above, all;
    if (sh.equal <= room) {                             // all of them are kept
        here += held ? sh.ties[threadIdx.x] * on : 0;
    } else if (b.ties > 0) {
        const u64 equal = held ? sh.ties[threadIdx.x] : 0, ties_upto = block_scan(sh, equal, all);
        ties_front = ties_upto - equal;
        here += (min(ties_upto, room) - min(ties_front, room)) * on;
    }
    const u64 upto = block_scan(sh, here, all);
    const u64 aim = (u64)((double)u * (double)all);
    if (upto - here <= aim && aim < upto) sh.chosen = threadIdx.x, sh.before = upto - here, sh.ties_before = (int)ties_front;
    __syncthreads();
    if (wave != sh.chosen % kWaves) return;
    const int c = sh.chosen / kWaves;
    float x[kPiece];
    row.values(c, x);
    u64 equal_here = 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) equal_here += x[i] == b.value;
    u64 number = sh.ties_before + wave_scan(equal_here) - equal_here;
    u64 w[kPiece], sum = 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        w[i] = x[i] >= low ? (weight.down(x[i]) >= least ? weight(x[i]) : 0) : x[i] == b.value && number < room ? on : 0;
        number += x[i] == b.value;
        sum += w[i];
    }
    u64 at = sh.before + wave_scan(sum) - sum;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
        if (at <= aim && aim < at + w[i]) {              // one token
            a.token[r] = (c * kBlock + threadIdx.x) * kPiece + i - row.skip;
            if (a.logprob) a.logprob[r] = (float)(weight.down(x[i]) - log((double)all / kOne));
        }
        at += w[i];
    }
}

}  // namespace

hipError_t launch_sample(const void* logits, int type, int64_t stride, int R, int V, const qail_sampling& s, const float* u, int32_t* token, float* logprob,
                         uint32_t* errors, hipStream_t st) {
    const SampleArgs a = {logits, stride, V, s, u, token, logprob, errors};
    const bool aligned = stride % (type == QAIL_LOGITS_BF16 ? 8 : 4) == 0 || R == 1;
    const int length = V + (aligned ? 0 : kPiece - 1);   // with what a row may skip
    const auto of_type = [&](auto bf16) {
        constexpr bool kBf16 = decltype(bf16)::value;
        return length <= kChunk ? sample_kernel<kBf16, 1> : length <= 4 * kChunk ? sample_kernel<kBf16, 4> : sample_kernel<kBf16, 0>;
    };
    const auto kernel = type == QAIL_LOGITS_BF16 ? of_type(std::true_type{}) : of_type(std::false_type{});
    hipLaunchKernelGGL(kernel, dim3((unsigned)R), dim3(kBlock), 0, st, a);
    return hipGetLastError();
}

}  // namespace qail
