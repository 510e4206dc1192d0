// The next token of each row of logits: temperature, top-k, top-p and min-p, then the inverse of the distribution at a given random number.
//
// With key(x) the bits of x in an order of unsigned numbers, every filter keeps a leading part of the tokens in the order (falling key, rising
// number), which is written as a border: all keys above `key` and the first `ties` tokens with that key.  The border is found without a sort:
// a histogram over at most kBins equal parts of the keys' range, the part in which the count or the weight passes its aim, then
// the same inside that part.  Weights are exp in 64 bits, as whole multiples of 2^-44: sums of whole numbers do not depend on their order,
// and a token is found as in exact arithmetic but for those 2^-44 (with weights of 32 bits one token in a few thousand rows is another one).
// One block a row; a row is read from memory again in every pass, and lies in L2 by then.
#include "qail_internal.h"

namespace qail {

namespace {

constexpr int kBlock = 1024, kWaves = kBlock / kWave;
constexpr int kPiece = 8;                          // neighbouring tokens of a thread
constexpr int kChunk = kBlock * kPiece;            // tokens of a pass over the block
constexpr int kMostChunks = (1 << 18) / kChunk;
constexpr int kBins = 2 * kBlock;
constexpr double kOne = 17592186044416.0;          // 2^44: the weight of the largest logit

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
    u64 wave_sum[kWaves];
    u64 segment[kMostChunks * kWaves];       // weight above the border of 512 neighbouring tokens each
    uint32_t ties[kMostChunks * kWaves];     // ... and how many lie on it
    uint32_t wave_key[kWaves];
    u64 before;                              // what the chosen bin or segment has in front of it
    int chosen, ties_before;
    uint32_t first;
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

template <bool kBf16, bool kAligned>
struct Row {
    const uint8_t* p;
    int V;
    // Keys of tokens j .. j + 7; kLowest behind the row.
    __device__ __forceinline__ void keys(int j, uint32_t* k) const {
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
};

struct Weight {
    double most, inverse;
    __device__ __forceinline__ double down(uint32_t key) const { return ((double)value_of(key) - most) * inverse; }
    __device__ __forceinline__ u64 operator()(uint32_t key) const { return (u64)(exp(down(key)) * kOne + 0.5); }
};

struct Border {
    uint32_t key;
    int ties;     // tokens with that key that are kept
};

// The shortest leading part of the tokens inside `in` whose count (kCount) or weight is at least `aim` (> 0 and no more than all of them have).
template <bool kCount, typename R>
__device__ Border narrow(Shared& sh, const R& row, int chunks, uint32_t top, uint32_t low, Border in, const Weight& weight, u64 aim) {
    uint32_t base = top;                              // the largest key of the range
    uint32_t width = top - low;                       // ... and how far it goes below
    for (;;) {
        const int shift = max(0, 21 - __builtin_clz(width | 1));   // width >> shift < kBins = 2^11
        for (int i = threadIdx.x; i < kBins; i += kBlock) sh.bins[i] = 0;
        __syncthreads();
        for (int c = 0; c < chunks; ++c) {
            uint32_t k[kPiece];
            row.keys(c * kChunk + threadIdx.x * kPiece, k);
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const bool here = k[i] <= base && base - k[i] <= width && k[i] > in.key;
                if (here) atomicAdd(&sh.bins[(base - k[i]) >> shift], kCount ? 1ull : weight(k[i]));
            }
        }
        __syncthreads();
        if (threadIdx.x == 0 && in.ties > 0 && in.key <= base && base - in.key <= width)
            sh.bins[(base - in.key) >> shift] += (u64)in.ties * (kCount ? 1ull : weight(in.key));
        __syncthreads();
        const u64 a = sh.bins[2 * threadIdx.x], b = sh.bins[2 * threadIdx.x + 1];
        u64 total;
        const u64 upto = block_scan(sh, a + b, total), front = upto - a - b;
        if (front < aim && aim <= upto) {             // one thread
            const bool second = front + a < aim;
            sh.chosen = 2 * threadIdx.x + second;
            sh.before = front + (second ? a : 0);
        }
        __syncthreads();
        const uint32_t bin = sh.chosen;
        aim -= sh.before;
        __syncthreads();
        base -= bin << shift;
        if (shift == 0) return {base, (int)(kCount ? aim : (aim - 1) / weight(base) + 1)};
        width = min(width - (bin << shift), (1u << shift) - 1);
    }
}

template <bool kBf16, bool kAligned>
__global__ __launch_bounds__(kBlock) void sample_kernel(const SampleArgs a) {
    __shared__ Shared sh;
    const int r = blockIdx.x, V = a.V, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int chunks = (V + kChunk - 1) / kChunk;
    const Row<kBf16, kAligned> row = {static_cast<const uint8_t*>(a.logits) + (long long)r * a.stride * (kBf16 ? 2 : 4), V};
    const float temperature = a.s.temperature ? a.s.temperature[r] : 1.f, top_p = a.s.top_p ? a.s.top_p[r] : 1.f, min_p = a.s.min_p ? a.s.min_p[r] : 0.f;
    const float u = a.u[r];
    const int top_k = a.s.top_k ? a.s.top_k[r] : 0;

    // the largest key, and where it stands first
    uint32_t most = 0, place = 0;
    for (int c = 0; c < chunks; ++c) {
        uint32_t k[kPiece];
        const int j = c * kChunk + threadIdx.x * kPiece;
        row.keys(j, k);
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (k[i] > most) most = k[i], place = j + i;
    }
    uint32_t m = most;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
    if (lane == 0) sh.wave_key[wave] = m;
    if (threadIdx.x == 0) sh.first = 0xFFFFFFFFu;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = max(m, sh.wave_key[w]);
    const bool numbers = m > kLowest && m < kHighest && temperature >= 0.f && temperature <= 3.4e38f && top_p == top_p && min_p == min_p;
    if (!numbers || (temperature > 0.f && !(u >= 0.f && u < 1.f))) {   // the same for the whole block
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = __builtin_nanf("");
            if (a.errors) atomicAdd(a.errors, 1u);
        }
        return;
    }
    if (most == m) atomicMin(&sh.first, place);
    __syncthreads();
    if (temperature == 0.f || min_p > 1.f) {
        if (threadIdx.x == 0) {
            a.token[r] = (int32_t)sh.first;
            if (a.logprob) a.logprob[r] = 0.f;
        }
        return;
    }

    const Weight weight = {(double)value_of(m), 1.0 / (double)temperature};
    Border b = {kLowest, 0};
    if (top_k > 0 && top_k < V) b = narrow<true>(sh, row, chunks, m, kLowest, {0, 0}, weight, (u64)top_k);
    if (top_p < 1.f) {
        u64 mine = 0, total;
        for (int c = 0; c < chunks; ++c) {
            uint32_t k[kPiece];
            row.keys(c * kChunk + threadIdx.x * kPiece, k);
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (k[i] > b.key) mine += weight(k[i]);
        }
        block_scan(sh, mine, total);
        total += (u64)b.ties * weight(b.key);
        const double share = ceil((double)top_p * (double)total);
        b = narrow<false>(sh, row, chunks, m, b.key, b, weight, share > 1.0 ? (u64)share : 1);
    }
    const double least = min_p > 0.f ? log((double)min_p) : -__builtin_inf();

    // the kept weight of every 512 neighbouring tokens, then the one in which the sum passes u
    const u64 on = b.ties > 0 && weight.down(b.key) >= least ? weight(b.key) : 0;
    for (int c = 0; c < chunks; ++c) {
        uint32_t k[kPiece];
        row.keys(c * kChunk + threadIdx.x * kPiece, k);
        u64 mine = 0;
        uint32_t ties = 0;
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
            if (k[i] > b.key && weight.down(k[i]) >= least) mine += weight(k[i]);
            ties += k[i] == b.key;
        }
        mine = shfl64(wave_scan(mine), kWave - 1);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) ties += __shfl_xor((int)ties, o, kWave);
        if (lane == 0) sh.segment[c * kWaves + wave] = mine, sh.ties[c * kWaves + wave] = ties;
    }
    __syncthreads();
    const int segments = chunks * kWaves;               // at most 512: one a thread
    const bool held = (int)threadIdx.x < segments;
    const u64 above = held ? sh.segment[threadIdx.x] : 0;
    const u64 equal = held ? sh.ties[threadIdx.x] : 0;
    u64 all;
    const u64 ties_upto = block_scan(sh, equal, all), ties_front = ties_upto - equal;
    const u64 room = b.ties;
    const u64 kept = above + ((ties_upto < room ? ties_upto : room) - (ties_front < room ? ties_front : room)) * on;
    const u64 upto = block_scan(sh, kept, all);
    const u64 aim = (u64)((double)u * (double)all);
    if (upto - kept <= aim && aim < upto) sh.chosen = threadIdx.x, sh.before = upto - kept, sh.ties_before = (int)ties_front;
    __syncthreads();
    if (wave != sh.chosen % kWaves) return;
    const int j = (sh.chosen / kWaves * kBlock + threadIdx.x) * kPiece;
    uint32_t k[kPiece];
    row.keys(j, k);
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
            a.token[r] = j + i;
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
    const auto kernel = type == QAIL_LOGITS_BF16 ? (aligned ? sample_kernel<true, true> : sample_kernel<true, false>)
                                                 : (aligned ? sample_kernel<false, true> : sample_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)R), dim3(kBlock), 0, st, a);
    return hipGetLastError();
}

}  // namespace qail
