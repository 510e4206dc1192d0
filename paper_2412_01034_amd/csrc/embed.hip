// Rows of a table of embeddings, and the gradient of that lookup.
//
// The gradient adds up the rows of dh that belong to a token.  Atomics would add them in any order, so the tokens are sorted first (stable: a token's rows stay
// in the order of their places), and whoever writes row v of the gradient reads its rows one after the other.  A token that comes more than kPart times is
// added up in parts of kPart sorted places by other blocks before, whose sums are then added in their order. What is sorted are pairs (token, place).  Up to
// kTile of them are ranked by comparing each with all others, a wave a pair, over the whole chip (2312 tokens 4.8 us, 4096 6.2; by digits in one block 9.8 and
// 10.8).  More of them are sorted in tiles of kTile, 8 bits of the token at a time, whose pairs stay in LDS for all digits: equal digits are found by comparing
// lanes.  Up to kMergeTiles tiles are then merged by rank: a pair's place is its own tile's plus how many pairs of each other tile come before it, 12 probes a
// tile (24577 tokens: 11.7 and 6.1 us).  More of them are sorted digit by digit over all tiles: their counts, the counts' sums, and the move.
#include <algorithm>

#include "qail_internal.h"

namespace qail {

namespace {

// ------------------------------------------------------------------------------------------------- lookup --

// 8 values a thread and access; `lanes` (a power of two, at most 256) threads a row.  Bound by HBM: 6181 rows of 4096 in 15.7 us (4.6 TB/s), 16 in 2.6, which is the launch.
__global__ __launch_bounds__(256) void embed_kernel(const uint16_t* __restrict__ table, int V, int pieces, int lanes, const int32_t* __restrict__ ids, int T,
                                                    float scale, uint16_t* __restrict__ h, uint32_t* __restrict__ errors) {
    const int t = blockIdx.x * (256 / lanes) + threadIdx.x / lanes, lane = threadIdx.x & (lanes - 1);
    if (t >= T) return;
    const int id = ids[t];
    if (id < 0) return;
    uint4* const to = reinterpret_cast<uint4*>(h) + (size_t)t * pieces;
    if (id >= V) {
        if (lane == 0 && errors) atomicAdd(errors, 1u);
        for (int i = lane; i < pieces; i += lanes) to[i] = make_uint4(0, 0, 0, 0);
        return;
    }
    const uint4* const from = reinterpret_cast<const uint4*>(table) + (size_t)id * pieces;
    for (int i = lane; i < pieces; i += lanes) {
        float v[8];
        unpack8(from[i], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
        to[i] = pack8(v);
    }
}

// --------------------------------------------------------------------------------------------------- sort --

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / kWave;
constexpr int kRounds = 4;                              // pairs of a thread
constexpr int kTile = kSortBlock * kRounds;
constexpr int kDigits = 256;

struct SortShared {
    uint32_t count[kSortWaves][kDigits];                // of a wave's pairs; then how many stand in front of them in the tile
    uint32_t wave_sum[kSortWaves];
};

// Wave w of a block has pairs 256 w .. 256 w + 255 of its tile, round i the 64 from 64 i on, so that waves, rounds and lanes go by the
// order of the pairs.  rank[i]: how many of the wave's earlier pairs have the digit.  Leaves the waves' counts in sh.count.
__device__ __forceinline__ void rank_digits(SortShared& sh, const uint32_t* digit, const bool* held, uint32_t* rank) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    for (int i = lane; i < kDigits; i += kWave) sh.count[wave][i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        unsigned long long same = __ballot(held[i]);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const unsigned long long ones = __ballot((digit[i] >> b) & 1u);
            same &= (digit[i] >> b) & 1u ? ones : ~ones;
        }
        const uint32_t earlier = held[i] ? sh.count[wave][digit[i]] : 0;
        const uint32_t below = __popcll(same & ((1ull << lane) - 1));
        rank[i] = earlier + below;
        __builtin_amdgcn_wave_barrier();
        if (held[i] && below == 0) sh.count[wave][digit[i]] = earlier + __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
}

// Per digit the counts of the waves in front; returns, in threads 0 .. 255, the tile's count of digit threadIdx.x.
__device__ __forceinline__ uint32_t sum_waves(SortShared& sh) {
    uint32_t n = 0;
    if (threadIdx.x < kDigits) {
        uint32_t c[kSortWaves];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) c[w] = sh.count[w][threadIdx.x];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            sh.count[w][threadIdx.x] = n;
            n += c[w];
        }
    }
    return n;
}

__device__ __forceinline__ uint32_t sum_before(SortShared& sh, uint32_t v, uint32_t* total) {   // exclusive sums over the block's threads
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    uint32_t in = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t t = __shfl_up(in, o, kWave);
        if (lane >= o) in += t;
    }
    if (lane == kWave - 1) sh.wave_sum[wave] = in;
    __syncthreads();
    uint32_t front = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t t = sh.wave_sum[w];
        front += w < wave ? t : 0;
        all += t;
    }
    __syncthreads();
    *total = all;
    return front + in - v;
}

// A token's key: itself, or V for what has no row of the table, behind all others.
__device__ __forceinline__ uint32_t token_key(int id, int V) { return id < 0 || id >= V ? (uint32_t)V : (uint32_t)id; }

__device__ __forceinline__ int place_in_tile(int i) { return threadIdx.x / kWave * (kWave * kRounds) + i * kWave + threadIdx.x % kWave; }

__device__ __forceinline__ void report(const int32_t* ids, int n, int V, uint32_t* errors) {
    if (!errors) return;
    for (int i = threadIdx.x; i < n; i += kSortBlock)
        if (ids[i] >= V) atomicAdd(errors, 1u);
}

// Every tile by itself, all digits.
__global__ __launch_bounds__(kSortBlock) void embed_sort_tiles_kernel(const int32_t* __restrict__ ids, int T, int V, int passes, uint32_t* __restrict__ keys,
                                                                      uint32_t* __restrict__ places, uint32_t* __restrict__ errors) {
    __shared__ SortShared sh;
    __shared__ uint32_t start[kDigits], pair[2][kTile];
    const int first = blockIdx.x * kTile, n = min(kTile, T - first);
    report(ids + first, n, V, errors);
    uint32_t key[kRounds], place[kRounds], digit[kRounds], rank[kRounds];
    bool held[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        place[i] = place_in_tile(i);
        held[i] = (int)place[i] < n;
        key[i] = held[i] ? token_key(ids[first + place[i]], V) : 0;
    }
    for (int pass = 0; pass < passes; ++pass) {
#pragma unroll
        for (int i = 0; i < kRounds; ++i) digit[i] = (key[i] >> (8 * pass)) & 255u;
        rank_digits(sh, digit, held, rank);
        uint32_t all;
        const uint32_t count = sum_waves(sh), before = sum_before(sh, count, &all);
        if (threadIdx.x < kDigits) start[threadIdx.x] = before;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kRounds; ++i)
            if (held[i]) {
                const uint32_t to = start[digit[i]] + sh.count[threadIdx.x / kWave][digit[i]] + rank[i];
                pair[0][to] = key[i];
                pair[1][to] = place[i];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kRounds; ++i)
            if (held[i]) key[i] = pair[0][place_in_tile(i)], place[i] = pair[1][place_in_tile(i)];
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kRounds; ++i)
        if (held[i]) keys[first + place_in_tile(i)] = key[i], places[first + place_in_tile(i)] = first + place[i];
}

// One tile: a wave compares a pair with all others.  Bound by the vector unit: T^2 comparisons of two instructions.
__global__ __launch_bounds__(kSortBlock) void embed_rank_kernel(const int32_t* __restrict__ ids, int T, int V, uint32_t* __restrict__ keys, uint32_t* __restrict__ places,
                                                                uint32_t* __restrict__ errors) {
    __shared__ __attribute__((aligned(16))) uint32_t all[kTile];
    if (blockIdx.x == 0) report(ids, T, V, errors);
    for (int i = threadIdx.x; i < (T + 3) / 4 * 4; i += kSortBlock) all[i] = i < T ? token_key(ids[i], V) : 0xFFFFFFFFu;
    __syncthreads();
    const int i = blockIdx.x * kSortWaves + threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (i >= T) return;
    const uint32_t key = all[i];
    uint32_t to = 0;
#pragma unroll 2
    for (int j = 4 * lane; j < T; j += 4 * kWave) {   // what stands in front counts if it is no larger, what stands behind if it is smaller
        const uint4 k = *reinterpret_cast<const uint4*>(&all[j]);
        to += (k.x < key + (j < i)) + (k.y < key + (j + 1 < i)) + (k.z < key + (j + 2 < i)) + (k.w < key + (j + 3 < i));
    }
#pragma unroll
    for (int o = 1; o < kWave; o *= 2) to += __shfl_xor(to, o, kWave);
    if (lane == 0) keys[to] = key, places[to] = i;
}

// How many of n ascending keys are below v.
__device__ __forceinline__ int below(const uint32_t* keys, int n, uint32_t v) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (keys[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

constexpr int kMergeTiles = 16;

// Sorted tiles into one list: kMergeTiles lanes a pair, each with a tile of its own, so that a pair waits for 12 trips to the L2 and not for as many per tile (24577 tokens
// 13.4 -> 6.1 us).
__global__ __launch_bounds__(256) void embed_merge_kernel(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ places, int T, uint32_t* __restrict__ keys_to,
                                                          uint32_t* __restrict__ places_to) {
    const int i = blockIdx.x * (256 / kMergeTiles) + threadIdx.x / kMergeTiles, s = threadIdx.x % kMergeTiles;
    if (i >= T) return;
    const int tile = i / kTile, first = s * kTile;
    const uint32_t key = keys[i];
    int to = s == tile ? i - first : first < T ? below(keys + first, min(kTile, T - first), s < tile ? key + 1 : key) : 0;
#pragma unroll
    for (int o = 1; o < kMergeTiles; o *= 2) to += __shfl_xor(to, o, kWave);
    if (s == 0) keys_to[to] = key, places_to[to] = places[i];
}

// Many tiles, one digit: the tiles' counts, [digit][tile] ...  (keys == NULL: the first digit, of ids)
__global__ __launch_bounds__(kSortBlock) void embed_count_kernel(const int32_t* __restrict__ ids, const uint32_t* __restrict__ keys, int T, int V, int shift,
                                                                 uint32_t* __restrict__ counts, uint32_t* __restrict__ errors) {
    __shared__ uint32_t count[kDigits];
    const int first = blockIdx.x * kTile, n = min(kTile, T - first);
    if (!keys) report(ids + first, n, V, errors);
    if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kSortBlock) {
        const uint32_t key = keys ? keys[first + i] : token_key(ids[first + i], V);
        atomicAdd(&count[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (threadIdx.x < kDigits) counts[(size_t)threadIdx.x * gridDim.x + blockIdx.x] = count[threadIdx.x];
}
// ... their sums in place (one block) ...
__global__ __launch_bounds__(kSortBlock) void embed_starts_kernel(uint32_t* __restrict__ counts, int n) {
    __shared__ SortShared sh;
    uint32_t front = 0;
    for (int i0 = 0; i0 < n; i0 += kSortBlock) {
        const int i = i0 + threadIdx.x;
        const uint32_t c = i < n ? counts[i] : 0;
        uint32_t all;
        const uint32_t before = sum_before(sh, c, &all);
        if (i < n) counts[i] = front + before;
        front += all;
    }
}
// ... and the move.
__global__ __launch_bounds__(kSortBlock) void embed_move_kernel(const int32_t* __restrict__ ids, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ places,
                                                                int T, int V, int shift, const uint32_t* __restrict__ starts, uint32_t* __restrict__ keys_to,
                                                                uint32_t* __restrict__ places_to) {
    __shared__ SortShared sh;
    uint32_t key[kRounds], place[kRounds], digit[kRounds], rank[kRounds];
    bool held[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int at = blockIdx.x * kTile + place_in_tile(i);
        held[i] = at < T;
        key[i] = !held[i] ? 0 : keys ? keys[at] : token_key(ids[at], V);
        place[i] = !held[i] ? 0 : keys ? places[at] : (uint32_t)at;
        digit[i] = (key[i] >> shift) & 255u;
    }
    rank_digits(sh, digit, held, rank);
    sum_waves(sh);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRounds; ++i)
        if (held[i]) {
            const uint32_t to = starts[(size_t)digit[i] * gridDim.x + blockIdx.x] + sh.count[threadIdx.x / kWave][digit[i]] + rank[i];
            keys_to[to] = key[i];
            places_to[to] = place[i];
        }
}

// --------------------------------------------------------------------------------------------------- sums --

constexpr int kPart = 32;       // sorted places of a part
constexpr int kMostRows = 16;   // rows of the gradient of a block, at most: with 64, 32000 x 4096 takes 147 us instead of 129 (24577 tokens), as blocks differ in their tokens
constexpr int kListed = 1024;   // places of a block's rows that it keeps in LDS

struct SumArgs {
    const uint32_t* keys;       // sorted
    const uint32_t* places;
    const uint16_t* dh;
    float* dtable;
    float* parts;               // [parts][2][K]
    int T, V, K, accumulate;
    float scale;
    int rows, lanes;            // of a block; threads that share a row, 4 columns each (a power of two)
};

// below() by a whole wave: 64 probes at a time, so three or four trips to memory instead of fifteen.
__device__ __forceinline__ int below_by_wave(const uint32_t* keys, int n, uint32_t v) {
    const int lane = threadIdx.x % kWave;
    int lo = 0, hi = n;
    while (lo < hi) {
        const int step = (hi - lo + kWave - 1) / kWave, at = lo + (lane + 1) * step - 1;   // the last of each of 64 runs
        const int c = __popcll(__ballot(at < hi && keys[at < hi ? at : hi - 1] < v));
        lo += c * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}

// The sum of the rows of dh at places[0 .. n), four columns a thread, eight rows requested at a time; behind the last one that row again (kShort: nothing, for
// sums of a row or two).
template <bool kShort, typename Places>
__device__ __forceinline__ f32x4_t sum_rows(const SumArgs& g, Places places, int n, int col) {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; i += 8) {
        uint2 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!kShort || i + e < n) v[e] = *reinterpret_cast<const uint2*>(g.dh + (size_t)places(kShort ? i + e : min(i + e, n - 1)) * g.K + col);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n)
                s += f32x4_t{__builtin_bit_cast(float, v[e].x << 16), __builtin_bit_cast(float, v[e].x & 0xFFFF0000u), __builtin_bit_cast(float, v[e].y << 16),
                             __builtin_bit_cast(float, v[e].y & 0xFFFF0000u)};
    }
    return s;
}

// Part i has sorted places kPart i .. and two sums: of the token that its first place belongs to, and of its last place's if that is another; each
// only where the token comes more than kPart times.
__global__ __launch_bounds__(256) void embed_parts_kernel(const SumArgs g) {
    const int across = (g.K + 1023) / 1024, part = blockIdx.x / across, lane = threadIdx.x % kWave;
    const int a = part * kPart, b = min(g.T, a + kPart);
    static_assert(kPart <= kWave, "a wave sees a part at once");
    const uint32_t key = g.keys[min(a + lane, b - 1)], head = __builtin_amdgcn_readfirstlane(key), tail = __builtin_amdgcn_readlane(key, kPart - 1);
    const int end = a + __popcll(__ballot(a + lane < b && key == head)), begin = b - __popcll(__ballot(a + lane < b && key == tail));   // in the part
    // more than kPart places of one token: the part's first or last and one kPart farther on
    const bool long_head = head < (uint32_t)g.V && ((end > kPart && g.keys[end - 1 - kPart] == head) || (a + kPart < g.T && g.keys[a + kPart] == head));
    const bool long_tail = tail != head && tail < (uint32_t)g.V && begin + kPart < g.T && g.keys[begin + kPart] == tail;
    const int col = blockIdx.x % across * 1024 + 4 * threadIdx.x;
    if (col >= g.K) return;
    const auto put = [&](int which, int from, int to) {
        *reinterpret_cast<f32x4_t*>(g.parts + ((size_t)part * 2 + which) * g.K + col) = sum_rows<false>(g, [&](int i) { return g.places[from + i]; }, to - from, col);
    };
    if (long_head) put(0, a, end);
    if (long_tail) put(1, begin, b);
}

// A block writes `rows` rows, whose tokens it finds by itself.  Bound by HBM: 32000 x 4096 with 2312 tokens in 100 us (5.4 TB/s), with 24577 in 128.  kStream:
// the gradient is written past the caches.
template <bool kStream>
__global__ __launch_bounds__(256, 8) void embed_rows_kernel(const SumArgs g) {
    __shared__ int start[kMostRows + 1], ends[2];
    __shared__ uint32_t listed[kListed];
    const int across = (g.K + 4 * g.lanes - 1) / (4 * g.lanes), v0 = blockIdx.x / across * g.rows, rows = min(g.rows, g.V - v0);
    // where the rows' tokens begin: the first and the last one's by two waves, the others' from the keys between
    if (threadIdx.x < 2 * kWave) {
        const int which = threadIdx.x / kWave, at = below_by_wave(g.keys, g.T, (uint32_t)(v0 + (which ? rows : 0)));
        if (threadIdx.x % kWave == 0) ends[which] = at;
    }
    __syncthreads();
    const int lo = ends[0], hi = ends[1];
    if (hi - lo <= kListed) {
        for (int i = lo + threadIdx.x; i <= hi; i += 256) {   // place i begins all rows above the key before it, up to its own
            const int from = i == lo ? 0 : (int)g.keys[i - 1] - v0 + 1, to = i == hi ? rows : (int)g.keys[i] - v0;
            for (int v = from; v <= to; ++v) start[v] = i;
            if (i < hi) listed[i - lo] = g.places[i];
        }
    } else if ((int)threadIdx.x <= rows) {
        start[threadIdx.x] = lo + below(g.keys + lo, hi - lo, (uint32_t)(v0 + threadIdx.x));
    }
    __syncthreads();
    const int col = 4 * (blockIdx.x % across * g.lanes + (threadIdx.x & (g.lanes - 1))), groups = 256 / g.lanes;
    if (col >= g.K) return;
    for (int i = threadIdx.x / g.lanes; i < rows; i += groups) {
        const int a = start[i], b = start[i + 1];
        if (a == b && g.accumulate) continue;
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
        if (b - a > kPart) {
            const int last = (b - 1) / kPart;
            for (int part = a / kPart; part <= last; part += 8) {
                f32x4_t t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = min(part + e, last), which = at * kPart < a;   // the token begins inside the part
                    t[e] = *reinterpret_cast<const f32x4_t*>(g.parts + ((size_t)at * 2 + which) * g.K + col);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (part + e <= last) s += t[e];
            }
        } else if (hi - lo <= kListed) {
            s = sum_rows<true>(g, [&](int k) { return listed[a - lo + k]; }, b - a, col);
        } else {
            s = sum_rows<true>(g, [&](int k) { return g.places[a + k]; }, b - a, col);
        }
        s *= g.scale;
        f32x4_t* const to = reinterpret_cast<f32x4_t*>(g.dtable + (size_t)(v0 + i) * g.K + col);
        if (g.accumulate) s += *to;
        if constexpr (kStream) __builtin_nontemporal_store(s, to);
        else *to = s;
    }
}

constexpr size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// A gradient that no cache holds (256 MB) is written past them, where it would push out dh: 32000 x 4096 with 2312 tokens 114 -> 103 us, the sums of parts before it
// 10 -> 7.
constexpr size_t kStreamFrom = (size_t)256 << 20;

struct Places {   // of the workspace
    int tiles, parts;
    size_t pairs, counts, sums, bytes;
    Places(int K, int T) {
        tiles = (T + kTile - 1) / kTile;
        parts = T > kPart ? (T + kPart - 1) / kPart : 0;
        pairs = round256((size_t)T * 4);                              // keys, places, and both again where several tiles are sorted
        counts = pairs * (tiles > 1 ? 4 : 2);
        sums = counts + (tiles > kMergeTiles ? round256((size_t)kDigits * tiles * 4) : 0);
        bytes = sums + (size_t)parts * 2 * K * 4;
    }
};

}  // namespace

hipError_t launch_embed(const uint16_t* table, int V, int K, const int32_t* ids, int T, float scale, uint16_t* h, uint32_t* errors, hipStream_t st) {
    const int pieces = K / 8;
    int lanes = 1;
    while (lanes < pieces && lanes < 256) lanes *= 2;
    const int rows = 256 / lanes;
    hipLaunchKernelGGL(embed_kernel, dim3((unsigned)((T + rows - 1) / rows)), dim3(256), 0, st, table, V, pieces, lanes, ids, T, scale, h, errors);
    return hipGetLastError();
}

size_t embed_back_workspace(int K, int T) { return std::max<size_t>(256, Places(K, T).bytes); }

hipError_t launch_embed_back(const int32_t* ids, const uint16_t* dh, int T, float scale, int V, int K, bool accumulate, float* dtable, uint32_t* errors, void* ws,
                             hipStream_t st) {
    const Places at(K, T);
    char* const w = static_cast<char*>(ws);
    uint32_t* pair[4];
    for (int i = 0; i < 4; ++i) pair[i] = reinterpret_cast<uint32_t*>(w + i * at.pairs);
    uint32_t* const counts = reinterpret_cast<uint32_t*>(w + at.counts);
    int passes = 1;
    while (passes < 4 && (V >> (8 * passes)) != 0) ++passes;   // keys are 0 .. V
    SumArgs g = {pair[0], pair[1], dh, dtable, reinterpret_cast<float*>(w + at.sums), T, V, K, accumulate, scale, 1, 1};
    while (4 * g.lanes < K && g.lanes < 256) g.lanes *= 2;
    // eight blocks a compute unit, and a row for each group of threads that shares one (below K = 64 there are more groups than rows: the others' threads have none)
    const int across = (K + 4 * g.lanes - 1) / (4 * g.lanes), groups = 256 / g.lanes;
    g.rows = (int)std::min<long long>(kMostRows, std::max<long long>(groups, (long long)V * across / (8 * device_cu_count())));
    if (at.tiles == 1) {
        hipLaunchKernelGGL(embed_rank_kernel, dim3((T + kSortWaves - 1) / kSortWaves), dim3(kSortBlock), 0, st, ids, T, V, pair[0], pair[1], errors);
    } else if (at.tiles > 1 && at.tiles <= kMergeTiles) {
        hipLaunchKernelGGL(embed_sort_tiles_kernel, dim3(at.tiles), dim3(kSortBlock), 0, st, ids, T, V, passes, pair[2], pair[3], errors);
        hipLaunchKernelGGL(embed_merge_kernel, dim3((T * kMergeTiles + 255) / 256), dim3(256), 0, st, pair[2], pair[3], T, pair[0], pair[1]);
    } else if (at.tiles > kMergeTiles) {
        for (int pass = 0; pass < passes; ++pass) {
            const uint32_t* const keys = pass ? pair[2 * (pass & 1)] : nullptr;
            const uint32_t* const places = pass ? pair[2 * (pass & 1) + 1] : nullptr;
            uint32_t* const keys_to = pair[2 * (~pass & 1)];
            uint32_t* const places_to = pair[2 * (~pass & 1) + 1];
            hipLaunchKernelGGL(embed_count_kernel, dim3(at.tiles), dim3(kSortBlock), 0, st, ids, keys, T, V, 8 * pass, counts, errors);
            hipLaunchKernelGGL(embed_starts_kernel, dim3(1), dim3(kSortBlock), 0, st, counts, kDigits * at.tiles);
            hipLaunchKernelGGL(embed_move_kernel, dim3(at.tiles), dim3(kSortBlock), 0, st, ids, keys, places, T, V, 8 * pass, counts, keys_to, places_to);
            g.keys = keys_to, g.places = places_to;
        }
    }
    if (at.parts) hipLaunchKernelGGL(embed_parts_kernel, dim3((unsigned)at.parts * ((K + 1023) / 1024)), dim3(256), 0, st, g);
    const auto rows_kernel = (size_t)V * K * sizeof(float) >= kStreamFrom ? embed_rows_kernel<true> : embed_rows_kernel<false>;
    hipLaunchKernelGGL(rows_kernel, dim3((unsigned)((V + g.rows - 1) / g.rows) * across), dim3(256), 0, st, g);
    return hipGetLastError();
}

}  // namespace qail
