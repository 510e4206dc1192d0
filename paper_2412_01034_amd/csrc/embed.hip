// Rows of a table of embeddings, and the gradient of that lookup.
//
// The gradient adds up the rows of dh that belong to a token.  Atomics would add them in any order, so the tokens are sorted first (stable: a
// token's rows stay in the order of their places), and whoever writes row v of the gradient reads its rows one after the other.  A token that comes
// more than kPart times is added up in parts of kPart sorted places by other blocks before, whose sums are then added in their order.
// What is sorted are pairs (token, place), 8 bits of the token at a time, in tiles of kTile: per tile the places of equal digits are
// counted by comparing lanes, the counts of all tiles are summed up, and the pairs move.  All tokens in one tile stay in LDS for all digits.
#include <algorithm>

#include "qail_internal.h"

namespace qail {

namespace {

// ------------------------------------------------------------------------------------------------- lookup --

// 8 values a thread and access; `lanes` (a power of two, at most 256) threads a row.  Bound by HBM.
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
    if (threadIdx.x < kDigits)
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = sh.count[w][threadIdx.x];
            sh.count[w][threadIdx.x] = n;
            n += c;
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

// All tokens in one tile: every digit in one launch.
__global__ __launch_bounds__(kSortBlock) void embed_sort_tile_kernel(const int32_t* __restrict__ ids, int T, int V, int passes, uint32_t* __restrict__ keys,
                                                                     uint32_t* __restrict__ places, uint32_t* __restrict__ errors) {
    __shared__ SortShared sh;
    __shared__ uint32_t start[kDigits], pair[2][kTile];
    report(ids, T, V, errors);
    uint32_t key[kRounds], place[kRounds], digit[kRounds], rank[kRounds];
    bool held[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        place[i] = place_in_tile(i);
        held[i] = (int)place[i] < T;
        key[i] = held[i] ? token_key(ids[place[i]], V) : 0;
    }
    for (int pass = 0; pass < passes; ++pass) {
#pragma unroll
        for (int i = 0; i < kRounds; ++i) digit[i] = (key[i] >> (8 * pass)) & 255u;
        rank_digits(sh, digit, held, rank);
        uint32_t all;
        const uint32_t n = sum_waves(sh), before = sum_before(sh, n, &all);
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
        if (held[i]) keys[place_in_tile(i)] = key[i], places[place_in_tile(i)] = place[i];
}

// Several tiles, one digit: the tiles' counts, [digit][tile] ...  (keys == NULL: the first digit, of ids)
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
constexpr int kRowsEach = 64;   // rows of the gradient of a block
constexpr int kCols = 1024;     // columns of a block: four a thread

struct SumArgs {
    const uint32_t* keys;       // sorted
    const uint32_t* places;
    const uint16_t* dh;
    float* dtable;
    float* parts;               // [parts][2][K]
    int T, V, K, accumulate;
    float scale;
};

// How many sorted keys are below v.
__device__ __forceinline__ int below(const uint32_t* keys, int T, uint32_t v) {
    int lo = 0, hi = T;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (keys[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// The sum of the rows at sorted places a .. b - 1, four columns a thread, eight rows requested at a time.
__device__ __forceinline__ float4 sum_rows(const SumArgs& g, int a, int b, int col) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = a; i < b; i += 8) {
        uint2 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = i + e < b ? i + e : b - 1;
            v[e] = *reinterpret_cast<const uint2*>(g.dh + (size_t)g.places[at] * g.K + col);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < b) {
                s.x += __builtin_bit_cast(float, v[e].x << 16);
                s.y += __builtin_bit_cast(float, v[e].x & 0xFFFF0000u);
                s.z += __builtin_bit_cast(float, v[e].y << 16);
                s.w += __builtin_bit_cast(float, v[e].y & 0xFFFF0000u);
            }
    }
    return s;
}

// Part i has sorted places kPart i .. and two sums: of the token that its first place belongs to, and of its last place's if that is another; each
// only where the token comes more than kPart times.
__global__ __launch_bounds__(256) void embed_parts_kernel(const SumArgs g) {
    __shared__ int at[6];
    const int across = (g.K + kCols - 1) / kCols, part = blockIdx.x / across;
    const int a = part * kPart, b = min(g.T, a + kPart);
    const uint32_t head = g.keys[a], tail = g.keys[b - 1];
    if (threadIdx.x < 4) {   // where both tokens begin and end
        const uint32_t v = threadIdx.x < 2 ? head : tail;
        at[threadIdx.x] = below(g.keys, g.T, v + threadIdx.x % 2);
    }
    __syncthreads();
    const int col = blockIdx.x % across * kCols + 4 * threadIdx.x;
    if (col >= g.K) return;
    float4* const to = reinterpret_cast<float4*>(g.parts + (size_t)part * 2 * g.K + col);
    if (head < (uint32_t)g.V && at[1] - at[0] > kPart) *to = sum_rows(g, a, min(b, at[1]), col);
    if (tail != head && tail < (uint32_t)g.V && at[3] - at[2] > kPart) to[g.K / 4] = sum_rows(g, at[2], b, col);
}

__global__ __launch_bounds__(256) void embed_rows_kernel(const SumArgs g) {
    __shared__ int start[kRowsEach + 1];
    const int across = (g.K + kCols - 1) / kCols, v0 = blockIdx.x / across * kRowsEach, rows = min(kRowsEach, g.V - v0);
    if ((int)threadIdx.x <= rows) start[threadIdx.x] = below(g.keys, g.T, (uint32_t)(v0 + threadIdx.x));
    __syncthreads();
    const int col = blockIdx.x % across * kCols + 4 * threadIdx.x;
    if (col >= g.K) return;
    for (int i = 0; i < rows; ++i) {
        const int a = start[i], b = start[i + 1];
        if (a == b && g.accumulate) continue;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (b - a <= kPart) {
            s = sum_rows(g, a, b, col);
        } else {
            for (int part = a / kPart; part * kPart < b; ++part) {
                const int which = part * kPart < a;   // the token begins inside the part
                const float4 t = *reinterpret_cast<const float4*>(g.parts + ((size_t)part * 2 + which) * g.K + col);
                s.x += t.x, s.y += t.y, s.z += t.z, s.w += t.w;
            }
        }
        s.x *= g.scale, s.y *= g.scale, s.z *= g.scale, s.w *= g.scale;
        float4* const to = reinterpret_cast<float4*>(g.dtable + (size_t)(v0 + i) * g.K + col);
        if (g.accumulate) {
            const float4 o = *to;
            s.x += o.x, s.y += o.y, s.z += o.z, s.w += o.w;
        }
        *to = s;
    }
}

constexpr size_t round256(size_t b) { return (b + 255) / 256 * 256; }

struct Places {   // of the workspace
    int tiles, parts;
    size_t pairs, counts, sums, bytes;
    Places(int K, int T) {
        tiles = (T + kTile - 1) / kTile;
        parts = T > kPart ? (T + kPart - 1) / kPart : 0;
        pairs = round256((size_t)T * 4);                              // keys, places, and both again where several tiles are sorted
        counts = pairs * (tiles > 1 ? 4 : 2);
        sums = counts + (tiles > 1 ? round256((size_t)kDigits * tiles * 4) : 0);
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
    SumArgs g = {pair[0], pair[1], dh, dtable, reinterpret_cast<float*>(w + at.sums), T, V, K, accumulate, scale};
    if (at.tiles == 1) {
        hipLaunchKernelGGL(embed_sort_tile_kernel, dim3(1), dim3(kSortBlock), 0, st, ids, T, V, passes, pair[0], pair[1], errors);
    } else if (at.tiles > 1) {
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
    const int across = (K + kCols - 1) / kCols;
    if (at.parts) hipLaunchKernelGGL(embed_parts_kernel, dim3((unsigned)at.parts * across), dim3(256), 0, st, g);
    hipLaunchKernelGGL(embed_rows_kernel, dim3((unsigned)((V + kRowsEach - 1) / kRowsEach) * across), dim3(256), 0, st, g);
    return hipGetLastError();
}

}  // namespace qail
