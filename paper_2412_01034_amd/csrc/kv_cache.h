// The cache of keys and values and the requests of a step, as the kernels see them.
#pragma once

#include "qail_internal.h"

namespace qail {

struct CacheArgs {
    void *k, *v;
    float *k_scale, *v_scale;
    const int32_t *table, *starts, *lens;
    uint32_t* errors;
    int num_pages, heads, page_shift, max_pages, requests, tokens;
};

inline CacheArgs cache_args(const qail_kv_cache& c, const qail_requests& b, uint32_t* errors) {
    return CacheArgs{c.k, c.v, c.k_scale, c.v_scale, b.page_table, b.q_start, b.kv_len, errors,
                     c.num_pages, c.heads, __builtin_ctz((unsigned)c.page_size), b.max_pages, b.requests, b.tokens};
}

__device__ __forceinline__ void report(const CacheArgs& a) {
    if (a.errors) atomicAdd(a.errors, 1u);
}

// A request's rows of the step's tensors and its length, with what the arrays may hold turned into something that stays inside
// the buffers: n = 0 where q_start is bad, len cut to what the page table can hold.  (This and what follows is for the host
// too, which walks through it in the tests.)
struct Request {
    int start, n, len;
};
__host__ __device__ __forceinline__ Request request(const CacheArgs& a, int r, bool& bad) {
    const int s = a.starts[r], e = a.starts[r + 1], len = a.lens[r];
    const long long room = (long long)a.max_pages << a.page_shift;
    const bool rows = s >= 0 && e >= s && e <= a.tokens, keys = len >= 0 && (long long)len <= room;
    bad = !rows || !keys;
    Request q{0, 0, 0};
    if (rows) q = Request{s, e - s, keys ? len : len < 0 ? 0 : (int)room};   // room < len fits 31 bits
    return q;
}

// The request that has row t: the last one whose rows start at or before it.  A wave looks at 64 starts at a time, with no load waiting
// for another (a binary search would wait for eight in a row at 256 requests).
__device__ __forceinline__ int request_of(const CacheArgs& a, int t) {
    int before = 0;
    for (int i = 0; i < a.requests; i += kWave) {
        const int r = i + (int)threadIdx.x % kWave;
        before += __popcll(__ballot(r < a.requests && a.starts[r] <= t));
    }
    return before - 1;
}

// Keys that rows row0 .. row0 + count - 1 of a request see (its last row's), `group` rows a token.
__host__ __device__ __forceinline__ int keys_of(const Request& q, int group, int row0, int count) {
    const int rows = q.n * group, last = row0 + count < rows ? row0 + count - 1 : rows - 1;
    const int keys = q.len - q.n + last / group + 1;
    return keys > 0 ? keys : 0;
}

// Tiles of `height` rows that a request's new tokens make, `group` rows each; none for fewer than min_rows.
__host__ __device__ __forceinline__ int tiles_of(const Request& q, int group, int min_rows, int height) {
    const int rows = q.n * group;
    return rows < min_rows ? 0 : (rows + height - 1) / height;
}

// Reports requests whose q_start is bad: they have no rows, so no block comes across them.
__device__ __forceinline__ void report_rows(const CacheArgs& a) {
    for (int r = threadIdx.x; r < a.requests; r += blockDim.x) {
        bool bad;
        const Request q = request(a, r, bad);
        if (bad && q.n == 0) report(a);
    }
}

// Few rows: the work of a request for one head of the cache, in steps of kStepKeys keys for a tile of kStreamRows rows.  (Every tile of a
// request counts as many steps as its last.)
constexpr int kStreamRows = 16, kStepKeys = 128;
struct Steps {
    int tiles, steps;   // steps of each tile: at least one, which writes zeros where there is no key
};
__host__ __device__ __forceinline__ Steps steps_of(const Request& q, int group, int max_rows) {
    const int rows = q.n * group;
    if (rows == 0 || rows > max_rows) return Steps{0, 0};
    const int keys = keys_of(q, group, 0, rows), steps = (keys + kStepKeys - 1) / kStepKeys;
    return Steps{(rows + kStreamRows - 1) / kStreamRows, steps > 1 ? steps : 1};
}
// The steps of all requests, heads and tiles in a row are cut into equal shares, one a block.
__host__ __device__ __forceinline__ long long steps_of_a_share(long long total, int blocks, int least) {
    const long long s = (total + blocks - 1) / blocks;
    return s > least ? s : least;
}
// Where block b leaves its part of a tile whose steps begin at `begin`, if that is not all of it: a block can have two such tiles, one
// that has begun before it and one that goes on after it.
__host__ __device__ __forceinline__ long long place_of(long long begin, long long b, long long share) { return 2 * b + (begin >= b * share ? 1 : 0); }

// The request and the first row of tile `tile` of all of them, counted in the order of the requests; false past the last one.
__device__ __forceinline__ bool tile_of(const CacheArgs& a, int group, int min_rows, int height, int tile, int& r, int& row0, Request& q, bool& bad) {
    const int lane = threadIdx.x % kWave;
    for (int r0 = 0; r0 < a.requests; r0 += kWave) {
        bool bad_here = false;
        const Request here = r0 + lane < a.requests ? request(a, r0 + lane, bad_here) : Request{0, 0, 0};
        const int mine = tiles_of(here, group, min_rows, height);
        int sum = mine;   // of this lane's request and those before it
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int left = __shfl_up(sum, o, kWave);
            if (lane >= o) sum += left;
        }
        const unsigned long long past = __ballot(sum > tile);
        if (past) {
            const int at = __builtin_ctzll(past);
            r = r0 + at;
            row0 = (tile - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(mine, at))) * height;
            q = Request{__builtin_amdgcn_readlane(here.start, at), __builtin_amdgcn_readlane(here.n, at), __builtin_amdgcn_readlane(here.len, at)};
            bad = (__ballot(bad_here) >> at) & 1;
            return true;
        }
        tile -= __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    return false;
}

// Whether a token of a request can be written: its position is one that the page table and the table of angles (positions; 0: none) reach.
__host__ __device__ __forceinline__ bool has_slot(const Request& q, int t, int positions, int& at) {
    at = q.len - q.n + (t - q.start);   // below len: inside the page table
    return t >= q.start && t < q.start + q.n && at >= 0 && (positions == 0 || at < positions);
}

// Shares that `keys` are divided into: `chunk` each, at most `most` of them, of which the last takes what is left.
__host__ __device__ __forceinline__ int shares(int keys, int chunk, int most) {
    const int n = (keys + chunk - 1) / chunk;
    return n < 1 ? 1 : n > most ? most : n;
}
struct Range {
    int begin, end;
};
__host__ __device__ __forceinline__ Range share_of(int keys, int chunk, int count, int i) {
    return Range{i * chunk, i == count - 1 ? keys : (i + 1) * chunk};
}

__host__ __device__ __forceinline__ bool is_page(int p, int num_pages) { return (unsigned)p < (unsigned)num_pages; }

// The entry of the page table, as it is; looked at (below) when it is used, so that no load waits for the one before.
__device__ __forceinline__ int page_entry(const CacheArgs& a, int r, int index) { return a.table[(size_t)r * a.max_pages + index]; }

// A page's number in the cache: page 0, and `bad`, where an entry is none.
__device__ __forceinline__ int page_of(const CacheArgs& a, int entry, bool& bad) {
    const bool in = is_page(entry, a.num_pages);
    bad = bad || !in;
    return in ? entry : 0;
}

}  // namespace qail
