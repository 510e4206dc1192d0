// Division of labour of the attention over the paged cache (paged_attention.hip): which kernels run, over how many blocks, and how they share
// the keys.  Apart from the kernels, so that the host can walk through it.
#pragma once

#include <algorithm>

#include "kv_cache.h"

namespace qail {

constexpr int kTileRows = 128, kTileKeys = 64;   // many rows: of a block, and keys that it takes at a time

constexpr int stream_blocks(int head_dim) { return head_dim == 64 ? 3 : 2; }   // few rows: that a compute unit holds, by registers

// How a step is divided among blocks, by what the host knows: which kernels run (both where requests of few rows and of many may come
// together) and how they share the keys.
struct AttentionPlan {
    bool stream, tiles;
    int stream_rows;            // requests of up to so many rows are the stream's
    int shared, blocks, least;  // the stream's
    unsigned join_tokens;
    int row_tiles, chunk, most; // the tiles'
};

inline AttentionPlan plan_attention(const qail_kv_cache& c, const qail_requests& b, int q_heads, int cus) {
    AttentionPlan p{};
    const int group = q_heads / c.heads;
    const long long keys = std::max<long long>(1, std::min<long long>(b.max_len, (long long)b.max_pages * c.page_size));   // at most 2^30
    const long long most_rows = (long long)std::min(b.max_new, b.tokens) * group;
    p.stream = most_rows <= kStreamRows;
    p.tiles = !p.stream;
    if (p.tiles && b.requests > 1 && (long long)b.requests * b.max_new != b.tokens && group <= kStreamRows) p.stream = true;
    p.stream_rows = p.tiles ? (p.stream ? kStreamRows : 0) : INT32_MAX;
    if (p.stream) {
        // Shared steps cost a join, about 4 us together with what the kernel does for it; a block for each request and head costs the time of the
        // longest one, 1.6 us per step.  us, one / shared, uniform lengths: 32 units, 512 keys 8.9 / 10.9, 1024 keys 14.5 / 12, 16384 keys 224 / 49;
        // 256 units, 2048 keys 31 / 33, 4096 keys 66 / 55; 512 units, 1024 keys 26 / 31, 8192 keys 192 / 203, but of 500 to 8000
        // keys 153 / 128.
        const long long units = (long long)b.requests * c.heads;
        p.shared = keys > std::min(2048ll, 512 + 6 * units);
        p.blocks = p.shared ? cus * stream_blocks(c.head_dim) : (int)units;
        p.join_tokens = (unsigned)std::max(1, std::min({b.max_new, b.tokens, kStreamRows}));
        p.least = 2;   // of 1, 2, 3 and 4 the best or next to it from 1024 to 16384 keys
    }
    if (p.tiles) {
        // Each request with rows has at most one tile that is not full, and no more requests than tokens have rows.  That keeps the grid below 2^24 blocks (2^32
        // threads): tokens * q_heads / 128 + requests * heads is at most 2^23 + 2^22, and where keys are shared, `work` times `most` is below four blocks a unit.
        p.row_tiles = (int)((long long)b.tokens * group / kTileRows) + std::min(b.requests, b.tokens);
        const long long work = std::max(1ll, (long long)b.tokens * group / kTileRows) * c.heads;
        // Shares until there are two blocks a unit, of 512 keys or more (us with 128 / 256 / 512 / 1024: one prompt of 1049, 4 heads to 1 22 / 19 / 20 / 23; 40 rows behind 2560
        // keys, 8 to 2 21 / 19 / 21 / 28; 200 behind 12000, 8 to 1 54 / 54 / 38 / 37; two of 64 behind 4000 keys of 8 bits, 32 to 8 47 / 34 / 34 / 45), and 64 at most: the
        // join reads them all (32 rows behind 40000 keys, 8 to 1, 48 with 64 and 61 with 256; behind 100000 67 and 123).
        const long long n = std::max(1ll, std::min({(2ll * cus + work - 1) / work, 64ll, (keys + 511) / 512}));
        p.most = (int)n;
        p.chunk = (int)((keys + n - 1) / n + kTileKeys - 1) / kTileKeys * kTileKeys;
    }
    return p;
}

// Partial results that a call may leave.
inline size_t attention_places(const AttentionPlan& p, const qail_requests& b, int q_heads) {
    const size_t stream = p.stream && p.shared ? (size_t)2 * p.blocks * kStreamRows : 0, tiles = p.tiles && p.most > 1 ? (size_t)b.tokens * q_heads * p.most : 0;
    return std::max(stream, tiles);
}

}  // namespace qail
