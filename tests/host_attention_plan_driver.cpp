// Walks through the plans of the attention over the paged cache (csrc/attention_plan.h) on the host: over everything that the interface
// accepts a launch stays below 2^32 threads, and the grid has a block for every tile of rows.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "attention_plan.h"

using namespace qail;

namespace {

#define CHECK(cond, ...)                                          \
    do {                                                          \
        if (!(cond)) {                                            \
            std::printf("failed: %s: ", #cond);                   \
            std::printf(__VA_ARGS__);                             \
            std::printf("\n");                                    \
            std::exit(1);                                         \
        }                                                         \
    } while (0)

// The limits that the interface states.
bool accepted(const qail_kv_cache& c, const qail_requests& b, int q_heads) {
    return b.tokens < (1 << 24) && b.requests <= (1 << 20) && (long long)b.max_pages * c.page_size <= (1 << 30) &&
           (long long)b.requests * c.heads <= (1 << 22) && (long long)b.tokens * q_heads <= (1 << 30) && q_heads <= 65535;
}

void threads(const qail_kv_cache& c, const qail_requests& b, int q_heads, int cus) {
    const AttentionPlan p = plan_attention(c, b, q_heads, cus);
    const long long limit = 1ll << 32;   // of a launch, in each direction
    const double tiles = p.tiles ? (double)p.row_tiles * c.heads * p.most * 256 : 0;
    CHECK(tiles < limit, "%d requests, %d tokens, %d heads to %d, up to %d of %d: %d tiles, %d shares", b.requests, b.tokens, q_heads, c.heads, b.max_new, b.max_len,
          p.row_tiles, p.most);
    CHECK(!p.stream || p.blocks * 256ll < limit, "%d requests, %d heads", b.requests, c.heads);
    CHECK(!p.stream || (p.join_tokens >= 1 && p.join_tokens <= 16), "%u", p.join_tokens);
    CHECK(!p.tiles || (p.row_tiles >= 1 && p.most >= 1 && p.most <= 64 && p.chunk > 0), "%d tiles, %d shares of %d", p.row_tiles, p.most, p.chunk);
    CHECK(p.tiles || p.stream, "%d tokens", b.tokens);
    // partial results: fp32 and at most 128 values each
    CHECK((double)attention_places(p, b, q_heads) * (128 * 4 + 8) < 1e13, "%d tokens", b.tokens);
}

// Tiles of rows of requests with so many new tokens.
void covered(const std::vector<int>& fresh, int group, int heads, int max_new, int cus) {
    qail_kv_cache c{};
    c.heads = heads;
    c.page_size = 64;
    c.head_dim = 128;
    qail_requests b{};
    b.requests = (int)fresh.size();
    b.max_pages = 100;
    b.max_len = 6400;
    b.max_new = max_new;
    for (int n : fresh) b.tokens += n;
    if (b.tokens == 0) return;
    const AttentionPlan p = plan_attention(c, b, heads * group, cus);
    if (!p.tiles) return;
    long long tiles = 0;
    for (int n : fresh) tiles += tiles_of(Request{0, n, 6400}, group, p.stream ? kStreamRows + 1 : 1, kTileRows);
    CHECK(tiles <= p.row_tiles, "%lld tiles of %d requests, %d planned", tiles, b.requests, p.row_tiles);
}

}  // namespace

int main() {
    std::mt19937 rng(11);
    auto pick = [&](long long lo, long long hi) { return std::uniform_int_distribution<long long>(lo, hi)(rng); };
    auto wide = [&](int bits) { return (int)pick(1, 1ll << pick(0, bits)); };   // spread over the logarithm
    const int steps[][5] = {   // requests, heads, tokens, max_new, max_len
        {32768, 8, 100, 100, 65536}, {65536, 8, 40, 17, 40000}, {1 << 20, 4, 100, 100, 1 << 20}, {1 << 20, 4, 17, 17, 1 << 30}, {1 << 20, 1, (1 << 24) - 1, 40, 1 << 30}, {1, 1, 17, 17, 1 << 30}};
    for (const auto& s : steps) {
        qail_kv_cache c{};
        c.heads = s[1];
        c.page_size = 1024;
        c.head_dim = 128;
        qail_requests b{};
        b.requests = s[0];
        b.max_pages = 1 << 20;
        b.tokens = s[2];
        b.max_new = s[3];
        b.max_len = s[4];
        CHECK(accepted(c, b, s[1]), "a step of the list is not accepted");
        threads(c, b, s[1], 256);
    }
    int seen = 0;
    for (int i = 0; i < 400000; ++i) {
        qail_kv_cache c{};
        c.heads = wide(15);
        c.page_size = 1 << pick(4, 10);
        c.head_dim = pick(0, 1) ? 64 : 128;
        qail_requests b{};
        b.requests = wide(20);
        b.max_pages = wide(26);
        b.tokens = wide(24);
        b.max_new = pick(0, 3) ? wide(24) : b.tokens;
        b.max_len = wide(30);
        const long long q_heads = (long long)c.heads * wide(6);
        if (q_heads > 65535 || !accepted(c, b, (int)q_heads)) continue;
        threads(c, b, (int)q_heads, 256);
        ++seen;
    }
    CHECK(seen > 10000, "%d plans", seen);
    for (int i = 0; i < 20000; ++i) {
        std::vector<int> fresh;
        const int kind = (int)pick(0, 3);   // many that wait, whole tiles, a token more than whole tiles, anything
        for (int r = (int)pick(1, 40); r > 0; --r) fresh.push_back(kind == 0 ? (pick(0, 7) ? 0 : wide(9)) : kind == 1 ? (int)pick(0, 3) * 128 : kind == 2 ? (int)pick(0, 3) * 128 + 1 : wide(9) - 1);
        int most = 0;
        for (int n : fresh) most = std::max(most, n);
        const int groups[] = {1, 2, 7, 16, 24};
        covered(fresh, groups[pick(0, 4)], (int)pick(1, 4), pick(0, 2) ? most : wide(10), 256);
    }
    std::printf("plans: ok\n");
    return 0;
}
