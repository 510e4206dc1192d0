// Walks through the index arithmetic of the paged cache's kernels (csrc/kv_cache.h) on the host: whatever the arrays of a step hold, rows,
// slots and shares of keys stay inside their buffers, and good arrays are taken as they are.
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "kv_cache.h"

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

struct Arrays {
    std::vector<int32_t> starts, lens;
    int tokens, max_pages, page_shift;
    CacheArgs args() const {
        CacheArgs a{};
        a.starts = starts.data();
        a.lens = lens.data();
        a.requests = (int)lens.size();
        a.tokens = tokens;
        a.max_pages = max_pages;
        a.page_shift = page_shift;
        return a;
    }
};

// The request that the kernels would find for row t.
int request_of(const Arrays& s, int t) {
    int before = 0;
    for (size_t r = 0; r < s.lens.size(); ++r) before += s.starts[r] <= t;
    return before - 1;
}

void walk(const Arrays& s, bool good) {
    const CacheArgs a = s.args();
    const long long room = (long long)s.max_pages << s.page_shift;
    for (int t = 0; t < s.tokens; ++t) {
        const int r = request_of(s, t);
        CHECK(r >= -1 && r < a.requests, "row %d", t);
        if (r < 0) {
            CHECK(!good, "row %d has no request", t);
            continue;
        }
        bool bad;
        const Request q = request(a, r, bad);
        int at;
        if (bad || !has_slot(q, t, 0, at)) {
            CHECK(!good || q.len < q.n, "row %d", t);
            continue;
        }
        CHECK(at >= 0 && at < room && at < s.lens[r], "row %d at %d of %lld", t, at, room);
        CHECK((at >> s.page_shift) < s.max_pages, "row %d", t);
        int same;
        CHECK(at == 0 || !has_slot(q, t, at, same), "row %d beyond the angles", t);
    }
    for (int group : {1, 7, 16, 24})   // the grid has so many tiles of rows
        for (int height : {128, 256}) {
            long long tiles = 0;
            bool bad;
            for (int r = 0; r < a.requests; ++r) tiles += tiles_of(request(a, r, bad), group, 1, height);
            CHECK(!good || tiles <= (long long)s.tokens * group / height + a.requests, "%lld tiles of %d", tiles, height);
        }
    for (int group : {1, 16, 24})   // the stream's steps: every one has one block, every part of a tile a place of its own
        for (int max_rows : {16, INT_MAX})
            for (int heads : {1, 3})
                for (int least : {1, 3}) {
                    const int blocks = 17;
                    std::vector<Steps> of;
                    long long total = 0;
                    bool bad;
                    for (int r = 0; r < a.requests; ++r) {
                        const Request q = request(a, r, bad);
                        of.push_back(steps_of(q, group, max_rows));
                        CHECK((of[r].tiles == 0) == (q.n == 0 || q.n * group > max_rows), "request %d", r);
                        CHECK(of[r].tiles * kStreamRows >= (of[r].tiles ? q.n * group : 0), "request %d", r);
                        CHECK(of[r].tiles == 0 || (long long)of[r].steps * kStepKeys >= keys_of(q, group, 0, q.n * group), "request %d", r);
                        total += (long long)of[r].tiles * of[r].steps * heads;
                    }
                    if (total > 100000) continue;
                    const long long share = steps_of_a_share(total, blocks, least);
                    CHECK(share * blocks >= total, "%lld steps, share %lld", total, share);
                    std::vector<int> used(2 * blocks, 0);
                    long long begin = 0;
                    for (int r = 0; r < a.requests; ++r)
                        for (int u = 0; u < of[r].tiles * heads; ++u, begin += of[r].steps) {
                            const long long b0 = begin / share, b1 = (begin + of[r].steps - 1) / share;
                            CHECK(b1 < blocks, "block %lld", b1);
                            for (long long b = b0; b0 != b1 && b <= b1; ++b) {
                                const long long at = place_of(begin, b, share);
                                CHECK(at >= 0 && at < 2 * blocks && !used[at]++, "place %lld of block %lld", at, b);
                            }
                        }
                }
    for (int r = 0; r < a.requests; ++r) {
        bool bad;
        const Request q = request(a, r, bad);
        CHECK(!good || !bad, "request %d", r);
        CHECK(q.n >= 0 && q.start >= 0 && (long long)q.start + q.n <= s.tokens, "request %d: rows %d + %d of %d", r, q.start, q.n, s.tokens);
        CHECK(q.len >= 0 && q.len <= room, "request %d: %d keys, room for %lld", r, q.len, room);
        for (int group : {1, 3, 16, 24})
            for (int tile : {16, 128, 256})
                for (int row0 = 0; row0 < q.n * group; row0 += tile) {
                    const int keys = keys_of(q, group, row0, tile);
                    CHECK(keys >= 0 && keys <= q.len, "request %d row %d: %d keys", r, row0, keys);
                    for (int chunk : {128, 256, 4096})
                        for (int most : {1, 3, 64}) {
                            const int count = shares(keys, chunk, most);
                            CHECK(count >= 1 && count <= most, "%d keys, chunk %d", keys, chunk);
                            int at = 0;
                            for (int i = 0; i < count; ++i) {   // they follow each other, none is empty unless there is no key
                                const Range k = share_of(keys, chunk, count, i);
                                CHECK(k.begin == at && (k.end > k.begin || keys == 0), "%d keys, chunk %d, share %d of %d", keys, chunk, i, count);
                                at = k.end;
                            }
                            CHECK(at == keys, "%d keys, chunk %d, %d shares", keys, chunk, count);
                        }
                }
    }
}

}  // namespace

int main() {
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return (int)std::uniform_int_distribution<long long>(lo, hi)(rng); };
    for (int round = 0; round < 1500; ++round) {
        Arrays s;
        const int R = pick(1, 6);
        s.page_shift = pick(4, 10);
        s.max_pages = pick(1, 20);
        s.starts = {0};
        for (int r = 0; r < R; ++r) {
            const int room = s.max_pages << s.page_shift, n = pick(0, 4) == 0 ? 0 : pick(1, 40);
            s.starts.push_back(s.starts.back() + n);
            s.lens.push_back(pick(0, 9) == 0 ? pick(0, n) : pick(n < room ? n : room, room));
        }
        s.tokens = s.starts.back();
        walk(s, true);
        // anything in any place
        const int strange[] = {INT_MIN, INT_MIN + 1, -1, 0, 1, s.tokens, s.tokens + 1, s.max_pages << s.page_shift, INT_MAX - 1, INT_MAX, pick(INT_MIN, INT_MAX)};
        for (int i = pick(1, 4); i > 0; --i) {
            const int v = strange[pick(0, 10)];
            if (pick(0, 1)) s.starts[pick(0, R)] = v;
            else s.lens[pick(0, R - 1)] = v;
        }
        walk(s, false);
    }
    for (int p : {INT_MIN, -1, 70000, INT_MAX}) CHECK(!is_page(p, 70000), "page %d", p);
    for (int p : {0, 1, 69999}) CHECK(is_page(p, 70000), "page %d", p);
    std::printf("cache: ok\n");
    return 0;
}
