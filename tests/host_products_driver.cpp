// How the products of the 16-bit linears are divided, on the host: every share of every tile is some block's, once, shares cover the
// steps of a tile, and none is empty.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "w16a16_plan.h"

using namespace qail;

#define CHECK(x)                                                                                       \
    do {                                                                                               \
        if (!(x)) {                                                                                    \
            std::printf("failed: %s  (P %lld Q %lld R %lld, %d units)\n", #x, P, Q, R, units);         \
            std::exit(1);                                                                              \
        }                                                                                              \
    } while (0)

static void walk(long long P, long long Q, long long R, bool turned, int units) {
    const ProductPlan pl = plan_product(P, Q, R, turned, units);
    CHECK(pl.tiles_p >= 1 && pl.tiles_q >= 1 && pl.splits >= 1 && pl.steps >= 1);
    CHECK((long long)pl.tiles_p * pl.bp >= P && (long long)(pl.tiles_p - 1) * pl.bp < P);
    CHECK((long long)pl.tiles_q * pl.bq >= Q && (long long)(pl.tiles_q - 1) * pl.bq < Q);
    CHECK((long long)pl.steps * kStepR >= R && (long long)(pl.steps - 1) * kStepR < R);
    CHECK(pl.first_step(0) == 0 && pl.first_step(pl.splits) == pl.steps);
    for (int s = 0; s < pl.splits; ++s) CHECK(pl.first_step(s) < pl.first_step(s + 1));
    CHECK((long long)pl.tiles_p * pl.tiles_q * pl.splits * 512 < (1ll << 32));
    if (pl.blocks() > 300000) return;
    std::vector<char> seen(pl.blocks());
    for (int b = 0; b < pl.blocks(); ++b) {
        const TilePlace t = tile_place(pl, b);
        CHECK(t.tp >= 0 && t.tp < pl.tiles_p && t.tq >= 0 && t.tq < pl.tiles_q && t.split >= 0 && t.split < pl.splits);
        char& c = seen[((size_t)t.split * pl.tiles_p + t.tp) * pl.tiles_q + t.tq];
        CHECK(!c);
        c = 1;
    }
}

int main() {
    const long long sizes[] = {1, 2, 8, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 289, 511, 513, 1000, 1024, 2056, 4096, 4097, 11008, 32000};
    for (const int units : {256, 304, 64, 1})
        for (const long long P : sizes)
            for (const long long Q : sizes)
                for (const long long R : sizes) walk(P, Q, R, false, units), walk(P, Q, R, true, units);
    const int units = 256;
    (void)units;
    walk(1 << 22, 2048, 8, false, 256);
    walk(2048, 1 << 22, 8, true, 256);
    walk(1, 8, 1 << 22, true, 256);
    std::printf("products: ok\n");
    return 0;
}
