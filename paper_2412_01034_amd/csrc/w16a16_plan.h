// How the products of the 16-bit linears (w16a16.hip) are divided: the tile, the shares of the contraction, and which block works on
// which of them; apart from the kernel so that the host can walk through it.
#ifndef QAIL_W16A16_PLAN_H
#define QAIL_W16A16_PLAN_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qail {

constexpr int kStepR = 64;   // r of a step: 128 bytes of a straight row

// C[P][Q] in tiles of bp x bq; the steps of a tile are divided among `splits` blocks (share s: [first_step(s), first_step(s + 1))).
struct ProductPlan {
    int bp, bq;
    int tiles_p, tiles_q, steps, splits;
    __host__ __device__ int blocks() const { return tiles_p * tiles_q * splits; }
    __host__ __device__ int first_step(int s) const { return (int)((long long)s * steps / splits); }
};

struct TilePlace {
    int tp, tq, split;
};

// Workgroup b of the launch runs on XCD b mod 8: the blocks of an XCD take consecutive places, so that tiles which share operands share
// an L2.  Consecutive places walk down kTallP row tiles, then to the next column tile.
constexpr int kTallP = 8;
__host__ __device__ inline TilePlace tile_place(const ProductPlan& pl, int b) {
    const int n = pl.blocks(), x = b & 7, each = n >> 3, rest = n & 7;
    int at = x * each + (x < rest ? x : rest) + (b >> 3);
    TilePlace t;
    const int tiles = pl.tiles_p * pl.tiles_q;
    t.split = at / tiles;
    at -= t.split * tiles;
    const int width = kTallP * pl.tiles_q, group = at / width, first = group * kTallP;
    const int tall = pl.tiles_p - first < kTallP ? pl.tiles_p - first : kTallP;
    at -= group * width;
    t.tp = first + at % tall;
    t.tq = at / tall;
    return t;
}

// turned: the operand of P lies row by row of r; parts: it is the sum of so many matrices, which the steps go through in turn.
//
// Up to 32 rows: tiles of 32 x 64, whose cost is the stream of the other operand; blocks for three a unit by shares of the contraction, which are
// not worth the second launch before a tile has eight steps for each.
// Beyond: the tile and the shares that cost least by what was measured (us a step, of two tiles that share a unit / of one that has it alone, and for the way in and out):
//     128 x 128   1.0 / 0.62, 7        192 x 128 (straight)   1.4 / 0.78, 9        256 x 256   1.65, 10 (one a unit)
// and for shares 3 for the second launch and their sums' way at 4 TB/s.  4096 x 4096 x 4096 takes 118 us with 256 x 256 tiles and 148 with 128 x 128, 2056 x 4096 x 1024 28
// with 192 x 128 and 33 with either other, 289 x 4096 x 4096 25 with five shares of 128 x 128 tiles and 42 with one.
inline ProductPlan plan_product(long long P, long long Q, long long R, bool turned, int units, int parts = 1) {
    ProductPlan pl;
    pl.steps = parts * (int)((R + kStepR - 1) / kStepR);
    const auto tiles_of = [&](int bp, int bq) {
        pl.bp = bp, pl.bq = bq;
        pl.tiles_p = (int)((P + bp - 1) / bp);
        pl.tiles_q = (int)((Q + bq - 1) / bq);
        return (long long)pl.tiles_p * pl.tiles_q;
    };
    if (P <= 32 && !turned) {
        const long long tiles = tiles_of(32, 64);
        long long splits = 3ll * units / tiles;
        if (splits > pl.steps / 8) splits = pl.steps / 8;
        pl.splits = splits < 1 ? 1 : (int)splits;
        return pl;
    }
    struct Tile {
        int bp, bq;
        double pair, alone, fixed;   // pair == 0: one a unit
    };
    const Tile kinds[] = {{128, 128, 1.0, 0.62, 7.}, {192, 128, 1.4, 0.78, 9.}, {256, 256, 0., 1.65, 10.}};
    double least = 1e300;
    const Tile* tile = kinds;
    int shares = 1;
    const int most = pl.steps / 4 < 1 ? 1 : pl.steps / 4 > 16 ? 16 : pl.steps / 4;
    for (int splits = 1; splits <= most; ++splits) {
        const double sums = splits == 1 ? 0. : 3. + splits * (double)P * (double)Q * 1e-6;
        const double steps = (double)((pl.steps + splits - 1) / splits);
        for (const Tile& k : kinds) {
            if (k.bp == 192 && turned) continue;
            const long long blocks = tiles_of(k.bp, k.bq) * splits, full = k.pair > 0. ? 2ll * units : units, rounds = blocks / full, rest = blocks % full;
            const double each = (k.pair > 0. ? k.pair : k.alone) * steps + k.fixed, alone = k.alone * steps + k.fixed;
            const double cost = sums + (double)rounds * each + (rest == 0 ? 0. : rest <= units ? alone : each);
            if (cost < least) least = cost, tile = &k, shares = splits;
        }
    }
    tiles_of(tile->bp, tile->bq);
    pl.splits = shares;
    return pl;
}

}  // namespace qail
#endif
