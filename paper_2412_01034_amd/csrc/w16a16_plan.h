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

// turned: the operand of P lies row by row of r.
//
// Up to 32 rows: tiles of 32 x 64, whose cost is the stream of the other operand; blocks for three a unit by shares of the contraction, which are
// not worth the second launch before a tile has sixteen steps for each.
// Beyond: the tile and the shares that cost least by what was measured (us): of 128 x 128 tiles two share a unit, 1.05 a step together and 0.62 alone, of 256 x 256 one
// has it, 1.7 a step; beside that 5 and 12 for the way in and out of a tile, and for shares 3 for the second launch and their sums' way at 4 TB/s.  4096 x 4096 x 4096 takes 126
// with 256 x 256 tiles and 148 with 128 x 128, 2056 x 4096 x 1024 33 with either, 289 x 4096 x 4096 25 with five shares of 128 x 128 tiles and 42 with one.
inline ProductPlan plan_product(long long P, long long Q, long long R, bool turned, int units) {
    ProductPlan pl;
    pl.steps = (int)((R + kStepR - 1) / kStepR);
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
    double least = 1e300;
    int tile = 128, shares = 1;
    const int most = pl.steps / 4 < 1 ? 1 : pl.steps / 4 > 16 ? 16 : pl.steps / 4;
    for (int splits = 1; splits <= most; ++splits) {
        const double sums = splits == 1 ? 0. : 3. + splits * (double)P * (double)Q * 1e-6;
        const double steps = (double)((pl.steps + splits - 1) / splits);
        const long long small = tiles_of(128, 128) * splits, large = tiles_of(256, 256) * splits;
        const long long pairs = small / (2 * units), rest = small % (2 * units);
        const double with_small = sums + (double)pairs * (1.05 * steps + 5.) + (rest == 0 ? 0. : rest <= units ? 0.62 * steps + 5. : 1.05 * steps + 5.);
        const double with_large = sums + (double)((large + units - 1) / units) * (1.7 * steps + 12.);
        if (with_small < least) least = with_small, tile = 128, shares = splits;
        if (with_large < least) least = with_large, tile = 256, shares = splits;
    }
    tiles_of(tile, tile);
    pl.splits = shares;
    return pl;
}

}  // namespace qail
#endif
