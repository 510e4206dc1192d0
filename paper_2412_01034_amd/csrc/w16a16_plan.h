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
inline ProductPlan plan_product(long long P, long long Q, long long R, bool turned, int units) {
    ProductPlan pl;
    pl.bp = P <= 32 && !turned ? 32 : 128;
    pl.bq = 128;
    pl.tiles_p = (int)((P + pl.bp - 1) / pl.bp);
    pl.tiles_q = (int)((Q + pl.bq - 1) / pl.bq);
    pl.steps = (int)((R + kStepR - 1) / kStepR);
    const long long tiles = (long long)pl.tiles_p * pl.tiles_q;
    long long splits = 2ll * units / tiles;
    if (splits > pl.steps / 4) splits = pl.steps / 4;
    pl.splits = splits < 1 ? 1 : (int)splits;
    return pl;
}

}  // namespace qail
#endif
