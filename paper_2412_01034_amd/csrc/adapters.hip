// Low-rank adapters of many requests beside a shared 4-bit linear: row m of x goes through adapter a = row_adapter[m],
//   t[m][j] = sum_k x[m][k] A[a][j][k],   y[m][n] += scaling[a] sum_j t[m][j] B[a][n][j].
// Two launches around the linears': both contractions run on the matrix cores, 16 rows of x at a time.  A tile's rows may belong to
// any number of adapters: each distinct one is multiplied with all 16 rows and only its own rows' columns are kept, by selection, so that
// nothing an adapter holds (an infinity included) reaches another's rows.  At decode sizes, where every row may have its own,
// the distinct adapters of a tile are spread over blocks (`slots`), since one after the other they would be a chain of round
// trips to memory.  The bytes are those of the adapters in use, r (K + N) bf16 each.
// y is rounded to bf16 twice, by the linear's launch and here (0.0023 of its norm from 64 bits, 0.0017 with one rounding): a linear in fp32 between the two would be
// written and read with twice the bytes, 170 MB more at 1000 rows of a 7B layer.
#include <algorithm>

#include "qail_internal.h"

namespace qail {

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kMaxItems = 8;    // linears that share the two launches
constexpr int kMaxSplits = 8, kSplitK = 1024;   // shares of K: one for 1024 (128 a wave), so that those of a long K take no longer
constexpr int kDownWaves = 8, kUpWaves = 4, kUpChunks = 4;
constexpr int kManyRows = 320, kManyTile = 64;   // more rows than kManyRows: kManyTile of them a block of the first launch

struct AdapterItem {
    const uint16_t *x, *A, *B;
    const float* scaling;
    float* t;      // fp32 [splits][M][r]
    uint16_t* y;
    int N, K, n, r, splits;
    int first;     // of the linear's blocks, where they are numbered through
};
struct AdapterArgs {
    AdapterItem it[kMaxItems];
    const int32_t* rows;
    int count, M, splits;   // splits: the most of a linear
    int slots;       // blocks that share the adapters of a tile of rows (the grid's y)
    int chunks;      // of 64 columns that a wave of the second launch takes
};

// Calls f(a, mine) for the distinct adapters of the tile that are this slot's; `mine`: whether the lane's column (row m0 + lane % 16) uses it.
template <typename F>
__device__ __forceinline__ void each_adapter(const AdapterArgs& a, const AdapterItem& it, int m0, int slot, int slots, F f) {
    const int m = m0 + (int)threadIdx.x % 16;
    const int id = m < a.M ? a.rows[m] : -1;
    unsigned long long left = __ballot(id >= 0 && id < it.n) & 0xFFFFull;   // the first 16 lanes hold the tile's rows
    for (int i = 0; left; ++i) {
        const int of = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const bool mine = id == of;
        left &= ~__ballot(mine);
        if (i % slots == slot) f(of, mine);
    }
}

// Products of kRows tiles of 16 rows (from x's row m0 on) with adapter `of`, for k0 <= k < k1: `part` has [row tile][rank tile].  Whole lines of memory to
// a wave, kAhead times 32 k requested at once.
template <int kRows, int kTiles, int kAhead>
__device__ __forceinline__ void multiply_down(const AdapterItem& it, int M, int m0, int of, int k0, int k1, f32x4_t (&part)[kRows][kTiles]) {
    const int lane = threadIdx.x % kWave, col = lane % 16, g = lane / 16, K = it.K, r = it.r;
    const uint16_t *xr[kRows], *ar[kTiles];
#pragma unroll
    for (int i = 0; i < kRows; ++i) xr[i] = it.x + (size_t)min(m0 + 16 * i + col, M - 1) * K;
#pragma unroll
    for (int j = 0; j < kTiles; ++j) ar[j] = it.A + ((size_t)of * r + min(16 * j + col, r - 1)) * K;   // rows past the rank are not stored
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int j = 0; j < kTiles; ++j) part[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int kb = k0; kb < k1; kb += 32 * kAhead) {
        const u32x4_t zero = {0u, 0u, 0u, 0u};
        u32x4_t xv[kAhead][kRows], av[kAhead][kTiles];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (kb + 32 * u >= k1) break;
            const int k = kb + 32 * u + 8 * g, at = k < k1 ? k : 0;   // past the end element 0 is read again and counts as 0
#pragma unroll
            for (int i = 0; i < kRows; ++i) xv[u][i] = *reinterpret_cast<const u32x4_t*>(xr[i] + at);
#pragma unroll
            for (int j = 0; j < kTiles; ++j) av[u][j] = *reinterpret_cast<const u32x4_t*>(ar[j] + at);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (kb + 32 * u >= k1) break;
            const bool in = kb + 32 * u + 8 * g < k1;
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const bf16x8_t x = __builtin_bit_cast(bf16x8_t, in ? xv[u][i] : zero);
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
                    part[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, in ? av[u][j] : zero), x, part[i][j], 0, 0, 0);
            }
        }
    }
}

// The piece of K of a wave: a multiple of a line, so that none is read by two compute units.
__device__ __forceinline__ void piece_of(int K, int pieces, int i, int& k0, int& k1) {
    const int piece = (((K + 31) / 32 + pieces - 1) / pieces + 1) / 2 * 64;
    k0 = i * piece;
    k1 = min(k0 + piece, K);
}

// The waves' sums of a tile of rows added up and stored; `mine`: the lane's row (m) uses the adapter.
template <int kTiles>
__device__ __forceinline__ void store_down(const AdapterItem& it, f32x4_t (*red)[kTiles][kWave], const f32x4_t (&part)[kTiles], int wave, size_t m, bool mine) {
    const int lane = threadIdx.x % kWave;
    __syncthreads();   // the sums before have been read
#pragma unroll
    for (int j = 0; j < kTiles; ++j) red[wave][j][lane] = part[j];
    __syncthreads();
    if (wave < kTiles && mine) {   // (mine: the row exists)
        f32x4_t sum = red[0][wave][lane];
#pragma unroll
        for (int w = 1; w < kDownWaves; ++w) sum += red[w][wave][lane];
        const int j = 16 * wave + lane / 16 * 4;
        if (j < it.r) *reinterpret_cast<f32x4_t*>(it.t + m * it.r + j) = sum;   // r % 8 == 0
    }
}

// A block takes 16 rows of x, all of the rank (kTiles tiles of 16) and a share of K, of which each wave has a piece of its own: with few rows the trips to
// memory are what counts, so that a piece (192 k at K = 11008) is requested at once.
template <int kTiles>
__global__ __launch_bounds__(kDownWaves* kWave) void adapters_down_kernel(const AdapterArgs a) {
    __shared__ f32x4_t red[kDownWaves][kTiles][kWave];
    const AdapterItem& it = a.it[blockIdx.z];
    const int split = blockIdx.x % a.splits, m0 = blockIdx.x / a.splits * 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (split >= it.splits) return;   // whole blocks
    int k0, k1;
    piece_of(it.K, it.splits * kDownWaves, split * kDownWaves + wave, k0, k1);
    each_adapter(a, it, m0, blockIdx.y, gridDim.y, [&](int of, bool mine) {
        f32x4_t part[1][kTiles];
        multiply_down<1, kTiles, 6>(it, a.M, m0, of, k0, k1, part);
        store_down<kTiles>(it, red, part[0], wave, (size_t)split * a.M + m0 + threadIdx.x % 16, mine);
    });
}

// The same for 64 rows, of which an adapter usually has all: A is read by a quarter as many blocks (at 1000 rows of a 7B layer 24 MB instead of 94 beside x's
// 46, 34 us instead of 54).  What took long there were tiles of several adapters at the longest K: so a second adapter has a block of its own, a long K more
// shares, and all 64 rows are multiplied at once unless only 16 are the adapter's.  The layer, this kernel / the one above: 257 rows 177 / 176 us, 400 rows
// 285 / 287, 1000 rows 493 / 510 with 3 adapters, 263 / 248, 372 / 373 and 575 / 569 with 64.
template <int kTiles>
__global__ __launch_bounds__(kDownWaves* kWave) void adapters_down_rows_kernel(const AdapterArgs a) {
    __shared__ f32x4_t red[kDownWaves][kTiles][kWave];
    int i = 0;
    while (i + 1 < a.count && (int)blockIdx.x >= a.it[i + 1].first) ++i;
    const AdapterItem& it = a.it[i];
    const int block = blockIdx.x - it.first, split = block % it.splits, m0 = block / it.splits * kManyTile, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lane = threadIdx.x % kWave, col = lane % 16;
    int k0, k1;
    piece_of(it.K, it.splits * kDownWaves, split * kDownWaves + wave, k0, k1);
    const int id = m0 + lane < a.M ? a.rows[m0 + lane] : -1;   // a lane a row
    unsigned long long left = __ballot(id >= 0 && id < it.n);
    for (int which = 0; left; ++which) {
        const int of = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const unsigned long long mine = __ballot(id == of);
        left &= ~mine;
        if (which % (int)gridDim.y != (int)blockIdx.y) continue;
        const int tile = __builtin_ctzll(mine) / 16;
        if (mine & ~(0xFFFFull << (16 * tile))) {
            f32x4_t part[4][kTiles];
            multiply_down<4, kTiles, kTiles <= 2 ? 6 : 4>(it, a.M, m0, of, k0, k1, part);
#pragma unroll
            for (int i = 0; i < 4; ++i) store_down<kTiles>(it, red, part[i], wave, (size_t)split * a.M + m0 + 16 * i + col, (mine >> (16 * i + col)) & 1);
        } else {
            f32x4_t part[1][kTiles];
            multiply_down<1, kTiles, 6>(it, a.M, m0 + 16 * tile, of, k0, k1, part);
            store_down<kTiles>(it, red, part[0], wave, (size_t)split * a.M + m0 + 16 * tile + col, (mine >> (16 * tile + col)) & 1);
        }
    }
}

// A wave adds to 16 rows of `chunks` times 64 columns.  Row i of tile t of the product is column 16 (i / 4) + 4 t + i % 4, so that a lane ends up with 16
// consecutive columns of one row.  t is split into two bf16 values (a relative 2^-16 may be lost, where one alone may lose 2^-8).
template <int kParts, bool kWide>   // of 32 of the rank; N % 8 == 0: rows of y are 16-byte aligned
__device__ __forceinline__ void add_up(const AdapterArgs& a, const AdapterItem& it, int m0, int n_begin, int slot) {
    const int lane = threadIdx.x % kWave, col = lane % 16, g = lane / 16;
    const int N = it.N, r = it.r, M = a.M, m = m0 + col;
    each_adapter(a, it, m0, slot, gridDim.y, [&](int of, bool mine) {
        const float scaling = it.scaling[of];
        bf16x8_t th[kParts], tl[kParts];   // of 32 j each
#pragma unroll
        for (int jt = 0; jt < kParts; ++jt) {
            const bool in = mine && 32 * jt + 8 * g < r;
            f32x4_t sum[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
#pragma unroll 1
            for (int k = 0; k < it.splits; k += 4) {   // four shares at a time
                f32x4_t part[4][2];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
                    const f32x4_t* p = reinterpret_cast<const f32x4_t*>(it.t + ((size_t)(k + u) * M + m) * r + 32 * jt + 8 * g);
                    const bool have = in && k + u < it.splits;
                    part[u][0] = have ? p[0] : zero;
                    part[u][1] = have ? p[1] : zero;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) sum[e] += (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
            }
            float s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = sum[e / 4][e % 4];
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                hi[e] = f32x2_to_bf16x2_rne(s[2 * e], s[2 * e + 1]);
                lo[e] = f32x2_to_bf16x2_rne(s[2 * e] - __builtin_bit_cast(float, hi[e] << 16), s[2 * e + 1] - __builtin_bit_cast(float, hi[e] & 0xFFFF0000u));
            }
            th[jt] = __builtin_bit_cast(bf16x8_t, u32x4_t{hi[0], hi[1], hi[2], hi[3]});
            tl[jt] = __builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], lo[2], lo[3]});
        }
        auto b_of = [&](int n0, int t, int jt) {
            const int row = min(n0 + col / 4 * 16 + 4 * t + col % 4, N - 1);
            return 32 * jt + 8 * g < r ? *reinterpret_cast<const u32x4_t*>(it.B + ((size_t)of * N + row) * r + 32 * jt + 8 * g) : u32x4_t{0u, 0u, 0u, 0u};
        };
        for (int n0 = n_begin, c = 0; c < a.chunks && n0 < N; ++c, n0 += 64) {
            const int n = n0 + 16 * g;
            uint16_t* const y = it.y + (size_t)min(m, M - 1) * N + n;
            u32x4_t old[2];
            if (kWide && mine) {   // on its way while the products are formed
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (n + 8 * half < N) old[half] = reinterpret_cast<u32x4_t*>(y)[half];
            }
            f32x4_t acc[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int jt = 0; jt < kParts; ++jt) {
                u32x4_t bv[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) bv[t] = b_of(n0, t, jt);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const bf16x8_t b = __builtin_bit_cast(bf16x8_t, bv[t]);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, tl[jt], acc[t], 0, 0, 0);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, th[jt], acc[t], 0, 0, 0);
                }
            }
            float odd = 0.f;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) odd = fmaf(acc[t][e], 0.f, odd);
            if (__builtin_expect(__any(mine && odd != 0.f), 0)) {   // NaN: an infinity of t or B is right times t's upper part; its product with the lower one is NaN or of either sign
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    f32x4_t high = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int jt = 0; jt < kParts; ++jt) high = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b_of(n0, t, jt)), th[jt], high, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t][e] = fabsf(acc[t][e]) < INFINITY ? acc[t][e] : high[e];
                }
            }
            if (!mine || n >= N) continue;
            if (kWide) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (n + 8 * half >= N) break;
                    u32x4_t w = old[half];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x4_t& d = acc[2 * half + e / 2];
                        const uint32_t was = w[e];
                        w[e] = f32x2_to_bf16x2_rne(fmaf(scaling, d[e % 2 * 2], __builtin_bit_cast(float, was << 16)),
                                                   fmaf(scaling, d[e % 2 * 2 + 1], __builtin_bit_cast(float, was & 0xFFFF0000u)));
                    }
                    reinterpret_cast<u32x4_t*>(y)[half] = w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (n + e < N) y[e] = (uint16_t)f32x2_to_bf16x2_rne(fmaf(scaling, acc[e / 4][e % 4], bf16_bits_to_f32(y[e])), 0.f);
            }
        }
    });
}

template <int kParts>
__global__ __launch_bounds__(kUpWaves* kWave) void adapters_up_kernel(const AdapterArgs a) {
    const AdapterItem& it = a.it[blockIdx.z];
    const int row_tiles = (a.M + 15) / 16;
    const int m0 = blockIdx.x % row_tiles * 16, n0 = (blockIdx.x / row_tiles * kUpWaves + (int)threadIdx.x / kWave) * 64 * a.chunks;
    if (n0 >= it.N) return;   // whole waves; no barrier below
    if (it.N % 8 == 0) add_up<kParts, true>(a, it, m0, n0, blockIdx.y);
    else add_up<kParts, false>(a, it, m0, n0, blockIdx.y);
}

int k_splits(int K) {
    const int s = (K + kSplitK - 1) / kSplitK;
    return s > kMaxSplits ? kMaxSplits : s;
}

}  // namespace

// fp32 values of workspace: the down-projections of every linear.
size_t adapters_workspace(const qail_w4a16_item* items, const qail_adapters* ad, int count, int M) {
    size_t n = 0;
    for (int i = 0; i < count; ++i) n += (size_t)k_splits(items[i].d.K) * M * ad[i].r;
    return n;
}

namespace {

template <typename F>
hipError_t in_groups(const qail_w4a16_item* items, const qail_adapters* ad, const int32_t* rows, int count, int M, float* t, F launch) {
    for (int i0 = 0; i0 < count; i0 += kMaxItems) {
        const int c = count - i0 < kMaxItems ? count - i0 : kMaxItems;
        AdapterArgs a{};
        int widest = 0, most = 1, rank = 0, blocks = 0;
        a.rows = rows;
        a.M = M;
        a.count = c;
        for (int i = 0; i < c; ++i) {
            const qail_w4a16_item& s = items[i0 + i];
            const qail_adapters& l = ad[i0 + i];
            const int splits = k_splits(s.d.K);
            a.it[i] = AdapterItem{s.x, l.A, l.B, l.scaling, t, s.y, s.d.N, s.d.K, l.n, l.r, splits, blocks};
            blocks += (M + kManyTile - 1) / kManyTile * splits;
            t += (size_t)splits * M * l.r;
            a.splits = splits > a.splits ? splits : a.splits;
            widest = s.d.N > widest ? s.d.N : widest;
            most = l.n > most ? l.n : most;
            rank = l.r > rank ? l.r : rank;
        }
        // as many as a tile can have adapters at decode sizes; with more rows the blocks of tiles that have one are in the way.  us of a 7B layer, 1 or 2 / 4 / 16
        // slots: 80 rows of 3 adapters 91 / 87 / 95, of 64 requests 190 / 151 / 138; 200 rows 153 / 156 / 164 and 235 / 210 / 218
        a.slots = std::min(most, M > kManyRows ? 2 : M > 64 ? 4 : std::min(M, 16));
        a.chunks = M > 64 ? kUpChunks : 1;
        launch(a, blocks, widest, (rank + 15) / 16);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_adapters_down(const qail_w4a16_item* items, const qail_adapters* ad, const int32_t* rows, int count, int M, float* t, hipStream_t st) {
    return in_groups(items, ad, rows, count, M, t, [&](const AdapterArgs& a, int blocks, int, int tiles) {
        auto* const few = tiles == 1 ? adapters_down_kernel<1> : tiles == 2 ? adapters_down_kernel<2> : tiles == 3 ? adapters_down_kernel<3> : adapters_down_kernel<4>;
        auto* const many = tiles == 1 ? adapters_down_rows_kernel<1> : tiles == 2 ? adapters_down_rows_kernel<2> : tiles == 3 ? adapters_down_rows_kernel<3> : adapters_down_rows_kernel<4>;
        if (M > kManyRows) hipLaunchKernelGGL(many, dim3(blocks, a.slots), dim3(kDownWaves * kWave), 0, st, a);
        else hipLaunchKernelGGL(few, dim3((M + 15) / 16 * a.splits, a.slots, a.count), dim3(kDownWaves * kWave), 0, st, a);
    });
}

hipError_t launch_adapters_up(const qail_w4a16_item* items, const qail_adapters* ad, const int32_t* rows, int count, int M, float* t, hipStream_t st) {
    return in_groups(items, ad, rows, count, M, t, [&](const AdapterArgs& a, int, int widest, int tiles) {
        auto* const kernel = tiles <= 2 ? adapters_up_kernel<1> : adapters_up_kernel<2>;
        const int columns = 64 * kUpWaves * a.chunks;   // of a block
        const int slots = M > kManyRows ? 1 : a.slots;   // (1000 rows of 3 adapters: 493 with 1, 500 with 2)
        hipLaunchKernelGGL(kernel, dim3((M + 15) / 16 * ((widest + columns - 1) / columns), slots, a.count), dim3(kUpWaves * kWave), 0, st, a);
    });
}

}  // namespace qail
