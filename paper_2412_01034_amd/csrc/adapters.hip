// Low-rank adapters of many requests beside a shared 4-bit linear: row m of x goes through adapter a = row_adapter[m],
//   t[m][j] = sum_k x[m][k] A[a][j][k],   y[m][n] += scaling[a] sum_j t[m][j] B[a][n][j].
// Two launches around the linears': both contractions run on the matrix cores, 16 rows of x at a time.  A tile's rows may belong to
// any number of adapters: each distinct one is multiplied with all 16 rows and only its own rows' columns are kept, by selection, so that
// nothing an adapter holds (an infinity included) reaches another's rows.  At decode sizes, where every row may have its own,
// the distinct adapters of a tile are spread over blocks (`slots`), since one after the other they would be a chain of round
// trips to memory.  The bytes are those of the adapters in use, r (K + N) bf16 each.
#include "qail_internal.h"

namespace qail {

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kMaxItems = 8;    // linears that share the two launches
constexpr int kMaxSplits = 4;   // shares of K
constexpr int kDownWaves = 8, kUpWaves = 4, kUpChunks = 4;

struct AdapterItem {
    const uint16_t *x, *A, *B;
    const float* scaling;
    float* t;      // fp32 [splits][M][r]
    uint16_t* y;
    int N, K, n, r;
};
struct AdapterArgs {
    AdapterItem it[kMaxItems];
    const int32_t* rows;
    int M, slots, splits;
    int chunks;   // of 64 columns that a wave of the second launch takes
};

// Calls f(a, mine) for the distinct adapters of the tile that are this slot's; `mine`: whether the lane's column (row m0 + lane % 16) uses it.
template <typename F>
__device__ __forceinline__ void each_adapter(const AdapterArgs& a, const AdapterItem& it, int m0, int slot, F f) {
    const int m = m0 + (int)threadIdx.x % 16;
    const int id = m < a.M ? a.rows[m] : -1;
    unsigned long long left = __ballot(id >= 0 && id < it.n) & 0xFFFFull;   // the first 16 lanes hold the tile's rows
    for (int i = 0; left; ++i) {
        const int of = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const bool mine = id == of;
        left &= ~__ballot(mine);
        if (i % a.slots == slot) f(of, mine);
    }
}

// A block takes 16 rows of x, all of the rank (kTiles tiles of 16) and a share of K, of which each wave has a piece of its own: whole lines of memory, so
// that none is read by two compute units.
template <int kTiles>
__global__ __launch_bounds__(kDownWaves* kWave) void adapters_down_kernel(const AdapterArgs a) {
    __shared__ f32x4_t red[kDownWaves][kTiles][kWave];
    const AdapterItem& it = a.it[blockIdx.z];
    const int split = blockIdx.x % a.splits, m0 = blockIdx.x / a.splits * 16;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, col = lane % 16, g = lane / 16;
    const int K = it.K, r = it.r, M = a.M;
    const int pieces = a.splits * kDownWaves, piece = (((K + 31) / 32 + pieces - 1) / pieces + 1) / 2 * 64;   // of K; a multiple of a line
    const int k0 = (split * kDownWaves + wave) * piece, k1 = min(k0 + piece, K);
    const uint16_t* xr = it.x + (size_t)min(m0 + col, M - 1) * K;
    each_adapter(a, it, m0, blockIdx.y, [&](int of, bool mine) {
        const uint16_t* ar[kTiles];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) ar[j] = it.A + ((size_t)of * r + min(16 * j + col, r - 1)) * K;   // rows past the rank are not stored
        constexpr int kAhead = 4;
        f32x4_t part[kTiles][2];   // two chains
#pragma unroll
        for (int j = 0; j < kTiles; ++j) part[j][0] = part[j][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int kb = k0; kb < k1; kb += 32 * kAhead) {
            u32x4_t xv[kAhead], av[kAhead][kTiles];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {   // past the end element 0 is read again and counts as 0
                const int k = kb + 32 * u + 8 * g, at = k < k1 ? k : 0;
                xv[u] = *reinterpret_cast<const u32x4_t*>(xr + at);
#pragma unroll
                for (int j = 0; j < kTiles; ++j) av[u][j] = *reinterpret_cast<const u32x4_t*>(ar[j] + at);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const bool in = kb + 32 * u + 8 * g < k1;
                const bf16x8_t x = __builtin_bit_cast(bf16x8_t, in ? xv[u] : u32x4_t{0u, 0u, 0u, 0u});
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
                    part[j][u % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, in ? av[u][j] : u32x4_t{0u, 0u, 0u, 0u}), x,
                                                                             part[j][u % 2], 0, 0, 0);
            }
        }
        __syncthreads();   // the sums of the adapter before have been read
#pragma unroll
        for (int j = 0; j < kTiles; ++j) red[wave][j][lane] = part[j][0] + part[j][1];
        __syncthreads();
        if (wave < kTiles && mine) {   // (mine: the row exists)
            f32x4_t sum = red[0][wave][lane];
#pragma unroll
            for (int w = 1; w < kDownWaves; ++w) sum += red[w][wave][lane];
            const int j = 16 * wave + 4 * g;
            if (j < r) *reinterpret_cast<f32x4_t*>(it.t + ((size_t)split * M + m0 + col) * r + j) = sum;   // r % 8 == 0
        }
    });
}

// A wave adds to 16 rows of `chunks` times 64 columns.  Row i of tile t of the product is column 16 (i / 4) + 4 t + i % 4, so that a lane ends up with 16
// consecutive columns of one row.  t is split into two bf16 values (a relative 2^-17 is lost, where one alone would lose 2^-9).
template <bool kWide>   // N % 8 == 0: rows of y are 16-byte aligned
__device__ __forceinline__ void add_up(const AdapterArgs& a, const AdapterItem& it, int m0, int n_begin, int slot) {
    const int lane = threadIdx.x % kWave, col = lane % 16, g = lane / 16;
    const int N = it.N, r = it.r, M = a.M, m = m0 + col;
    each_adapter(a, it, m0, slot, [&](int of, bool mine) {
        const float scaling = it.scaling[of];
        bf16x8_t th[2], tl[2];   // of 32 j each
#pragma unroll
        for (int jt = 0; jt < 2; ++jt) {
            const bool in = mine && 32 * jt + 8 * g < r;
            f32x4_t part[kMaxSplits][2];
#pragma unroll
            for (int k = 0; k < kMaxSplits; ++k) {
                const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
                const f32x4_t* p = reinterpret_cast<const f32x4_t*>(it.t + ((size_t)k * M + m) * r + 32 * jt + 8 * g);
                const bool have = in && k < a.splits;
                part[k][0] = have ? p[0] : zero;
                part[k][1] = have ? p[1] : zero;
            }
            float s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = (part[0][e / 4][e % 4] + part[1][e / 4][e % 4]) + (part[2][e / 4][e % 4] + part[3][e / 4][e % 4]);
            static_assert(kMaxSplits == 4, "four parts are added up");
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                hi[e] = f32x2_to_bf16x2_rne(s[2 * e], s[2 * e + 1]);
                lo[e] = f32x2_to_bf16x2_rne(s[2 * e] - __builtin_bit_cast(float, hi[e] << 16), s[2 * e + 1] - __builtin_bit_cast(float, hi[e] & 0xFFFF0000u));
            }
            th[jt] = __builtin_bit_cast(bf16x8_t, u32x4_t{hi[0], hi[1], hi[2], hi[3]});
            tl[jt] = __builtin_bit_cast(bf16x8_t, u32x4_t{lo[0], lo[1], lo[2], lo[3]});
        }
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
            for (int jt = 0; jt < 2; ++jt) {
                if (32 * jt >= r) break;
                u32x4_t bv[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int row = min(n0 + col / 4 * 16 + 4 * t + col % 4, N - 1);
                    bv[t] = 32 * jt + 8 * g < r ? *reinterpret_cast<const u32x4_t*>(it.B + ((size_t)of * N + row) * r + 32 * jt + 8 * g) : u32x4_t{0u, 0u, 0u, 0u};
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const bf16x8_t b = __builtin_bit_cast(bf16x8_t, bv[t]);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, tl[jt], acc[t], 0, 0, 0);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, th[jt], acc[t], 0, 0, 0);
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

__global__ __launch_bounds__(kUpWaves* kWave) void adapters_up_kernel(const AdapterArgs a) {
    const AdapterItem& it = a.it[blockIdx.z];
    const int row_tiles = (a.M + 15) / 16;
    const int m0 = blockIdx.x % row_tiles * 16, n0 = (blockIdx.x / row_tiles * kUpWaves + (int)threadIdx.x / kWave) * 64 * a.chunks;
    if (n0 >= it.N) return;   // whole waves; no barrier below
    if (it.N % 8 == 0) add_up<true>(a, it, m0, n0, blockIdx.y);
    else add_up<false>(a, it, m0, n0, blockIdx.y);
}

// Shares of K: more where the tiles alone leave the chip empty.
int k_splits(int M, int count) {
    const long long blocks = (long long)((M + 15) / 16) * count, s = 2ll * device_cu_count() / blocks;
    return s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : (int)s;
}

}  // namespace

// fp32 values of workspace: the down-projections of every linear.
size_t adapters_workspace(const qail_adapters* ad, int count, int M) {
    size_t n = 0;
    for (int i = 0; i < count; ++i) {
        const int first = i / kMaxItems * kMaxItems;
        n += (size_t)k_splits(M, count - first < kMaxItems ? count - first : kMaxItems) * M * ad[i].r;
    }
    return n;
}

namespace {

template <typename F>
hipError_t in_groups(const qail_w4a16_item* items, const qail_adapters* ad, const int32_t* rows, int count, int M, float* t, F launch) {
    for (int i0 = 0; i0 < count; i0 += kMaxItems) {
        const int c = count - i0 < kMaxItems ? count - i0 : kMaxItems;
        AdapterArgs a{};
        int widest = 0, most = 1, rank = 0;
        a.rows = rows;
        a.M = M;
        a.splits = k_splits(M, c);
        for (int i = 0; i < c; ++i) {
            const qail_w4a16_item& s = items[i0 + i];
            const qail_adapters& l = ad[i0 + i];
            a.it[i] = AdapterItem{s.x, l.A, l.B, l.scaling, t, s.y, s.d.N, s.d.K, l.n, l.r};
            t += (size_t)a.splits * M * l.r;
            widest = s.d.N > widest ? s.d.N : widest;
            most = l.n > most ? l.n : most;
            rank = l.r > rank ? l.r : rank;
        }
        const int in_tile = M < 16 ? M : 16;   // distinct adapters of a tile, at most
        a.slots = most < in_tile ? most : in_tile;
        if (M > 64) a.slots = 1;
        a.chunks = M > 64 ? kUpChunks : 1;
        launch(a, c, widest, (rank + 15) / 16);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_adapters_down(const qail_w4a16_item* items, const qail_adapters* ad, const int32_t* rows, int count, int M, float* t, hipStream_t st) {
    return in_groups(items, ad, rows, count, M, t, [&](const AdapterArgs& a, int c, int, int tiles) {
        auto* const kernel = tiles == 1 ? adapters_down_kernel<1> : tiles == 2 ? adapters_down_kernel<2> : tiles == 3 ? adapters_down_kernel<3> : adapters_down_kernel<4>;
        hipLaunchKernelGGL(kernel, dim3((M + 15) / 16 * a.splits, a.slots, c), dim3(kDownWaves * kWave), 0, st, a);
    });
}

hipError_t launch_adapters_up(const qail_w4a16_item* items, const qail_adapters* ad, const int32_t* rows, int count, int M, float* t, hipStream_t st) {
    return in_groups(items, ad, rows, count, M, t, [&](const AdapterArgs& a, int c, int widest, int) {
        hipLaunchKernelGGL(adapters_up_kernel, dim3((M + 15) / 16 * ((widest + 64 * kUpWaves * a.chunks - 1) / (64 * kUpWaves * a.chunks)), a.slots, c), dim3(kUpWaves * kWave), 0, st, a);
    });
}

}  // namespace qail
