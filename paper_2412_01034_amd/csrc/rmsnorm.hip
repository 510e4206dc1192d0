// Root-mean-square norm of rows with the residual's addition, to bf16 or to 8-bit codes with a step per row, and its gradient.
//
// Both directions are bound by memory: a handful of operations per element.  The forward kernel holds a row in the registers of
// kGroup threads from its first to its last use, so that everything is read once and written once; both reductions of a row (its
// sum of squares, the largest |h * weight|) go through one exchange.  The codes do not depend on r = 1 / rms: q = rint(u / s) with
// u = h * weight and s = max |u| / 127, and r goes into the scale that is written beside them.  Two machines or two orders of
// summation then agree on every code.  With the residual 2048 x 4096 to codes take 13.8 us (59 MB, 4.3 TB/s), 7 rows 3.2; the gradient of
// 4096 x 4096 26.8 us (134 MB, 5.0 TB/s) and 4.8 for the weight's sums, 289 rows 5.9 and 3.7.
#include "qail_internal.h"

namespace qail {

namespace {

constexpr int kNormMaxK = 32768;   // 1024 threads hold a row as four pieces of eight values each

// Sum of a and maximum (of magnitudes) or sum of b over the kGroup threads that share a row; every thread gets them.
template <int kGroup, bool kMax>
__device__ __forceinline__ void row_reduce(float& a, float& b, float2* red) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        a += __shfl_xor(a, o, kWave);
        const float c = __shfl_xor(b, o, kWave);
        b = kMax ? max_magnitude(b, c) : b + c;
    }
    if constexpr (kGroup > kWave) {
        constexpr int waves = kGroup / kWave;
        if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = make_float2(a, b);
        __syncthreads();
        float2 t = red[0];
#pragma unroll
        for (int w = 1; w < waves; ++w) {
            t.x += red[w].x;
            t.y = kMax ? max_magnitude(t.y, red[w].y) : t.y + red[w].y;
        }
        a = t.x;
        b = t.y;
    }
}

struct NormArgs {
    const uint16_t *x, *residual, *weight;   // none of the row tensors is __restrict__: outputs may lie on inputs
    uint16_t *h_out, *y;
    uint32_t* y_s8;
    float* y_scale;
    float eps, inv_k;
    int M, K;
};

template <int kGroup, int kPer, bool kEight>
__global__ __launch_bounds__(kGroup < 256 ? 256 : kGroup) void rmsnorm_kernel(const NormArgs a) {
    constexpr int kBlock = kGroup < 256 ? 256 : kGroup;
    __shared__ float2 red[kBlock / kWave];
    const int m = blockIdx.x * (kBlock / kGroup) + threadIdx.x / kGroup, t = threadIdx.x % kGroup;
    if (m >= a.M) return;   // whole waves, and only where a row has no barrier
    const int n8 = a.K / 8;
    const size_t base = (size_t)m * n8;
    const uint4* x = reinterpret_cast<const uint4*>(a.x) + base;
    const uint4* res = reinterpret_cast<const uint4*>(a.residual) + base;
    const uint4* weight = reinterpret_cast<const uint4*>(a.weight);
    uint4 xv[kPer], rv[kPer], wv[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {   // every load is issued before the first is used
        const int i = t + u * kGroup;
        xv[u] = rv[u] = wv[u] = uint4{0u, 0u, 0u, 0u};
        if (i < n8) {
            xv[u] = x[i];
            if (a.residual) rv[u] = res[i];
            wv[u] = weight[i];
        }
    }
    float h[kPer][8], ss = 0.f, most = 0.f;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        float r[8], w[8];
        unpack8(xv[u], h[u]);
        unpack8(rv[u], r);
        unpack8(wv[u], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (a.residual) h[u][e] += r[e];
            ss = fmaf(h[u][e], h[u][e], ss);
            if constexpr (kEight) most = max_magnitude(most, fabsf(h[u][e] * w[e]));
        }
        const int i = t + u * kGroup;
        if (a.h_out && i < n8) reinterpret_cast<uint4*>(a.h_out)[base + i] = pack8(h[u]);
    }
    row_reduce<kGroup, true>(ss, most, red);
    const float r = 1.0f / sqrtf(fmaf(ss, a.inv_k, a.eps));
    if constexpr (kEight) {
        const float s = most > 0.f ? most / 127.0f : 1.0f;
        if (t == 0) a.y_scale[m] = most < INFINITY ? s * r : __builtin_nanf("");   // no code could say that a u is not finite
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int i = t + u * kGroup;
            float w[8];
            unpack8(wv[u], w);
            uint32_t word[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = fminf(fmaxf(rintf(h[u][e] * w[e] / s), -127.f), 127.f);
                word[e / 4] |= ((uint32_t)(int)q & 255u) << (8 * (e % 4));
            }
            if (i < n8) reinterpret_cast<uint2*>(a.y_s8)[base + i] = uint2{word[0], word[1]};
        }
    }
    if (a.y) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int i = t + u * kGroup;
            float w[8];
            unpack8(wv[u], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] *= h[u][e] * r;
            if (i < n8) reinterpret_cast<uint4*>(a.y)[base + i] = pack8(w);
        }
    }
}

struct NormBackArgs {
    const uint16_t *h, *weight, *dy, *dres;
    uint16_t* dx;
    float* partial;   // [blocks][K]
    float eps, inv_k;
    int M, K;
};

// A block takes rows blockIdx, blockIdx + blocks, ...: the weight's gradient stays in its registers until the end and costs one row of
// fp32 a block.  The next row is on its way while the sums of the present one are exchanged.
template <int kGroup, int kPer>
__global__ __launch_bounds__(kGroup) void rmsnorm_back_kernel(const NormBackArgs a) {
    __shared__ float2 red[2][kGroup / kWave + 1];
    const int t = threadIdx.x, n8 = a.K / 8;
    const uint4* H = reinterpret_cast<const uint4*>(a.h);
    const uint4* DY = reinterpret_cast<const uint4*>(a.dy);
    const uint4* DR = reinterpret_cast<const uint4*>(a.dres);
    uint4 wv[kPer], hv[kPer], gv[kPer], rv[kPer];
    float dw[kPer][8] = {};
    auto load = [&](int m) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int i = t + u * kGroup;
            hv[u] = gv[u] = rv[u] = uint4{0u, 0u, 0u, 0u};
            if (i < n8) {
                const size_t at = (size_t)m * n8 + i;
                hv[u] = H[at];
                gv[u] = DY[at];
                if (a.dres) rv[u] = DR[at];
            }
        }
    };
#pragma unroll
    for (int u = 0; u < kPer; ++u) wv[u] = t + u * kGroup < n8 ? reinterpret_cast<const uint4*>(a.weight)[t + u * kGroup] : uint4{0u, 0u, 0u, 0u};
    load(blockIdx.x);   // blocks <= M
    for (int m = blockIdx.x, turn = 0; m < a.M; m += gridDim.x, turn ^= 1) {
        uint4 h_now[kPer], g_now[kPer], r_now[kPer];
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            h_now[u] = hv[u];
            g_now[u] = gv[u];
            r_now[u] = rv[u];
            float h[8], g[8], w[8];
            unpack8(h_now[u], h);
            unpack8(g_now[u], g);
            unpack8(wv[u], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ss = fmaf(h[e], h[e], ss);
                dot = fmaf(g[e] * w[e], h[e], dot);
            }
        }
        if (m + (int)gridDim.x < a.M) load(m + gridDim.x);
        row_reduce<kGroup, false>(ss, dot, red[turn]);   // two places in turn: one barrier a row
        const float r = 1.0f / sqrtf(fmaf(ss, a.inv_k, a.eps));
        const float c = dot * a.inv_k * r * r;           // mean(dy * w * n) * r
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            float h[8], g[8], w[8], d[8], out[8];
            unpack8(h_now[u], h);
            unpack8(g_now[u], g);
            unpack8(wv[u], w);
            unpack8(r_now[u], d);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                out[e] = r * (g[e] * w[e] - h[e] * c);
                if (a.dres) out[e] += d[e];
                dw[u][e] = fmaf(g[e], h[e] * r, dw[u][e]);
            }
            const int i = t + u * kGroup;
            if (i < n8) reinterpret_cast<uint4*>(a.dx)[(size_t)m * n8 + i] = pack8(out);
        }
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int i = t + u * kGroup;
        float4* out = reinterpret_cast<float4*>(a.partial + (size_t)blockIdx.x * a.K) + 2 * i;
        if (i < n8) {
            out[0] = make_float4(dw[u][0], dw[u][1], dw[u][2], dw[u][3]);
            out[1] = make_float4(dw[u][4], dw[u][5], dw[u][6], dw[u][7]);
        }
    }
}

// dweight[k] = sum over blocks of partial[block][k]: kSlices threads a column of four, eight loads of each on their way, in a fixed order.
constexpr int kSlices = 64;
__global__ __launch_bounds__(16 * kSlices) void rmsnorm_weight_kernel(const float* __restrict__ partial, int blocks, int K, float* __restrict__ dw) {
    __shared__ f32x4_t red[kSlices][16];
    const int c = threadIdx.x % 16, s = threadIdx.x / 16, n4 = K / 4;
    const int col = blockIdx.x * 16 + c;
    const f32x4_t* p = reinterpret_cast<const f32x4_t*>(partial) + min(col, n4 - 1);
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    for (int b0 = s; b0 < blocks; b0 += 8 * kSlices) {
        f32x4_t v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = p[(size_t)min(b0 + u * kSlices, blocks - 1) * n4];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (b0 + u * kSlices < blocks) sum += v[u];
    }
    red[s][c] = sum;
    __syncthreads();
#pragma unroll
    for (int o = kSlices / 2; o >= 1; o >>= 1) {
        if (s < o) red[s][c] = sum = sum + red[s + o][c];
        __syncthreads();
    }
    if (s == 0 && col < n4) reinterpret_cast<f32x4_t*>(dw)[col] = sum;
}

// Two blocks a unit: more have more rows on their way and leave more sums of the weight.  us with 1 / 2 / 4 / 8: 4096 x 4096 31 / 31 / 37 / 43, 289 x 4096 9.5 / 9.3 / 9.0 / 9.1,
// 2000 x 8192 32 / 36 / 45 / 54, 6964 x 392 25 / 17 / 14 / 16, 6396 x 1024 27 / 19 / 17 / 21, 301 x 16384 22 / 23 / 23 / 23.
int back_blocks(int M) {
    const int most = 2 * device_cu_count();
    return M < most ? M : most;
}

template <bool kEight>
void launch_norm(const NormArgs& a, hipStream_t st) {
    const int n8 = a.K / 8;
#define QAIL_NORM(group, per)                                                                                                      \
    hipLaunchKernelGGL((rmsnorm_kernel<group, per, kEight>), dim3(group < 256 ? (a.M + 256 / group - 1) / (256 / group) : a.M),    \
                       dim3(group < 256 ? 256 : group), 0, st, a)
    if (n8 <= 64) QAIL_NORM(64, 1);
    else if (n8 <= 128) QAIL_NORM(64, 2);
    else if (n8 <= 256) QAIL_NORM(256, 1);
    else if (n8 <= 512) QAIL_NORM(256, 2);
    else if (n8 <= 1024) QAIL_NORM(256, 4);
    else if (n8 <= 2048) QAIL_NORM(1024, 2);
    else QAIL_NORM(1024, 4);
#undef QAIL_NORM
}

}  // namespace

bool rmsnorm_supports(int K) { return K <= kNormMaxK; }

hipError_t launch_rmsnorm(const uint16_t* x, const uint16_t* residual, const uint16_t* weight, float eps, int M, int K, uint16_t* h_out,
                          uint16_t* y, uint32_t* y_s8, float* y_scale, hipStream_t st) {
    const NormArgs a{x, residual, weight, h_out, y, y_s8, y_scale, eps, 1.0f / (float)K, M, K};
    if (y_s8) launch_norm<true>(a, st);
    else launch_norm<false>(a, st);
    return hipGetLastError();
}

size_t rmsnorm_back_workspace(int M, int K) { return (size_t)back_blocks(M) * K * sizeof(float); }

hipError_t launch_rmsnorm_back(const uint16_t* h, const uint16_t* weight, float eps, const uint16_t* dy, const uint16_t* dres, int M, int K,
                               uint16_t* dx, float* dweight, float* ws, hipStream_t st) {
    const NormBackArgs a{h, weight, dy, dres, dx, ws, eps, 1.0f / (float)K, M, K};
    const int n8 = K / 8, blocks = back_blocks(M);
#define QAIL_BACK(group, per) hipLaunchKernelGGL((rmsnorm_back_kernel<group, per>), dim3(blocks), dim3(group), 0, st, a)
    if (n8 <= 64) QAIL_BACK(64, 1);
    else if (n8 <= 256) QAIL_BACK(256, 1);
    else if (n8 <= 512) QAIL_BACK(256, 2);
    else if (n8 <= 1024) QAIL_BACK(1024, 1);
    else if (n8 <= 2048) QAIL_BACK(1024, 2);
    else QAIL_BACK(1024, 4);
#undef QAIL_BACK
    hipLaunchKernelGGL(rmsnorm_weight_kernel, dim3((K / 4 + 15) / 16), dim3(16 * kSlices), 0, st, ws, blocks, K, dweight);
    return hipGetLastError();
}

}  // namespace qail
