// The writer of the paged cache: rotates a step's new keys and queries and stores keys and values in their requests' pages.
//
// Bound by memory, or at a few tokens by the latency of finding a token's place: q_start -> request -> kv_len and page -> slot.
// head_dim / 16 lanes share a head, each with eight values of either half, so that a lane has both values of its rotations and
// a head's largest magnitude is three exchanges away.  Where the cache has bytes, codes are decided in fp32 without fused
// multiply-adds: the same codes come out of any correct fp32 implementation of the formulas.  16 tokens of 32 heads of 128 take 3.0 us,
// 5512 into a cache of bytes 56 us (228 MB, 4.1 TB/s), with the vector unit busy for 78 % of them.
#include "kv_cache.h"

namespace qail {

namespace {

struct AppendArgs {
    CacheArgs c;
    const uint16_t *k, *v, *q;
    uint16_t* q_out;
    const float *cos, *sin;
    long long k_stride, v_stride, q_stride;
    int q_heads, positions;
};

// A block's heads of a token.
template <int D, bool kEight>
__device__ __forceinline__ void append_token(const AppendArgs& a) {
    constexpr int kLanes = D / 16, kHalf = D / 2;
    const int t = blockIdx.x, H = a.c.heads;
    const int unit = blockIdx.y * (256 / kLanes) + threadIdx.x / kLanes;   // head: keys, values, then queries
    const int i = threadIdx.x % kLanes * 8;
    const int r = request_of(a.c, t);
    bool bad = r < 0;
    Request q{0, 0, 0};
    if (!bad) q = request(a.c, r, bad);
    int at = 0;
    if (bad || !has_slot(q, t, a.positions, at)) {   // the whole block
        if (threadIdx.x == 0 && blockIdx.y == 0) report(a.c);
        return;
    }
    if (unit >= 2 * H + a.q_heads) return;   // no exchange crosses a head's lanes
    const bool key = unit < H, value = !key && unit < 2 * H;
    const uint16_t* src = key ? a.k + t * a.k_stride + unit * D : value ? a.v + t * a.v_stride + (unit - H) * D : a.q + t * a.q_stride + (unit - 2 * H) * D;
    const uint4 lo = *reinterpret_cast<const uint4*>(src + i), hi = *reinterpret_cast<const uint4*>(src + kHalf + i);
    float x[8], y[8];
    unpack8(lo, x);
    unpack8(hi, y);
    if (a.cos && !value) {
#pragma clang fp contract(off)
        float c[8], s[8];
        const float4* cp = reinterpret_cast<const float4*>(a.cos + (size_t)at * kHalf + i);
        const float4* sp = reinterpret_cast<const float4*>(a.sin + (size_t)at * kHalf + i);
        *reinterpret_cast<float4*>(c) = cp[0];
        *reinterpret_cast<float4*>(c + 4) = cp[1];
        *reinterpret_cast<float4*>(s) = sp[0];
        *reinterpret_cast<float4*>(s + 4) = sp[1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = x[e] * c[e] - y[e] * s[e], w = y[e] * c[e] + x[e] * s[e];
            x[e] = u;
            y[e] = w;
        }
    }
    if (!key && !value) {
        uint16_t* out = a.q_out + ((size_t)t * a.q_heads + (unit - 2 * H)) * D;
        *reinterpret_cast<uint4*>(out + i) = pack8(x);
        *reinterpret_cast<uint4*>(out + kHalf + i) = pack8(y);
        return;
    }
    const int page = a.c.table[(size_t)r * a.c.max_pages + (at >> a.c.page_shift)];
    if (!is_page(page, a.c.num_pages)) {
        report(a.c);
        return;
    }
    const size_t slot = ((((size_t)page * H + (key ? unit : unit - H)) << a.c.page_shift) + (at & ((1 << a.c.page_shift) - 1)));
    if constexpr (kEight) {
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max_magnitude(most, max_magnitude(fabsf(x[e]), fabsf(y[e])));
#pragma unroll
        for (int o = kLanes / 2; o >= 1; o >>= 1) most = max_magnitude(most, __shfl_xor(most, o, kWave));
        const float s = most > 0.f ? most / 127.0f : 1.0f;
        auto codes = [&](const float* f) {
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e / 4] |= ((uint32_t)(int)fminf(fmaxf(rintf(f[e] / s), -127.f), 127.f) & 255u) << (8 * (e % 4));
            return uint2{w[0], w[1]};
        };
        uint8_t* out = static_cast<uint8_t*>(key ? a.c.k : a.c.v) + slot * D;
        *reinterpret_cast<uint2*>(out + i) = codes(x);
        *reinterpret_cast<uint2*>(out + kHalf + i) = codes(y);
        if (i == 0) (key ? a.c.k_scale : a.c.v_scale)[slot] = most < INFINITY ? s : __builtin_nanf("");   // no code could say that a value is not finite
    } else {
        uint16_t* out = static_cast<uint16_t*>(key ? a.c.k : a.c.v) + slot * D;
        *reinterpret_cast<uint4*>(out + i) = pack8(x);
        *reinterpret_cast<uint4*>(out + kHalf + i) = pack8(y);
    }
}

template <int D, bool kEight>
__global__ __launch_bounds__(256) void kv_append_kernel(const AppendArgs a) {
    append_token<D, kEight>(a);
    if (blockIdx.x == 0 && blockIdx.y == 0) report_rows(a.c);   // at the end: after an atomic the arrays' loads are no scalar ones (55 -> 65 us at 5512 tokens)
}

}  // namespace

hipError_t launch_kv_append(const qail_kv_cache& c, const qail_requests& b, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                            const uint16_t* q, int64_t q_stride, int q_heads, uint16_t* q_out, const float* cos, const float* sin, int positions,
                            uint32_t* errors, hipStream_t st) {
    const AppendArgs a{cache_args(c, b, errors), k, v, q, q_out, cos, sin, k_stride, v_stride, q_stride, q ? q_heads : 0, cos ? positions : 0};
    const int units = 2 * c.heads + a.q_heads, per = 256 / (c.head_dim / 16);
    const dim3 grid(b.tokens, (units + per - 1) / per);
    const bool eight = c.type == QAIL_KV_S8;
    auto* const kernel = c.head_dim == 128 ? (eight ? kv_append_kernel<128, true> : kv_append_kernel<128, false>)
                                           : (eight ? kv_append_kernel<64, true> : kv_append_kernel<64, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qail
