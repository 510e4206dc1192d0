// Causal attention of new tokens over a paged cache.
//
// Scores are computed transposed, S^T = K Q^T, so that a lane of the result holds one row's (query's) scores for several keys: a row's maximum
// and sum are a few exchanges between the lanes that share a column, its rescaling factor is where its output column
// O^T = V^T P^T is, and the scores' registers are the second product's operand as they are.  The keys that a lane holds are
// chosen by the order in which rows of K enter the first product, which is free.
//
// Rows of one request and one head of the cache: row i is token i / group, head i % group, so grouped heads share every key that is loaded.
#include "attention_plan.h"

namespace qail {

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(8))) short s16x8_t;
typedef __attribute__((ext_vector_type(2))) int i32x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;   // (arrays of HIP's own uint4 end up in scratch memory)

struct AttentionArgs {
    CacheArgs c;
    const uint16_t* q;
    uint16_t* out;
    float* part_o;      // partial results, D values each, not yet divided by their sum,
    float2* part_ml;    // and their maximum and sum: [places][16] of the stream, [tokens][q_heads][most] of the tiles
    long long q_stride;
    float scale;        // times log2(e)
    int q_heads, group;
    // stream: requests of at most max_rows rows; all steps shared by `blocks` blocks, `least` of them each, or a block for each request and head
    int max_rows, shared, blocks, least;
    // tiles: requests of at least min_rows rows, in at most `tiles` tiles; the keys of a tile in shares of `chunk`, at most `most`
    int min_rows, tiles, chunk, most;
};

__device__ __forceinline__ bf16x8_t as_bf16x8(const u32x4_t& v) { return __builtin_bit_cast(bf16x8_t, v); }

// Eight signed bytes as bf16 (exact).
__device__ __forceinline__ bf16x8_t codes_to_bf16(uint32_t lo, uint32_t hi) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t src = i < 2 ? lo : hi;
        const int sh = i % 2 * 16;
        const float x = (float)(int)(int8_t)(src >> sh), y = (float)(int)(int8_t)(src >> (sh + 8));
        w[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, x), 0x07060302u);   // upper halves
    }
    return __builtin_bit_cast(bf16x8_t, u32x4_t{w[0], w[1], w[2], w[3]});
}

// One row by one wave, which reads no key behind the row's last: keys k0 .. last of request r and head h.  The products on the matrix cores
// multiply by a p of zero the values of keys that a row does not see, and the last key's in every place behind it; zero times an infinity or NaN is
// NaN: where that may have happened (a result that is not finite, of a row whose sum is) the row is computed again, here.
// A lane takes a key of 64 for the scores, then D / 64 values of every key.  o, m and l as in the kernels: not yet divided by l.
template <int D, bool kEight>
__device__ __forceinline__ void attend_row_alone(const AttentionArgs& a, int r, int h, const uint16_t* q, int k0, int last, float* o, float& m, float& l) {
    constexpr int kRowBytes = kEight ? D : 2 * D, kPer = D / kWave;
    const int lane = threadIdx.x % kWave, slots = 1 << a.c.page_shift;
    bool bad = false;   // (has been reported)
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.f;
#pragma unroll 1
    for (int kt = k0; kt <= last; kt += kWave) {
        const int key = min(kt + lane, last);
        const size_t slot = (((size_t)page_of(a.c, page_entry(a.c, r, key >> a.c.page_shift), bad) * a.c.heads + h) << a.c.page_shift) + (key & (slots - 1));
        const uint8_t* const k = static_cast<const uint8_t*>(a.c.k) + slot * kRowBytes;
        float s = 0.f;
#pragma unroll 1
        for (int d = 0; d < D; d += 8) {
            bf16x8_t kd;
            if constexpr (kEight) {
                const uint2 c = *reinterpret_cast<const uint2*>(k + d);
                kd = codes_to_bf16(c.x, c.y);
            } else {
                kd = as_bf16x8(*reinterpret_cast<const u32x4_t*>(k + 2 * d));
            }
            const bf16x8_t qd = as_bf16x8(*reinterpret_cast<const u32x4_t*>(q + d));
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf((float)kd[e], (float)qd[e], s);
        }
        if constexpr (kEight) s *= a.c.k_scale[slot];
        if (kt + lane > last) s = -INFINITY;
        float top = s;
#pragma unroll
        for (int i = 32; i >= 1; i >>= 1) top = fmaxf(top, __shfl_xor(top, i, kWave));
        const float m_new = fmaxf(m, top), off = m_new == -INFINITY ? 0.f : m_new * a.scale;
        const float alpha = __builtin_amdgcn_exp2f(m * a.scale - off);   // 0 where there was no key yet
        float p = __builtin_amdgcn_exp2f(fmaf(s, a.scale, -off)), sum = p;
#pragma unroll
        for (int i = 32; i >= 1; i >>= 1) sum += __shfl_xor(sum, i, kWave);
        l = fmaf(l, alpha, sum);
        m = m_new;
        if constexpr (kEight) p *= a.c.v_scale[slot];
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] *= alpha;
        const int held = min(kWave, last + 1 - kt);
#pragma unroll 1
        for (int i0 = 0; i0 < held; i0 += 8) {
            float x[8][kPer];
#pragma unroll
            for (int u = 0; u < 8; ++u) {   // past the end the last is read again and not counted
                const uint8_t* const v = static_cast<const uint8_t*>(a.c.v) + (size_t)__shfl((long long)slot, min(i0 + u, held - 1), kWave) * kRowBytes;
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    if constexpr (kEight) x[u][e] = (float)reinterpret_cast<const int8_t*>(v)[lane * kPer + e];
                    else x[u][e] = bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(v)[lane * kPer + e]);
                }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float pi = __shfl(p, min(i0 + u, held - 1), kWave);
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (i0 + u < held) o[e] = fmaf(pi, x[u][e], o[e]);
            }
        }
    }
}

// 1 / l for a row at position `pos`.  A row that sees no key is zeros; one whose keys all have a score of minus infinity has no largest: NaN.
__device__ __forceinline__ float inverse(float l, int pos) { return l > 0.f ? 1.0f / l : l == 0.f && pos < 0 ? 0.f : __builtin_nanf(""); }

// That row's result to `out`, or to place `at` of the partial ones where there is one.
template <int D>
__device__ __forceinline__ void store_row_alone(const AttentionArgs& a, const float* o, float m, float l, int pos, uint16_t* out, long long at) {
    constexpr int kPer = D / kWave;
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        if (at < 0) out[lane * kPer + e] = (uint16_t)f32x2_to_bf16x2_rne(o[e] * inverse(l, pos), 0.f);
        else a.part_o[at * D + lane * kPer + e] = o[e];
    }
    if (at >= 0 && lane == 0) a.part_ml[at] = make_float2(m, l);
}

// ---------------------------------------------------------------------------- few rows: a stream of keys --
//
// Up to 16 rows (a decode step: the heads that share a head of the cache) against all keys: bound by the cache's bytes, each read
// once.  A wave takes 32 keys at a time, on its own: K goes from memory into the registers that the first product reads,
// V through the wave's part of LDS, which is read transposed.  The four waves of a block take tiles in turn and add up at the end.
// Rows past the last key repeat it (its slot holds a token, which slots behind it need not) and get a score of minus infinity.  64 requests of
// 500 to 8000 8-bit keys, 32 heads to 8: 589 MB in 133 us with the join, 4.4 TB/s; one of 295 bf16 keys 7.2 us, which are trips to memory.
constexpr int kStreamWaves = 4, kStreamKeys = 32;   // a step (kStepKeys) is a tile of keys for each wave
static_assert(kStreamWaves * kStreamKeys == kStepKeys, "a step is a tile of keys for each wave");

template <int D, bool kEight>
struct Stream {
    static constexpr int kRowBytes = kEight ? D : 2 * D;
    static constexpr int kSteps = D / 32;                          // of the first product
    static constexpr int kLoadsK = kEight ? D / 64 : D / 32;       // 16-byte loads of a lane per tile of 16 keys
    static constexpr int kLanesV = kRowBytes / 16;                 // lanes that load a row of V
    static constexpr int kSlots = kWave / kLanesV;                 // rows a load instruction covers
    static constexpr int kLoadsV = kStreamKeys / kSlots;
    static constexpr int kPadO = D + 4;
    static constexpr int kLds = kStreamWaves * (kStreamKeys * kRowBytes > 16 * kPadO * 4 ? kStreamKeys * kRowBytes : 16 * kPadO * 4);

    // V's rows lie in LDS with their 16-byte pieces exchanged so that the rows read together lie in different banks.
    __device__ static __forceinline__ int swizzle(int row, int piece) {
        if constexpr (kEight) return kRowBytes == 128 ? piece ^ ((row >> 1) & 7) : piece ^ ((row >> 2) & 3);
        else return kRowBytes == 256 ? piece ^ (((row & 3) | ((row >> 1) & 4)) << 1) : piece ^ ((((row >> 1) & 1) | ((row >> 2) & 2)) << 1);
    }
};

// Keys k0 .. k1 - 1 of request r and head h for its rows from row0.  place < 0: these are all keys, the outputs are written; else they are left
// in that place, with their maximum and sum, for the join.
template <int D, bool kEight>
__device__ __forceinline__ void attend_rows(const AttentionArgs& a, uint8_t* lds, float2 (*ml)[kStreamRows], const Request& rq, int r, int h, int row0, int k0, int k1,
                                            long long place, bool& bad) {
    using S = Stream<D, kEight>;
    const int H = a.c.heads, rows = rq.n * a.group, before = rq.len - rq.n;   // keys in front of the new ones; may be negative
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, col = lane % 16, g = lane / 16;
    uint8_t* const lds_v = lds + wave * kStreamKeys * S::kRowBytes;
    float* const lds_o = reinterpret_cast<float*>(lds);
    {
        const int row = row0 + col, token = row / a.group, head = h * a.group + row % a.group;
        const int pos = row < rows ? before + token : -1;

        bf16x8_t q[S::kSteps];
#pragma unroll
        for (int s = 0; s < S::kSteps; ++s) {   // bytes: a lane's 16 codes of K are two steps
            const int d = kEight ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
            q[s] = as_bf16x8(row < rows ? *reinterpret_cast<const u32x4_t*>(a.q + (rq.start + token) * a.q_stride + head * D + d) : u32x4_t{0u, 0u, 0u, 0u});
        }
        f32x4_t o[D / 16];
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;

        // Of the 32 keys from `kt`, lane group g has keys 8 g .. 8 g + 7 after the first product: row 4 g' + i of tile t is key 8 g' + 4 t + i.
        const int key_k = 8 * (col / 4) + col % 4;
        const int slot_v = lane / S::kLanesV, row_v = 8 * (slot_v / (S::kSlots / 4)) + slot_v % (S::kSlots / 4) * S::kLoadsV;
        u32x4_t kv[2][S::kLoadsK], vv[S::kLoadsV];
        float ks[8], vs[8];
        int entry_k, entry_v, entry_s;   // of the page table, for the tile that is loaded next
        auto entries = [&](int kt) {     // eight keys never lie in two pages
            entry_k = page_entry(a.c, r, min(kt + 8 * (col / 4), k1 - 1) >> a.c.page_shift);
            entry_v = page_entry(a.c, r, min(kt + row_v / 8 * 8, k1 - 1) >> a.c.page_shift);
            if constexpr (kEight) entry_s = page_entry(a.c, r, min(kt + 8 * g, k1 - 1) >> a.c.page_shift);
        };
        const int slots = 1 << a.c.page_shift;
        auto load_k = [&](int kt) {
            const uint8_t* base = static_cast<const uint8_t*>(a.c.k) + ((((size_t)page_of(a.c, entry_k, bad) * H + h) << a.c.page_shift) * S::kRowBytes);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint8_t* p = base + (min(kt + key_k + 4 * t, k1 - 1) & (slots - 1)) * S::kRowBytes;
#pragma unroll
                for (int s = 0; s < S::kLoadsK; ++s) kv[t][s] = *reinterpret_cast<const u32x4_t*>(p + 64 * s + 16 * g);
            }
        };
        auto load_v = [&](int kt) {
            const uint8_t* base = static_cast<const uint8_t*>(a.c.v) + ((((size_t)page_of(a.c, entry_v, bad) * H + h) << a.c.page_shift) * S::kRowBytes) + lane % S::kLanesV * 16;
#pragma unroll
            for (int n = 0; n < S::kLoadsV; ++n)
                vv[n] = *reinterpret_cast<const u32x4_t*>(base + (min(kt + row_v + n, k1 - 1) & (slots - 1)) * S::kRowBytes);
        };
        auto load_steps = [&](int kt) {
            const size_t base = (((size_t)page_of(a.c, entry_s, bad) * H + h) << a.c.page_shift);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const size_t at = base + (min(kt + 8 * g + i, k1 - 1) & (slots - 1));
                ks[i] = a.c.k_scale[at];
                vs[i] = a.c.v_scale[at];
            }
        };
        constexpr int kStride = kStepKeys;
        int kt = k0 + wave * kStreamKeys;
        if (kt < k1) {
            entries(kt);
            load_v(kt);
            load_k(kt);
            if constexpr (kEight) load_steps(kt);
            entries(kt + kStride);   // (the last key's beyond the end)
        }
        for (; kt < k1; kt += kStride) {
            const bool more = kt + kStride < k1;
#pragma unroll
            for (int n = 0; n < S::kLoadsV; ++n)
                *reinterpret_cast<u32x4_t*>(lds_v + (row_v + n) * S::kRowBytes + S::swizzle(row_v + n, lane % S::kLanesV) * 16) = vv[n];
            if (more) load_v(kt + kStride);
            f32x4_t sc[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                sc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < S::kSteps; ++s) {
                    bf16x8_t kf;
                    if constexpr (kEight) kf = s % 2 ? codes_to_bf16(kv[t][s / 2].z, kv[t][s / 2].w) : codes_to_bf16(kv[t][s / 2].x, kv[t][s / 2].y);
                    else kf = as_bf16x8(kv[t][s]);
                    sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[s], sc[t], 0, 0, 0);
                }
            }
            if (more) load_k(kt + kStride);
            float p[8], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = sc[i / 4][i % 4];
                if constexpr (kEight) p[i] *= ks[i];
                const int key = kt + 8 * g + i;
                p[i] = key <= pos && key < k1 ? p[i] : -INFINITY;
                top = fmaxf(top, p[i]);
            }
            top = fmaxf(top, __shfl_xor(top, 16, kWave));
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float m_new = fmaxf(m, top), off = m_new == -INFINITY ? 0.f : m_new * a.scale;
            if (__any(m_new > m)) {
                const float alpha = __builtin_amdgcn_exp2f(m * a.scale - off);   // 0 where there was no key yet
                l *= alpha;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) o[d] *= alpha;
                m = m_new;
            }
            // p in two parts, each rounded to bf16: 2^-16 of it may be lost instead of 2^-8, for D / 16 more products of 32 keys (one request of 295 keys 7.0 -> 7.2 us,
            // 64 of 8-bit keys 129 -> 133)
            uint32_t ph[4], pl[4];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], a.scale, -off));
                l += p[i];
                if constexpr (kEight) p[i] *= vs[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ph[i] = f32x2_to_bf16x2_rne(p[2 * i], p[2 * i + 1]);
                pl[i] = f32x2_to_bf16x2_rne(p[2 * i] - __builtin_bit_cast(float, ph[i] << 16), p[2 * i + 1] - __builtin_bit_cast(float, ph[i] & 0xFFFF0000u));
            }
            const bf16x8_t upper = as_bf16x8(u32x4_t{ph[0], ph[1], ph[2], ph[3]}), lower = as_bf16x8(u32x4_t{pl[0], pl[1], pl[2], pl[3]});
            if (more) {
                if constexpr (kEight) load_steps(kt + kStride);
                entries(kt + 2 * kStride);
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                bf16x8_t vf;
                if constexpr (kEight) {
                    const int rv = 8 * g + col / 2;
                    const i32x2_t c = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                        (__attribute__((address_space(3))) i32x2_t*)(lds_v + rv * S::kRowBytes + S::swizzle(rv, d) * 16 + col % 2 * 8));
                    vf = codes_to_bf16((uint32_t)c[0], (uint32_t)c[1]);
                } else {
                    s16x4_t part[2];
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int rv = 8 * g + 4 * t + col / 4;
                        part[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(
                            lds_v + rv * S::kRowBytes + S::swizzle(rv, 2 * d + col % 4 / 2) * 16 + col % 2 * 8));
                    }
                    const s16x8_t both = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    vf = __builtin_bit_cast(bf16x8_t, both);
                }
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, upper, o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lower, o[d], 0, 0, 0);
            }
        }
        l += __shfl_xor(l, 16, kWave);
        l += __shfl_xor(l, 32, kWave);

        // the waves' shares, added up: o[d][i] of lane (col, g) is output 16 d + 4 g + i of row col
        __syncthreads();   // no wave reads V any more
        if (g == 0) ml[wave][col] = make_float2(m, l);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4_t*>(lds_o + (wave * 16 + col) * S::kPadO + 16 * d + 4 * g) = o[d];
        __syncthreads();
        constexpr int kLanesO = D / 8;   // of an output row, eight values each
        static_assert(kStreamWaves * kWave / kLanesO >= kStreamRows, "the block's threads cover all rows");
        const int i = threadIdx.x / kLanesO, d = threadIdx.x % kLanesO * 8, n = min(kStreamRows, rows - row0);
        float top = -INFINITY, sum = 0.f, acc[8] = {}, odd = 0.f;
        if (i < n) {
#pragma unroll
            for (int w = 0; w < kStreamWaves; ++w) top = fmaxf(top, ml[w][i].x);
#pragma unroll
            for (int w = 0; w < kStreamWaves; ++w) {
                const float f = ml[w][i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[w][i].x - top) * a.scale);
                sum = fmaf(f, ml[w][i].y, sum);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = fmaf(f, lds_o[(w * 16 + i) * S::kPadO + d + e], acc[e]);
            }
        }
        // where a row's result goes, and whether that is a partial one
        auto out_of = [&](int row) { return (size_t)(rq.start + (row0 + row) / a.group) * a.q_heads + h * a.group + (row0 + row) % a.group; };
        if (i < n && sum == sum)   // its own scores are no NaN
#pragma unroll
            for (int e = 0; e < 8; ++e) odd = fmaf(acc[e], 0.f, odd);
        unsigned long long left = __ballot(odd != 0.f);   // NaN
        const bool again = (left >> (lane / kLanesO * kLanesO)) & ((1ull << kLanesO) - 1);
        if (i < n && !again) {
            if (place < 0) {
                const float inv = inverse(sum, before + (row0 + i) / a.group);
                u32x4_t w;
                w.x = f32x2_to_bf16x2_rne(acc[0] * inv, acc[1] * inv);
                w.y = f32x2_to_bf16x2_rne(acc[2] * inv, acc[3] * inv);
                w.z = f32x2_to_bf16x2_rne(acc[4] * inv, acc[5] * inv);
                w.w = f32x2_to_bf16x2_rne(acc[6] * inv, acc[7] * inv);
                *reinterpret_cast<u32x4_t*>(a.out + out_of(i) * D + d) = w;
            } else {
                const long long to = place * kStreamRows + i;
                float4* out = reinterpret_cast<float4*>(a.part_o + to * D + d);
                out[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                out[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
                if (d == 0) a.part_ml[to] = make_float2(top, sum);
            }
        }
        while (__builtin_expect(left != 0, 0)) {   // the wave's rows that are computed again
            const int which = __builtin_ctzll(left) / kLanesO, row = wave * (kWave / kLanesO) + which, token = (row0 + row) / a.group;
            left &= ~(((1ull << kLanesO) - 1) << (which * kLanesO));
            float again_o[D / kWave], again_m, again_l;
            attend_row_alone<D, kEight>(a, r, h, a.q + (rq.start + token) * a.q_stride + (h * a.group + (row0 + row) % a.group) * D, k0, min(before + token, k1 - 1), again_o, again_m, again_l);
            store_row_alone<D>(a, again_o, again_m, again_l, before + token, a.out + out_of(row) * D, place < 0 ? -1 : place * kStreamRows + row);
        }
        __syncthreads();
    }
}

// The steps of 64 requests and those before them in the same 64: what lane i holds is request first + i's.
struct Scan {
    long long mine, sum;
};
__device__ __forceinline__ Scan scan_steps(const AttentionArgs& a, int first) {
    const int r = first + (int)threadIdx.x % kWave;
    bool bad;
    const Steps s = r < a.c.requests ? steps_of(request(a.c, r, bad), a.group, a.max_rows) : Steps{0, 0};
    Scan v;
    v.mine = v.sum = (long long)s.tiles * s.steps * a.c.heads;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const long long left = __shfl_up(v.sum, o, kWave);
        if ((int)threadIdx.x % kWave >= o) v.sum += left;
    }
    return v;
}
__device__ __forceinline__ long long value_of_lane(long long v, int lane) {
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (unsigned)__builtin_amdgcn_readlane((int)v, lane));
}

template <int D, bool kEight>
__global__ __launch_bounds__(kStreamWaves* kWave, stream_blocks(D)) void attend_stream_kernel(const AttentionArgs a) {
    using S = Stream<D, kEight>;
    __shared__ __attribute__((aligned(16))) uint8_t lds[S::kLds];
    __shared__ float2 ml[kStreamWaves][kStreamRows];
    const int H = a.c.heads;
    bool bad;
    if (!a.shared) {   // a block for each request and head
        const int r = blockIdx.x / H, h = blockIdx.x % H;
        const Request rq = request(a.c, r, bad);
        if (bad && h == 0 && threadIdx.x == 0) report(a.c);
        bad = false;   // from here on: a page
        const Steps s = steps_of(rq, a.group, a.max_rows);
        for (int t = 0; t < s.tiles; ++t)
            attend_rows<D, kEight>(a, lds, ml, rq, r, h, t * kStreamRows, 0, keys_of(rq, a.group, t * kStreamRows, kStreamRows), -1, bad);
        if (bad) report(a.c);
        return;
    }
    const Scan near = scan_steps(a, 0);
    long long total = value_of_lane(near.sum, kWave - 1);
    for (int r0 = kWave; r0 < a.c.requests; r0 += kWave) total += value_of_lane(scan_steps(a, r0).sum, kWave - 1);
    const long long share = steps_of_a_share(total, gridDim.x, a.least), end = min((blockIdx.x + 1ll) * share, total);
    bool page_bad = false;
    for (long long p = blockIdx.x * share; p < end;) {
        int r = 0;
        long long first = 0;   // step of the request's beginning
        for (int r0 = 0; r0 < a.c.requests; r0 += kWave) {   // p < total: one is found
            const Scan v = r0 == 0 ? near : scan_steps(a, r0);
            const unsigned long long past = __ballot(first + v.sum > p);
            if (past) {
                const int at = __builtin_ctzll(past);
                r = r0 + at;
                first += value_of_lane(v.sum, at) - value_of_lane(v.mine, at);
                break;
            }
            first += value_of_lane(v.sum, kWave - 1);
        }
        const Request rq = request(a.c, r, bad);
        const Steps s = steps_of(rq, a.group, a.max_rows);
        if (bad && p == first && threadIdx.x == 0) report(a.c);
        const int unit = (int)((p - first) / s.steps), step = (int)((p - first) % s.steps), h = unit / s.tiles, row0 = unit % s.tiles * kStreamRows;
        const int steps = (int)min((long long)(s.steps - step), end - p);
        const int keys = keys_of(rq, a.group, row0, kStreamRows);
        attend_rows<D, kEight>(a, lds, ml, rq, r, h, row0, min(step * kStepKeys, keys), min((step + steps) * kStepKeys, keys),
                               steps == s.steps ? -1 : place_of(p - step, blockIdx.x, share), page_bad);
        p += steps;
    }
    if (page_bad) report(a.c);
    if (blockIdx.x == 0) report_rows(a.c);
}

// Adds up what the stream's blocks have left: a wave per output row.
constexpr int kJoinWaves = 4;

// The sum of `count` partial results of a row at position `pos`, the i-th in place(i), as bf16 to `out`.
template <int D, typename F>
__device__ __forceinline__ void join_row(const AttentionArgs& a, long long count, int pos, uint16_t* out, F place) {
    const int lane = threadIdx.x % kWave;
    float top = -INFINITY;
    for (long long i = lane; i < count; i += kWave) top = fmaxf(top, a.part_ml[place(i)].x);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    // D / 4 lanes take a partial result, the wave several at a time and four times as many on their way
    constexpr int kLanes = D / 4, kAtOnce = kWave / kLanes;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    for (long long i0 = 0; i0 < count; i0 += 4 * kAtOnce) {
        f32x4_t v[4];
        float2 ml[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {   // past the end the last is read again and not counted
            const long long at = place(min(i0 + u * kAtOnce + lane / kLanes, count - 1));
            v[u] = reinterpret_cast<const f32x4_t*>(a.part_o + at * D)[lane % kLanes];
            ml[u] = a.part_ml[at];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + u * kAtOnce + lane / kLanes >= count || ml[u].y == 0.f) continue;   // no key; scores that are all NaN leave a maximum of -inf too, and a sum of NaN
            const float w = __builtin_amdgcn_exp2f((ml[u].x - top) * a.scale);
            sum = fmaf(w, ml[u].y, sum);
            acc += v[u] * w;
        }
    }
#pragma unroll
    for (int o = kLanes; o < kWave; o <<= 1) {
        sum += __shfl_xor(sum, o, kWave);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o, kWave);
    }
    const float inv = inverse(sum, pos);
    if (lane < kLanes) reinterpret_cast<uint2*>(out)[lane] = uint2{f32x2_to_bf16x2_rne(acc[0] * inv, acc[1] * inv), f32x2_to_bf16x2_rne(acc[2] * inv, acc[3] * inv)};
}

template <int D>
__global__ __launch_bounds__(kJoinWaves* kWave) void join_stream_kernel(const AttentionArgs a) {
    const int r = blockIdx.x, head = blockIdx.y * kJoinWaves + threadIdx.x / kWave;
    if (head >= a.q_heads) return;   // whole waves
    long long total = 0, first = 0;
    for (int r0 = 0; r0 < a.c.requests; r0 += kWave) {
        const Scan v = scan_steps(a, r0);
        if (r >= r0 && r < r0 + kWave) first = total + value_of_lane(v.sum, r - r0) - value_of_lane(v.mine, r - r0);
        total += value_of_lane(v.sum, kWave - 1);
    }
    const long long share = steps_of_a_share(total, a.blocks, a.least);
    bool bad;
    const Request rq = request(a.c, r, bad);
    const Steps s = steps_of(rq, a.group, a.max_rows);
    if (s.tiles == 0) return;
    for (int token = blockIdx.z; token < rq.n; token += gridDim.z) {
        const int row = token * a.group + head % a.group;
        const long long begin = first + ((long long)(head / a.group) * s.tiles + row / kStreamRows) * s.steps;
        const long long b0 = begin / share, count = (begin + s.steps - 1) / share - b0 + 1;
        if (count == 1) continue;
        join_row<D>(a, count, rq.len - rq.n + token, a.out + ((size_t)(rq.start + token) * a.q_heads + head) * D,
                    [&](long long i) { return place_of(begin, b0 + i, share) * kStreamRows + row % kStreamRows; });
    }
}

// ---------------------------------------------------------------------------- many rows: tiles on the matrix cores --
//
// A block takes 128 rows, a wave 32 of them, against 64 keys at a time.  Both operands of the keys go through LDS, twice 64 keys: from memory
// straight into it (bytes through registers, as bf16 codes, their steps beside them), while the waves work on the 64 keys before.
// Bound by the vector unit next to the matrix cores: of 64 keys a wave has 32 products of 32 cycles each, and for every score a
// multiply-add, an exponential and three halves of an instruction for the maximum, the sum (two rounded p at a time) and
// the rounding.  So nothing else is left in the loop: places in LDS are registers and immediates (the loop has a copy for either half), places in memory
// scalars, but for the last 64 keys.  Four prompts to 2500 tokens (111 GFLOP) take 158 us, 700 TFLOP/s, three chunks behind 7000 to 13000 keys 790: the
// matrix cores are busy 36 and 40 % of the time and the vector unit 41 and 39 %, next to each other for little of it; a quarter of a wave's time is waiting.
// 32 keys at a time and three blocks a compute unit instead of two: prompts the same, chunks 171 -> 213.
constexpr int kTileWaves = 4;
static_assert(kTileRows == kTileWaves * 32, "a wave takes 32 rows");

template <int D, bool kEight>
struct Tile {
    static constexpr int kRowBytes = 2 * D;                        // of LDS
    static constexpr int kPieces = kEight ? D / 16 : D / 8;        // 16-byte pieces of a row in memory
    static constexpr int kPass = kTileWaves * kWave / kPieces;     // rows that the block loads at once
    static constexpr int kLoads = kTileKeys / kPass;
    static constexpr int kV = kTileKeys * kRowBytes, kSteps = 2 * kV;                 // K, V, their steps
    static constexpr int kBuffer = 2 * kV + (kEight ? 2 * kTileKeys * 4 : 0);
    static constexpr int kLds = 2 * kBuffer;

    // Pieces of a row are exchanged so that what is read together lies in different banks: K by 16 rows and one piece, V by
    // four rows and two neighbouring pieces of 32 bytes.
    __device__ static __forceinline__ int swizzle_k(int row, int piece) { return D == 128 ? piece ^ (row & 15) : piece ^ ((row >> 1) & 7); }
    __device__ static __forceinline__ int swizzle_v(int row, int piece) { return D == 128 ? piece ^ ((row & 3) << 2) : piece ^ ((row & 2) << 1); }
};

// The larger of a value and its counterpart in the other half of the wave.
__device__ __forceinline__ float max_of_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned a = r[0], b = r[1];   // (a bit cast of r[1] itself gives r[0])
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

constexpr int kVector = 0x002, kProducts = 0x008, kReads = 0x100;   // kinds of instructions, for the scheduler
typedef __attribute__((address_space(3))) uint8_t lds_t;
typedef __attribute__((address_space(1))) uint8_t global_t;

// 16 bytes of each lane from memory into LDS, lane i's to to + 16 i.
__device__ __forceinline__ void load_to_lds(const uint8_t* from, lds_t* to) {
#ifdef __HIP_DEVICE_COMPILE__   // (the host pass does not know the size)
    __builtin_amdgcn_global_load_lds((const global_t*)from, to, 16, 0, 0);
#endif
}

template <int D, bool kEight>
__global__ __launch_bounds__(kTileWaves* kWave, 2) void attend_tile_kernel(const AttentionArgs a) {
    using T = Tile<D, kEight>;
    __shared__ __attribute__((aligned(16))) uint8_t half0[T::kBuffer], half1[T::kBuffer];
    lds_t* const lds0 = (lds_t*)half0;
    lds_t* const lds1 = (lds_t*)half1;
    const int H = a.c.heads;
    const int h = blockIdx.x % H, split = blockIdx.x / H % a.most, tile = a.tiles - 1 - blockIdx.x / H / a.most;   // a request's longest first
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, col = lane % 32, half = lane / 32;
    int r, row0;
    if (blockIdx.x == 0) report_rows(a.c);
    bool bad;
    Request rq;
    if (!tile_of(a.c, a.group, a.min_rows, kTileRows, tile, r, row0, rq, bad)) return;
    if (bad && h == 0 && split == 0 && row0 == 0 && threadIdx.x == 0) report(a.c);
    const int rows = rq.n * a.group, before = rq.len - rq.n;
    const int keys = keys_of(rq, a.group, row0, kTileRows), count = shares(keys, a.chunk, a.most);
    if (split >= count) return;
    bad = false;   // from here on: a page
    const Range range = share_of(keys, a.chunk, count, split);
    const int k1 = range.end;

    bf16x8_t q[D / 16];
    f32x16_t o[D / 32];
    const int row = row0 + wave * 32 + col, token = row / a.group;
    const int lim = row < rows ? min(before + token, k1 - 1) : k1 - 1;   // the last key that the row sees; rows past the end are not stored
    const int lim_first = __builtin_amdgcn_readfirstlane(lim), lim_last = __builtin_amdgcn_readlane(lim, 31);   // they ascend
    {
        const uint16_t* p = a.q + (rq.start + (row < rows ? token : 0)) * a.q_stride + (h * a.group + row % a.group) * D + 8 * half;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) q[s] = as_bf16x8(row < rows ? *reinterpret_cast<const u32x4_t*>(p + 16 * s) : u32x4_t{0u, 0u, 0u, 0u});
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    // From memory: the block's threads cover kPass rows at a time; 16 rows never lie in two pages, so that a wave's rows begin at a scalar place.
    const int piece = threadIdx.x % T::kPieces, row_in = threadIdx.x / T::kPieces, group_in = wave * (kWave / T::kPieces) / 16 * 16;
    const int slots = 1 << a.c.page_shift;
    constexpr int kMemoryRow = T::kPieces * 16;
    const int from_k = (kEight ? piece : T::swizzle_k(row_in, piece)) * 16, from_v = (kEight ? piece : T::swizzle_v(row_in, piece)) * 16;
    u32x4_t kv[kEight ? T::kLoads : 1], vv[kEight ? T::kLoads : 1];
    float step;
    int entry[T::kLoads], entry_s;   // of the page table, for the keys that are loaded next
    auto entries = [&](int kt) {
#pragma unroll
        for (int n = 0; n < T::kLoads; ++n) entry[n] = page_entry(a.c, r, min(kt + n * T::kPass + group_in, k1 - 1) >> a.c.page_shift);
        if constexpr (kEight) entry_s = page_entry(a.c, r, min(kt + (int)threadIdx.x % kTileKeys, k1 - 1) >> a.c.page_shift);
    };
    auto load = [&](int kt, lds_t* to) {
        const bool whole = kt + kTileKeys <= k1;
#pragma unroll
        for (int n = 0; n < T::kLoads; ++n) {
            const size_t page = (size_t)(unsigned)__builtin_amdgcn_readfirstlane(page_of(a.c, entry[n], bad)) * H + h;
            const int first = (kt + n * T::kPass + group_in) & (slots - 1);
            // rows past the last key repeat it (its slot holds a token, which slots behind it need not) and are masked
            const int slot = whole ? row_in % 16 : (min(kt + n * T::kPass + row_in, k1 - 1) & (slots - 1)) - first;
            const size_t base = ((page << a.c.page_shift) + first) * kMemoryRow;
            const uint8_t* const kp = static_cast<const uint8_t*>(a.c.k) + base + slot * kMemoryRow + from_k;
            const uint8_t* const vp = static_cast<const uint8_t*>(a.c.v) + base + slot * kMemoryRow + from_v;
            if constexpr (kEight) {
                kv[n] = *reinterpret_cast<const u32x4_t*>(kp);
                vv[n] = *reinterpret_cast<const u32x4_t*>(vp);
            } else {
                lds_t* const at = to + (n * T::kPass + wave * (kWave / T::kPieces)) * T::kRowBytes;   // of the wave; lane i's 16 bytes go to i * 16
                load_to_lds(kp, at);
                load_to_lds(vp, at + T::kV);
            }
        }
        if constexpr (kEight) {
            if (threadIdx.x < 2 * kTileKeys) {   // threads 0 .. 63 a step of K each, 64 .. 127 of V
                const int key = min(kt + (int)threadIdx.x % kTileKeys, k1 - 1);
                const size_t at = (((size_t)page_of(a.c, entry_s, bad) * H + h) << a.c.page_shift) + (key & (slots - 1));
                step = (threadIdx.x < kTileKeys ? a.c.k_scale : a.c.v_scale)[at];
            }
        }
    };
    auto store = [&](lds_t* to) {   // what has been loaded is in LDS when the block's barrier is passed
        if constexpr (kEight) {
#pragma unroll
            for (int n = 0; n < T::kLoads; ++n) {
                const int at = n * T::kPass + row_in;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const bf16x8_t kc = i ? codes_to_bf16(kv[n].z, kv[n].w) : codes_to_bf16(kv[n].x, kv[n].y);
                    const bf16x8_t vc = i ? codes_to_bf16(vv[n].z, vv[n].w) : codes_to_bf16(vv[n].x, vv[n].y);
                    *(__attribute__((address_space(3))) bf16x8_t*)(to + at * T::kRowBytes + T::swizzle_k(at, 2 * piece + i) * 16) = kc;
                    *(__attribute__((address_space(3))) bf16x8_t*)(to + T::kV + at * T::kRowBytes + T::swizzle_v(at, 2 * piece + i) * 16) = vc;
                }
            }
            if (threadIdx.x < 2 * kTileKeys) ((__attribute__((address_space(3))) float*)(to + T::kSteps))[threadIdx.x] = step;
        } else {
            __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
        }
    };

    // From LDS: K's row 32 u + col, piece 2 s + half; V's row 16 st + 8 j + 4 half + lane % 16 / 4, pieces 4 d + 2 (lane / 16 % 2) and the next.
    int at_k[D / 16], at_v[D / 32];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) at_k[s] = col * T::kRowBytes + T::swizzle_k(col, 2 * s + half) * 16;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        const int first = 4 * half + lane % 16 / 4;
        at_v[d] = T::kV + first * T::kRowBytes + T::swizzle_v(first, 4 * d + 2 * (lane / 16 % 2) + lane % 4 / 2) * 16 + lane % 2 * 8;
    }
    auto compute = [&](int kt, const lds_t* from) {
        if (kt > lim_last) return;   // no row of the wave sees a key
        f32x16_t sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[u][e] = 0.f;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                const bf16x8_t kf = *(const __attribute__((address_space(3))) bf16x8_t*)(from + at_k[s] + 32 * u * T::kRowBytes);
                sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[s], sc[u], 0, 0, 0);
            }
        }
        // six reads ahead of the products
        __builtin_amdgcn_sched_group_barrier(kReads, 6, 0);
#pragma unroll
        for (int i = 0; i < D / 8 - 6; ++i) {
            __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kReads, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kProducts, 6, 0);
        // element e of half u is key kt + 32 u + 8 (e / 4) + 4 half + e % 4
        const __attribute__((address_space(3))) f32x4_t* const steps = (const __attribute__((address_space(3))) f32x4_t*)(from + T::kSteps) + half;
        if constexpr (kEight) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4_t k4 = steps[8 * u + e / 2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[u][e + i] *= k4[i];
                }
        }
        if (kt + kTileKeys - 1 > lim_first) {
            const int left = lim - kt - 4 * half;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * u + 8 * (e / 4) + e % 4 > left) sc[u][e] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[u][e]);
        top = max_of_halves(top);
        // the maximum is followed only where it has grown by more than 2^8: p stays far from overflow, and a tile rarely rescales
        if (__any((top - m) * a.scale > 8.f)) {
            const float m_new = fmaxf(m, top), alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m_new) * a.scale);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[d] *= alpha;
        }
        const float off = m == -INFINITY ? 0.f : m * a.scale;
        __builtin_amdgcn_s_setprio(1);   // the other wave of the SIMD gets what these products leave: 181 -> 177 us at 384 rows behind 13000 keys
        bf16x8_t pf[4];
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            // p is rounded to bf16 once: in two parts, as with few rows, the error against 64 bits would be 0.0016 of the result's norm instead of 0.0021 (prompts) and
            // 0.0024 (chunks), and the kernel takes 161 -> 195 us and 168 -> 210.  Without steps the sum is fp32 of the rounded p, so that weights add up to one.
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = 8 * (st % 2) + 2 * e;
                float x = __builtin_amdgcn_exp2f(fmaf(sc[st / 2][at], a.scale, -off)), y = __builtin_amdgcn_exp2f(fmaf(sc[st / 2][at + 1], a.scale, -off));
                if constexpr (kEight) {
                    l += x + y;
                    const f32x4_t v4 = steps[kTileKeys / 4 + 8 * (st / 2) + at / 4 * 2];
                    x *= v4[at % 4];
                    y *= v4[at % 4 + 1];
                }
                w[e] = f32x2_to_bf16x2_rne(x, y);
                if constexpr (!kEight) {
                    const uint32_t ones = 0x3F803F80u;
                    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[e]), __builtin_bit_cast(bf16x2_t, ones), l, false);
                }
            }
            pf[st] = as_bf16x8(u32x4_t{w[0], w[1], w[2], w[3]});
        }
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int d = 0; d < D / 32; ++d) {
                const lds_t* const at = from + at_v[d] + 16 * st * T::kRowBytes;
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)at);
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(at + 8 * T::kRowBytes));
                const s16x8_t both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, both), pf[st], o[d], 0, 0, 0);
            }
        // the exponentials of the next 16 keys between the products of these
        constexpr int kAhead = D / 32, kBetween = (kEight ? 40 : 28) / kAhead;
        __builtin_amdgcn_sched_group_barrier(kReads, 2 * kAhead, 0);
        __builtin_amdgcn_sched_group_barrier(kVector, kAhead * kBetween, 0);
#pragma unroll
        for (int i = 0; i < 4 * kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
            if (i < 3 * kAhead) {
                __builtin_amdgcn_sched_group_barrier(kReads, 2, 0);
                __builtin_amdgcn_sched_group_barrier(kVector, kBetween, 0);
            }
        }
    };
    auto turn = [&](int kt, lds_t* mine, lds_t* next) {
        __syncthreads();
        const bool more = kt + kTileKeys < k1;
        if (more) {
            load(kt + kTileKeys, next);
            entries(kt + 2 * kTileKeys);
        }
        compute(kt, mine);
        __builtin_amdgcn_s_setprio(0);
        if (more) store(next);
    };
    if (range.begin < k1) {
        entries(range.begin);
        load(range.begin, lds0);
        entries(range.begin + kTileKeys);   // (the last key's beyond the end)
        store(lds0);
        for (int kt = range.begin; kt < k1; kt += 2 * kTileKeys) {
            turn(kt, lds0, lds1);
            if (kt + kTileKeys < k1) turn(kt + kTileKeys, lds1, lds0);
        }
    }
    if (bad) report(a.c);

    const float sum = l + __shfl_xor(l, 32, kWave);
    const size_t at = (size_t)(rq.start + token) * a.q_heads + h * a.group + row % a.group;
    float odd = 0.f;
    if (row < rows && sum == sum)   // its own scores are no NaN
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) odd = fmaf(o[d][e], 0.f, odd);
    odd += __shfl_xor(odd, 32, kWave);
    unsigned left = (unsigned)__ballot(odd != 0.f);   // NaN
    if (row < rows && !((left >> col) & 1)) {
        if (count == 1) {
            const float inv = inverse(sum, before + token);
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *reinterpret_cast<uint2*>(a.out + at * D + 32 * d + 2 * e + 4 * half) =
                        uint2{f32x2_to_bf16x2_rne(o[d][e] * inv, o[d][e + 1] * inv), f32x2_to_bf16x2_rne(o[d][e + 2] * inv, o[d][e + 3] * inv)};
        } else {
            float* out = a.part_o + (at * a.most + split) * D;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *reinterpret_cast<float4*>(out + 32 * d + 2 * e + 4 * half) = make_float4(o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]);
            if (half == 0) a.part_ml[at * a.most + split] = make_float2(m, sum);
        }
    }
    for (; __builtin_expect(left != 0, 0); left &= left - 1) {   // rows that are computed again
        const int again = row0 + wave * 32 + __builtin_ctz(left), new_token = again / a.group, head = h * a.group + again % a.group;
        const size_t to = (size_t)(rq.start + new_token) * a.q_heads + head;
        float again_o[D / kWave], again_m, again_l;
        attend_row_alone<D, kEight>(a, r, h, a.q + (rq.start + new_token) * a.q_stride + head * D, range.begin, min(before + new_token, k1 - 1), again_o, again_m, again_l);
        store_row_alone<D>(a, again_o, again_m, again_l, before + new_token, a.out + to * D, count == 1 ? -1 : (long long)(to * a.most + split));
    }
}

// Adds up the shares of the keys of a tile of rows: D / 4 lanes a row, a block the heads of a token.
template <int D>
__global__ __launch_bounds__(kJoinWaves* kWave) void join_tiles_kernel(const AttentionArgs a) {
    constexpr int kLanes = D / 4;
    const int r = request_of(a.c, blockIdx.x), head = blockIdx.y * (kJoinWaves * kWave / kLanes) + threadIdx.x / kLanes;
    if (r < 0 || head >= a.q_heads) return;
    bool bad;
    const Request rq = request(a.c, r, bad);
    const int token = (int)blockIdx.x - rq.start;
    if (token >= rq.n || rq.n * a.group < a.min_rows) return;   // (token >= n: q_start is bad)
    const int row0 = (token * a.group + head % a.group) / kTileRows * kTileRows;
    const int count = shares(keys_of(rq, a.group, row0, kTileRows), a.chunk, a.most);
    if (count == 1) return;
    const size_t at = (size_t)blockIdx.x * a.q_heads + head;
    const float2* ml = a.part_ml + at * a.most;
    const f32x4_t* part = reinterpret_cast<const f32x4_t*>(a.part_o + at * a.most * D) + threadIdx.x % kLanes;
    float top = -INFINITY;
    for (int i = 0; i < count; ++i) top = fmaxf(top, ml[i].x);
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    for (int i0 = 0; i0 < count; i0 += 4) {
        f32x4_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = part[min(i0 + u, count - 1) * kLanes];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float2 x = ml[min(i0 + u, count - 1)];
            if (i0 + u >= count || x.y == 0.f) continue;   // no key; scores that are all NaN leave a maximum of -inf too, and a sum of NaN
            const float w = __builtin_amdgcn_exp2f((x.x - top) * a.scale);
            sum = fmaf(w, x.y, sum);
            acc += v[u] * w;
        }
    }
    const float inv = inverse(sum, rq.len - rq.n + token);
    reinterpret_cast<uint2*>(a.out + at * D)[threadIdx.x % kLanes] =
        uint2{f32x2_to_bf16x2_rne(acc[0] * inv, acc[1] * inv), f32x2_to_bf16x2_rne(acc[2] * inv, acc[3] * inv)};
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

template <int D, bool kEight>
hipError_t launch_step(const AttentionPlan& p, const qail_kv_cache& c, const qail_requests& b, const AttentionArgs& a, hipStream_t st) {
    const unsigned head_blocks = (unsigned)((a.q_heads + kJoinWaves - 1) / kJoinWaves);
    if (p.tiles) {   // the longer kernel first
        hipLaunchKernelGGL((attend_tile_kernel<D, kEight>), dim3((unsigned)((long long)p.row_tiles * c.heads * p.most)), dim3(kTileWaves * kWave), 0, st, a);
        if (p.most > 1) hipLaunchKernelGGL(join_tiles_kernel<D>, dim3((unsigned)b.tokens, (unsigned)((a.q_heads * (D / 4) + kJoinWaves * kWave - 1) / (kJoinWaves * kWave))), dim3(kJoinWaves * kWave), 0, st, a);
    }
    if (p.stream) {   // (its partial results may lie where the tiles' were)
        hipLaunchKernelGGL((attend_stream_kernel<D, kEight>), dim3((unsigned)p.blocks), dim3(kStreamWaves * kWave), 0, st, a);
        if (p.shared) hipLaunchKernelGGL(join_stream_kernel<D>, dim3((unsigned)b.requests, head_blocks, p.join_tokens), dim3(kJoinWaves * kWave), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace

size_t paged_attention_workspace(const qail_kv_cache& c, const qail_requests& b, int q_heads) {
    const size_t n = attention_places(plan_attention(c, b, q_heads, device_cu_count()), b, q_heads);
    return align256(n * c.head_dim * sizeof(float)) + align256(n * sizeof(float2));
}

hipError_t launch_paged_attention(const qail_kv_cache& c, const qail_requests& b, const uint16_t* q, int64_t q_stride, int q_heads, float scale,
                                  uint16_t* out, uint32_t* errors, void* ws, hipStream_t st) {
    const AttentionPlan p = plan_attention(c, b, q_heads, device_cu_count());
    AttentionArgs a{};
    a.c = cache_args(c, b, errors);
    a.q = q;
    a.out = out;
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + align256(attention_places(p, b, q_heads) * c.head_dim * sizeof(float)));
    a.q_stride = q_stride;
    a.scale = scale * 1.44269504088896340736f;
    a.q_heads = q_heads;
    a.group = q_heads / c.heads;
    a.max_rows = p.stream_rows;
    a.shared = p.shared;
    a.blocks = p.blocks;
    a.least = p.least;
    a.min_rows = p.stream ? kStreamRows + 1 : 1;
    a.tiles = p.row_tiles;
    a.chunk = p.chunk;
    a.most = p.most;
    const bool eight = c.type == QAIL_KV_S8;
    if (c.head_dim == 128) return eight ? launch_step<128, true>(p, c, b, a, st) : launch_step<128, false>(p, c, b, a, st);
    return eight ? launch_step<64, true>(p, c, b, a, st) : launch_step<64, false>(p, c, b, a, st);
}

}  // namespace qail
