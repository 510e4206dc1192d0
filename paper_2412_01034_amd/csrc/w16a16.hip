// Linears whose weights stay in 16 bits, with bias, activation and residual in the epilogue, and their gradients:
//     y = act(x W^T + b) + residual,   dz = dy act'(z),   dx = dz W,   dW = dz^T x,   db = sum of dz over the rows.
//
// All three products are C[p][q] = sum_r A(p, r) B(q, r), whose operands either have r contiguous ("straight": x and W of the
// forward product, dz of dx) or lie row by row of r ("turned": W of dx, dz and x of dW).  One kernel computes them: 64 r at a time go from
// memory straight into LDS, and a turned operand is read from there transposed by the hardware, so that nothing is transposed in memory.
//
// dz is computed in fp32 and the matrix cores take bf16: it enters its products as the sum of two bf16 numbers, which takes about twice as long as rounding it once (289 x 4096 x
// 4096 77 us for 54, 4096 x 4096 x 4096 500 for 270) and leaves the gradients their own rounding alone (0.0017 of their norm from 64 bits; 0.0023 with dz rounded).  The
// caller may ask for the rounded one; where dz has 8 bits anyway (a bf16 dy, no activation or RELU) there is one part.
#include <algorithm>

#include "qail_internal.h"
#include "w16a16_plan.h"

namespace qail {

namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(8))) short s16x8_t;
typedef __attribute__((address_space(3))) uint8_t lds_t;

// s_waitcnt immediate: vmcnt(n), lgkmcnt(0), expcnt untouched.
__host__ __device__ constexpr int waitcnt_vm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4); }

// ------------------------------------------------------------------------------------------------ activations --

// A tile has as many outputs as its waves have cycles to spare, so these are short: products and sums with one rounding, the hardware's 2^x and 1 / x
// (1 ulp each).  The arguments of exponentials are kept in two parts, since 2^x loses 2^-24 x.  Relative errors are below 2^-20, but for the short GELU (2^-14.3, below) and
// tanh-GELU of far negative z (2^-15.5: its argument has 2^-22 of itself, which is 88 there).  Results below 2^-119 may be 0: the hardware's 2^x and 1 / x have no subnormal ones.

// exp(x): 0 below -87.3, infinity beyond 88.7.  (The argument's clamp is farther out: it keeps infinities out of `lo`.)
__device__ __forceinline__ float exp_of(float x) {
    constexpr float k = 1.44269504f, k_lo = 1.92596299e-8f;   // log2(e)
    x = __builtin_amdgcn_fmed3f(x, -126.f, 126.f);
    const float hi = x * k, lo = fmaf(x, k, -hi) + x * k_lo;
    return __builtin_amdgcn_exp2f(hi) * fmaf(lo, 0.693147181f, 1.f);
}

// x = |z| <= 20: exp(-z^2 / 2), and beside it erfc(x / sqrt(2)) / 2, the share of the normal distribution beyond x.  erfc(v) exp(v^2) is t P(t), t = 1 / (1 + 0.3 v), with
// a polynomial that is fitted to v <= 10 with the least largest relative error: of degree 8 (2^-25.6), or where the result is rounded to bf16 (2^-8) of degree 5 (2^-14.7), the
// argument of the exponential in one part (2^-16.5).  The shorter form saves a quarter of an epilogue's instructions with the exact GELU (2056 x 4096 x 1024: 51.7 -> 49.8 us).
template <bool kShort>
__device__ __forceinline__ float normal_tail(float x, float& bell) {
    constexpr float k = -0.721347520f, k_lo = -9.62981495e-9f;   // -log2(e) / 2
    const float s = x * x, hi = s * k, t = __builtin_amdgcn_rcpf(fmaf(x, 0.212132034f, 1.f));
    float q;
    if constexpr (kShort) {
        bell = __builtin_amdgcn_exp2f(hi);
        q = 0.385530733f;
        q = fmaf(q, t, -0.497444498f);
        q = fmaf(q, t, 0.500339436f);
        q = fmaf(q, t, -0.0889795918f);
        q = fmaf(q, t, 0.118597002f);
        q = fmaf(q, t, 0.0819387143f);
    } else {
        const float s_lo = fmaf(x, x, -s), lo = fmaf(s, k, -hi) + fmaf(s_lo, k, s * k_lo);
        bell = __builtin_amdgcn_exp2f(hi) * fmaf(lo, 0.693147181f, 1.f);
        q = -0.0647618126f;
        q = fmaf(q, t, 0.242783429f);
        q = fmaf(q, t, -0.256142925f);
        q = fmaf(q, t, 0.273864594f);
        q = fmaf(q, t, -0.0473286336f);
        q = fmaf(q, t, 0.107464472f);
        q = fmaf(q, t, 0.0741692019f);
        q = fmaf(q, t, 0.0853576683f);
        q = fmaf(q, t, 0.0845939992f);
    }
    return q * t * bell;
}

__device__ __forceinline__ float gelu_tanh_argument(float z) { return z * fmaf(0.0713548163f * z, z, 1.59576912f); }   // (1 + tanh(v / 2)) / 2 = 1 / (1 + exp(-v))

template <bool kShort>
__device__ __forceinline__ float activated(int act, float z) {
    switch (act) {
        case QAIL_ACT_RELU: return z < 0.f ? 0.f : z;
        case QAIL_ACT_GELU: {
            float bell;
            const float x = fminf(fabsf(z), 20.f), h = normal_tail<kShort>(x, bell);
            return z > 0.f ? fmaf(-x, h, z) : z * h;   // (h is 0 from 14 on: not -z, or infinity would meet it)
        }
        case QAIL_ACT_GELU_TANH: return z * __builtin_amdgcn_rcpf(1.f + exp_of(-gelu_tanh_argument(z)));
        case QAIL_ACT_SILU: return z * __builtin_amdgcn_rcpf(1.f + exp_of(-z));
        default: return z;
    }
}

// act'(z).  Terms that vanish far out are taken at the ends of the range in which they do not, so that no infinity meets a zero.
__device__ __forceinline__ float slope(int act, float z) {
    float r;
    switch (act) {
        case QAIL_ACT_RELU: return z > 0.f ? 1.f : z != z ? z : 0.f;
        case QAIL_ACT_GELU: {
            float bell;
            const float near = __builtin_amdgcn_fmed3f(z, -20.f, 20.f), h = normal_tail<false>(fabsf(near), bell);
            r = fmaf(0.398942280f * near, bell, z > 0.f ? 1.f - h : h);
            break;
        }
        case QAIL_ACT_GELU_TANH:
        case QAIL_ACT_SILU: {
            const float near = __builtin_amdgcn_fmed3f(z, -80.f, 80.f);
            const float v = act == QAIL_ACT_SILU ? near : __builtin_amdgcn_fmed3f(gelu_tanh_argument(near), -80.f, 80.f);
            const float dv = act == QAIL_ACT_SILU ? 1.f : fmaf(0.214064449f * near, near, 1.59576912f);
            const float e = exp_of(-v), share = __builtin_amdgcn_rcpf(1.f + e);
            r = fmaf(near * dv, share * (e * share), share);
            break;
        }
        default: return 1.f;
    }
    return z != z ? z : r;
}

// ------------------------------------------------------------------------------------------------- epilogue --

struct Epilogue {
    const uint16_t* bias;       // [Q] or NULL
    const uint16_t* residual;   // [P][Q] or NULL
    uint16_t* z;                // [P][Q] or NULL
    uint16_t* y;                // [P][Q], or y32
    float* y32;
    int act, Q;
};

// 8 values at any address that their type allows, in loads and stores of 16 bytes all the same (rows of an odd number of values; value by value the kernel of dz took
// 67 us for 3468 x 5073, now 34, and 310 x 4096 x 14905 96 us, 17 more than 14904).
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef u32x4_t any_half8_t __attribute__((aligned(2)));
typedef f32x4_t any_float4_t __attribute__((aligned(4)));
__device__ __forceinline__ void load8(const uint16_t* p, float* v) {
    const u32x4_t t = *reinterpret_cast<const any_half8_t*>(p);
    unpack8(make_uint4(t.x, t.y, t.z, t.w), v);
}
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
    const uint4 t = pack8(v);
    *reinterpret_cast<any_half8_t*>(p) = u32x4_t{t.x, t.y, t.z, t.w};
}

// Outputs p, q .. q + 7 from their sums; the last ones of a row, fewer than 8, value by value.
__device__ __forceinline__ void finish8(const Epilogue& e, long long p, int q, float* v) {
    const size_t at = (size_t)p * e.Q + q;
    if (q + 8 <= e.Q) {
        float t[8];
        if (e.bias) {
            load8(e.bias + q, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (e.z) store8(e.z + at, v);
        if (e.act != QAIL_ACT_NONE) {
            if (e.y) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = activated<true>(e.act, v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = activated<false>(e.act, v[i]);
            }
        }
        if (e.residual) {
            load8(e.residual + at, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (e.y) {
            store8(e.y + at, v);
        } else {
            reinterpret_cast<any_float4_t*>(e.y32 + at)[0] = f32x4_t{v[0], v[1], v[2], v[3]};
            reinterpret_cast<any_float4_t*>(e.y32 + at)[1] = f32x4_t{v[4], v[5], v[6], v[7]};
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (q + i >= e.Q) return;
        float t = v[i];
        if (e.bias) t += bf16_bits_to_f32(e.bias[q + i]);
        if (e.z) e.z[at + i] = (uint16_t)f32x2_to_bf16x2_rne(t, 0.f);
        if (e.act != QAIL_ACT_NONE) t = e.y ? activated<true>(e.act, t) : activated<false>(e.act, t);   // the same function as in whole groups
        if (e.residual) t += bf16_bits_to_f32(e.residual[at + i]);
        if (e.y) e.y[at + i] = (uint16_t)f32x2_to_bf16x2_rne(t, 0.f);
        else e.y32[at + i] = t;
    }
}

// ------------------------------------------------------------------------------------------------- products --

struct ProductArgs {
    const uint16_t* a;      // straight: [P][lda], turned: [R][lda] (lda >= P rounded up to 8)
    const uint16_t* b;      // likewise with Q
    long long lda, ldb;
    long long low;          // where a's second parts begin, elements from a; 0: it has none.  Their steps come first, and the plan has them
    int P, Q, R;            // R: of a straight operand a multiple of 8 that its rows have
    ProductPlan plan;
    float* partial;         // [splits][P][Q rounded up to 8], where splits > 1
    Epilogue e;
};

__device__ const uint4 kNothing = {0, 0, 0, 0};   // what is loaded beyond the end of r

// 16 bytes of each lane from memory into LDS, lane i's at lds + 16 i.  As assembly: the compiler would make every LDS read wait for all
// copies in flight, since it does not see that the slots of the ring differ.  The waits are the explicit s_waitcnt vmcnt(n).
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }
__device__ __forceinline__ void copy16(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy16_from(const void* p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}

// One operand's part of a step in LDS: kB rows (p or q) of 64 r.  Straight: kB rows of 128 bytes, piece s (16 bytes) of row i at s ^ (i & 7) ^ (i / 8 & 1),
// so that the 16 lanes that are served together, 16 consecutive rows of one s, hit 16 places of 256 bytes (with i & 7 alone rows 8 apart met, four cycles a read:
// 3000 x 4096 x 2048 took 54.5 us instead of 52.3).  Turned: 64 rows (r) of 2 kB bytes, piece s of row i at s ^ ((i & 3) << 2): a transposed read takes
// 64 bytes of each of four rows, which lie in four places of 256 bytes then (of 128, two rows, where kB is 64).
template <int kB, bool kTurned, int kThreads>
struct Operand {
    static constexpr int kBytes = kB * 2 * kStepR;
    static constexpr int kLoads = kBytes / 16 / kThreads;
    static constexpr int kPieces = kTurned ? kB / 8 : kStepR / 8;   // of a row
    static_assert(kLoads * 16 * kThreads == kBytes && (!kTurned || kB >= 64), "whole loads, whole swizzles");
    __device__ static __forceinline__ int place(int row, int piece) {
        return piece ^ (!kTurned ? (row & 7) ^ (row >> 3 & 1) : kB == 64 ? (row & 2) << 1 : (row & 3) << 2);
    }

    const uint16_t* base;     // row 0 of the tile (straight) or its column 0 in row 0 (turned), at r = 0
    long long ld;
    uint32_t off[kLoads];     // bytes of a thread's pieces of a step from there
    int R;

    __device__ __forceinline__ Operand(const uint16_t* m, long long ld_, int first, int count, int R_) : ld(ld_), R(R_) {
        base = kTurned ? m + first : m + (long long)first * ld;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int id = i * kThreads + threadIdx.x, row = id / kPieces, piece = place(row, id % kPieces);
            if constexpr (kTurned) {
                const int last = (count - 1 - first) / 8;   // pieces behind the matrix repeat its last one: outputs that nobody writes
                off[i] = (uint32_t)((long long)row * ld * 2) + 16u * (piece < last ? piece : last);
            } else {
                const int last = count - 1 - first;
                off[i] = (uint32_t)((long long)(row < last ? row : last) * ld * 2) + 16u * piece;
            }
        }
    }
    // Step `step` of the matrix that begins `part` elements farther on into LDS at `lds` (of the block); what lies beyond R is zero.
    __device__ __forceinline__ void load(int step, uint32_t lds, long long part) const {
        const int r0 = step * kStepR;
        const uint16_t* const from = base + part + (kTurned ? (long long)r0 * ld : (long long)r0);
        const uint32_t to = lds + (threadIdx.x / kWave) * (16 * kWave);
        if (r0 + kStepR <= R) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) copy16(from, off[i], __builtin_amdgcn_readfirstlane(to + i * kThreads * 16));
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int id = i * kThreads + threadIdx.x, row = id / kPieces;
                const int r = kTurned ? r0 + row : r0 + 8 * place(row, id % kPieces);
                const void* const p = r < R ? reinterpret_cast<const char*>(from) + off[i] : reinterpret_cast<const char*>(&kNothing);
                copy16_from(p, __builtin_amdgcn_readfirstlane(to + i * kThreads * 16));
            }
        }
    }
    // The fragment of rows first .. first + 31 and r 16 kk .. 16 kk + 15: lane l has row l % 32 and 8 r from 8 (l / 32) on.
    __device__ static __forceinline__ bf16x8_t fragment(const uint8_t* s, int first, int kk, int lane) {
        if constexpr (!kTurned) {
            const int row = first + lane % 32;
            return *reinterpret_cast<const bf16x8_t*>(s + row * 128 + place(row, 2 * kk + lane / 32) * 16);
        } else {
            s16x4_t part[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int row = 16 * kk + 8 * (lane / 32) + 4 * t + lane % 16 / 4, col = first + lane % 32 / 16 * 16 + lane % 4 * 4;
                part[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4_t*)(lds_t*)(s + row * (2 * kB) + place(row, col / 8) * 16 + col % 8 * 2));
            }
            const s16x8_t both = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8_t, both);
        }
    }
};

// kWP x kWQ waves share a tile of kBP x kBQ; kSlots steps lie in LDS, all but one of them on their way while one is multiplied. The matrix cores get B's rows
// as rows: a lane then has one p and groups of four neighbouring q.  Where the chip is full bound by the matrix pipe (61 to 66 % busy) and by what runs beside no product, a tile's way in and its
// epilogue, as a unit has one tile at a time (a 4096 x 4096 x 4096 gradient 115 to 125 us with dz in one part, 224 to 264 in two: 1040 to 1230 TFLOP/s of 1450 that a
// library product reaches), by the other operand's way from memory with few rows (16 x 4096 x 32000: 55 us, 4.8 TB/s),
// by the epilogue with short contractions (2056 x 4096 x 1024 with GELU, z and bias 40 us, 28 without them).
template <int kBP, int kBQ, int kWP, int kWQ, bool kTA, bool kTB, int kSlots>
__global__ __launch_bounds__(kWP* kWQ* kWave, (kWP * kWQ > 4 ? 2 : 1)) void w16a16_product_kernel(const ProductArgs g) {
    constexpr int kThreads = kWP * kWQ * kWave, FP = kBP / kWP / 32, FQ = kBQ / kWQ / 32;
    using A = Operand<kBP, kTA, kThreads>;
    using Bo = Operand<kBQ, kTB, kThreads>;
    constexpr int kSlot = A::kBytes + Bo::kBytes, kLoads = A::kLoads + Bo::kLoads;
    extern __shared__ __attribute__((aligned(16))) uint8_t ring[];
    const TilePlace t = tile_place(g.plan, blockIdx.x);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int p0 = t.tp * kBP, q0 = t.tq * kBQ, wp = wave / kWQ * (32 * FP), wq = wave % kWQ * (32 * FQ);
    const A a(g.a, g.lda, p0, g.P, g.R);
    const Bo b(g.b, g.ldb, q0, g.Q, g.R);
    const int first = g.plan.first_step(t.split), steps = g.plan.first_step(t.split + 1) - first;
    const uint32_t lds = lds_addr(ring);

    f32x16_t acc[FP][FQ] = {};
    bf16x8_t fa[2][FP] = {}, fb[2][FQ] = {};
    // The gradients' products (B turned) have dz in two parts, whose sum it is: first the steps of the second parts, then the same ones of the first parts.
    const int low_steps = kTB && g.low != 0 ? g.plan.steps / 2 : 0, low = kTB ? max(0, min(low_steps - first, steps)) : 0;   // in all, and of this block's
    auto load = [&](int i) {
        const int slot = i % kSlots, step = first + i - (i < low ? 0 : low_steps);
        a.load(step, lds + slot * kSlot, i < low ? g.low : 0);
        b.load(step, lds + slot * kSlot + A::kBytes, 0);
    };
    // All of the steps up to i have arrived (at most kSlots - 1 later ones are on their way), and nobody reads the step in front of them.
    auto wait_for = [&](int i, int issued) {
        const int later = min(issued, steps) - 1 - i;
        static_assert(kSlots == 2 || kSlots == 4, "");
        if (kSlots == 4 && later >= 3) __builtin_amdgcn_s_waitcnt(waitcnt_vm(3 * kLoads));
        else if (kSlots == 4 && later == 2) __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * kLoads));
        else if (later >= 1) __builtin_amdgcn_s_waitcnt(waitcnt_vm(kLoads));
        else __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        asm volatile("s_barrier" ::: "memory");
    };
    auto multiply = [&](int set) {
#pragma unroll
        for (int x = 0; x < FP; ++x)
#pragma unroll
            for (int y = 0; y < FQ; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[set][y], fa[set][x], acc[x][y], 0, 0, 0);
    };
    // The second parts add 2^-8 of the sums at most.  Where an infinity or NaN of B met them the sum is the first parts' alone: of opposite infinities, or of an infinity and
    // the 0 that an exact dz has for its second part, it would be NaN where the product's is infinite.
    auto drop = [&]() {
#pragma unroll
        for (int x = 0; x < FP; ++x)
#pragma unroll
            for (int y = 0; y < FQ; ++y)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[x][y][e] = fabsf(acc[x][y][e]) <= 3.4028235e38f ? acc[x][y][e] : 0.f;
    };
#pragma unroll
    for (int i = 0; i < kSlots; ++i)
        if (i < steps) load(i);
    wait_for(0, kSlots);
    // The fragments of 16 r are read while those before them are multiplied, the first ones of a step beside the last products of the step before
    // (zeros at the beginning), so that the matrix cores do not wait for the barrier's reads.
    for (int i = 0; i < steps; ++i) {
        if (kTB && i == low && low > 0) {
            multiply(1);
            drop();
#pragma unroll
            for (int j = 0; j < FP; ++j) fa[1][j] = bf16x8_t{};
#pragma unroll
            for (int j = 0; j < FQ; ++j) fb[1][j] = bf16x8_t{};
        }
        const uint8_t* const sa = ring + i % kSlots * kSlot;
        const uint8_t* const sb = sa + A::kBytes;
#pragma unroll
        for (int kk = 0; kk < kStepR / 16; ++kk) {
#pragma unroll
            for (int j = 0; j < FQ; ++j) fb[kk % 2][j] = Bo::fragment(sb, wq + 32 * j, kk, lane);
#pragma unroll
            for (int j = 0; j < FP; ++j) fa[kk % 2][j] = A::fragment(sa, wp + 32 * j, kk, lane);
            multiply((kk + 1) % 2);
            constexpr int kReads = FP * (kTA ? 2 : 1) + FQ * (kTB ? 2 : 1), kProducts = FP * FQ;
#pragma unroll
            for (int j = 0; j < kProducts; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a product, then its share of the reads
                if (kReads * (j + 1) / kProducts > kReads * j / kProducts) {
                    if (kReads * (j + 1) / kProducts - kReads * j / kProducts == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    else __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
            }
        }
        if (i + 1 < steps) {
            wait_for(i + 1, i + kSlots);
            if (i + kSlots < steps) load(i + kSlots);
        }
    }
    multiply(1);
    if (kTB && low == steps) drop();

    // Out through LDS, 32 rows of a wave at a time: the lanes then have 8 neighbouring outputs of a row, a row's lanes lie beside each other, and the
    // epilogue is a loop (unrolled over the registers its code is far longer than the instruction cache).  Piece c (16 bytes) of row p lies at c ^ (p & 15).
    constexpr int kRow = 32 * FQ, kPiecesOut = kRow / 4, kLanes = kRow / 8;   // floats and pieces of a row; lanes that share one
    static_assert(kWP * kWQ * 32 * kRow * 4 <= kSlots * kSlot && kPiecesOut >= 8, "the waves' rows fit the ring");
    constexpr int kMask = kPiecesOut < 16 ? kPiecesOut - 1 : 15;
    float4* const mine = reinterpret_cast<float4*>(ring + wave * (32 * kRow * 4));
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");           // nobody reads the last step any more
#pragma unroll
    for (int x = 0; x < FP; ++x) {
        const int row = lane % 32;
#pragma unroll
        for (int y = 0; y < FQ; ++y)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                mine[row * kPiecesOut + ((8 * y + 2 * i + lane / 32) ^ (row & kMask))] =
                    make_float4(acc[x][y][4 * i], acc[x][y][4 * i + 1], acc[x][y][4 * i + 2], acc[x][y][4 * i + 3]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int c = lane % kLanes, q = q0 + wq + 8 * c, Q8 = (g.Q + 7) / 8 * 8;
#pragma unroll 1
        for (int r = lane / kLanes; r < 32; r += kWave / kLanes) {
            const int p = p0 + wp + 32 * x + r;
            const float4 lo = mine[r * kPiecesOut + ((2 * c) ^ (r & kMask))], hi = mine[r * kPiecesOut + ((2 * c + 1) ^ (r & kMask))];
            if (p >= g.P || q >= g.Q) continue;
            if (g.plan.splits == 1) {
                float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                finish8(g.e, p, q, v);
            } else {
                float4* const to = reinterpret_cast<float4*>(g.partial + ((size_t)t.split * g.P + p) * Q8 + q);
                to[0] = lo;
                to[1] = hi;
            }
        }
        asm volatile("" ::: "memory");
    }
}

// The shares of the contraction added up, in their order, and the epilogue: 8 outputs a thread.
__global__ __launch_bounds__(256) void w16a16_sum_kernel(const float* __restrict__ partial, int splits, int P, const Epilogue e) {
    const int n8 = (e.Q + 7) / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, all = (long long)P * n8;
    if (i >= all) return;
    float v[8] = {};
    const float4* const from = reinterpret_cast<const float4*>(partial) + 2 * i;
    for (int s = 0; s < splits; s += 4) {   // four shares requested at a time; behind the last one that one again
        float4 lo[4], hi[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const float4* const share = from + 2 * all * min(s + t, splits - 1);
            lo[t] = share[0], hi[t] = share[1];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (s + t < splits) {
                v[0] += lo[t].x, v[1] += lo[t].y, v[2] += lo[t].z, v[3] += lo[t].w;
                v[4] += hi[t].x, v[5] += hi[t].y, v[6] += hi[t].z, v[7] += hi[t].w;
            }
    }
    finish8(e, i / n8, (int)(i % n8) * 8, v);
}

// -------------------------------------------------------------------------------------------- dz and db --

constexpr int kDzCols = 256;   // columns of a block: 32 threads of 8; 8 threads share a column's rows
constexpr int kDzSlices = 8;
constexpr float kMostHalf = 3.38953139e38f;   // the largest number of bf16

// The rows of a block: 8 a thread where that leaves eight blocks a compute unit, fewer for short batches.
inline int dz_rows(int M, int across, int units) {
    const long long rows = (long long)M * across / (8ll * units);
    return kDzSlices * (int)std::max(1ll, std::min(8ll, rows / kDzSlices));
}

// dz = bf16(dy act'(z)), or that and bf16 of what it leaves over (low), rows of ld values (N rounded up to 8, zeros behind N), and the sums of the unrounded dz over a
// block's rows.  Bound by HBM and, with either GELU, as much by its slope: 4096 x 4096 in two parts in 32 us (4.1 TB/s), in one in 26.
__global__ __launch_bounds__(256) void w16a16_dz_kernel(const uint16_t* __restrict__ z, const uint16_t* __restrict__ dy, const float* __restrict__ dy32, int act,
                                                        int M, int N, int ld, int rows, uint16_t* __restrict__ dz, uint16_t* __restrict__ low, float* __restrict__ sums) {
    __shared__ float part[kDzSlices][kDzCols + 8];
    const int across = (ld + kDzCols - 1) / kDzCols, bx = blockIdx.x % across, by = blockIdx.x / across;
    const int c = threadIdx.x % 32, n = bx * kDzCols + 8 * c, slice = threadIdx.x / 32;
    const int m0 = by * rows, m1 = min(M, m0 + rows);
    float sum[8] = {};
    const auto add = [&](int m, float* v, const float* s) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (act != QAIL_ACT_NONE) v[i] *= slope(act, s[i]);
            sum[i] += v[i];
        }
        if (!dz) return;
        const size_t at = (size_t)m * ld + n;
        if (!low) {
            *reinterpret_cast<uint4*>(dz + at) = pack8(v);
            return;
        }
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = fabsf(v[i]) <= 3.4028235e38f ? __builtin_amdgcn_fmed3f(v[i], -kMostHalf, kMostHalf) : v[i];
        const uint4 high = pack8(t);
        *reinterpret_cast<uint4*>(dz + at) = high;
        unpack8(high, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = fabsf(v[i]) <= 3.4028235e38f ? v[i] - t[i] : 0.f;   // an infinity has no second part
        *reinterpret_cast<uint4*>(low + at) = pack8(t);
    };
    if (n + 8 <= N) {
#pragma unroll 2
        for (int m = m0 + slice; m < m1; m += kDzSlices) {
            const size_t at = (size_t)m * N + n;
            float v[8], s[8];
            u32x4_t kept;
            if (act != QAIL_ACT_NONE) kept = *reinterpret_cast<const any_half8_t*>(z + at);
            if (dy) load8(dy + at, v);
            else {
                const f32x4_t lo = reinterpret_cast<const any_float4_t*>(dy32 + at)[0], hi = reinterpret_cast<const any_float4_t*>(dy32 + at)[1];
                v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
            }
            if (act != QAIL_ACT_NONE) unpack8(make_uint4(kept.x, kept.y, kept.z, kept.w), s);
            add(m, v, s);
        }
    } else if (n < N) {
        for (int m = m0 + slice; m < m1; m += kDzSlices) {
            const size_t at = (size_t)m * N + n;
            float v[8], s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = n + i < N;
                v[i] = !in ? 0.f : dy ? bf16_bits_to_f32(dy[at + i]) : dy32[at + i];
                s[i] = in && act != QAIL_ACT_NONE ? bf16_bits_to_f32(z[at + i]) : 0.f;
            }
            add(m, v, s);   // (slopes at 0 are finite: what lies behind N stays 0)
        }
    }
    if (!sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[slice][8 * c + i] = sum[i];
    __syncthreads();
    const int col = bx * kDzCols + threadIdx.x;
    if (col >= N) return;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kDzSlices; ++i) t += part[i][threadIdx.x];
    sums[(size_t)by * N + col] = t;
}

// The blocks' sums added up: 32 columns a block, 8 threads a column.
__global__ __launch_bounds__(256) void w16a16_bias_kernel(const float* __restrict__ sums, int count, int N, float* __restrict__ dbias) {
    __shared__ float part[8][32];
    const int c = threadIdx.x % 32, slice = threadIdx.x / 32, n = blockIdx.x * 32 + c;
    float t = 0.f;
    if (n < N) {
#pragma unroll 8
        for (int i = slice; i < count; i += 8) t += sums[(size_t)i * N + n];
    }
    part[slice][c] = t;
    __syncthreads();
    if (slice != 0 || n >= N) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) t += part[i][c];
    dbias[n] = t;
}

// --------------------------------------------------------------------------------------------- launches --

constexpr size_t round256(size_t b) { return (b + 255) / 256 * 256; }

template <int kBP, int kBQ, int kWP, int kWQ, bool kTA, bool kTB, int kSlots>
hipError_t launch_tiles(const ProductArgs& g, hipStream_t st) {
    constexpr int lds = kSlots * (kBP + kBQ) * 2 * kStepR;
    static_assert(lds <= 160 * 1024, "the ring fits LDS");
    const auto kernel = w16a16_product_kernel<kBP, kBQ, kWP, kWQ, kTA, kTB, kSlots>;
    if (lds > 64 * 1024) {   // needs an opt-in, on every device
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)g.plan.blocks()), dim3(kWP * kWQ * kWave), lds, st, g);
    return hipGetLastError();
}

template <bool kTA, bool kTB>
hipError_t launch_product(ProductArgs g, float* partial, hipStream_t st) {
    g.plan = plan_product(g.P, g.Q, g.R, kTA, device_cu_count(), g.low != 0 ? 2 : 1);
    g.partial = partial;
    g.e.Q = g.Q;
    hipError_t e = hipErrorInvalidValue;
    if (g.plan.bp == 256) e = launch_tiles<256, 256, 2, 4, kTA, kTB, 2>(g, st);
    // A tile that has its unit to itself may keep four steps in LDS, which cover the way from memory: 3468 x 64 x 5072 (a gradient) 14.8 -> 12.8 us, 310 x 4096 x 14904 81 -> 73;
    // not where many row tiles share a column's lines, which the first of them brings into L2: 1500 x 4096 x 4096, eight of 192, 58 -> 61.
    const bool deep = g.plan.blocks() <= device_cu_count() && (g.plan.bp == 128 || g.plan.tiles_p <= 4);
    if (g.plan.bp == 128) e = deep ? launch_tiles<128, 128, 2, 2, kTA, kTB, 4>(g, st) : launch_tiles<128, 128, 2, 2, kTA, kTB, 2>(g, st);
    if constexpr (!kTA)
        if (g.plan.bp == 192) e = deep ? launch_tiles<192, 128, 2, 2, kTA, kTB, 4>(g, st) : launch_tiles<192, 128, 2, 2, kTA, kTB, 2>(g, st);
    if constexpr (!kTA)
        if (g.plan.bp == 32) e = launch_tiles<32, 64, 1, 2, kTA, kTB, 4>(g, st);
    if (e != hipSuccess || g.plan.splits == 1) return e;
    const long long threads = (long long)g.P * ((g.Q + 7) / 8);
    hipLaunchKernelGGL(w16a16_sum_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, partial, g.plan.splits, g.P, g.e);
    return hipGetLastError();
}

size_t partial_bytes(long long P, long long Q, long long R, bool turned, int parts = 1) {
    const ProductPlan pl = plan_product(P, Q, R, turned, device_cu_count(), parts);
    return pl.splits == 1 ? 0 : (size_t)pl.splits * P * ((Q + 7) / 8 * 8) * sizeof(float);
}

}  // namespace

size_t w16a16_workspace(const qail_w16a16& d, int M) { return partial_bytes(M, d.N, d.K, false); }

hipError_t launch_w16a16(const qail_w16a16& d, const uint16_t* x, int M, const uint16_t* residual, uint16_t* z_out, uint16_t* y, float* y_f32, void* ws,
                         hipStream_t st) {
    ProductArgs g = {};
    g.a = x, g.b = d.weight, g.lda = g.ldb = d.K;
    g.P = M, g.Q = d.N, g.R = d.K;
    g.e = {d.bias, residual, z_out, y, y_f32, d.activation, 0};
    return launch_product<false, false>(g, static_cast<float*>(ws), st);
}

// The workspace of the backward call: dz and its second parts, the sums of dz over the blocks' rows, then the shares of the two products in turn.
struct BackPlaces {
    int ld, across, rows, row_blocks;
    size_t low, sums, partial, bytes;
    BackPlaces(const qail_w16a16& d, int M) {
        ld = (d.N + 7) / 8 * 8;
        across = (ld + kDzCols - 1) / kDzCols;
        rows = dz_rows(M, across, device_cu_count());
        row_blocks = (M + rows - 1) / rows;
        low = round256((size_t)M * ld * 2);
        sums = d.round_dz ? low : 2 * low;
        partial = sums + round256((size_t)row_blocks * d.N * sizeof(float));
        size_t shares = 0;   // in either number of parts, which the type of dy decides
        for (int parts = 1; parts <= (d.round_dz ? 1 : 2); ++parts)
            shares = std::max({shares, partial_bytes(M, d.K, d.N, false, parts), partial_bytes(d.N, d.K, M, true, parts)});
        bytes = partial + round256(shares);
    }
};

size_t w16a16_back_workspace(const qail_w16a16& d, int M) { return BackPlaces(d, M).bytes; }

hipError_t launch_w16a16_back(const qail_w16a16& d, const uint16_t* x, const uint16_t* z, const uint16_t* dy, const float* dy_f32, int M, uint16_t* dx,
                              uint16_t* dweight, float* dbias, void* ws, hipStream_t st) {
    const BackPlaces at(d, M);
    char* const w = static_cast<char*>(ws);
    uint16_t* const dz = reinterpret_cast<uint16_t*>(w);
    float* const sums = reinterpret_cast<float*>(w + at.sums);
    float* const partial = reinterpret_cast<float*>(w + at.partial);
    const bool as_it_is = d.activation == QAIL_ACT_NONE && dy && d.N % 8 == 0;   // dz is dy
    const bool products = dx || dweight;
    // dz has no more than 8 bits where dy has no more and the slopes are 0 and 1
    const bool two_parts = !d.round_dz && (dy_f32 || (d.activation != QAIL_ACT_NONE && d.activation != QAIL_ACT_RELU));
    if ((products && !as_it_is) || dbias) {
        hipLaunchKernelGGL(w16a16_dz_kernel, dim3((unsigned)at.across * (unsigned)at.row_blocks), dim3(256), 0, st, z, dy, dy_f32, d.activation, M, d.N, at.ld, at.rows,
                           products && !as_it_is ? dz : nullptr, products && two_parts ? dz + at.low / 2 : nullptr, dbias ? sums : nullptr);
        if (dbias) hipLaunchKernelGGL(w16a16_bias_kernel, dim3((unsigned)((d.N + 31) / 32)), dim3(256), 0, st, sums, at.row_blocks, d.N, dbias);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const uint16_t* const from = as_it_is ? dy : dz;
    ProductArgs g = {};
    g.low = two_parts ? (long long)(at.low / 2) : 0;
    if (dx) {
        g.a = from, g.lda = at.ld, g.b = d.weight, g.ldb = d.K;
        g.P = M, g.Q = d.K, g.R = d.N;
        g.e = {nullptr, nullptr, nullptr, dx, nullptr, QAIL_ACT_NONE, 0};
        const hipError_t e = launch_product<false, true>(g, partial, st);
        if (e != hipSuccess) return e;
    }
    if (dweight) {
        g.a = from, g.lda = at.ld, g.b = x, g.ldb = d.K;
        g.P = d.N, g.Q = d.K, g.R = M;
        g.e = {nullptr, nullptr, nullptr, dweight, nullptr, QAIL_ACT_NONE, 0};
        const hipError_t e = launch_product<true, true>(g, partial, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace qail
