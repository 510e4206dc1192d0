// C entry points of the policy's ends in 16 bits: argument checks and dispatch.  As in api.hip, every check is done on the host before the
// first HIP call.
#include <initializer_list>

#include "qail_internal.h"

using namespace qail;

namespace {

template <int kBytes = 16>
bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & (kBytes - 1)) == 0; }   // NULL is
int hip_status(hipError_t e) { return e == hipSuccess ? QAIL_OK : QAIL_ERR_HIP; }

int check_embed(int32_t V, int32_t K, int32_t T) {
    if (V < 1 || K < 8 || K % 8 != 0 || T < 0) return QAIL_ERR_SHAPE;
    // 256 threads a token, or for 16 rows of the table and 1024 columns, stay below 2^32
    if (K > 65536 || V >= (1 << 24) || T >= (1 << 24) || (long long)V * K > (1ll << 36) || (long long)T * K > (1ll << 36)) return QAIL_ERR_UNSUPPORTED;
    return QAIL_OK;
}
bool finite(float v) { return v >= -3.4028235e38f && v <= 3.4028235e38f; }

int check_linear(const qail_w16a16* d, int32_t M) {
    if (!d) return QAIL_ERR_NULL;
    if (d->activation < QAIL_ACT_NONE || d->activation > QAIL_ACT_SILU) return QAIL_ERR_UNSUPPORTED;
    if (M < 1 || d->N < 1 || d->K < 8 || d->K % 8 != 0) return QAIL_ERR_SHAPE;
    // 256 rows of an operand are reached by 32-bit offsets, and 256 threads for 8 outputs, or for a tile, stay below 2^32
    constexpr int kMostSize = 1 << 22;
    constexpr long long kMost = 1ll << 33;
    static_assert(257ll * kMostSize * (int)sizeof(uint16_t) < (1ll << 32), "offsets of a tile's rows");
    if (M > kMostSize || d->N > kMostSize || d->K > kMostSize || (long long)M * d->N > kMost || (long long)M * d->K > kMost || (long long)d->N * d->K > kMost)
        return QAIL_ERR_UNSUPPORTED;
    return QAIL_OK;
}

// No output is an input or another output (NULL is neither).
bool apart(std::initializer_list<const void*> in, std::initializer_list<const void*> out) {
    for (auto o = out.begin(); o != out.end(); ++o) {
        if (!*o) continue;
        for (const void* i : in)
            if (i == *o) return false;
        for (auto p = out.begin(); p != o; ++p)
            if (*p == *o) return false;
    }
    return true;
}

}  // namespace

extern "C" {

int qail_embed(const uint16_t* table, int32_t V, int32_t K, const int32_t* ids, int32_t T, float scale, uint16_t* h, uint32_t* errors, void* stream) {
    const int e = check_embed(V, K, T);
    if (e != QAIL_OK) return e;
    if (!finite(scale)) return QAIL_ERR_SHAPE;
    if (!table || (T > 0 && (!ids || !h))) return QAIL_ERR_NULL;   // an empty tensor has no address
    if (!aligned(table) || !aligned<4>(ids) || !aligned(h) || !aligned<4>(errors)) return QAIL_ERR_ALIGN;
    if (h == table) return QAIL_ERR_SHAPE;
    if (T == 0) return QAIL_OK;
    return hip_status(launch_embed(table, V, K, ids, T, scale, h, errors, static_cast<hipStream_t>(stream)));
}

int qail_embed_backward_workspace(int32_t V, int32_t K, int32_t T, size_t* bytes) {
    const int e = check_embed(V, K, T);
    if (e != QAIL_OK) return e;
    if (!bytes) return QAIL_ERR_NULL;
    *bytes = embed_back_workspace(K, T);
    return QAIL_OK;
}

int qail_embed_backward(const int32_t* ids, const uint16_t* dh, int32_t T, float scale, int32_t V, int32_t K, int32_t accumulate, float* dtable,
                        uint32_t* errors, void* workspace, size_t workspace_bytes, void* stream) {
    const int e = check_embed(V, K, T);
    if (e != QAIL_OK) return e;
    if (!finite(scale)) return QAIL_ERR_SHAPE;
    if (!dtable || (T > 0 && (!ids || !dh))) return QAIL_ERR_NULL;
    if (!aligned<4>(ids) || !aligned(dh) || !aligned(dtable) || !aligned<4>(errors)) return QAIL_ERR_ALIGN;
    if (T > 0 && !apart({ids, dh}, {dtable})) return QAIL_ERR_SHAPE;
    if (T == 0 && accumulate) return QAIL_OK;
    if (!workspace || workspace_bytes < embed_back_workspace(K, T)) return QAIL_ERR_WORKSPACE;
    if (!aligned<256>(workspace)) return QAIL_ERR_ALIGN;
    return hip_status(launch_embed_back(ids, dh, T, scale, V, K, accumulate != 0, dtable, errors, workspace, static_cast<hipStream_t>(stream)));
}

int qail_w16a16_workspace(const qail_w16a16* d, int32_t M, size_t* bytes) {
    const int e = check_linear(d, M);
    if (e != QAIL_OK) return e;
    if (!bytes) return QAIL_ERR_NULL;
    *bytes = w16a16_workspace(*d, M);
    return QAIL_OK;
}

int qail_w16a16_linear(const qail_w16a16* d, const uint16_t* x, int32_t M, const uint16_t* residual, uint16_t* z_out, uint16_t* y, float* y_f32,
                       void* workspace, size_t workspace_bytes, void* stream) {
    const int e = check_linear(d, M);
    if (e != QAIL_OK) return e;
    if (!d->weight || !x || !y == !y_f32) return QAIL_ERR_NULL;
    if (!aligned(d->weight) || !aligned(d->bias) || !aligned(x) || !aligned(residual) || !aligned(z_out) || !aligned(y) || !aligned(y_f32)) return QAIL_ERR_ALIGN;
    if (!apart({x, d->weight, d->bias}, {z_out, y, y_f32}) || !apart({residual}, {z_out, y_f32})) return QAIL_ERR_SHAPE;   // y may be the residual
    const size_t need = w16a16_workspace(*d, M);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return QAIL_ERR_WORKSPACE;
        if (!aligned<256>(workspace)) return QAIL_ERR_ALIGN;
    }
    return hip_status(launch_w16a16(*d, x, M, residual, z_out, y, y_f32, workspace, static_cast<hipStream_t>(stream)));
}

int qail_w16a16_backward_workspace(const qail_w16a16* d, int32_t M, size_t* bytes) {
    const int e = check_linear(d, M);
    if (e != QAIL_OK) return e;
    if (!bytes) return QAIL_ERR_NULL;
    *bytes = w16a16_back_workspace(*d, M);
    return QAIL_OK;
}

int qail_w16a16_backward(const qail_w16a16* d, const uint16_t* x, const uint16_t* z, const uint16_t* dy, const float* dy_f32, int32_t M, uint16_t* dx,
                         uint16_t* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    const int e = check_linear(d, M);
    if (e != QAIL_OK) return e;
    if (!d->weight || !dy == !dy_f32 || (!dx && !dweight && !dbias) || (dweight && !x) || (d->activation != QAIL_ACT_NONE && !z)) return QAIL_ERR_NULL;
    if (!aligned(d->weight) || !aligned(x) || !aligned(z) || !aligned(dy) || !aligned(dy_f32) || !aligned(dx) || !aligned(dweight) || !aligned(dbias))
        return QAIL_ERR_ALIGN;
    if (!apart({x, z, dy, dy_f32, d->weight}, {dx, dweight, dbias})) return QAIL_ERR_SHAPE;
    if (!workspace || workspace_bytes < w16a16_back_workspace(*d, M)) return QAIL_ERR_WORKSPACE;
    if (!aligned<256>(workspace)) return QAIL_ERR_ALIGN;
    return hip_status(launch_w16a16_back(*d, x, z, dy, dy_f32, M, dx, dweight, dbias, workspace, static_cast<hipStream_t>(stream)));
}

int qail_sample(const void* logits, int32_t type, int64_t stride, int32_t R, int32_t V, const qail_sampling* s, const float* u, int32_t* token,
                float* logprob, uint32_t* errors, void* stream) {
    if (type != QAIL_LOGITS_BF16 && type != QAIL_LOGITS_F32) return QAIL_ERR_UNSUPPORTED;
    if (R < 0 || V < 1 || stride < V) return QAIL_ERR_SHAPE;
    if (R > (1 << 20) || V > (1 << 18) || stride > (1ll << 36)) return QAIL_ERR_UNSUPPORTED;
    if (!s || (R > 0 && (!logits || !u || !token))) return QAIL_ERR_NULL;
    if (!aligned(logits) || !aligned<4>(u) || !aligned<4>(token) || !aligned<4>(logprob) || !aligned<4>(errors) || !aligned<4>(s->temperature) ||
        !aligned<4>(s->top_k) || !aligned<4>(s->top_p) || !aligned<4>(s->min_p))
        return QAIL_ERR_ALIGN;
    if (R == 0) return QAIL_OK;
    return hip_status(launch_sample(logits, type, stride, R, V, *s, u, token, logprob, errors, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
