// C entry points of what lies between a decoder's linears: argument checks and dispatch.  As in api.hip, every check is done on the
// host before the first HIP call.
#include <algorithm>

#include "qail_internal.h"

using namespace qail;

namespace {

template <int kBytes = 16>
bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & (kBytes - 1)) == 0; }   // NULL is
int hip_status(hipError_t e) { return e == hipSuccess ? QAIL_OK : QAIL_ERR_HIP; }
size_t round256(size_t b) { return (b + 255) / 256 * 256; }

int check_norm(int32_t M, int32_t K, float eps) {
    if (M < 1 || K < 8 || K % 8 != 0 || !(eps > 0.f && eps <= 3.0e38f)) return QAIL_ERR_SHAPE;
    if ((long long)M * K > 0x7FFFFFFFll || M >= (1 << 26) || !rmsnorm_supports(K)) return QAIL_ERR_UNSUPPORTED;   // 64 threads a row, below 2^32
    return QAIL_OK;
}

int check_cache(const qail_kv_cache* c) {
    if (!c) return QAIL_ERR_NULL;
    if (c->type != QAIL_KV_BF16 && c->type != QAIL_KV_S8) return QAIL_ERR_UNSUPPORTED;
    if (c->num_pages < 1 || c->heads < 1 || c->page_size < 16 || (c->page_size & (c->page_size - 1)) != 0 || c->head_dim < 1)
        return QAIL_ERR_SHAPE;
    if (c->page_size > 1024 || (c->head_dim != 64 && c->head_dim != 128) || c->heads > 65535) return QAIL_ERR_UNSUPPORTED;
    return QAIL_OK;
}

// The cache's pointers and the requests.
int check_step(const qail_kv_cache* c, const qail_requests* b) {
    const int e = check_cache(c);
    if (e != QAIL_OK) return e;
    if (!b) return QAIL_ERR_NULL;
    if (b->requests < 1 || b->max_pages < 1 || b->tokens < 0 || b->max_new < 0 || b->max_len < 0) return QAIL_ERR_SHAPE;
    // positions and rows are 32-bit values in the kernels, and 256 threads a token stay below 2^32
    if ((long long)b->max_pages * c->page_size > (1 << 30) || b->tokens >= (1 << 24) || b->requests > (1 << 20)) return QAIL_ERR_UNSUPPORTED;
    if (!c->k || !c->v || !b->page_table || !b->q_start || !b->kv_len) return QAIL_ERR_NULL;
    if (c->type == QAIL_KV_S8 && (!c->k_scale || !c->v_scale)) return QAIL_ERR_NULL;
    if (!aligned(c->k) || !aligned(c->v) || !aligned(c->k_scale) || !aligned(c->v_scale) || !aligned<4>(b->page_table) || !aligned<4>(b->q_start) ||
        !aligned<4>(b->kv_len))
        return QAIL_ERR_ALIGN;
    return QAIL_OK;
}

int check_rows(int64_t stride, int heads, int head_dim) {
    if (stride % 8 != 0 || stride < (int64_t)heads * head_dim) return QAIL_ERR_SHAPE;
    return stride > (1ll << 36) ? QAIL_ERR_UNSUPPORTED : QAIL_OK;   // 64-bit offsets with room to spare
}

int check_heads(const qail_kv_cache* c, const qail_requests* b, int32_t q_heads) {
    if (q_heads < 1 || q_heads % c->heads != 0) return QAIL_ERR_SHAPE;
    if (q_heads > 65535 || (long long)b->tokens * q_heads > (1 << 30) || (long long)b->requests * c->heads > (1 << 22)) return QAIL_ERR_UNSUPPORTED;
    return QAIL_OK;
}

int check_adapters(const qail_w4a16_item* items, const qail_adapters* ad, int32_t count, int32_t M, size_t* base) {
    if (count > 0 && !ad) return QAIL_ERR_NULL;
    const int e = qail_w4a16_batch_workspace(items, count, M, base);
    if (e != QAIL_OK) return e;
    for (int i = 0; i < count; ++i) {
        if (ad[i].r < 8 || ad[i].r > 64 || ad[i].r % 8 != 0 || ad[i].n < 1) return QAIL_ERR_SHAPE;
        if ((long long)M * items[i].d.N > 0x7FFFFFFFll || (long long)M * items[i].d.K > 0x7FFFFFFFll || M > (1 << 24) || count > 65535)
            return QAIL_ERR_UNSUPPORTED;
    }
    return QAIL_OK;
}

}  // namespace

extern "C" {

int qail_rmsnorm(const uint16_t* x, const uint16_t* residual, const uint16_t* weight, float eps, int32_t M, int32_t K, uint16_t* h_out,
                 uint16_t* y, uint32_t* y_s8, float* y_scale, void* stream) {
    const int e = check_norm(M, K, eps);
    if (e != QAIL_OK) return e;
    if (!x || !weight || (!h_out && !y && !y_s8) || !y_s8 != !y_scale) return QAIL_ERR_NULL;
    if (!y && !y_s8 && !residual) return QAIL_ERR_NULL;   // h_out alone would be a copy
    if (!aligned(x) || !aligned(residual) || !aligned(weight) || !aligned(h_out) || !aligned(y) || !aligned(y_s8) || !aligned<4>(y_scale))
        return QAIL_ERR_ALIGN;
    if (h_out && h_out == y) return QAIL_ERR_SHAPE;
    return hip_status(launch_rmsnorm(x, residual, weight, eps, M, K, h_out, y, y_s8, y_scale, static_cast<hipStream_t>(stream)));
}

int qail_rmsnorm_backward_workspace(int32_t M, int32_t K, size_t* bytes) {
    const int e = check_norm(M, K, 1.f);
    if (e != QAIL_OK) return e;
    if (!bytes) return QAIL_ERR_NULL;
    *bytes = rmsnorm_back_workspace(M, K);
    return QAIL_OK;
}

int qail_rmsnorm_backward(const uint16_t* h, const uint16_t* weight, float eps, const uint16_t* dy, const uint16_t* dres, int32_t M, int32_t K,
                          uint16_t* dx, float* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    const int e = check_norm(M, K, eps);
    if (e != QAIL_OK) return e;
    if (!h || !weight || !dy || !dx || !dweight) return QAIL_ERR_NULL;
    if (!aligned(h) || !aligned(weight) || !aligned(dy) || !aligned(dres) || !aligned(dx) || !aligned(dweight)) return QAIL_ERR_ALIGN;
    if (!workspace || workspace_bytes < rmsnorm_back_workspace(M, K)) return QAIL_ERR_WORKSPACE;
    if (!aligned(workspace)) return QAIL_ERR_ALIGN;
    return hip_status(launch_rmsnorm_back(h, weight, eps, dy, dres, M, K, dx, dweight, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
}

int qail_kv_cache_sizes(const qail_kv_cache* c, size_t* data_bytes, size_t* scale_bytes) {
    const int e = check_cache(c);
    if (e != QAIL_OK) return e;
    const size_t slots = (size_t)c->num_pages * c->heads * c->page_size;   // < 2^57
    if (data_bytes) *data_bytes = slots * c->head_dim * (c->type == QAIL_KV_S8 ? 1 : 2);
    if (scale_bytes) *scale_bytes = c->type == QAIL_KV_S8 ? slots * sizeof(float) : 0;
    return QAIL_OK;
}

int qail_kv_append(const qail_kv_cache* c, const qail_requests* b, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                   const uint16_t* q, int64_t q_stride, int32_t q_heads, uint16_t* q_out, const float* cos, const float* sin, int32_t positions,
                   uint32_t* errors, void* stream) {
    int e = check_step(c, b);
    if (e != QAIL_OK) return e;
    if ((e = check_rows(k_stride, c->heads, c->head_dim)) != QAIL_OK || (e = check_rows(v_stride, c->heads, c->head_dim)) != QAIL_OK) return e;
    if (!k || !v || !q != !q_out || !cos != !sin || (q && !cos)) return QAIL_ERR_NULL;
    if (q) {
        if (q_heads < 1) return QAIL_ERR_SHAPE;
        if (q_heads > 65535) return QAIL_ERR_UNSUPPORTED;
        if ((e = check_rows(q_stride, q_heads, c->head_dim)) != QAIL_OK) return e;
        if (q == q_out && q_stride != (int64_t)q_heads * c->head_dim) return QAIL_ERR_SHAPE;
    }
    if (cos && positions < 1) return QAIL_ERR_SHAPE;
    if (!aligned(k) || !aligned(v) || !aligned(q) || !aligned(q_out) || !aligned(cos) || !aligned(sin) || !aligned<4>(errors)) return QAIL_ERR_ALIGN;
    if (b->tokens == 0) return QAIL_OK;
    return hip_status(launch_kv_append(*c, *b, k, k_stride, v, v_stride, q, q_stride, q_heads, q_out, cos, sin, positions, errors,
                                       static_cast<hipStream_t>(stream)));
}

int qail_paged_attention_workspace(const qail_kv_cache* c, const qail_requests* b, int32_t q_heads, size_t* bytes) {
    int e = check_step(c, b);
    if (e != QAIL_OK) return e;
    if ((e = check_heads(c, b, q_heads)) != QAIL_OK) return e;
    if (!bytes) return QAIL_ERR_NULL;
    *bytes = b->tokens == 0 ? 0 : paged_attention_workspace(*c, *b, q_heads);
    return QAIL_OK;
}

int qail_paged_attention(const qail_kv_cache* c, const qail_requests* b, const uint16_t* q, int64_t q_stride, int32_t q_heads, float scale,
                         uint16_t* out, uint32_t* errors, void* workspace, size_t workspace_bytes, void* stream) {
    int e = check_step(c, b);
    if (e != QAIL_OK) return e;
    if ((e = check_heads(c, b, q_heads)) != QAIL_OK || (e = check_rows(q_stride, q_heads, c->head_dim)) != QAIL_OK) return e;
    if (!(scale > 0.f && scale <= 1.0e38f)) return QAIL_ERR_SHAPE;
    if (!q || !out) return QAIL_ERR_NULL;
    if (!aligned(q) || !aligned(out) || !aligned<4>(errors)) return QAIL_ERR_ALIGN;
    if (b->tokens == 0) return QAIL_OK;
    const size_t need = paged_attention_workspace(*c, *b, q_heads);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return QAIL_ERR_WORKSPACE;
        if (!aligned<256>(workspace)) return QAIL_ERR_ALIGN;
    }
    return hip_status(launch_paged_attention(*c, *b, q, q_stride, q_heads, scale, out, errors, workspace, static_cast<hipStream_t>(stream)));
}

int qail_w4a16_adapters_workspace(const qail_w4a16_item* items, const qail_adapters* adapters, int32_t count, int32_t M, size_t* bytes) {
    size_t base = 0;
    const int e = check_adapters(items, adapters, count, M, &base);
    if (e != QAIL_OK) return e;
    if (!bytes) return QAIL_ERR_NULL;
    *bytes = round256(base) + round256(adapters_workspace(items, adapters, count, M) * sizeof(float));
    return QAIL_OK;
}

int qail_w4a16_linear_adapters_batch(const qail_w4a16_item* items, const qail_adapters* adapters, const int32_t* row_adapter, int32_t count,
                                     int32_t M, void* workspace, size_t workspace_bytes, void* stream) {
    size_t base = 0;
    const int e = check_adapters(items, adapters, count, M, &base);
    if (e != QAIL_OK) return e;
    if (count == 0) return QAIL_OK;
    if (!row_adapter) return QAIL_ERR_NULL;
    bool sixteen = aligned<4>(row_adapter);
    for (int i = 0; i < count; ++i) {
        const qail_w4a16_item& it = items[i];
        const qail_adapters& ad = adapters[i];
        if (!it.qweight || !it.scales || !it.zeros || !it.x || !it.y || !ad.A || !ad.B || !ad.scaling) return QAIL_ERR_NULL;
        sixteen = sixteen && aligned(it.qweight) && aligned(it.scales) && aligned(it.zeros) && aligned(it.x) && aligned(it.y) && aligned(ad.A) &&
                  aligned(ad.B) && aligned(ad.scaling);
    }
    if (!sixteen) return QAIL_ERR_ALIGN;
    const size_t need = round256(base) + round256(adapters_workspace(items, adapters, count, M) * sizeof(float));
    if (!workspace || workspace_bytes < need) return QAIL_ERR_WORKSPACE;
    if (!aligned<256>(workspace)) return QAIL_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* const t = reinterpret_cast<float*>(static_cast<char*>(workspace) + round256(base));
    if (launch_adapters_down(items, adapters, row_adapter, count, M, t, st) != hipSuccess) return QAIL_ERR_HIP;
    const int el = qail_w4a16_linear_batch(items, count, M, workspace, round256(base), stream);
    if (el != QAIL_OK) return el;
    return hip_status(launch_adapters_up(items, adapters, row_adapter, count, M, t, st));
}

}  // extern "C"
