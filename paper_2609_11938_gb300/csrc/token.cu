// token.cu -- attention of one new token of each sequence over the paged cache
// (opattr_cache_attention).
#include <math.h>

#include "serve.cuh"

namespace opattr {

bool cache_ok(const opattr_cache *k);

template <typename T>
__global__ void __launch_bounds__(256) k_token_rows(opattr_cache kv, const int32_t *seqs, int n, int q_heads,
                                                    opattr_rows q, opattr_rows out, float *lse, float scale,
                                                    unsigned *err) {
    pdl_wait();
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (item >= (int64_t)n * q_heads) return;
    const int b = (int)(item / q_heads), h = (int)(item % q_heads), g = h / (q_heads / kv.kv_heads);
    const int seq = seqs ? seqs[b] : b;
    int64_t len = 0;
    if (seq >= 0 && seq < kv.n_seqs) len = kv.length[seq];
    else if (lane_id() == 0) atomicOr(err, SERVE_INVALID);
    if (len < 0 || len > (int64_t)kv.pages_per_seq * kv.page_size) {
        if (lane_id() == 0) atomicOr(err, SERVE_INVALID);
        len = 0;
    }
    const T *x0 = (const T *)q.data + b * q.token_stride + h * q.head_stride;
    const int e = 4 * lane_id(), on = e < kv.head_dim;
    float x[4] = {}, o[4] = {}, m = -INFINITY, l = 0.f;
    for (int i = 0; on && i < 4; ++i) x[i] = (float)x0[e + i] * (scale * LOG2E);
    for (int64_t j = 0; j < len; ++j) {
        const int page = kv.table[(int64_t)seq * kv.pages_per_seq + j / kv.page_size];
        if (page < 0 || page >= kv.n_pages) {
            if (lane_id() == 0) atomicOr(err, SERVE_INVALID);
            continue;
        }
        const int64_t at = (((int64_t)page * kv.kv_heads + g) * kv.page_size + j % kv.page_size) * kv.head_dim;
        const T *k = (const T *)kv.k_pages + at, *v = (const T *)kv.v_pages + at;
        float s = 0.f;
        for (int i = 0; on && i < 4; ++i) s = __fmaf_rn(x[i], (float)k[e + i], s);
        s = warp_sum(s);
        const float top = fmaxf(m, s);
        const float keep = top == -INFINITY ? 1.f : exp2f(m - top), p = top == -INFINITY ? 0.f : exp2f(s - top);
        m = top;
        l = __fmaf_rn(l, keep, p);
        for (int i = 0; on && i < 4; ++i) o[i] = __fmaf_rn(o[i], keep, p * (float)v[e + i]);
    }
    T *y = (T *)out.data + b * out.token_stride + h * out.head_stride;
    for (int i = 0; on && i < 4; ++i) y[e + i] = (T)(l == 0.f ? 0.f : o[i] / l);
    if (lse && lane_id() == 0) lse[item] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

opattr_status do_cache_attention(Ctx &c, Serve &s, const opattr_cache *kv, const int32_t *seqs, int32_t n,
                                 int32_t q_heads, const opattr_rows *q, const opattr_rows *out, float *lse,
                                 float scale) {
    if (!cache_ok(kv) || n < 0 || q_heads < 1 || q_heads % kv->kv_heads || !isfinite(scale)) return OPATTR_E_INVALID_ARG;
    if (!rows_ok(*q, n, q_heads, kv->head_dim) || !rows_ok(*out, n, q_heads, kv->head_dim)) return OPATTR_E_INVALID_ARG;
    if (!seqs && n > kv->n_seqs) return OPATTR_E_INVALID_ARG;
    if (n == 0) return OPATTR_OK;
    opattr_status st = serve_ready(c, s, 0);
    if (st) return st;
    const int64_t items = (int64_t)n * q_heads;
    const dim3 grid((unsigned)((items + 7) / 8));
    if (kv->dtype == OPATTR_BF16)
        launch(c, "token", k_token_rows<__nv_bfloat16>, grid, dim3(256), 0, *kv, seqs, n, q_heads, *q, *out, lse, scale, s.err);
    else
        launch(c, "token", k_token_rows<__half>, grid, dim3(256), 0, *kv, seqs, n, q_heads, *q, *out, lse, scale, s.err);
    return cuda_status(c, c.last_error);
}

}  // namespace opattr
