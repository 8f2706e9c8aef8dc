// prompt.cu -- attention over whole prompts: packed sequences of any lengths,
// grouped heads, causal or not (opattr_attention).
//
//   s_ij = scale * q_i . k_j,  j seen by i: j < Lk and, causal, j <= i + Lk - Lq
//   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i),  lse_i = m_i + log of that sum
// A row that sees no key gets o = 0 and lse = -inf.
#include <math.h>

#include "serve.cuh"

namespace opattr {

bool rows_ok(const opattr_rows &r, int64_t tokens, int heads, int dim) {
    if (tokens == 0) return true;
    if (!r.data || (reinterpret_cast<uintptr_t>(r.data) & 15)) return false;
    if (tokens > 1 && (r.token_stride < 0 || r.token_stride % 8)) return false;
    if (heads > 1 && (r.head_stride < 0 || r.head_stride % 8)) return false;
    return dim % 8 == 0;
}

template <typename T>
__global__ void __launch_bounds__(256) k_prompt_rows(opattr_prompt a, unsigned *err) {
    pdl_wait();
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b < a.n_seqs; b += 256)
            if (a.q_offsets[b + 1] < a.q_offsets[b] || a.k_offsets[b + 1] < a.k_offsets[b]) atomicOr(err, SERVE_INVALID);
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (item >= a.q_tokens * a.q_heads) return;
    const int t = (int)(item / a.q_heads), h = (int)(item % a.q_heads), g = h / (a.q_heads / a.kv_heads);
    if (a.q_offsets[0] != 0 || a.q_offsets[a.n_seqs] != a.q_tokens || a.k_offsets[0] != 0 ||
        a.k_offsets[a.n_seqs] != a.k_tokens) {
        if (item == 0 && lane_id() == 0) atomicOr(err, SERVE_INVALID);
        return;
    }
    const int b = seq_of_row(a.q_offsets, a.n_seqs, t);
    const int q0 = a.q_offsets[b], lq = a.q_offsets[b + 1] - q0;
    const int k0 = a.k_offsets[b], lk = a.k_offsets[b + 1] - k0;
    if (lq < 0 || t < q0 || t >= q0 + lq || lk < 0 || k0 < 0 || (int64_t)k0 + lk > a.k_tokens) {
        if (lane_id() == 0) atomicOr(err, SERVE_INVALID);
        return;
    }
    int64_t seen = lk;
    if (a.causal) seen = min(seen, (int64_t)(t - q0) + lk - lq + 1);
    const T *q = (const T *)a.q.data + t * a.q.token_stride + h * a.q.head_stride;
    const int e = 4 * lane_id(), on = e < a.head_dim;
    float x[4] = {}, o[4] = {}, m = -INFINITY, l = 0.f;
    const float s2 = a.scale * LOG2E;
    for (int i = 0; on && i < 4; ++i) x[i] = (float)q[e + i] * s2;
    for (int64_t j = 0; j < seen; ++j) {
        const T *k = (const T *)a.k.data + (k0 + j) * a.k.token_stride + g * a.k.head_stride;
        const T *v = (const T *)a.v.data + (k0 + j) * a.v.token_stride + g * a.v.head_stride;
        float s = 0.f;
        for (int i = 0; on && i < 4; ++i) s = __fmaf_rn(x[i], (float)k[e + i], s);
        s = warp_sum(s);
        const float top = fmaxf(m, s);
        const float keep = top == -INFINITY ? 1.f : exp2f(m - top), p = top == -INFINITY ? 0.f : exp2f(s - top);
        m = top;
        l = __fmaf_rn(l, keep, p);
        for (int i = 0; on && i < 4; ++i) o[i] = __fmaf_rn(o[i], keep, p * (float)v[e + i]);
    }
    T *out = (T *)a.out.data + t * a.out.token_stride + h * a.out.head_stride;
    for (int i = 0; on && i < 4; ++i) out[e + i] = (T)(l == 0.f ? 0.f : o[i] / l);
    if (a.lse && lane_id() == 0) a.lse[item] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

opattr_status do_attention(Ctx &c, Serve &s, const opattr_prompt *a) {
    if (a->dtype != OPATTR_BF16 && a->dtype != OPATTR_F16) return OPATTR_E_INVALID_ARG;
    if (a->n_seqs < 0 || a->q_tokens < 0 || a->k_tokens < 0 || a->q_tokens > INT32_MAX || a->k_tokens > INT32_MAX)
        return OPATTR_E_INVALID_ARG;
    if (a->kv_heads < 1 || a->q_heads < 1 || a->q_heads % a->kv_heads) return OPATTR_E_INVALID_ARG;
    if (a->head_dim < 8 || a->head_dim > 128 || !isfinite(a->scale)) return OPATTR_E_INVALID_ARG;
    if (!rows_ok(a->q, a->q_tokens, a->q_heads, a->head_dim) || !rows_ok(a->out, a->q_tokens, a->q_heads, a->head_dim) ||
        !rows_ok(a->k, a->k_tokens, a->kv_heads, a->head_dim) || !rows_ok(a->v, a->k_tokens, a->kv_heads, a->head_dim))
        return OPATTR_E_INVALID_ARG;
    if (a->q_tokens == 0) return OPATTR_OK;
    if (a->n_seqs == 0 || !a->q_offsets || !a->k_offsets) return OPATTR_E_INVALID_ARG;
    opattr_status st = serve_ready(c, s, 0);
    if (st) return st;
    const int64_t items = a->q_tokens * a->q_heads;
    if (items > 8ll * INT32_MAX) return OPATTR_E_INVALID_ARG;
    const dim3 grid((unsigned)((items + 7) / 8));
    if (a->dtype == OPATTR_BF16) launch(c, "prompt", k_prompt_rows<__nv_bfloat16>, grid, dim3(256), 0, *a, s.err);
    else launch(c, "prompt", k_prompt_rows<__half>, grid, dim3(256), 0, *a, s.err);
    return cuda_status(c, c.last_error);
}

}  // namespace opattr
