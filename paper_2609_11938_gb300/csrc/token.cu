// token.cu -- attention of one new token of each sequence over the paged cache: the calls, and the
// kernel of token.cuh for pages of 16 bits of which every token is seen.
#include "token.cuh"

namespace opattr {

bool cache_ok(const opattr_cache *k);

opattr_status token_plain(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return token_of<false, false, false>(c, s, p, dtype);
}

opattr_status do_cache_attention(Ctx &c, Serve &s, const opattr_cache *kv, const int32_t *seqs, int32_t n,
                                 int32_t q_heads, const opattr_rows *q, const opattr_rows *out, float *lse,
                                 float scale, int32_t window, int32_t sinks) {
    if (window < 0 || sinks < 0 || (window == 0 && sinks > 0)) return OPATTR_E_INVALID_ARG;
    if (!cache_ok(kv) || n < 0 || q_heads < 1 || q_heads % kv->kv_heads || !isfinite(scale)) return OPATTR_E_INVALID_ARG;
    if (!rows_ok(*q, n, q_heads, kv->head_dim) || !rows_ok(*out, n, q_heads, kv->head_dim)) return OPATTR_E_INVALID_ARG;
    if (n > MOST_SEQS || (!seqs && n > kv->n_seqs)) return OPATTR_E_INVALID_ARG;
    if (n == 0) return OPATTR_OK;
    TokenArgs p{};
    p.kv = *kv;
    p.window = window;
    p.sinks = sinks;
    const opattr_cache8 *e8 = cache8(kv);
    // (a block of a pool has a number of 30 bits; more would not fit the memory of a GPU)
    if (e8 && kv->n_pages * kv->kv_heads >= (int64_t)PARTLY / (kv->page_size / OPATTR_SCALE_TOKENS)) return OPATTR_E_INVALID_ARG;
    if (e8) p.k_scales = e8->k_scales, p.v_scales = e8->v_scales;
    p.seqs = seqs;
    p.n = n;
    p.q_heads = q_heads;
    p.group = q_heads / kv->kv_heads;
    p.blocks_of_heads = p.group <= 8 ? 1 : (p.group + 15) / 16;
    p.q = *q;
    p.out = *out;
    p.lse = lse;
    p.scale = scale;
    while ((1 << p.shift) < kv->page_size) ++p.shift;
    const int dtype = e8 ? e8->rows : kv->dtype;
    if (e8 && kv->head_dim != 64 && kv->head_dim != 128) return window ? token8_window_odd(c, s, p, dtype) : token8_plain_odd(c, s, p, dtype);
    if (e8) return window ? token8_window(c, s, p, dtype) : token8_plain(c, s, p, dtype);
    return window ? token_window(c, s, p, dtype) : token_plain(c, s, p, dtype);
}

}  // namespace opattr
