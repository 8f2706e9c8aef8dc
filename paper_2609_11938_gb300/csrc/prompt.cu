// prompt.cu -- attention over whole prompts (opattr_attention, opattr_attention_window): checks,
// tile copies' maps, and the kernels of prompt.cuh without a window.
#include "prompt.cuh"

namespace opattr {

bool rows_ok(const opattr_rows &r, int64_t tokens, int heads, int dim) {
    if (tokens == 0) return true;
    if (!r.data || (reinterpret_cast<uintptr_t>(r.data) & 15)) return false;
    if (tokens > 1 && (r.token_stride < 8 || r.token_stride % 8)) return false;
    if (heads > 1 && (r.head_stride < 0 || r.head_stride % 8)) return false;
    return dim % 8 == 0;
}

opattr_status prompt_plain(Ctx &c, Serve &s, PromptArgs &p, const Maps<true> &m) {
    return p.a.dtype == OPATTR_BF16 ? prompt_of<__nv_bfloat16, false>(c, s, p, m) : prompt_of<__half, false>(c, s, p, m);
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}

// Boxes of 64 elements of `pack` heads of `span` rows; past a head's width or the last row: zeros.
static bool row_map(CUtensorMap *m, int dtype, const opattr_rows &r, int64_t tokens, int heads, int dim, int pack, int span) {
    const bool one = heads == 1 || r.head_stride == 0;
    const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)(one ? 1 : heads), (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {2 * (cuuint64_t)(one ? dim : r.head_stride),
                                   2 * (cuuint64_t)(tokens == 1 ? dim : r.token_stride)};
    const cuuint32_t box[3] = {64, (cuuint32_t)pack, (cuuint32_t)span}, step[3] = {1, 1, 1};
    return encode_tiled()(m, dtype == OPATTR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                          r.data, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

opattr_status do_attention(Ctx &c, Serve &s, const opattr_prompt *a, int32_t window, int32_t sinks) {
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
    opattr_status st = serve_ready(c, s);
    if (st) return st;
    PromptArgs p{};
    p.a = *a;
    const int group = a->q_heads / a->kv_heads;
    p.q_mul = a->q_heads > 1 && a->q.head_stride != 0;
    // Heads that share keys share a sub-tile: as many of a group as leave at most 8 of its rows
    // over, so that short runs of queries fill it too (five pieces of prompts of 60 .. 1,021
    // queries, 20 heads on 4: 143 us, by 256 queries of a head 160)
    p.pack = 1;
    for (int k = 2; k <= ROWS && p.q_mul; ++k)
        if (group % k == 0 && k * (ROWS / k) >= ROWS - 8) p.pack = k;
    p.span = ROWS / p.pack;
    p.heads_x = a->q_heads / p.pack;
    const int64_t tiles = a->q_tokens / (2 * p.span) + a->n_seqs;
    if (tiles * p.heads_x > INT32_MAX) return OPATTR_E_INVALID_ARG;
    p.tiles = (int)tiles;
    p.window = window;
    p.sinks = sinks;
    p.silent = s.silent;
    p.limit_us = s.silent ? SILENT_WAIT_US : WAIT_US + TILE_WAIT_US * (unsigned)(a->k_tokens / KEYS);
    s.silent = 0;
    p.next = s.err + 16;                                 // its own line
    p.wide = a->head_dim % 64 == 0 && (reinterpret_cast<uintptr_t>(a->out.data) & 31) == 0 &&
             (a->q_tokens == 1 || a->out.token_stride % 16 == 0) && (a->q_heads == 1 || a->out.head_stride % 16 == 0);
    p.k_mul = a->kv_heads > 1 && a->k.head_stride != 0;
    p.v_mul = a->kv_heads > 1 && a->v.head_stride != 0;
    if (!encode_tiled()) return OPATTR_E_CUDA;
    // without keys there is nothing to copy, and any rows stand in for them
    Maps<true> m;
    const opattr_rows &k = a->k_tokens ? a->k : a->q, &v = a->k_tokens ? a->v : a->q;
    const int64_t keys = a->k_tokens ? a->k_tokens : 1;
    if (!row_map(&m.q, a->dtype, a->q, a->q_tokens, a->q_heads, a->head_dim, p.pack, p.span) ||
        !row_map(&m.k, a->dtype, k, keys, a->kv_heads, a->head_dim, 1, KEYS) ||
        !row_map(&m.v, a->dtype, v, keys, a->kv_heads, a->head_dim, 1, KEYS))
        return OPATTR_E_INVALID_ARG;
    if (sinks > 0 && (!row_map(&m.k16, a->dtype, k, keys, a->kv_heads, a->head_dim, 1, SIXTEEN) ||
                      !row_map(&m.v16, a->dtype, v, keys, a->kv_heads, a->head_dim, 1, SIXTEEN)))
        return OPATTR_E_INVALID_ARG;
    if (window && sinks == 0) m.k16 = m.k, m.v16 = m.v;  // (no copy goes by them)
    return window ? prompt_window(c, s, p, m) : prompt_plain(c, s, p, m);
}

}  // namespace opattr
