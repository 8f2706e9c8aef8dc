// pages.cu -- the paged key-value cache: appending tokens, sharing pages between
// sequences, freeing them, and moving the live ones together.
//
// The cache's state is the caller's: a table of each sequence's pages, its
// length, and for each page how many sequences hold it (a page held by none is
// free).  Every call reads that state, checks its own arguments against it in
// one block (`*_plan`), and changes it in a second launch only where they hold;
// otherwise the call changes nothing and opattr_check reports it.  What a call
// does is defined without reference to the order in which threads run: pages
// are given out from the lowest free one on, sequence after sequence.
//
// There is nothing to compute: large calls are bound by the rows' way through memory, small
// ones by launches and a plan's chain of dependent loads.  Measured on one GB300 (400
// sequences of 200 .. 3,100 tokens in pages of 32, 8 heads of 128): an eighth of them appended
// anew, 55,000 tokens: 70 us, 6.4 TB/s; their freed places closed by compaction: 71 us; freeing
// them 6, the plan of the append 7.  Of 24 sequences the three calls take 16.6 us, and the
// host 23.
//
// Pages of 8 bits (opattr_cache8): 16 tokens of a head share a scale, so a warp takes these 16 rows at
// once: their largest element, the scale, the codes, and what the scale's growth means for the codes before
// them.  A block of threads looks up where 16 tokens go once for all heads.  58,650 tokens to 50 empty sequences, 8 heads
// of 128: 59 us, 6.1 TB/s read and written (a lookup for every head: 113; three blocks of threads to an SM in the place of four: 63); one token to each of 200, 16 heads of 64: 8 us;
// to 48 sequences that share pages of 8, 8 heads of 128: 12 us (their copies one after another: 25).
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "serve.cuh"

namespace opattr {

constexpr int PLAN_THREADS = 1024;         // at most: a plan of few sequences has fewer
constexpr int COPY_THREADS = 256;
// tokens whose pieces a thread has under way (four, with half the threads, took 97 us for
// 55,000 tokens of 8 heads of 128, two 70)
constexpr int ROWS_AHEAD = 2;

bool cache_ok(const opattr_cache *k) {
    const opattr_cache8 *e8 = cache8(k);
    const int rows = e8 ? e8->rows : k->dtype;
    if (rows != OPATTR_BF16 && rows != OPATTR_F16) return false;
    if (e8 && (k->head_dim % 16 || !e8->k_scales || !e8->v_scales ||
               ((reinterpret_cast<uintptr_t>(e8->k_scales) | reinterpret_cast<uintptr_t>(e8->v_scales)) & 3)))
        return false;
    if (k->page_size < 16 || k->page_size > 1024 || (k->page_size & (k->page_size - 1))) return false;
    if (k->kv_heads < 1 || k->head_dim < 8 || k->head_dim > 128 || k->head_dim % 8) return false;
    if (k->n_seqs < 1 || k->pages_per_seq < 1 || k->n_pages < 1 || k->n_pages > INT32_MAX) return false;
    if ((int64_t)k->pages_per_seq * k->page_size > INT32_MAX) return false;
    if (!k->k_pages || !k->v_pages || !k->table || !k->length || !k->refs || !k->low) return false;
    return ((reinterpret_cast<uintptr_t>(k->k_pages) | reinterpret_cast<uintptr_t>(k->v_pages)) & 15) == 0;
}

opattr_status serve_ready(Ctx &c, Serve &s) {
    if (s.err) return OPATTR_OK;
    if (capturing(c)) return OPATTR_E_OOM;               // as for the scratch
    const size_t bytes = 256 + sizeof(uint32_t) * ALL_TICKETS;
    cudaError_t e = cudaMalloc(&s.err, bytes);
    if (e == cudaErrorMemoryAllocation) {
        cudaGetLastError();
        s.err = nullptr;
        return OPATTR_E_OOM;
    }
    if (e != cudaSuccess) return cuda_status(c, e);
    s.tickets = s.err + 64;
    const char *fault = getenv("OPATTR_FAULT");
    if (fault && strncmp(fault, "prompt:", 7) == 0) s.silent = atoi(fault + 7);
    e = cudaMemsetAsync(s.err, 0, bytes, c.stream);
    return e == cudaSuccess ? OPATTR_OK : cuda_status(c, e);
}

void serve_free(Serve &s) {
    if (s.err) cudaFree(s.err);
    s = Serve{};
}

__host__ __device__ __forceinline__ int pages_for(int tokens, int page) { return (tokens + page - 1) / page; }

// ---------------------------------------------------------------- checks of a plan
// Every block-wide check ends in `bad` (shared): whether the call is void.
__device__ __forceinline__ bool any_bad(bool mine, unsigned bit, unsigned *err) {
    const bool bad = __syncthreads_or(mine);
    if (bad && threadIdx.x == 0) atomicOr(err, bit);
    return bad;
}
// A sequence that is there twice: `mark` has a word per table row, in which a
// sequence's entries store their index; one is the last to do so, the others see it.
__device__ __forceinline__ bool marks_bad(const int32_t *seqs, int n, const int32_t *mark, unsigned *err) {
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += blockDim.x) bad = bad || mark[seqs[i]] != i;
    return any_bad(bad, SERVE_INVALID, err);
}
__device__ __forceinline__ bool length_bad(const opattr_cache &kv, int seq) {
    const int len = kv.length[seq];
    return len < 0 || len > kv.pages_per_seq * kv.page_size;
}

// ---------------------------------------------------------------- append
// What the plan leaves for the launch that moves the rows.
struct AppendPlan {
    int32_t *go;        // [1] 1: the call holds; 2: and pages are copied
    int32_t *old;       // [n] lengths before
    int32_t *from, *to; // [n] a partly filled page that is copied first, and where to; -1 none
    int32_t *late;      // [n] a page that this sequence keeps and shortens for one that copies it; -1 none
    int32_t *mark;      // [n_seqs]
    int32_t *first;     // [n + 1] new pages before this sequence's
    int32_t *fresh;     // new pages in the order they are given out
    int32_t room;       // entries of fresh
};

// `align`: a sequence that appends writes from a multiple of it on (pages of 8 bits: the block
// that its first row falls into may get a new scale).
// One block: a call has few sequences, and their new pages are found where the
// lowest free ones are (`low`: none below it is free), four reference counts to a
// thread at a time.
__global__ void __launch_bounds__(PLAN_THREADS)
k_append_plan(opattr_cache kv, const int32_t *seqs, int n, const int32_t *offsets, int tokens, AppendPlan p,
              int align, unsigned *err) {
    constexpr int HELD = 2048;
    __shared__ int warp_buf[33], held_page[HELD];
    __shared__ uint16_t held_part[HELD];
    pdl_wait();
    if (threadIdx.x == 0) *p.go = 0;
    // (asked for before anything else, since the others wait on one another)
    const int64_t low = max(0, *kv.low);
    int early[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) early[q] = low + 4 * threadIdx.x + q < kv.n_pages ? kv.refs[low + 4 * threadIdx.x + q] : 1;
    // each sequence's length, and the page that it is about to write into where that is filled in part
    bool bad = threadIdx.x == 0 && (offsets[0] != 0 || offsets[n] != tokens);
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int s = seqs[i], more = offsets[i + 1] - offsets[i];
        int old = 0, last = -1, refs = 0;
        bad = bad || more < 0 || offsets[i] < 0;
        if (s < 0 || s >= kv.n_seqs) bad = true;
        else {
            p.mark[s] = i;
            old = kv.length[s];
            if (old < 0 || (int64_t)old + max(0, more) > (int64_t)kv.pages_per_seq * kv.page_size) bad = true;
            else if (more > 0 && old % kv.page_size) {
                last = kv.table[(int64_t)s * kv.pages_per_seq + old / kv.page_size];
                if (last < 0 || last >= kv.n_pages) bad = true;
                else refs = kv.refs[last];
            }
        }
        p.old[i] = old;
        p.to[i] = last;
        p.from[i] = refs;
        if (i < HELD) held_page[i] = last, held_part[i] = (uint16_t)(old % kv.page_size);
    }
    if (any_bad(bad, SERVE_INVALID, err)) return;
    if (marks_bad(seqs, n, p.mark, err)) return;
    int total = 0;
    bool any_late = false, any_copied = false;
    for (int i0 = 0; i0 < n; i0 += blockDim.x) {
        const int i = i0 + threadIdx.x;
        int need = 0;
        if (i < n) {
            const int old = p.old[i], more = offsets[i + 1] - offsets[i], last = p.to[i];
            need = pages_for(old + more, kv.page_size) - pages_for(old, kv.page_size);
            int from = -1, late = -1;
            int held = p.from[i];
            if (held > 1) {
                // one after another: those before it have copied theirs and let go
                int longest = 0;
                const int near = min(i, HELD);
#pragma unroll 8
                for (int k = 0; k < near; ++k)
                    if (held_page[k] == last) --held, longest = max(longest, (int)held_part[k]);
                for (int k = HELD; k < i; ++k)
                    if (p.to[k] == last) --held, longest = max(longest, p.old[k] % kv.page_size);
                if (held > 1) from = last;
                else if (longest > old % kv.page_size / align * align) late = last;
            }
            p.from[i] = from;
            p.late[i] = late;
            any_late = any_late || late >= 0;
            any_copied = any_copied || from >= 0;
            need += from >= 0;
        }
        int sum;
        const int before = block_exclusive_scan(need, warp_buf, &sum);
        if (i < n) p.first[i] = total + before;
        total += sum;
        if (total > p.room) break;       // (also keeps the sum from running over)
    }
    if (threadIdx.x == 0) p.first[n] = total;
    if (any_bad(total > p.room, SERVE_PAGES, err)) return;
    // the lowest `total` free pages
    int found = 0;
    for (int64_t at = low; found < total && at < kv.n_pages; at += 4 * blockDim.x) {
        const int64_t i = at + 4 * threadIdx.x;
        int r[4], mine = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            r[q] = at == low ? early[q] : i + q < kv.n_pages ? kv.refs[i + q] : 1;
            mine += r[q] == 0;
        }
        int sum, rank = found + block_exclusive_scan(mine, warp_buf, &sum);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (r[q] == 0 && rank < total) p.fresh[rank++] = (int)(i + q);
        found += sum;
    }
    __syncthreads();
    if (any_bad(found < total, SERVE_PAGES, err)) return;
    // it holds: the tables change
    const int32_t *first = p.first;
    if (n < HELD) {                      // (the shared pages have been ranked)
        for (int i = threadIdx.x; i <= n; i += blockDim.x) held_page[i] = p.first[i];
        __syncthreads();
        first = held_page;
    }
    for (int k = threadIdx.x; k < total; k += blockDim.x) {
        const int i = seq_of_row(first, n, k), s = seqs[i], page = p.fresh[k];
        const int have = pages_for(p.old[i], kv.page_size), copied = p.from[i] >= 0;
        kv.table[(int64_t)s * kv.pages_per_seq + have - copied + (k - first[i])] = page;
        kv.refs[page] = 1;
    }
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        p.to[i] = -1;
        if (p.from[i] >= 0) {
            p.to[i] = p.fresh[p.first[i]];
            atomicSub(&kv.refs[p.from[i]], 1);
        }
        kv.length[seqs[i]] = p.old[i] + (offsets[i + 1] - offsets[i]);
    }
    any_copied = __syncthreads_or(any_copied);
    if (__syncthreads_or(any_late)) {
        // the sequence that keeps such a page copies it for the others before it writes there
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            int page = p.late[i];
            if (p.from[i] >= 0)
                for (int k = i + 1; k < n && page < 0; ++k)
                    if (p.late[k] == p.from[i]) page = p.late[k];
            if (page >= 0) p.from[i] = -2 - page;
        }
    }
    if (threadIdx.x == 0) {
        if (total > 0) *kv.low = p.fresh[total - 1] + 1;
        *p.go = any_copied ? 2 : 1;
    }
}

// Rows into their pages, 16 bytes at a time, keys and values side by side; the
// blocks past `row_blocks` copy the pages that were shared, each sequence its own.
// Where the one that is left with the page in place begins to write before the end
// of what another copies (from below -1), it does both, one after the other.
__global__ void __launch_bounds__(COPY_THREADS)
k_append_rows(opattr_cache kv, const int32_t *seqs, int n, const int32_t *offsets, int tokens, opattr_rows k,
              opattr_rows v, AppendPlan p, unsigned row_blocks) {
    pdl_wait();
    if (*p.go == 0) return;
    const int per = kv.head_dim / 8;                              // pieces of a head's row
    uint4 *kp = reinterpret_cast<uint4 *>(kv.k_pages), *vp = reinterpret_cast<uint4 *>(kv.v_pages);
    if (blockIdx.x >= row_blocks) {
        if (*p.go == 1) return;
        // a sequence's head at a time, as many threads as its filled rows have pieces
        const int64_t all = (int64_t)n * kv.kv_heads, block = (int64_t)kv.page_size * per;
        for (int64_t x = blockIdx.x - row_blocks; x < all; x += gridDim.x - row_blocks) {
            const int i = (int)(x / kv.kv_heads), g = (int)(x % kv.kv_heads);
            const int from = p.from[i];
            auto copy = [&](int entry, int page) {
                const int live = (p.old[entry] % kv.page_size) * per;
                const int64_t src = (page * (int64_t)kv.kv_heads + g) * block, dst = (p.to[entry] * (int64_t)kv.kv_heads + g) * block;
                for (int e = threadIdx.x; e < live; e += COPY_THREADS) {
                    const uint4 k4 = kp[src + e], v4 = vp[src + e];
                    kp[dst + e] = k4;
                    vp[dst + e] = v4;
                }
            };
            if (from >= 0) copy(i, from);
            if (from >= -1 || p.to[i] >= 0) continue;
            const int page = -2 - from, part = p.old[i] % kv.page_size;
#pragma unroll 4
            for (int e = 0; e < i; ++e)
                if (p.from[e] == from && p.to[e] >= 0) copy(e, page);
            __syncthreads();
            const int rows = min(offsets[i + 1] - offsets[i], kv.page_size - part);
            for (int e = threadIdx.x; e < rows * per; e += COPY_THREADS) {
                const int64_t t = offsets[i] + e / per, d = 8 * (e % per), dst = (page * (int64_t)kv.kv_heads + g) * block + part * per + e;
                kp[dst] = *reinterpret_cast<const uint4 *>((const uint16_t *)k.data + t * k.token_stride + g * k.head_stride + d);
                vp[dst] = *reinterpret_cast<const uint4 *>((const uint16_t *)v.data + t * v.token_stride + g * v.head_stride + d);
            }
        }
        return;
    }
    // a thread keeps its piece of a row and goes from token to token, so that nothing is divided
    // on the way (that cost more than the copies)
    const int row = kv.kv_heads * per, side = max(1, COPY_THREADS / row), sub = threadIdx.x / row;
    if (sub >= side) return;
    for (int r = threadIdx.x % row; r < row; r += COPY_THREADS) {
        const int g = r / per, e = r % per;
        const uint16_t *kr = (const uint16_t *)k.data + g * k.head_stride + 8 * e;
        const uint16_t *vr = (const uint16_t *)v.data + g * v.head_stride + 8 * e;
        const int64_t step = (int64_t)row_blocks * side;
        for (int64_t t0 = (int64_t)blockIdx.x * side + sub; t0 < tokens; t0 += ROWS_AHEAD * step) {
            uint4 k4[ROWS_AHEAD], v4[ROWS_AHEAD];
#pragma unroll
            for (int q = 0; q < ROWS_AHEAD; ++q) {
                const int64_t t = t0 + q * step;
                if (t >= tokens) break;
                k4[q] = *reinterpret_cast<const uint4 *>(kr + t * k.token_stride);
                v4[q] = *reinterpret_cast<const uint4 *>(vr + t * v.token_stride);
            }
#pragma unroll
            for (int q = 0; q < ROWS_AHEAD; ++q) {
                const int64_t t = t0 + q * step;
                if (t >= tokens) break;
                const int i = seq_of_row(offsets, n, (int)t), pos = p.old[i] + (int)t - offsets[i];
                const int page = kv.table[(int64_t)seqs[i] * kv.pages_per_seq + pos / kv.page_size];
                if (page < 0 || page >= kv.n_pages) continue;     // a table that was not consistent before the call
                if (pos - pos % kv.page_size < p.old[i] && p.from[i] < -1 && p.to[i] < 0) continue;
                const int64_t dst = ((page * (int64_t)kv.kv_heads + g) * kv.page_size + pos % kv.page_size) * per + e;
                kp[dst] = k4[q];
                vp[dst] = v4[q];
            }
        }
    }
}

// ---------------------------------------------------------------- rows into pages of 8 bits
constexpr int BLOCK = OPATTR_SCALE_TOKENS;

// Two values to codes, `lo` in the low byte: nearest even, at most 448, NaN stays.
__device__ __forceinline__ uint32_t codes2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 values2(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
    return Type2<__half>::up(r);
}
// The least power of two, from 2^-126 to 2^119, that takes `top` (finite) to 448 = 1.75 * 2^8 at most.
__device__ __forceinline__ float scale_for(float top) {
    const int bits = __float_as_int(top), e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000);
    return __int_as_float((min(119, max(-126, e)) + 127) << 23);
}

// What a warp does for a block of one head, of keys or of values: rows x (`count` of them, the
// first at place `first`) after the block's first `first` tokens, whose codes and scale are at
// src and src_scale (the same as dst, or in a page that is being copied).
template <typename T, int DP>
__device__ __forceinline__ void append_block(const T *x, int64_t stride, int first, int count, int dim, const uint8_t *src, const float *src_scale,
                                             uint8_t *dst, float *dst_scale) {
    constexpr int PIECES = DP / 8, SIDE = 32 / PIECES, N = BLOCK / SIDE;
    constexpr uint32_t INF = std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u;
    const int lane = lane_id(), sub = lane / PIECES, d = 8 * (lane % PIECES);
    const bool mine = d < dim;
    const float was = first > 0 ? *src_scale : 0.f;
    uint4 v[N];
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const int r = sub + q * SIDE;
        v[q] = mine && r < count ? __ldcs(reinterpret_cast<const uint4 *>(x + r * stride + d)) : make_uint4(0, 0, 0, 0);
    }
    uint32_t *w = &v[0].x, most = 0;
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) most = __vmaxu2(most, w[i] & 0x7fff7fffu);
    uint32_t top = __reduce_max_sync(0xffffffffu, max(most >> 16, most & 0xffffu));
    if (top >= INF) {
        // what is not finite has no say in the scale, and becomes NaN
        most = 0;
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) {
            const uint32_t size = w[i] & 0x7fff7fffu, bad = __vcmpgeu2(size, INF << 16 | INF);
            most = __vmaxu2(most, size & ~bad);
            w[i] |= bad & 0x7fff7fffu;
        }
        top = __reduce_max_sync(0xffffffffu, max(most >> 16, most & 0xffffu));
    }
    const float2 t2 = Type2<T>::up(top);
    const float need = scale_for(t2.x), now = was > need ? was : need;
    const bool grown = first > 0 && !(was >= now);
    // (a scale that this library chose is a power of two, and so is its inverse)
    const bool power = (__float_as_int(now) & 0x7fffff) == 0 && now >= __int_as_float(1 << 23);
    const float inverse = 1.f / now;
    auto store = [&](auto &&by) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int r = sub + q * SIDE;
            uint32_t y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 z = Type2<T>::up(w[4 * q + i]);
                y[i] = codes2(by(z.x), by(z.y));
            }
            if (mine && r < count) *reinterpret_cast<uint2 *>(dst + (first + r) * dim + d) = make_uint2(y[0] | y[1] << 16, y[2] | y[3] << 16);
        }
    };
    if (power) store([&](float z) { return z * inverse; });
    else store([&](float z) { return __fdiv_rn(z, now); });
    if (first > 0 && (grown || src != dst)) {
        const float share = grown ? __fdiv_rn(was, now) : 1.f;
        for (int r = sub; r < first; r += SIDE) {
            if (!mine) continue;
            uint2 y = *reinterpret_cast<const uint2 *>(src + r * dim + d);
            if (grown) {
                uint32_t *z = &y.x;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float2 a = values2(z[i] & 0xffffu), b = values2(z[i] >> 16);
                    z[i] = codes2(a.x * share, a.y * share) | codes2(b.x * share, b.y * share) << 16;
                }
            }
            *reinterpret_cast<uint2 *>(dst + r * dim + d) = y;
        }
    }
    __syncwarp();
    if (lane == 0) *dst_scale = now;
}

// As k_append_rows, a warp to 16 tokens of a head's keys or values at a time.  Sequence i has the
// places from offsets[i] / 16 + 2 i on, enough for its blocks wherever they begin; those it does not
// need are passed over.  A block of threads looks a place up once for `1 / parts` of its heads.  The
// tokens that a sequence's new rows share a scale with, where their page is copied, are put together from both
// by whoever writes the rows; the copying blocks have the full sixteens.
template <typename T, int DP>
__global__ void __launch_bounds__(COPY_THREADS, 4)
k_append_rows8(opattr_cache8 c8, const int32_t *seqs, int n, const int32_t *offsets, int tokens, opattr_rows k,
               opattr_rows v, AppendPlan p, unsigned row_blocks, int parts) {
    pdl_wait();
    if (*p.go == 0) return;
    const opattr_cache &kv = c8.pages;
    constexpr int WARPS = COPY_THREADS / 32;
    const int dim = kv.head_dim, warp = threadIdx.x / 32, lane = lane_id(), subs = kv.page_size / BLOCK;
    // rows of entry i from its old length `old` or from block b of its sequence on, up to `all`; its tokens before them are in page `src`
    auto block = [&](int i, int old, int all, int b, int g, int what, int src, int dst) {
        const int lo = max(old, b * BLOCK), hi = min(all, b * BLOCK + BLOCK);
        const int64_t at = ((int64_t)dst * kv.kv_heads + g) * subs + b % subs, from = ((int64_t)src * kv.kv_heads + g) * subs + b % subs;
        const opattr_rows &x = what ? v : k;
        uint8_t *pool = (uint8_t *)(what ? kv.v_pages : kv.k_pages);
        float *scales = what ? c8.v_scales : c8.k_scales;
        append_block<T, DP>((const T *)x.data + (int64_t)(offsets[i] + lo - old) * x.token_stride + g * x.head_stride, x.token_stride,
                            lo - b * BLOCK, hi - lo, dim, pool + from * BLOCK * dim, scales + from, pool + at * BLOCK * dim, scales + at);
    };
    if (blockIdx.x >= row_blocks) {
        if (*p.go == 1) return;
        const int64_t all = (int64_t)n * kv.kv_heads;
        for (int64_t x = blockIdx.x - row_blocks; x < all; x += gridDim.x - row_blocks) {
            const int i = (int)(x / kv.kv_heads), g = (int)(x % kv.kv_heads);
            const int from = p.from[i];
            // the full sixteens of an entry's keys or values, by threads t, t + step, ..
            auto copy = [&](int entry, int page, int what, int t, int step) {
                const int full = p.old[entry] % kv.page_size / BLOCK;
                const int64_t src = ((int64_t)page * kv.kv_heads + g) * subs, dst = ((int64_t)p.to[entry] * kv.kv_heads + g) * subs;
                uint8_t *pool = (uint8_t *)(what ? kv.v_pages : kv.k_pages);
                float *scales = what ? c8.v_scales : c8.k_scales;
                const uint4 *xs = (const uint4 *)(pool + src * BLOCK * dim);
                uint4 *xd = (uint4 *)(pool + dst * BLOCK * dim);
#pragma unroll 4
                for (int e = t; e < full * dim; e += step) xd[e] = xs[e];
                for (int e = t; e < full; e += step) scales[dst + e] = scales[src + e];
            };
            if (from >= 0) copy(i, from, threadIdx.x & 1, threadIdx.x >> 1, COPY_THREADS / 2);
            if (from >= -1 || p.to[i] >= 0) continue;
            // the page stays with this sequence: first those that copy it, with what they have in its last block, a
            // warp to keys or values of each
            const int page = -2 - from;
            for (int e0 = 0, task = 0; e0 < i; e0 += 32) {
                const int e = e0 + lane;
                unsigned theirs = __ballot_sync(0xffffffffu, e < i && p.from[e] == from && p.to[e] >= 0);
                for (; theirs; theirs &= theirs - 1)
                    for (int what = 0; what < 2; ++what, ++task) {
                        if (task % WARPS != warp) continue;
                        const int y = e0 + __ffs(theirs) - 1, old = p.old[y];
                        copy(y, page, what, lane, 32);
                        if (old % BLOCK) block(y, old, old + offsets[y + 1] - offsets[y], old / BLOCK, g, what, page, p.to[y]);
                    }
            }
            __syncthreads();
            const int old = p.old[i], end = old + offsets[i + 1] - offsets[i];
            const int first = old / BLOCK, last = min(end - 1, old - old % kv.page_size + kv.page_size - 1) / BLOCK;
            for (int w = warp; w < 2 * (last - first + 1); w += WARPS) block(i, old, end, first + w / 2, g, w % 2, page, page);
        }
        return;
    }
    const int64_t all = (tokens / BLOCK + 2ll * n) * parts;
    for (int64_t x = blockIdx.x; x < all; x += row_blocks) {
        const int64_t place = x / parts;
        const int part = (int)(x - place * parts);
        // the last sequence whose places begin there or before, 32 at a time
        int i = 0;
        for (int m = n; m > 1;) {
            const int step = (m + 31) / 32, e = i + step * lane;
            const bool le = step * lane < m && offsets[e] / BLOCK + 2ll * e <= place;
            const int at = 31 - __clz(__ballot_sync(0xffffffffu, le));
            i += at * step;
            m = min(step, m - at * step);
        }
        const int old = p.old[i], more = offsets[i + 1] - offsets[i], b = (int)(old / BLOCK + place - (offsets[i] / BLOCK + 2ll * i));
        if (more == 0 || b > (old + more - 1) / BLOCK) continue;
        const int j = b / subs, page = kv.table[(int64_t)seqs[i] * kv.pages_per_seq + j];
        if (page < 0 || page >= kv.n_pages) continue;             // a table that was not consistent before the call
        const int from = p.from[i];
        const bool shared = b * BLOCK < old;                      // (with tokens before the call)
        if (from < -1 && (p.to[i] < 0 ? j * kv.page_size < old : shared)) continue;
        for (int u = part * WARPS + warp; u < 2 * kv.kv_heads; u += parts * WARPS)
            block(i, old, old + more, b, u >> 1, u & 1, shared && from >= 0 ? from : page, page);
    }
}

// One thread to a sequence, or to four new pages; of few, a block that is quick to begin.
static unsigned plan_threads(int64_t n) { return n <= 256 ? 256 : PLAN_THREADS; }
static opattr_status seqs_ok(const opattr_cache *kv, const int32_t *seqs, int32_t n) {
    return cache_ok(kv) && n >= 0 && n <= std::min(kv->n_seqs, MOST_SEQS) && (n == 0 || seqs) ? OPATTR_OK : OPATTR_E_INVALID_ARG;
}

template <typename T>
static opattr_status rows8_of(Ctx &c, const opattr_cache8 &c8, const int32_t *seqs, int n, const int32_t *offsets, int tokens,
                              const opattr_rows &k, const opattr_rows &v, const AppendPlan &p) {
    const opattr_cache &kv = c8.pages;
    // few places: their heads are shared out, so that every SM has some
    const int64_t places = tokens / BLOCK + 2ll * n, wave = 8 * sm_count(c);
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(wave / places, (2 * kv.kv_heads + COPY_THREADS / 32 - 1) / (COPY_THREADS / 32)));
    const unsigned rows = (unsigned)std::min<int64_t>(places * parts, 2 * wave);
    const unsigned shared = (unsigned)std::min<int64_t>((int64_t)n * kv.kv_heads, 2 * sm_count(c));
    if (kv.head_dim <= 64)
        launch(c, "append_rows8", k_append_rows8<T, 64>, dim3(rows + shared), dim3(COPY_THREADS), 0, c8, seqs, n, offsets, tokens, k, v, p, rows, parts);
    else
        launch(c, "append_rows8", k_append_rows8<T, 128>, dim3(rows + shared), dim3(COPY_THREADS), 0, c8, seqs, n, offsets, tokens, k, v, p, rows, parts);
    return cuda_status(c, c.last_error);
}

opattr_status do_cache_append(Ctx &c, Serve &s, const opattr_cache *kv, const int32_t *seqs, int32_t n,
                              const int32_t *offsets, int64_t tokens, const opattr_rows *k, const opattr_rows *v) {
    opattr_status st = seqs_ok(kv, seqs, n);
    if (st) return st;
    const opattr_cache8 *e8 = cache8(kv);
    if (tokens < 0 || tokens > INT32_MAX || (n == 0 && tokens > 0) || (n > 0 && !offsets)) return OPATTR_E_INVALID_ARG;
    if (!rows_ok(*k, tokens, kv->kv_heads, kv->head_dim) || !rows_ok(*v, tokens, kv->kv_heads, kv->head_dim))
        return OPATTR_E_INVALID_ARG;
    if (n == 0) return OPATTR_OK;
    if ((st = serve_ready(c, s))) return st;
    // at most: a page copied and one begun by each sequence, and the full ones
    const int64_t most = std::min<int64_t>(kv->n_pages, 2ll * n + tokens / kv->page_size);
    if ((st = ensure_lasting_arena(c, Need().add<int32_t>(1).add<int32_t>(n).add<int32_t>(n).add<int32_t>(n).add<int32_t>(n).add<int32_t>(n + 1)
                                  .add<int32_t>(kv->n_seqs).add<int32_t>(most).bytes)))
        return st;
    Arena a(c);
    AppendPlan p{};
    p.go = a.take<int32_t>(1);
    p.old = a.take<int32_t>(n);
    p.from = a.take<int32_t>(n);
    p.to = a.take<int32_t>(n);
    p.late = a.take<int32_t>(n);
    p.first = a.take<int32_t>(n + 1);
    p.mark = a.take<int32_t>(kv->n_seqs);
    p.fresh = a.take<int32_t>(most);
    p.room = (int32_t)most;
    launch(c, "append_plan", k_append_plan, dim3(1), dim3(plan_threads(std::max<int64_t>(n, most / 4))), 0, *kv, seqs, n, offsets, (int)tokens, p,
           e8 ? BLOCK : 1, s.err);
    if (e8) return e8->rows == OPATTR_BF16 ? rows8_of<__nv_bfloat16>(c, *e8, seqs, n, offsets, (int)tokens, *k, *v, p)
                                           : rows8_of<__half>(c, *e8, seqs, n, offsets, (int)tokens, *k, *v, p);
    const int row = kv->kv_heads * (kv->head_dim / 8);
    const unsigned rows = grid_for(tokens, std::max(1, COPY_THREADS / row), 8u * sm_count(c));
    const unsigned shared = (unsigned)std::min<int64_t>((int64_t)n * kv->kv_heads, 2 * sm_count(c));
    launch(c, "append_rows", k_append_rows, dim3(rows + shared), dim3(COPY_THREADS), 0, *kv, seqs, n, offsets, (int)tokens,
           *k, *v, p, rows);
    return cuda_status(c, c.last_error);
}

// ---------------------------------------------------------------- fork and trim
// The plan's block makes the change itself where the sequences' tables have few
// entries, a thread to an entry (a warp to a sequence took 17 us more for fork and trim
// of 138 sequences of four pages at most).  A second launch costs the host 2 us, and the GPU what
// the block takes for 2,500 entries: fork and trim of 40 sequences of 63 pages 8.0 us here,
// 7.8 in two launches each; of 16 pages 7.1 and 7.3; of 100 (two launches) 10.1 and 7.9.
constexpr int64_t SMALL_ENTRIES = 4096;

// Page j of sequence s to sequence d; a source is no destination, its length stands.
__device__ __forceinline__ void fork_page(const opattr_cache &kv, int s, int d, int len, int j) {
    const int page = kv.table[(int64_t)s * kv.pages_per_seq + j];
    kv.table[(int64_t)d * kv.pages_per_seq + j] = page;
    if (page >= 0 && page < kv.n_pages) atomicAdd(&kv.refs[page], 1);
    if (j == 0) kv.length[d] = len;
}
__global__ void __launch_bounds__(PLAN_THREADS)
k_fork_plan(opattr_cache kv, const int32_t *src, const int32_t *dst, int n, int32_t *mark, int32_t *go, int small,
            unsigned *err) {
    pdl_wait();
    if (threadIdx.x == 0) *go = 0;
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int s = src[i], d = dst[i];
        if (s < 0 || s >= kv.n_seqs || d < 0 || d >= kv.n_seqs) bad = true;
        else {
            mark[d] = i;
            bad = bad || length_bad(kv, s) || kv.length[d] != 0;
        }
    }
    if (any_bad(bad, SERVE_INVALID, err)) return;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        // a source is no destination (its mark, where it has one, names its entry in dst)
        const int m = mark[src[i]];
        bad = bad || mark[dst[i]] != i || (m >= 0 && m < n && dst[m] == src[i]);
    }
    if (any_bad(bad, SERVE_INVALID, err)) return;
    if (small) {
        for (int x = threadIdx.x; x < n * kv.pages_per_seq; x += blockDim.x) {
            const int i = x / kv.pages_per_seq, j = x - i * kv.pages_per_seq, s = src[i], len = kv.length[s];
            if (j < pages_for(len, kv.page_size)) fork_page(kv, s, dst[i], len, j);
        }
    } else if (threadIdx.x == 0) {
        *go = 1;
    }
}
__global__ void __launch_bounds__(COPY_THREADS)
k_fork(opattr_cache kv, const int32_t *src, const int32_t *dst, const int32_t *go) {
    pdl_wait();
    if (*go == 0) return;
    const int s = src[blockIdx.x], d = dst[blockIdx.x], len = kv.length[s], held = pages_for(len, kv.page_size);
    for (int j = blockIdx.y * COPY_THREADS + threadIdx.x; j < held; j += gridDim.y * COPY_THREADS) fork_page(kv, s, d, len, j);
}

opattr_status do_cache_fork(Ctx &c, Serve &s, const opattr_cache *kv, const int32_t *src, const int32_t *dst, int32_t n) {
    opattr_status st = seqs_ok(kv, dst, n);
    if (st || n == 0) return st;
    if (!src) return OPATTR_E_INVALID_ARG;
    if ((st = serve_ready(c, s))) return st;
    if ((st = ensure_lasting_arena(c, Need().add<int32_t>(1).add<int32_t>(kv->n_seqs).bytes))) return st;
    Arena a(c);
    int32_t *go = a.take<int32_t>(1), *mark = a.take<int32_t>(kv->n_seqs);
    const int64_t entries = (int64_t)n * kv->pages_per_seq;
    const bool small = entries <= SMALL_ENTRIES;
    launch(c, "fork_plan", k_fork_plan, dim3(1), dim3(plan_threads(small ? std::max<int64_t>(n, entries / 4) : n)), 0, *kv, src, dst, n, mark, go,
           (int)small, s.err);
    if (!small)
        launch(c, "fork", k_fork, dim3(n, grid_for(kv->pages_per_seq, 4 * COPY_THREADS, 64)), dim3(COPY_THREADS), 0, *kv, src,
               dst, (const int32_t *)go);
    return cuda_status(c, c.last_error);
}

// Page j of sequence s is let go; the lowest that is free now.
__device__ __forceinline__ int trim_page(const opattr_cache &kv, int s, int j, int low) {
    int32_t *e = &kv.table[(int64_t)s * kv.pages_per_seq + j];
    const int page = *e;
    *e = -1;
    return page >= 0 && page < kv.n_pages && atomicSub(&kv.refs[page], 1) == 1 ? min(low, page) : low;
}
__device__ __forceinline__ void trim_low(const opattr_cache &kv, int low) {
    __syncwarp();
    low = __reduce_min_sync(0xffffffffu, low);
    if (lane_id() == 0 && low < INT32_MAX) atomicMin(kv.low, low);
}
__global__ void __launch_bounds__(PLAN_THREADS)
k_trim_plan(opattr_cache kv, const int32_t *seqs, const int32_t *lengths, int n, int32_t *mark, int32_t *old,
            int32_t *kept, int32_t *go, int small, unsigned *err) {
    pdl_wait();
    if (threadIdx.x == 0) *go = 0;
    bool bad = false;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int s = seqs[i], to = lengths ? lengths[i] : 0;
        if (s < 0 || s >= kv.n_seqs) bad = true;
        else {
            mark[s] = i;
            const int len = kv.length[s];
            bad = bad || length_bad(kv, s) || to < 0 || to > len;
            old[i] = len;
            kept[i] = to;        // (`lengths` may be the cache's own, which change below)
        }
    }
    if (any_bad(bad, SERVE_INVALID, err)) return;
    if (marks_bad(seqs, n, mark, err)) return;
    for (int i = threadIdx.x; i < n; i += blockDim.x) kv.length[seqs[i]] = kept[i];
    if (small) {
        int low = INT32_MAX;
        for (int x = threadIdx.x; x < n * kv.pages_per_seq; x += blockDim.x) {
            const int i = x / kv.pages_per_seq, j = x - i * kv.pages_per_seq;
            if (j >= pages_for(kept[i], kv.page_size) && j < pages_for(old[i], kv.page_size)) low = trim_page(kv, seqs[i], j, low);
        }
        trim_low(kv, low);
    } else if (threadIdx.x == 0) {
        *go = 1;
    }
}
__global__ void __launch_bounds__(COPY_THREADS)
k_trim(opattr_cache kv, const int32_t *seqs, const int32_t *kept, const int32_t *old, const int32_t *go) {
    pdl_wait();
    if (*go == 0) return;
    const int i = blockIdx.x, s = seqs[i], keep = pages_for(kept[i], kv.page_size), held = pages_for(old[i], kv.page_size);
    int low = INT32_MAX;
    for (int j = keep + blockIdx.y * COPY_THREADS + threadIdx.x; j < held; j += gridDim.y * COPY_THREADS) low = trim_page(kv, s, j, low);
    trim_low(kv, low);
}

opattr_status do_cache_trim(Ctx &c, Serve &s, const opattr_cache *kv, const int32_t *seqs, const int32_t *lengths,
                            int32_t n) {
    opattr_status st = seqs_ok(kv, seqs, n);
    if (st || n == 0) return st;
    if ((st = serve_ready(c, s))) return st;
    if ((st = ensure_lasting_arena(c, Need().add<int32_t>(1).add<int32_t>(n).add<int32_t>(n).add<int32_t>(kv->n_seqs).bytes))) return st;
    Arena a(c);
    int32_t *go = a.take<int32_t>(1), *old = a.take<int32_t>(n), *kept = a.take<int32_t>(n), *mark = a.take<int32_t>(kv->n_seqs);
    const int64_t entries = (int64_t)n * kv->pages_per_seq;
    const bool small = entries <= SMALL_ENTRIES;
    launch(c, "trim_plan", k_trim_plan, dim3(1), dim3(plan_threads(small ? std::max<int64_t>(n, entries / 4) : n)), 0, *kv, seqs, lengths, n, mark,
           old, kept, go, (int)small, s.err);
    if (!small)
        launch(c, "trim", k_trim, dim3(n, grid_for(kv->pages_per_seq, 4 * COPY_THREADS, 64)), dim3(COPY_THREADS), 0, *kv, seqs,
               (const int32_t *)kept, (const int32_t *)old, (const int32_t *)go);
    return cuda_status(c, c.last_error);
}

// ---------------------------------------------------------------- compact
// L pages are live.  The live ones at L and past it, in order, move into the
// free ones below L, in order: as many of the one as of the other, so no page
// is read after it was written and none moves twice.
constexpr int TILE_PAGES = 4096;

__device__ __forceinline__ int live_in(const opattr_cache &kv, int64_t from, int64_t to, int *warp_buf) {
    int mine = 0;
    for (int64_t i = from + threadIdx.x; i < to; i += blockDim.x) mine += kv.refs[i] > 0;
    return block_sum(mine, warp_buf);
}
__global__ void __launch_bounds__(PLAN_THREADS) k_compact_count(opattr_cache kv, int32_t *tile_live) {
    __shared__ int warp_buf[33];
    pdl_wait();
    const int64_t at = (int64_t)blockIdx.x * TILE_PAGES;
    const int live = live_in(kv, at, min(at + TILE_PAGES, kv.n_pages), warp_buf);
    if (threadIdx.x == 0) tile_live[blockIdx.x] = live;
}
// rank[page] of the pages that move, hole[rank] where they go.
// A pool of one tile counts it here; others' counts come from k_compact_count.
__global__ void __launch_bounds__(PLAN_THREADS)
k_compact_place(opattr_cache kv, const int32_t *tile_live, int tiles, int32_t *rank, int32_t *hole, int32_t *mover,
                int32_t *counts, int32_t *out_live) {
    __shared__ int warp_buf[33];
    pdl_wait();
    const int tile = blockIdx.x;
    const int64_t at = (int64_t)tile * TILE_PAGES + 4 * threadIdx.x;
    int r[4], mine = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        r[q] = at + q < kv.n_pages ? kv.refs[at + q] : 0;
        mine += r[q] > 0;
    }
    int L, below = 0;                                    // live pages, and those of them below L
    int live = block_exclusive_scan(mine, warp_buf, &L);
    if (tiles > 1) {
        int all = 0, before = 0;
        for (int t = threadIdx.x; t < tiles; t += blockDim.x) {
            all += tile_live[t];
            if (t < tile) before += tile_live[t];
        }
        L = block_sum(all, warp_buf);
        live += block_sum(before, warp_buf);
        const int edge = L / TILE_PAGES;
        for (int t = threadIdx.x; t < edge; t += blockDim.x) below += tile_live[t];
        below = block_sum(below, warp_buf) + live_in(kv, (int64_t)edge * TILE_PAGES, L, warp_buf);
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) below += at + q < L && r[q] > 0;
        below = block_sum(below, warp_buf);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t i = at + q;
        // (every page is live or a hole, a count below 0 too: as many holes as pages that move)
        if (i < L && r[q] <= 0) hole[i - live] = (int)i;
        if (i >= L && r[q] > 0) {
            rank[i] = live - below;
            mover[live - below] = (int)i;
        }
        live += r[q] > 0;
    }
    if (tile == 0 && threadIdx.x == 0) {
        counts[0] = L - below;
        counts[1] = L;
        if (out_live) *out_live = L;
    }
}
constexpr int MOVE = 4 * COPY_THREADS;          // pieces of 16 bytes of a run
// Pages over the grid; then the tables.
__global__ void __launch_bounds__(COPY_THREADS)
k_compact_move(opattr_cache kv, float *k_scales, float *v_scales, const int32_t *rank, const int32_t *hole, const int32_t *mover, const int32_t *counts) {
    pdl_wait();
    const int moves = counts[0], L = counts[1];
    const int page = kv.kv_heads * (k_scales ? kv.page_size / BLOCK * kv.head_dim : kv.page_size * (kv.head_dim / 8)), runs = (page + MOVE - 1) / MOVE;
    const int64_t t0 = (int64_t)blockIdx.x * COPY_THREADS + threadIdx.x, step = (int64_t)gridDim.x * COPY_THREADS;
    uint4 *kp = reinterpret_cast<uint4 *>(kv.k_pages), *vp = reinterpret_cast<uint4 *>(kv.v_pages);
    // runs of a page's pieces, a block to each: every thread has all its loads under way before it stores
    for (int64_t u = blockIdx.x; u < (int64_t)moves * runs; u += gridDim.x) {
        const int m = (int)(u / runs), first = (int)(u % runs) * MOVE + threadIdx.x;
        const int64_t src = mover[m] * (int64_t)page, dst = hole[m] * (int64_t)page;
        uint4 k4[MOVE / COPY_THREADS], v4[MOVE / COPY_THREADS];
#pragma unroll
        for (int q = 0; q < MOVE / COPY_THREADS; ++q) {
            const int e = first + q * COPY_THREADS;
            if (e < page) k4[q] = kp[src + e], v4[q] = vp[src + e];
        }
#pragma unroll
        for (int q = 0; q < MOVE / COPY_THREADS; ++q) {
            const int e = first + q * COPY_THREADS;
            if (e < page) kp[dst + e] = k4[q], vp[dst + e] = v4[q];
        }
    }
    if (k_scales) {
        const int each = kv.kv_heads * (kv.page_size / BLOCK);
        for (int64_t x = t0; x < (int64_t)moves * each; x += step) {
            const int m = (int)(x / each), e = (int)(x - (int64_t)m * each);
            const int64_t src = (int64_t)mover[m] * each + e, dst = (int64_t)hole[m] * each + e;
            const float a = k_scales[src], b = v_scales[src];
            k_scales[dst] = a;
            v_scales[dst] = b;
        }
    }
    for (int64_t m = t0; m < moves; m += step) {
        kv.refs[hole[m]] = kv.refs[mover[m]];
        kv.refs[mover[m]] = 0;
    }
    const int64_t entries = (int64_t)kv.n_seqs * kv.pages_per_seq;
    for (int64_t x = t0; x < entries; x += step) {
        const int e = kv.table[x];
        if (e >= L && e < kv.n_pages) {
            const int r = rank[e];
            if (r >= 0 && r < moves && mover[r] == e) kv.table[x] = hole[r];
        }
    }
    if (t0 == 0) *kv.low = L;
}

opattr_status do_cache_compact(Ctx &c, Serve &s, const opattr_cache *kv, int32_t *live) {
    if (!cache_ok(kv)) return OPATTR_E_INVALID_ARG;
    opattr_status st = serve_ready(c, s);
    if (st) return st;
    const opattr_cache8 *e8 = cache8(kv);
    const int tiles = (int)((kv->n_pages + TILE_PAGES - 1) / TILE_PAGES);
    if ((st = ensure_lasting_arena(c, Need().add<int32_t>(2).add<int32_t>(tiles).add<int32_t>(kv->n_pages).add<int32_t>(kv->n_pages)
                                  .add<int32_t>(kv->n_pages).bytes)))
        return st;
    Arena a(c);
    int32_t *counts = a.take<int32_t>(2), *tile_live = a.take<int32_t>(tiles), *rank = a.take<int32_t>(kv->n_pages);
    int32_t *hole = a.take<int32_t>(kv->n_pages), *mover = a.take<int32_t>(kv->n_pages);
    if (tiles > 1) launch(c, "compact_count", k_compact_count, dim3(tiles), dim3(PLAN_THREADS), 0, *kv, tile_live);
    launch(c, "compact_place", k_compact_place, dim3(tiles), dim3(PLAN_THREADS), 0, *kv, (const int32_t *)tile_live, tiles,
           rank, hole, mover, counts, live);
    launch(c, "compact_move", k_compact_move, dim3(8 * sm_count(c)), dim3(COPY_THREADS), 0, *kv,
           e8 ? e8->k_scales : nullptr, e8 ? e8->v_scales : nullptr, (const int32_t *)rank,
           (const int32_t *)hole, (const int32_t *)mover, (const int32_t *)counts);
    return cuda_status(c, c.last_error);
}

}  // namespace opattr
