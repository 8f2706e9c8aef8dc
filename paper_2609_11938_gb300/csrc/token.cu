// token.cu -- attention of one new token of each sequence over the paged cache
// (opattr_cache_attention).
//
// The cache is read once and there is little to compute on it, so what counts is
// that every SM has enough loads under way until the last one is done.  All
// (sequence, key head) pairs' tokens are laid end to end and cut into equal runs,
// one per block, whatever the lengths (short pairs stay whole; a pair counts one
// step more than it has, for what beginning and ending it costs: without that, a
// block whose run is of many short sequences ended 25 us after the others at 64
// sequences of 1 .. 16,000 tokens); a pair that is cut is joined by the block that
// finishes its part last, over the parts in order (so the bits do not depend on who
// that is).
//
// A warp takes 16 keys at a time straight from memory into the registers that
// the products want them in, without shared memory: the products' inner
// dimension may come in any order, so a lane takes 16 bytes (eight elements) of
// a key's row where the instruction would have four pairs, and the queries are
// laid out alike.  Values are paired across two rows by byte selection.
//   scores   S^T [16 keys x 8 queries] = K [16 x D] Q^T
//   result   O^T [D x 8 queries]      += V^T [D x 16 keys] P^T
// The queries of a key head (up to 8 or 16; more go round again) share its loads.
// P is rounded to the inputs' type, which the products take, as in prompt.cu: against 64 bits the
// results are 1.1 to 1.4 times as far off as their own rounding makes them.  As two terms, the
// rounded weight and what that left, on the same registers of values, it took 0 to 2.4 % longer and
// lost that factor, but an infinite value that is seen came out as NaN, since the second term may be 0.
//
// Measured on one GB300, whose memory copies at 6.8 TB/s (bytes of live keys and values
// over the time of a call among others): 2 sequences of 260,000 tokens, 40 heads of 128
// on 8: 316 us, 6.8 TB/s; 64 of 1 .. 16,001, 32 heads on 8: 67.7 us, 6.0, where the
// beginning and the end of the one launch, about 7 us, show; one of 700, 12 heads of 64:
// 7.7 us of the host's 12.  48 sequences that share the pages of 8 read them 48 times, from the
// second level cache: 30 us.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "serve.cuh"

namespace opattr {

bool cache_ok(const opattr_cache *k);

constexpr int TOKEN_WARPS = 4, TOKEN_THREADS = 32 * TOKEN_WARPS;
// Pairs are cut as far as there are blocks, but not so far that a longer join takes what
// shorter parts give: a part more costs 0.13 us to join, a step of a block by itself 0.5 to 1,
// and c / x + 0.13 x, of c steps in x parts, is least where x is the root of 8 c (12 measured
// best): 60,000 tokens, 8 heads of 128 on one: 68 us in parts of two steps, 29 of nine.  Pairs of
// few steps are whole, and belong to the block that they begin in: 13 of 1 .. 596
// tokens, 8 heads of 64 on 2: 10.7 us with every pair cut, 6.4; up to four steps 7.1, and
// 293 of 148 .. 444, 16 heads of 128 on 4, 37.6 for 36.8.
constexpr int WHOLE_STEPS = 3;
constexpr float JOIN_STEPS = 12.f;

struct TokenArgs {
    opattr_cache kv;
    const int32_t *seqs;
    int n, q_heads, group, blocks_of_heads;   // query heads; of a key head; and runs of them that share loads
    opattr_rows q, out;
    float *lse;
    float scale;
    int shift;                                // log2 of the page size
    float *parts;                             // [grid][2] partial results
    uint32_t *tickets;                        // [grid]
};

__device__ __forceinline__ uint4 load16(const void *p, bool on) {
    uint4 r = make_uint4(0, 0, 0, 0);
    if (on)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
__device__ __forceinline__ float root(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <typename T>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (std::is_same<T, __nv_bfloat16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit values, two of a row in a lane, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// DP: the padded head width; NT: eights of queries; FR: sixteens of keys that a
// warp takes at a time.
template <typename T, int DP, int NT, int FR>
__global__ void __launch_bounds__(TOKEN_THREADS, NT == 1 ? 3 : 2) k_token(const __grid_constant__ TokenArgs p, unsigned *err) {
    constexpr bool BF = std::is_same<T, __nv_bfloat16>::value;
    // as in prompt.cu: weights up to 2^(OFFSET + SLACK), rescaled when a maximum outgrows SLACK
    constexpr float OFFSET = BF ? 0.f : 8.f, SLACK = BF ? 8.f : 7.f;
    constexpr int KC = DP / 32, VC = DP / 64, STEP = 16 * FR * TOKEN_WARPS, NQ = 8 * NT, ROW = DP + 4;
    __shared__ float so[TOKEN_WARPS][NQ][ROW];
    __shared__ float sm[TOKEN_WARPS][NQ], sl[TOKEN_WARPS][NQ];
    __shared__ long long warp_buf[33];
    __shared__ long long first_at;
    __shared__ int first_seq, last_one;
    pdl_wait();
    const opattr_cache &kv = p.kv;
    const int lane = lane_id(), warp = threadIdx.x >> 5, row = lane >> 2, col = lane & 3;
    const int units = kv.kv_heads * p.blocks_of_heads;

    // ---- this block's run
    auto seq_of = [&](int b) { return p.seqs ? p.seqs[b] : b; };
    auto len_of = [&](int seq) {
        if (seq < 0 || seq >= kv.n_seqs) return -1;
        const int len = kv.length[seq];
        return len > kv.pages_per_seq << p.shift ? -1 : len;
    };
    auto steps_of = [](int len) { return len <= 0 ? 1 : (len - 1) / STEP + 1; };
    auto cost_of = [](int steps) { return steps + 1; };        // place 0 of a pair stands for no keys
    const int per = (p.n + TOKEN_THREADS - 1) / TOKEN_THREADS, b0 = min(p.n, (int)threadIdx.x * per), b1 = min(p.n, b0 + per);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) {
        const int len = len_of(seq_of(b));
        if (len < 0 && blockIdx.x == 0) atomicOr(err, SERVE_INVALID);
        mine += (long long)cost_of(steps_of(len)) * units;
    }
    long long total;
    long long at = block_exclusive_scan(mine, warp_buf, &total);
    const long long pairs = (long long)p.n * units;
    // (in 32 bits, where no grid comes near their end: 64 took 0.3 us of every launch)
    const int blocks = (int)gridDim.x, few = (int)min(total, 1ll << 30), few_pairs = (int)min(pairs, 1ll << 30);
    const long long W = min(min(few, blocks), (int)fminf(1e6f, root(JOIN_STEPS * (float)few * (float)few_pairs)));
    if (blockIdx.x >= W) return;
    const long long s0 = blockIdx.x * total / W, s1 = (blockIdx.x + 1) * total / W;
    if (s0 >= at && s0 < at + mine) {
        int b = b0;
        for (;; ++b) {
            const long long of = (long long)cost_of(steps_of(len_of(seq_of(b)))) * units;
            if (s0 < at + of) break;
            at += of;
        }
        first_seq = b;
        first_at = at;
    }
    __syncthreads();

    // ---- its pairs, one after another
    int b = first_seq;
    long long base = first_at;                    // where sequence b's steps begin
    const float c = p.scale * LOG2E;
    for (long long s = s0; s < s1;) {
        const int seq = seq_of(b), len = max(0, len_of(seq)), steps = steps_of(len), cost = cost_of(steps);
        if (s >= base + (long long)cost * units) {
            base += (long long)cost * units;
            ++b;
            continue;
        }
        const int unit = (int)((s - base) / cost), g = unit / p.blocks_of_heads, hb = unit % p.blocks_of_heads;
        const long long unit_at = base + (long long)unit * cost + 1;   // of its first step
        int from = (int)max(0ll, s - unit_at), to = (int)min((long long)steps, s1 - unit_at);
        if (steps <= WHOLE_STEPS) {
            // a short pair is whole, and belongs to the block that it begins in
            to = s < unit_at ? steps : from;
            from = min(from, to);
        }
        s = unit_at + steps;
        if (from >= to) continue;
        const int heads = min(NQ, p.group - hb * NQ), head0 = g * p.group + hb * NQ;
        const int32_t *table = kv.table + (long long)seq * kv.pages_per_seq;

        uint32_t qf[NT][KC][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < KC; ++i) {
                const int d = 32 * i + 8 * col, h = 8 * t + row;
                const uint4 x = load16((const T *)p.q.data + b * p.q.token_stride + (head0 + h) * p.q.head_stride + d,
                                       h < heads && d < kv.head_dim);
                qf[t][i][0] = x.x, qf[t][i][1] = x.y, qf[t][i][2] = x.z, qf[t][i][3] = x.w;
            }
        float o[NT][DP / 16][4] = {}, m[NT][2], l[NT][2] = {};
#pragma unroll
        for (int t = 0; t < NT; ++t) m[t][0] = m[t][1] = -INFINITY;
        // (unsigned where a step past a length near 2^31 is counted)
        const int last = (int)min((unsigned)len, (unsigned)to * STEP);  // keys of this run: from * STEP .. last
        uint4 kr[FR][2][KC], vr[FR][4][VC];
        // pages of this warp's coming keys, one to a lane: lane i has those of step held + i
        int held = 0, pages[FR];
        auto page_of = [&](int step, int f) -> int {
            if (step >= held + 32 || step < held || step == from) {
                held = step;
#pragma unroll
                for (int x = 0; x < FR; ++x) {
                    const unsigned key = (unsigned)(step + lane) * STEP + 16 * (warp * FR + x);
                    pages[x] = key < (unsigned)last ? table[key >> p.shift] : 0;
                }
            }
            return __shfl_sync(0xffffffffu, pages[f], step - held);
        };
        // where the rows of a step's keys are; none past the run's end or of a page that is none
        auto rows_at = [&](int step, int f, int &lim) -> long long {
            const int key = step * STEP + 16 * (warp * FR + f), page = page_of(step, f);
            lim = last - key;
            if (lim > 0 && (page < 0 || page >= kv.n_pages)) {
                atomicOr(err, SERVE_INVALID);
                lim = 0;
            }
            return (((long long)page * kv.kv_heads + g << p.shift) + (key & (kv.page_size - 1))) * kv.head_dim;
        };
        long long kat[FR], vat[FR];
        int klim[FR], vlim[FR];
        auto load_keys = [&](int step) {
#pragma unroll
            for (int f = 0; f < FR; ++f) {
                kat[f] = rows_at(step, f, klim[f]);
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < KC; ++i)
                        kr[f][r][i] = load16((const T *)kv.k_pages + kat[f] + (row + 8 * r) * kv.head_dim + 32 * i + 8 * col,
                                             row + 8 * r < klim[f] && 32 * i + 8 * col < kv.head_dim);
            }
        };
        auto load_values = [&]() {
#pragma unroll
            for (int f = 0; f < FR; ++f) {
                vat[f] = kat[f], vlim[f] = klim[f];
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < VC; ++i) {
                        const int key = 2 * col + (r & 1) + 8 * (r >> 1), d = 64 * i + 8 * row;
                        vr[f][r][i] = load16((const T *)kv.v_pages + vat[f] + key * kv.head_dim + d, key < vlim[f] && d < kv.head_dim);
                    }
            }
        };
        load_keys(from);
        load_values();
        for (int step = from; step < to; ++step) {
            float x[FR][NT][4] = {};
#pragma unroll
            for (int f = 0; f < FR; ++f)
#pragma unroll
                for (int i = 0; i < KC; ++i) {
                    const uint4 u = kr[f][0][i], w = kr[f][1][i];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        mma16<T>(x[f][t], u.x, w.x, u.y, w.y, qf[t][i][0], qf[t][i][1]);
                        mma16<T>(x[f][t], u.z, w.z, u.w, w.w, qf[t][i][2], qf[t][i][3]);
                    }
                }
            if (step + 1 < to) load_keys(step + 1);
            float top[NT][2];
            bool more = false;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                top[t][0] = top[t][1] = -INFINITY;
#pragma unroll
                for (int f = 0; f < FR; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[f][t][i] = row + 8 * (i >> 1) < vlim[f] ? x[f][t][i] * c : -INFINITY;
                        top[t][i & 1] = fmaxf(top[t][i & 1], x[f][t][i]);
                    }
                more = more || top[t][0] - m[t][0] > SLACK || top[t][1] - m[t][1] > SLACK;
            }
            if (__any_sync(0xffffffffu, more)) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float y = fmaxf(m[t][q], top[t][q]);
#pragma unroll
                        for (int e = 4; e < 32; e <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, e));
                        const float keep = y == m[t][q] ? 1.f : exp2_fast(m[t][q] - y);
                        m[t][q] = y;
                        l[t][q] *= keep;
#pragma unroll
                        for (int i = 0; i < DP / 16; ++i) o[t][i][q] *= keep, o[t][i][q + 2] *= keep;
                    }
            }
#pragma unroll
            for (int f = 0; f < FR; ++f) {
                uint32_t pb[NT][2];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float ref = m[t][i & 1];
                        y[i] = exp2_fast(x[f][t][i] - (ref == -INFINITY ? -OFFSET : ref - OFFSET));
                        l[t][i & 1] += y[i];
                    }
                    pb[t][0] = transpose8(Type2<T>::down(y[0], y[1]));
                    pb[t][1] = transpose8(Type2<T>::down(y[2], y[3]));
                }
#pragma unroll
                for (int i = 0; i < VC; ++i) {
                    const uint32_t *v0 = &vr[f][0][i].x, *v1 = &vr[f][1][i].x, *v2 = &vr[f][2][i].x, *v3 = &vr[f][3][i].x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t a0 = __byte_perm(v0[e], v1[e], 0x5410), a1 = __byte_perm(v0[e], v1[e], 0x7632);
                        const uint32_t a2 = __byte_perm(v2[e], v3[e], 0x5410), a3 = __byte_perm(v2[e], v3[e], 0x7632);
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma16<T>(o[t][4 * i + e], a0, a1, a2, a3, pb[t][0], pb[t][1]);
                    }
                }
            }
            if (step + 1 < to) load_values();
        }

        // ---- the warps' parts together
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float y = l[t][q];
#pragma unroll
                for (int e = 4; e < 32; e <<= 1) y += __shfl_xor_sync(0xffffffffu, y, e);
                const int h = 8 * t + 2 * col + q;
                if (row == 0) sm[warp][h] = m[t][q], sl[warp][h] = y;
#pragma unroll
                for (int i = 0; i < VC; ++i) {
                    float *at = &so[warp][h][64 * i + 8 * row];
                    *reinterpret_cast<float4 *>(at) = make_float4(o[t][4 * i][q], o[t][4 * i][q + 2], o[t][4 * i + 1][q], o[t][4 * i + 1][q + 2]);
                    *reinterpret_cast<float4 *>(at + 4) = make_float4(o[t][4 * i + 2][q], o[t][4 * i + 2][q + 2], o[t][4 * i + 3][q], o[t][4 * i + 3][q + 2]);
                }
            }
        __syncthreads();
        const bool whole = from == 0 && to == steps;
        // a pair's parts: the block it begins in keeps its own in place 1, later ones in place 0
        const int block1 = (int)(((unit_at + 1) * W - 1) / total), block2 = (int)(((unit_at + steps) * W - 1) / total);
        constexpr int PART = NQ * (DP + 2);
        auto finish = [&](int h, int d, float top, float sum, const float *y) {
            const float share = sum == 0.f ? 0.f : 1.f / sum;
            uint4 r;
            r.x = sum == 0.f ? 0u : Type2<T>::down(y[0] * share, y[1] * share);
            r.y = sum == 0.f ? 0u : Type2<T>::down(y[2] * share, y[3] * share);
            r.z = sum == 0.f ? 0u : Type2<T>::down(y[4] * share, y[5] * share);
            r.w = sum == 0.f ? 0u : Type2<T>::down(y[6] * share, y[7] * share);
            *reinterpret_cast<uint4 *>((T *)p.out.data + b * p.out.token_stride + (head0 + h) * p.out.head_stride + d) = r;
            if (p.lse && d == 0)
                p.lse[(long long)b * p.q_heads + head0 + h] =
                    sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) - OFFSET + log2f(sum)) * LN2;
        };
        float *part = p.parts + ((long long)blockIdx.x * 2 + (from == 0)) * PART;
        for (int i = threadIdx.x; i < NQ * (DP / 8); i += TOKEN_THREADS) {
            const int h = i / (DP / 8), d = i % (DP / 8) * 8;
            float top = -INFINITY, sum = 0.f, y[8] = {};
#pragma unroll
            for (int w = 0; w < TOKEN_WARPS; ++w) top = fmaxf(top, sm[w][h]);
#pragma unroll
            for (int w = 0; w < TOKEN_WARPS; ++w) {
                const float keep = sm[w][h] == top ? 1.f : exp2_fast(sm[w][h] - top);
                sum = __fmaf_rn(sl[w][h], keep, sum);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __fmaf_rn(so[w][h][d + e], keep, y[e]);
            }
            if (h >= heads || d >= kv.head_dim) continue;
            if (whole) finish(h, d, top, sum, y);
            else {
                __stcg(reinterpret_cast<float4 *>(part + h * DP + d), make_float4(y[0], y[1], y[2], y[3]));
                __stcg(reinterpret_cast<float4 *>(part + h * DP + d + 4), make_float4(y[4], y[5], y[6], y[7]));
                if (d == 0) __stcg(reinterpret_cast<float2 *>(part + NQ * DP) + h, make_float2(top, sum));
            }
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) last_one = atomicAdd(&p.tickets[block1], 1u) == (unsigned)(block2 - block1);
            __syncthreads();
            if (last_one) {
                __threadfence();
                for (int i = threadIdx.x; i < NQ * (DP / 8); i += TOKEN_THREADS) {
                    const int h = i / (DP / 8), d = i % (DP / 8) * 8;
                    if (h >= heads || d >= kv.head_dim) continue;
                    float top = -INFINITY, sum = 0.f, y[8] = {};
#pragma unroll 4
                    for (int k = block1; k <= block2; ++k) {
                        const float *at = p.parts + ((long long)k * 2 + (k == block1)) * PART;
                        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(at + NQ * DP) + h);
                        const float4 u = __ldcg(reinterpret_cast<const float4 *>(at + h * DP + d));
                        const float4 w = __ldcg(reinterpret_cast<const float4 *>(at + h * DP + d + 4));
                        const float t = fmaxf(top, ml.x), a = top == t ? 1.f : exp2_fast(top - t), z = ml.x == t ? 1.f : exp2_fast(ml.x - t);
                        top = t;
                        sum = __fmaf_rn(ml.y, z, sum * a);
                        y[0] = __fmaf_rn(u.x, z, y[0] * a), y[1] = __fmaf_rn(u.y, z, y[1] * a);
                        y[2] = __fmaf_rn(u.z, z, y[2] * a), y[3] = __fmaf_rn(u.w, z, y[3] * a);
                        y[4] = __fmaf_rn(w.x, z, y[4] * a), y[5] = __fmaf_rn(w.y, z, y[5] * a);
                        y[6] = __fmaf_rn(w.z, z, y[6] * a), y[7] = __fmaf_rn(w.w, z, y[7] * a);
                    }
                    finish(h, d, top, sum, y);
                }
                if (threadIdx.x == 0) p.tickets[block1] = 0;
            }
        }
        __syncthreads();
    }
}

template <typename T, int DP, int NT, int FR>
static opattr_status run_token(Ctx &c, Serve &s, TokenArgs &p) {
    const int64_t most = (int64_t)p.n * p.kv.kv_heads * p.blocks_of_heads *
                         (((int64_t)p.kv.pages_per_seq * p.kv.page_size + 16 * FR * TOKEN_WARPS - 1) / (16 * FR * TOKEN_WARPS));
    const int grid = (int)std::min<int64_t>((NT == 1 ? 3 : 2) * (int64_t)sm_count(c), most);
    opattr_status st = serve_ready(c, s);
    if (st) return st;
    const int64_t part = (int64_t)8 * NT * (DP + 2);
    if ((st = ensure_lasting_arena(c, Need().add<float>(2 * grid * part).bytes))) return st;
    Arena a(c);
    p.parts = a.take<float>(2 * grid * part);
    p.tickets = s.tickets;
    launch(c, "token", k_token<T, DP, NT, FR>, dim3(grid), dim3(TOKEN_THREADS), 0, p, s.err);
    return cuda_status(c, c.last_error);
}
template <typename T>
static opattr_status token_of(Ctx &c, Serve &s, TokenArgs &p) {
    if (p.kv.head_dim <= 64) return p.group <= 8 ? run_token<T, 64, 1, 2>(c, s, p) : run_token<T, 64, 2, 2>(c, s, p);
    return p.group <= 8 ? run_token<T, 128, 1, 1>(c, s, p) : run_token<T, 128, 2, 1>(c, s, p);
}

opattr_status do_cache_attention(Ctx &c, Serve &s, const opattr_cache *kv, const int32_t *seqs, int32_t n,
                                 int32_t q_heads, const opattr_rows *q, const opattr_rows *out, float *lse,
                                 float scale) {
    if (!cache_ok(kv) || n < 0 || q_heads < 1 || q_heads % kv->kv_heads || !isfinite(scale)) return OPATTR_E_INVALID_ARG;
    if (!rows_ok(*q, n, q_heads, kv->head_dim) || !rows_ok(*out, n, q_heads, kv->head_dim)) return OPATTR_E_INVALID_ARG;
    if (!seqs && n > kv->n_seqs) return OPATTR_E_INVALID_ARG;
    if (n == 0) return OPATTR_OK;
    TokenArgs p{};
    p.kv = *kv;
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
    return kv->dtype == OPATTR_BF16 ? token_of<__nv_bfloat16>(c, s, p) : token_of<__half>(c, s, p);
}

}  // namespace opattr
