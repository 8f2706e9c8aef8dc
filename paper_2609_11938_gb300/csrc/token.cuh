// token.cuh -- attention of one new token of each sequence over the paged cache
// (opattr_cache_attention, opattr_cache_attention_window).
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
// P is rounded to the inputs' type, which the products take, as in prompt.cuh: against 64 bits the
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
//
// Pages of 8 bits (E8): half the bytes, so that what is done for each of them counts.  Codes become halves, exactly,
// on the way into the products (a query of bfloat16 is brought into half's range by a power of
// two); the scale of 16 keys multiplies their scores, and the sums of their values' products.  No weight carries a
// scale, so that blocks may be far apart, but not as far as they like: a weight that is rounded to half is off by 2^-33 of
// its row's largest at most, and below that it is 0, however large its block's values are.  (Weights of 16 keys brought to
// their own power of two would keep them; their maximum is three exchanges between lanes, in every step.)  Where a warp's keys are whole sixteens, which
// is checked once for a lane's 32 coming steps, its loads have no conditions; those of heads 64 or 128 wide have their
// offsets in the instruction (2 sequences of 500,000 tokens, 40 heads of 128 on 8: 374 us with the conditions, 304
// without), those of other widths add them, in kernels of their own (16 of 30,000, 32 heads of 96 on 8: 160, 150).  Where
// pairs are many each warp has some of its own, and nobody waits for a block.
// Through a window (WIN) the sixteens of keys that are not seen are left out of a sequence's steps; the first
// ones have the sinks, the others begin where the window does.
//   8 bits, bytes as above: 2 of 500,000, 40 heads of 128 on 8: 304 to 308 us, 6.7 TB/s; 64 of 1 .. 16,001, 32 heads on 8: 44 us,
//   4.7, of which about 13 are the launch, first loads and joins; 200 of 4,096, 16 heads of 64: 276 us, 6.1.
//   A window of 4,096 and 4 sinks, 16 bits: 96 of 1 .. 20,001, 32 heads of 128 on 8: 80 us, 6.2.
// Tried for 8 bits: a ring of copies in shared memory, three to six steps ahead, in the place of loads into registers: 350 us
// for the 304 at every depth, and 77 for 79 at 200 sequences of 64 wide heads.
#pragma once
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "serve.cuh"

namespace opattr {

constexpr int TOKEN_WARPS = 4, TOKEN_THREADS = 32 * TOKEN_WARPS;
// Pairs are cut as far as there are blocks, but not so far that a longer join takes what
// shorter parts give: a part more costs 0.13 us to join, a step of a block by itself 0.5 to 1,
// and c / x + 0.13 x, of c steps in x parts, is least where x is the root of 8 c (12 measured
// best): 60,000 tokens, 8 heads of 128 on one: 68 us in parts of two steps, 29 of nine.  Pairs of
// few steps are whole, and belong to the block that they begin in: 13 of 1 .. 596
// tokens, 8 heads of 64 on 2: 10.7 us with every pair cut, 6.4; up to four steps 7.1, and
// 293 of 148 .. 444, 16 heads of 128 on 4, 37.6 for 36.8.
constexpr unsigned PARTLY = 1u << 30;
constexpr int WHOLE_STEPS = 3;
constexpr float JOIN_STEPS = 12.f;
// A warp by itself (TW below) takes 0.2 us to join a part more, 0.4 of 128 wide heads, and a sequence that is long among
// many short ones has hundreds.  Past GROUP parts it joins in two stages, groups of about their root, whose last warps do it side by
// side: one of 200,000 tokens among 1,500 of 300, 8 bits, 8 heads of 64 on one: 160 us in one stage, 37; among 2,300 of 1,000, 128 wide
// 160, 119; through a window of 100,000, 16 bits, among 2,300 of 300, 64 wide 75, 49.
constexpr int GROUP = 8;

// Pages of 8 bits: a warp takes two sixteens of keys at a time, and an SM holds so many blocks (by registers).
// Of 64 wide heads, 200 sequences of 1,028 tokens, 16 heads: two sixteens in four blocks 79 us, one in five 84, four in
// three 94; of 128 wide, 2 sequences of 500,000, 40 heads on 8: two in three blocks 307 us, one in four 318, two in four (which do
// not fit) 454.
template <int DP, int NT>
struct Eight {
    static constexpr int BLOCKS = NT > 1 ? 2 : DP == 64 ? 4 : 3;
};
// (pages of 8 bits) A weight stands at 2^15 at most, and a row's sums are divided by that of its weights at the end: sums of
// values from 2^113 on may leave 32 bits before.  A warp whose results come out at LARGE or more, or not finite, makes
// them again, LOWERED times as large: 2^31 tokens of 2^128 stay below 2^(15 + 31 + 128 - 64) so, and small values beside them
// lose 2^-86 a token.  Values below 2^49 are LARGE in no sum of 2^31 tokens.  All other calls pay a product for each 16
// keys and a look at the results, 0 to 4 % (114 sequences of 2,060 tokens, 16 heads of 64: 87.1 us without, 89.5; half through a
// window, 128 wide, 31.0 and 33.6).  Scales watched on the way took registers that are not there: 18 % where 12 heads of 128 share
// keys.
constexpr float LARGE = 0x1p96f, LOWERED = 0x1p-64f;
// Pairs for each SM from which on a warp has pairs of its own (TW below; pages of 8 bits, and windows).  It pays where pairs are
// short: a warp's time as a share of a block's, bfloat16, tokens (or window) a pair  256  1,024  4,096  32,768
//   8 bits, 16 heads of 64, 1,232 pairs                                              1.08   0.99   1.02   1.02
//                           3,664                                                    0.89   0.94   1.00   1.02
//   32 of 128 on 8, 1,832                                                            0.99   1.01   1.02   1.02
//                   3,656                                                            0.91   1.00   1.02   1.02
//   64 of 64 on 4, 48 of 128 on 4, 3,652                                             0.79   0.90   0.97   1.00
//   32 of 96 on 8, 3,656 (half 0.98 .. 1.10)                                         0.84   0.89   0.93   0.94
//   through windows, those of 3,650 (96 wide 0.79 .. 1.12; 128 in half 0.74 .. 0.93) 0.72   0.89   0.97   1.01
//   16 bits, windows, 16 of 64 and 32 of 128 on 8, 3,660                             0.84   0.98   1.00   1.00
// (608 pairs of 64 wide 1,028 tokens 1.14; 912 of 128 through a window of 256 1.03.)  The host knows the room of a table, not what is in it:
// to go by that too would cost short sequences in a large table up to a quarter, for 2 % of long ones.  Pages of 16 bits
// without a window read with conditions in any case, and a warp by itself only loses: 64 wide 1.10 from 1,024 tokens on, 128 1.01.
constexpr int own_pairs(int dp) { return dp == 64 ? 8 : 12; }

struct TokenArgs {
    opattr_cache kv;
    const int32_t *seqs;
    int n, q_heads, group, blocks_of_heads;   // query heads; of a key head; and runs of them that share loads
    opattr_rows q, out;
    float *lse;
    float scale;
    int shift;                                // log2 of the page size
    float *parts;                             // [grid][2] partial results
    uint32_t *tickets;                        // [TICKETS] of pairs, then [2 TICKETS] of groups of their parts
    const float *k_scales, *v_scales;         // (pages of 8 bits)
    int window, sinks;                        // (through a window) last tokens that are seen, and first ones
};

__device__ __forceinline__ uint4 load16(const void *p, bool on) {
    uint4 r = make_uint4(0, 0, 0, 0);
    if (on)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
__device__ __forceinline__ uint2 load8(const void *p, bool on) {
    uint2 r = make_uint2(0, 0);
    if (on) asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ float root(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// The nearest finite number; NaN stays.
__device__ __forceinline__ float within(float x) {
    float r;
    asm("min.NaN.f32 %0, %1, 0f7f7fffff;\n max.NaN.f32 %0, %0, 0fff7fffff;" : "=f"(r) : "f"(x));
    return r;
}
// The larger of two, NaN where one is.
__device__ __forceinline__ float max_nan(float x, float y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
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
// The same of halves, and of sums that begin with it.
__device__ __forceinline__ void mma16_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("{\n .reg .f32 z;\n mov.f32 z, 0f00000000;\n"
        " mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {z, z, z, z};\n}"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit values, two of a row in a lane, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// Two codes of 8 bits, in the low or the high half of x, as two halves: exact.
__device__ __forceinline__ uint32_t half_lo(uint32_t x) {
    uint32_t r;
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t half_hi(uint32_t x) {
    uint32_t r;
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, hi;\n}" : "=r"(r) : "r"(x));
    return r;
}

// A query's row, 16 elements of it in a lane, as halves for the products with codes of 8
// bits; four lanes (xor 1, 2) have all of it.  bfloat16 is brought within half's range by a power of
// two, which `back` undoes: exact, but for elements below 2^-31 of the row's largest.
template <typename T, int KC>
__device__ __forceinline__ void query_halves(uint32_t (&r)[KC][8], float &back) {
    back = 1.f;
    if (std::is_same<T, __half>::value) return;
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned lo = r[i][j] << 16 & 0x7fffffffu, hi = r[i][j] & 0x7fff0000u;
            top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
        }
#pragma unroll
    for (int e = 1; e < 4; e <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, e));
    // the largest comes to 2^14 .. 2^15; both powers are normal numbers, and so is `back` times the call's scale down to
    // 2^-14 of that (rows below 2^-98 stay smaller: their least element, 2^-133, comes to 2^-21, which half has)
    const int e = max(-98, (int)(top >> 23) - 127);
    const float up = __int_as_float((14 - e + 127) << 23);
    back = __int_as_float((e - 14 + 127) << 23);
#pragma unroll
    for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 x = Type2<__nv_bfloat16>::up(r[i][j]);
            r[i][j] = Type2<__half>::down(x.x * up, x.y * up);
        }
}

// Loads that nothing holds back: no zeros beforehand, and the offset within the instruction.
template <int OFF>
__device__ __forceinline__ uint4 get16(const uint8_t *p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4 + %5];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p), "n"(OFF));
    return r;
}
template <int OFF>
__device__ __forceinline__ uint2 get8(const uint8_t *p) {
    uint2 r;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2 + %3];" : "=r"(r.x), "=r"(r.y) : "l"(p), "n"(OFF));
    return r;
}
__device__ __forceinline__ void fma_pair(float &a, float &b, float x, float y, float f) {
    asm("{\n .reg .b64 s, u, v;\n mov.b64 s, {%0, %1};\n mov.b64 u, {%2, %3};\n mov.b64 v, {%4, %4};\n fma.rn.f32x2 s, u, v, s;\n mov.b64 {%0, %1}, s;\n}"
        : "+f"(a), "+f"(b) : "f"(x), "f"(y), "f"(f));
}

// DP: the padded head width; NT: eights of queries; FR: sixteens of keys that a
// warp takes at a time; E8: pages of 8 bits; WIN: through a window.  TW: warps that share a pair's
// keys: all of a block, or each by itself.  FULL: heads are as wide as they are padded to.
template <typename T, int DP, int NT, int FR, bool E8, bool WIN, int TW, bool FULL>
__global__ void __launch_bounds__(TOKEN_THREADS, E8 ? Eight<DP, NT>::BLOCKS : NT == 1 ? 3 : 2) k_token(const __grid_constant__ TokenArgs p, unsigned *err) {
    using P = std::conditional_t<E8, __half, T>;          // what the products take
    constexpr bool BF = std::is_same<P, __nv_bfloat16>::value;
    // as in prompt.cuh: weights up to 2^(OFFSET + SLACK), rescaled when a maximum outgrows SLACK
    constexpr float OFFSET = BF ? 0.f : 8.f, SLACK = BF ? 8.f : 7.f;
    constexpr int KC = DP / (E8 ? 64 : 32), VC = DP / 64, STEP = 16 * FR * TW, NQ = 8 * NT, ROW = DP + 4;
    __shared__ float so[TOKEN_WARPS][NQ][ROW];
    __shared__ float sm[TOKEN_WARPS][NQ], sl[TOKEN_WARPS][NQ];
    __shared__ long long warp_buf[33];
    constexpr int TEAMS = TOKEN_WARPS / TW;                    // of a block
    __shared__ long long first_at[TEAMS];
    __shared__ int first_seq[TEAMS], last_one;
    pdl_wait();
    const opattr_cache &kv = p.kv;
    const int lane = lane_id(), warp = threadIdx.x >> 5, row = lane >> 2, col = lane & 3;
    const int mate = TW == 1 ? 0 : warp, own = TW == 1 ? warp : 0, me = TW == 1 ? lane : (int)threadIdx.x;
    const int team = TW == 1 ? (int)blockIdx.x * TOKEN_WARPS + warp : (int)blockIdx.x;
    auto together = [] {
        if (TW == 1) __syncwarp();
        else __syncthreads();
    };
    const int units = kv.kv_heads * p.blocks_of_heads;

    // ---- this block's run
    auto seq_of = [&](int b) { return p.seqs ? p.seqs[b] : b; };
    auto len_of = [&](int seq) {
        if (seq < 0 || seq >= kv.n_seqs) return -1;
        const int len = kv.length[seq];
        return len > kv.pages_per_seq << p.shift ? -1 : len;
    };
    // Steps of a length.  Through a window, sixteens of keys that nobody sees are left out: the first
    // `head` ones have the sinks, and later ones are `gap` further on.
    auto steps_of = [&](int len, int &head, int &gap) {
        head = gap = 0;
        if (!WIN) return len <= 0 ? 1 : (len - 1) / STEP + 1;
        const int low = max(0, len - p.window), first = low >> 4, few = min(p.sinks, low);
        head = min(first, (int)(((unsigned)few + 15) >> 4));
        gap = first - head;
        const int all = len <= 0 ? 1 : ((len - 1) >> 4) + 1 - gap;
        return (all - 1) / (STEP / 16) + 1;
    };
    auto count_of = [&](int len) {
        int head, gap;
        return steps_of(len, head, gap);
    };
    auto cost_of = [](int steps) { return steps + 1; };        // place 0 of a pair stands for no keys
    const int per = (p.n + TOKEN_THREADS - 1) / TOKEN_THREADS, b0 = min(p.n, (int)threadIdx.x * per), b1 = min(p.n, b0 + per);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) {
        const int len = len_of(seq_of(b));
        if (len < 0 && blockIdx.x == 0) atomicOr(err, SERVE_INVALID);
        mine += (long long)cost_of(count_of(len)) * units;
    }
    long long total;
    long long at = block_exclusive_scan(mine, warp_buf, &total);
    const long long pairs = (long long)p.n * units;
    // (in 32 bits, where no grid comes near their end: 64 took 0.3 us of every launch)
    const int blocks = (int)gridDim.x * TEAMS, few = (int)min(total, 1ll << 30), few_pairs = (int)min(pairs, 1ll << 30);
    const long long W = min(min(few, blocks), (int)fminf(1e6f, root(JOIN_STEPS * (float)few * (float)few_pairs)));
    if ((long long)blockIdx.x * TEAMS >= W) return;
#pragma unroll
    for (int x = 0; x < TEAMS; ++x) {
        const long long begin = ((long long)blockIdx.x * TEAMS + x) * total / W;
        if (begin >= at && begin < at + mine) {
            int b = b0;
            long long here = at;
            for (;; ++b) {
                const long long of = (long long)cost_of(count_of(len_of(seq_of(b)))) * units;
                if (begin < here + of) break;
                here += of;
            }
            first_seq[x] = b;
            first_at[x] = here;
        }
    }
    const long long s0 = team * total / W, s1 = (team + 1ll) * total / W;
    __syncthreads();
    if (TW == 1 && team >= W) return;

    // ---- its pairs, one after another
    int b = first_seq[own];
    long long base = first_at[own];                    // where sequence b's steps begin
    const float c = p.scale * LOG2E;
    for (long long s = s0; s < s1;) {
        int head, gap;
        const int seq = seq_of(b), len = max(0, len_of(seq)), steps = steps_of(len, head, gap), cost = cost_of(steps);
        if (s >= base + (long long)cost * units) {
            base += (long long)cost * units;
            ++b;
            continue;
        }
        const long long past = s - base;
        const int unit = past <= INT32_MAX ? (int)past / cost : (int)(past / cost), g = unit / p.blocks_of_heads, hb = unit % p.blocks_of_heads;
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

        uint32_t qf[NT][KC][E8 ? 8 : 4];
        float cq[NT][2];                                  // of the queries that this lane has scores of
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < KC; ++i)
#pragma unroll
                for (int j = 0; j < (E8 ? 2 : 1); ++j) {
                    const int d = E8 ? 64 * i + 16 * col + 8 * j : 32 * i + 8 * col, h = 8 * t + row;
                    const uint4 x = load16((const T *)p.q.data + b * p.q.token_stride + (head0 + h) * p.q.head_stride + d,
                                           h < heads && d < kv.head_dim);
                    qf[t][i][4 * j] = x.x, qf[t][i][4 * j + 1] = x.y, qf[t][i][4 * j + 2] = x.z, qf[t][i][4 * j + 3] = x.w;
                }
            cq[t][0] = cq[t][1] = c;
            if constexpr (E8) {
                float back;
                query_halves<T, KC>(qf[t], back);
#pragma unroll
                for (int q = 0; q < 2; ++q) cq[t][q] = c * __shfl_sync(0xffffffffu, back, 4 * (2 * col + q));
            }
        }
        float o[NT][DP / 16][4] = {}, m[NT][2], l[NT][2] = {};
        float level = 1.f;                                // (pages of 8 bits) o is that many times what it stands for
#pragma unroll
        for (int t = 0; t < NT; ++t) m[t][0] = m[t][1] = -INFINITY;
        // (unsigned where a step past a length near 2^31 is counted)
        const int last = WIN ? len : (int)min((unsigned)len, (unsigned)to * STEP);  // keys of this run: from * STEP .. last
        // the first of the keys that this warp's f-th lot of a step has
        auto key_at = [&](int step, int f) {
            unsigned x = (unsigned)step * (STEP / 16) + (mate * FR + f);
            if (WIN && x >= (unsigned)head) x += gap;
            return 16 * x;
        };
        // of the rows up to `lim`, the keys from the window's first on, or the sinks
        const int near = min(p.window, len), far = p.sinks - len;
        auto seen = [&](int r, int lim) { return r < lim && (!WIN || r >= lim - near || r < lim + far); };
        uint4 kr[FR][2][KC];
        std::conditional_t<E8 && DP == 64, uint2, uint4> vr[FR][4][E8 ? 1 : VC];
        float ks[FR], vs[FR], vs_next[FR];                // (pages of 8 bits) their blocks' scales
        // (pages of 8 bits) which block of 16 tokens of the pools has a warp's keys: -1 where none is seen
        // or the page is none, and PARTLY added where not all of them are
        auto lot_of = [&](unsigned key, int page) -> int {
            const int lim = (int)min(16u, (unsigned)last - key);
            if (key >= (unsigned)last) return -1;
            if (WIN && !((int)key + lim > len - near || (int)key < p.sinks)) return -1;
            if (page < 0 || page >= kv.n_pages) {
                atomicOr(err, SERVE_INVALID);
                return -1;
            }
            const bool whole = lim == 16 && (!WIN || (int)key >= len - near || (int)key <= p.sinks - 16);
            return ((page * kv.kv_heads + g) << (p.shift - 4)) + ((int)key >> 4 & (kv.page_size / 16 - 1)) + (whole ? 0 : PARTLY);
        };
        // pages of this warp's coming keys, one to a lane: lane i has those of step held + i
        int held = 0, pages[FR];
        auto page_of = [&](int step, int f) -> int {
            if (step >= held + 32 || step < held || step == from) {
                held = step;
#pragma unroll
                for (int x = 0; x < FR; ++x) {
                    const unsigned key = key_at(step + lane, x);
                    pages[x] = key < (unsigned)last ? table[key >> p.shift] : 0;
                    if constexpr (E8) pages[x] = lot_of(key, pages[x]);
                }
            }
            return __shfl_sync(0xffffffffu, pages[f], step - held);
        };
        // where the rows of a step's keys are; none past the run's end or of a page that is none
        auto rows_at = [&](int step, int f, int &lim) -> long long {
            const int key = key_at(step, f), page = page_of(step, f);
            lim = (int)((unsigned)last - (unsigned)key);
            if (WIN) lim = lim > 0 && (lim - near < 16 || lim + far > 0) ? lim : 0;
            if (lim > 0 && (page < 0 || page >= kv.n_pages)) {
                atomicOr(err, SERVE_INVALID);
                lim = 0;
            }
            const long long at = ((long long)page * kv.kv_heads + g << p.shift) + (key & (kv.page_size - 1));
            return at * kv.head_dim;
        };
        long long kat[FR], vat[FR];
        int klim[FR], vlim[FR];
        // (pages of 8 bits) blocks of the keys, whether there is nothing to leave out of their rows, and whether there is nothing in them
        int lot[FR];
        bool kall = false, vall = false, knone = false, vnone = false;
        const uint8_t *k_lane = (const uint8_t *)kv.k_pages + (row * DP + 16 * col), *v_lane = (const uint8_t *)kv.v_pages + (2 * col * DP + DP / 8 * row);
        auto load_keys = [&](int step) {
            if constexpr (E8) {
                int any = -1, all = 0;
#pragma unroll
                for (int f = 0; f < FR; ++f) {
                    lot[f] = page_of(step, f);
                    any &= lot[f];
                    all |= lot[f];
                }
                kall = (!FULL || kv.head_dim == DP) && (unsigned)all < PARTLY;   // (left out, registers run out)
                knone = any == -1;
                if (kall) {
#pragma unroll
                    for (int f = 0; f < FR; ++f) {
                        if (FULL) {
                            const uint8_t *at = k_lane + (uint64_t)(unsigned)lot[f] * (16 * DP);
                            kr[f][0][0] = get16<0>(at);
                            kr[f][1][0] = get16<8 * DP>(at);
                            if constexpr (DP == 128) {
                                kr[f][0][KC - 1] = get16<64>(at);
                                kr[f][1][KC - 1] = get16<8 * DP + 64>(at);
                            }
                        } else {
                            // (in the place of elements that a row does not have its first ones: the queries have
                            // zeros there, and a code that is NaN makes the row's score NaN in its own place as well)
                            const uint8_t *at = (const uint8_t *)kv.k_pages + (uint64_t)(unsigned)lot[f] * (16 * kv.head_dim) + row * kv.head_dim;
#pragma unroll
                            for (int i = 0; i < KC; ++i) {
                                const int d = 64 * i + 16 * col < kv.head_dim ? 64 * i + 16 * col : 0;
                                kr[f][0][i] = get16<0>(at + d);
                                kr[f][1][i] = get16<0>(at + d + 8 * kv.head_dim);
                            }
                        }
                        ks[f] = p.k_scales[(unsigned)lot[f]];
                        vs_next[f] = p.v_scales[(unsigned)lot[f]];
                    }
                } else {
#pragma unroll
                    for (int f = 0; f < FR; ++f) {
                        const bool on = lot[f] >= 0;
                        klim[f] = on ? last - (int)key_at(step, f) : 0;
                        lot[f] = on ? lot[f] & (PARTLY - 1) : 0;
                        const uint8_t *at = (const uint8_t *)kv.k_pages + (uint64_t)(unsigned)lot[f] * (16 * kv.head_dim);
#pragma unroll
                        for (int r = 0; r < 2; ++r)
#pragma unroll
                            for (int i = 0; i < KC; ++i)
                                kr[f][r][i] = load16(at + (row + 8 * r) * kv.head_dim + 64 * i + 16 * col,
                                                     seen(row + 8 * r, klim[f]) && 64 * i + 16 * col < kv.head_dim);
                        ks[f] = on ? p.k_scales[(unsigned)lot[f]] : 0.f;
                        vs_next[f] = on ? p.v_scales[(unsigned)lot[f]] : 0.f;
                    }
                }
            } else {
                if constexpr (WIN) {
                    kall = true;
#pragma unroll
                    for (int f = 0; f < FR; ++f) {
                        kat[f] = rows_at(step, f, klim[f]);
                        kall = kall && klim[f] >= 16 && (klim[f] <= near || klim[f] + far >= 16);
                    }
                }
                if (WIN && kall && !FULL) {
#pragma unroll
                    for (int f = 0; f < FR; ++f)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
#pragma unroll
                            for (int i = 0; i < KC; ++i)
                                kr[f][r][i] = load16((const T *)kv.k_pages + kat[f] + (row + 8 * r) * kv.head_dim + 32 * i + 8 * col, 32 * i + 8 * col < kv.head_dim);
                    return;
                }
                if (WIN && kall) {
#pragma unroll
                    for (int f = 0; f < FR; ++f) {
                        const uint8_t *at = (const uint8_t *)((const T *)kv.k_pages + kat[f] + (row * DP + 8 * col));
                        kr[f][0][0] = get16<0>(at), kr[f][1][0] = get16<16 * DP>(at);
                        kr[f][0][1] = get16<64>(at), kr[f][1][1] = get16<16 * DP + 64>(at);
                        if constexpr (DP == 128) {
                            kr[f][0][KC - 2] = get16<128>(at), kr[f][1][KC - 2] = get16<16 * DP + 128>(at);
                            kr[f][0][KC - 1] = get16<192>(at), kr[f][1][KC - 1] = get16<16 * DP + 192>(at);
                        }
                    }
                    return;
                }
#pragma unroll
                for (int f = 0; f < FR; ++f) {
                    if (!WIN) kat[f] = rows_at(step, f, klim[f]);
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int i = 0; i < KC; ++i)
                            kr[f][r][i] = load16((const T *)kv.k_pages + kat[f] + (row + 8 * r) * kv.head_dim + 32 * i + 8 * col,
                                                     seen(row + 8 * r, klim[f]) && 32 * i + 8 * col < kv.head_dim);
                }
            }
        };
        auto load_values = [&]() {
            if constexpr (E8) {
                vall = kall, vnone = knone;
#pragma unroll
                for (int f = 0; f < FR; ++f) {
                    vlim[f] = klim[f], vs[f] = vs_next[f];
                    if (vall && FULL) {
                        const uint8_t *at = v_lane + (uint64_t)(unsigned)lot[f] * (16 * DP);
                        if constexpr (DP == 64) {
                            vr[f][0][0] = get8<0>(at), vr[f][1][0] = get8<DP>(at), vr[f][2][0] = get8<8 * DP>(at), vr[f][3][0] = get8<9 * DP>(at);
                        } else {
                            vr[f][0][0] = get16<0>(at), vr[f][1][0] = get16<DP>(at), vr[f][2][0] = get16<8 * DP>(at), vr[f][3][0] = get16<9 * DP>(at);
                        }
                        continue;
                    }
                    if (vall) {
                        // (results past the width are nobody's)
                        const int d = DP / 8 * row < kv.head_dim ? DP / 8 * row : 0;
                        const uint8_t *at = (const uint8_t *)kv.v_pages + (uint64_t)(unsigned)lot[f] * (16 * kv.head_dim) + 2 * col * kv.head_dim + d;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint8_t *x = at + ((r & 1) + 8 * (r >> 1)) * kv.head_dim;
                            if constexpr (DP == 64) vr[f][r][0] = get8<0>(x);
                            else vr[f][r][0] = get16<0>(x);
                        }
                        continue;
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = 2 * col + (r & 1) + 8 * (r >> 1), d = DP / 8 * row;
                        const bool on = seen(key, vlim[f]) && d < kv.head_dim;
                        const uint8_t *at = (const uint8_t *)kv.v_pages + (uint64_t)(unsigned)lot[f] * (16 * kv.head_dim) + key * kv.head_dim + d;
                        if constexpr (DP == 64) vr[f][r][0] = load8(at, on);
                        else vr[f][r][0] = load16(at, on);
                    }
                }
            } else {
                if (WIN) vall = kall;
#pragma unroll
                for (int f = 0; f < FR; ++f) {
                    vat[f] = kat[f], vlim[f] = klim[f];
                    if (WIN && vall && FULL) {
                        const uint8_t *at = (const uint8_t *)((const T *)kv.v_pages + kat[f] + (2 * col * DP + 8 * row));
                        vr[f][0][0] = get16<0>(at), vr[f][1][0] = get16<2 * DP>(at), vr[f][2][0] = get16<16 * DP>(at), vr[f][3][0] = get16<18 * DP>(at);
                        if constexpr (DP == 128) {
                            vr[f][0][VC - 1] = get16<128>(at), vr[f][1][VC - 1] = get16<2 * DP + 128>(at);
                            vr[f][2][VC - 1] = get16<16 * DP + 128>(at), vr[f][3][VC - 1] = get16<18 * DP + 128>(at);
                        }
                        continue;
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = 2 * col + (r & 1) + 8 * (r >> 1);
                        const bool on = (WIN && vall) || seen(key, vlim[f]);
#pragma unroll
                        for (int i = 0; i < VC; ++i) {
                            const int d = 64 * i + 8 * row;
                            vr[f][r][i] = load16((const T *)kv.v_pages + vat[f] + key * kv.head_dim + d, on && d < kv.head_dim);
                        }
                    }
                }
            }
        };
        for (;;) {
            load_keys(from);
            load_values();
            for (int step = from; step < to; ++step) {
                if (E8 && vnone) {                            // (of a warp: nothing of this step is its own)
                    if (step + 1 < to) load_keys(step + 1), load_values();
                    continue;
                }
                float x[FR][NT][4] = {};
#pragma unroll
                for (int f = 0; f < FR; ++f)
#pragma unroll
                    for (int i = 0; i < KC; ++i) {
                        const uint4 u = kr[f][0][i], w = kr[f][1][i];
                        if constexpr (E8) {
                            const uint32_t *u4 = &u.x, *w4 = &w.x;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t a0 = half_lo(u4[j]), a1 = half_lo(w4[j]), a2 = half_hi(u4[j]), a3 = half_hi(w4[j]);
#pragma unroll
                                for (int t = 0; t < NT; ++t) mma16<P>(x[f][t], a0, a1, a2, a3, qf[t][i][2 * j], qf[t][i][2 * j + 1]);
                            }
                        } else {
#pragma unroll
                            for (int t = 0; t < NT; ++t) {
                                mma16<T>(x[f][t], u.x, w.x, u.y, w.y, qf[t][i][0], qf[t][i][1]);
                                mma16<T>(x[f][t], u.z, w.z, u.w, w.w, qf[t][i][2], qf[t][i][3]);
                            }
                        }
                    }
                if constexpr (E8) {
#pragma unroll
                    for (int f = 0; f < FR; ++f)
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            float k0 = ks[f] * cq[t][0], k1 = ks[f] * cq[t][1];
                            // (past 32 bits, where products of zero stay zero)
                            if (level != 1.f) k0 = within(k0), k1 = within(k1);
                            x[f][t][0] *= k0, x[f][t][1] *= k1, x[f][t][2] *= k0, x[f][t][3] *= k1;
                        }
                    if (!vall) {
#pragma unroll
                        for (int f = 0; f < FR; ++f)
#pragma unroll
                            for (int t = 0; t < NT; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i) x[f][t][i] = seen(row + 8 * (i >> 1), vlim[f]) ? x[f][t][i] : -INFINITY;
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
                            if (!E8) x[f][t][i] = (WIN && vall) || seen(row + 8 * (i >> 1), vlim[f]) ? x[f][t][i] * c : -INFINITY;
                            top[t][i & 1] = fmaxf(top[t][i & 1], x[f][t][i]);
                        }
                    more = more || top[t][0] - m[t][0] > SLACK || top[t][1] - m[t][1] > SLACK;
                }
                if constexpr (E8)
#pragma unroll
                    for (int f = 0; f < FR; ++f) vs[f] *= level;
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
                        pb[t][0] = transpose8(Type2<P>::down(y[0], y[1]));
                        pb[t][1] = transpose8(Type2<P>::down(y[2], y[3]));
                    }
                    if constexpr (E8) {
                        // a block's products by themselves, times its scale: scales may lie too far apart for
                        // weights that carry them
                        const uint32_t *v0 = &vr[f][0][0].x, *v1 = &vr[f][1][0].x, *v2 = &vr[f][2][0].x, *v3 = &vr[f][3][0].x;
#pragma unroll
                        for (int j = 0; j < DP / 32; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint32_t u = __byte_perm(v0[j], v1[j], e ? 0x7362 : 0x5140), w = __byte_perm(v2[j], v3[j], e ? 0x7362 : 0x5140);
                                const uint32_t a0 = half_lo(u), a1 = half_hi(u), a2 = half_lo(w), a3 = half_hi(w);
#pragma unroll
                                for (int t = 0; t < NT; ++t) {
                                    float z[4];
                                    mma16_new(z, a0, a1, a2, a3, pb[t][0], pb[t][1]);
                                    float (&y)[4] = o[t][2 * j + e];
                                    fma_pair(y[0], y[1], z[0], z[1], vs[f]);
                                    fma_pair(y[2], y[3], z[2], z[3], vs[f]);
                                }
                            }
                    } else
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
            if constexpr (!E8) break;
            float most = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) most = max_nan(most, fabsf(o[t][i][q]));
            if (__all_sync(0xffffffffu, level != 1.f || most < LARGE)) break;
            level = LOWERED;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int i = 0; i < DP / 16; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) o[t][i][q] = 0.f;
                m[t][0] = m[t][1] = -INFINITY;
                l[t][0] = l[t][1] = 0.f;
            }
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
                // (a sum is at least 0; its sign says whether the results are lowered)
                if (row == 0) sm[warp][h] = m[t][q], sl[warp][h] = E8 && level != 1.f ? -y : y;
#pragma unroll
                for (int i = 0; i < VC; ++i) {
                    float *at = &so[warp][h][E8 ? DP / 8 * row + 8 * i : 64 * i + 8 * row];
                    *reinterpret_cast<float4 *>(at) = make_float4(o[t][4 * i][q], o[t][4 * i][q + 2], o[t][4 * i + 1][q], o[t][4 * i + 1][q + 2]);
                    *reinterpret_cast<float4 *>(at + 4) = make_float4(o[t][4 * i + 2][q], o[t][4 * i + 2][q + 2], o[t][4 * i + 3][q], o[t][4 * i + 3][q + 2]);
                }
            }
        together();
        const bool whole = from == 0 && to == steps;
        constexpr int PART = NQ * (DP + 2);
        auto is_low = [](float sum) { return E8 && __float_as_int(sum) < 0; };
        auto finish = [&](int h, int d, float top, float sum, float (&y)[8], bool lowered) {
            const float share = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = lowered ? y[e] * share * (1.f / LOWERED) : y[e] * share;
            uint4 r;
            r.x = sum == 0.f ? 0u : Type2<T>::down(y[0], y[1]);
            r.y = sum == 0.f ? 0u : Type2<T>::down(y[2], y[3]);
            r.z = sum == 0.f ? 0u : Type2<T>::down(y[4], y[5]);
            r.w = sum == 0.f ? 0u : Type2<T>::down(y[6], y[7]);
            *reinterpret_cast<uint4 *>((T *)p.out.data + b * p.out.token_stride + (head0 + h) * p.out.head_stride + d) = r;
            if (p.lse && d == 0)
                p.lse[(long long)b * p.q_heads + head0 + h] =
                    sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) - OFFSET + log2f(sum)) * LN2;
        };
        auto put_part = [&](float *part, int h, int d, float top, float sum, float (&y)[8], bool any_low) {
            __stcg(reinterpret_cast<float4 *>(part + h * DP + d), make_float4(y[0], y[1], y[2], y[3]));
            __stcg(reinterpret_cast<float4 *>(part + h * DP + d + 4), make_float4(y[4], y[5], y[6], y[7]));
            if (d == 0) __stcg(reinterpret_cast<float2 *>(part + NQ * DP) + h, make_float2(top, any_low ? -sum : sum));
        };
        for (int i = me; i < NQ * (DP / 8); i += 32 * TW) {
            const int h = i / (DP / 8), d = i % (DP / 8) * 8;
            if (h >= heads || d >= kv.head_dim) continue;
            float top = -INFINITY, sum = 0.f, y[8] = {};
            bool any_low = false;
#pragma unroll
            for (int w = own; w < own + TW; ++w) top = fmaxf(top, sm[w][h]), any_low = any_low || is_low(sl[w][h]);
#pragma unroll
            for (int w = own; w < own + TW; ++w) {
                const float keep = sm[w][h] == top ? 1.f : exp2_fast(sm[w][h] - top);
                sum = __fmaf_rn(fabsf(sl[w][h]), keep, sum);
                const float share = any_low && !is_low(sl[w][h]) ? keep * LOWERED : keep;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __fmaf_rn(so[w][h][d + e], share, y[e]);
            }
            if (whole) finish(h, d, top, sum, y, any_low);
            else put_part(p.parts + ((long long)team * 2 + (from == 0)) * PART, h, d, top, sum, y, any_low);
        }
        if (!whole) {
            // a pair's parts: the block it begins in keeps its own in place 1, later ones in place 0
            const int block1 = (int)(((unit_at + 1) * W - 1) / total), block2 = (int)(((unit_at + steps) * W - 1) / total);
            auto place = [&](int k) { return 2ll * k + (k == block1); };
            // whether this is the last of `count` that come here, which has what the others brought
            auto last_of = [&](uint32_t *ticket, int count) {
                __threadfence();
                together();
                int last = 0;
                if (me == 0) last = atomicAdd(ticket, 1u) == (unsigned)(count - 1);
                if (TW == 1) {
                    last = __shfl_sync(0xffffffffu, last, 0);
                } else {
                    if (me == 0) last_one = last;
                    together();
                    last = last_one;
                }
                if (last) {
                    __threadfence();
                    if (me == 0) *ticket = 0;
                }
                return last != 0;
            };
            // parts k0, k0 + by .. k1, in order: their sums, to put
            auto join = [&](int k0, int k1, int by, auto &&put) {
                for (int i = me; i < NQ * (DP / 8); i += 32 * TW) {
                    const int h = i / (DP / 8), d = i % (DP / 8) * 8;
                    const bool on = h < heads && d < kv.head_dim;
                    float top = -INFINITY, sum = 0.f, y[8] = {};
                    bool any_low = false;
                    if (on)
#pragma unroll 4
                        for (int k = k0; k <= k1; k += by) {
                            const float *at = p.parts + place(k) * PART;
                            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(at + NQ * DP) + h);
                            const float4 u = __ldcg(reinterpret_cast<const float4 *>(at + h * DP + d));
                            const float4 w = __ldcg(reinterpret_cast<const float4 *>(at + h * DP + d + 4));
                            const float t = fmaxf(top, ml.x);
                            float a = top == t ? 1.f : exp2_fast(top - t), z = ml.x == t ? 1.f : exp2_fast(ml.x - t);
                            top = t;
                            sum = __fmaf_rn(fabsf(ml.y), z, sum * a);
                            // (parts that are not lowered, where others are)
                            if (E8 && is_low(ml.y) != any_low) (any_low ? z : a) *= LOWERED, any_low = true;
                            y[0] = __fmaf_rn(u.x, z, y[0] * a), y[1] = __fmaf_rn(u.y, z, y[1] * a);
                            y[2] = __fmaf_rn(u.z, z, y[2] * a), y[3] = __fmaf_rn(u.w, z, y[3] * a);
                            y[4] = __fmaf_rn(w.x, z, y[4] * a), y[5] = __fmaf_rn(w.y, z, y[5] * a);
                            y[6] = __fmaf_rn(w.z, z, y[6] * a), y[7] = __fmaf_rn(w.w, z, y[7] * a);
                        }
                    __syncwarp();                         // (put may write where the warp has read)
                    if (on) put(h, d, top, sum, y, any_low);
                }
            };
            // A warp by itself joins a long pair in two stages, groups first: their last warps do it side by side.
            const int count = block2 - block1 + 1;
            int group = count, groups = 1, k0 = block1;
            if (TW == 1 && count > GROUP) {
                for (group = GROUP; group * group < count;) group *= 2;
                groups = (count + group - 1) / group;
                k0 = block1 + (team - block1) / group * group;
            }
            if (groups == 1) {
                if (last_of(&p.tickets[block1], count)) join(block1, block2, 1, finish);
            } else if (last_of(&p.tickets[TICKETS + place(k0)], min(group, block2 - k0 + 1))) {
                join(k0, min(block2, k0 + group - 1), 1, [&](int h, int d, float top, float sum, float (&y)[8], bool any_low) {
                    put_part(p.parts + place(k0) * PART, h, d, top, sum, y, any_low);
                });
                if (last_of(&p.tickets[block1], groups)) join(block1, block2, group, finish);
            }
        }
        together();
    }
}

template <typename T, int DP, int NT, int FR, bool E8, bool WIN, int TW, bool FULL>
static opattr_status run_teams(Ctx &c, Serve &s, TokenArgs &p) {
    const int64_t most = (int64_t)p.n * p.kv.kv_heads * p.blocks_of_heads *
                         (((int64_t)p.kv.pages_per_seq * p.kv.page_size + 16 * FR * TW - 1) / (16 * FR * TW));
    constexpr int TEAMS = TOKEN_WARPS / TW;
    const int grid = (int)std::min<int64_t>((E8 ? Eight<DP, NT>::BLOCKS : NT == 1 ? 3 : 2) * (int64_t)sm_count(c), std::min<int64_t>((most + TEAMS - 1) / TEAMS, TICKETS / TEAMS));
    opattr_status st = serve_ready(c, s);
    if (st) return st;
    const int64_t part = (int64_t)8 * NT * (DP + 2);
    if ((st = ensure_lasting_arena(c, Need().add<float>(2 * (int64_t)grid * TEAMS * part).bytes))) return st;
    Arena a(c);
    p.parts = a.take<float>(2 * (int64_t)grid * TEAMS * part);
    p.tickets = s.tickets;
    launch(c, E8 ? "token8" : "token", k_token<T, DP, NT, FR, E8, WIN, TW, FULL>, dim3(grid), dim3(TOKEN_THREADS), 0, p, s.err);
    return cuda_status(c, c.last_error);
}
template <typename T, int DP, int NT, int FR, bool E8, bool WIN, bool FULL>
static opattr_status run_token(Ctx &c, Serve &s, TokenArgs &p) {
    if constexpr (E8 || WIN) {
        if ((int64_t)p.n * p.kv.kv_heads * p.blocks_of_heads >= own_pairs(DP) * (int64_t)sm_count(c)) return run_teams<T, DP, NT, FR, E8, WIN, 1, FULL>(c, s, p);
    }
    return run_teams<T, DP, NT, FR, E8, WIN, TOKEN_WARPS, FULL>(c, s, p);
}
template <typename T, bool E8, bool WIN, bool FULL>
static opattr_status token_of(Ctx &c, Serve &s, TokenArgs &p) {
    constexpr int F64 = 2, F128 = E8 ? 2 : 1;
    if (p.kv.head_dim <= 64) return p.group <= 8 ? run_token<T, 64, 1, F64, E8, WIN, FULL>(c, s, p) : run_token<T, 64, 2, F64, E8, WIN, FULL>(c, s, p);
    return p.group <= 8 ? run_token<T, 128, 1, F128, E8, WIN, FULL>(c, s, p) : run_token<T, 128, 2, F128, E8, WIN, FULL>(c, s, p);
}
template <bool E8, bool WIN, bool FULL>
static opattr_status token_of(Ctx &c, Serve &s, TokenArgs &p, int dtype) {
    return dtype == OPATTR_BF16 ? token_of<__nv_bfloat16, E8, WIN, FULL>(c, s, p) : token_of<__half, E8, WIN, FULL>(c, s, p);
}

// By the type of the queries; each in a file of its own, which compiles beside the others.
opattr_status token_plain(Ctx &c, Serve &s, TokenArgs &p, int dtype);
opattr_status token_window(Ctx &c, Serve &s, TokenArgs &p, int dtype);
opattr_status token8_plain(Ctx &c, Serve &s, TokenArgs &p, int dtype);
opattr_status token8_window(Ctx &c, Serve &s, TokenArgs &p, int dtype);
// and of widths other than 64 and 128
opattr_status token8_plain_odd(Ctx &c, Serve &s, TokenArgs &p, int dtype);
opattr_status token8_window_odd(Ctx &c, Serve &s, TokenArgs &p, int dtype);

}  // namespace opattr
