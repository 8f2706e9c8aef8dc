// prompt.cu -- attention over whole prompts: packed sequences of any lengths,
// grouped heads, causal or not (opattr_attention).
//
//   s_ij = scale * q_i . k_j,  j seen by i: j < Lk and, causal, j <= i + Lk - Lq
//   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i),  lse_i = m_i + log of that sum
// A row that sees no key gets o = 0 and lse = -inf.
//
// One pass over the keys with a running maximum and sum.  A block holds two sub-tiles
// of 128 rows (queries; heads that share keys side by side) and takes their keys 128
// at a time:
//   S [128 x 128] = Q K^T       both from shared memory, into tensor memory
//   P = 2^(S c - m)             a thread per row, back into tensor memory in 16 bits
//   O [128 x D]  += P V         P from tensor memory, V as it lies (its rows are keys)
// with a row's m raised, and O and the sum rescaled, only when a new maximum is more
// than a few powers of two above it.  Tensor memory is full: two S and two O of 128
// columns each, P in the place of S.  While one sub-tile's softmax runs, the tensor
// cores have the other's products to do.  Warps: 0 .. 3 and 4 .. 7 the two softmax
// groups, 8 issues the products, 9 the tile copies into a ring of five (width 128) or
// eight tiles, 10 looks over value tiles that a mask cuts, 11 looks up work items.
// P is rounded to the inputs' type, which is what the products take: an error of the
// size of the result's own rounding.
//
// Measured on one GB300 (bfloat16, causal unless said): 12,301 tokens, 32 heads of 128 on 8:
// 821 us among other calls, 1,510 TFLOP/s (790 in short bursts, 815 held for seconds); 9,728, 16
// heads on 4, all keys seen: 504 us, 1,540.  The power limit is active there, at 1.86 GHz; of
// the 3,040 cycles that a tile of both sub-tiles takes the products have 2,048.  16 heads of 64:
// 383 us, 1,010: a tile's 2,320 cycles have 1,024 of products and 1,024 of the special function
// unit, and the chain from scores through tensor memory to weights sets the pace.  Short prompts
// wait for it: 8 x 512 tokens, 8 heads of 64, all seen, 17,000 cycles, 4,300 of them before
// the first product, 11,700 for four tiles one after another.
#include <math.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "tc.cuh"

namespace opattr {

bool rows_ok(const opattr_rows &r, int64_t tokens, int heads, int dim) {
    if (tokens == 0) return true;
    if (!r.data || (reinterpret_cast<uintptr_t>(r.data) & 15)) return false;
    if (tokens > 1 && (r.token_stride < 8 || r.token_stride % 8)) return false;
    if (heads > 1 && (r.head_stride < 0 || r.head_stride % 8)) return false;
    return dim % 8 == 0;
}

constexpr int KEYS = 128;                // keys of a tile
constexpr int ROWS = 128;                // rows of a sub-tile: one thread and one lane of tensor memory each
constexpr int THREADS = 384;             // two warpgroups for the softmax of two sub-tiles, one for the rest
constexpr int MMA_WARP = 8, LOAD_WARP = 9, TAIL_WARP = 10;   // and the last one looks up items
// registers: 384 x 168 at launch = 256 x 208 + 128 x 88
constexpr int REGS_SOFTMAX = 208, REGS_OTHERS = 88;
constexpr int CUTS = 4;                  // value tiles cut by a mask that can be under way: half the ring's stages
constexpr int SHORT = 4;                 // key tiles that take as long as the lookup of an item
// What a wait may take before its block gives up (opattr_check then returns OPATTR_E_TIMEOUT): the
// look-up waits for all tiles of an item, so long ones have several times what a tile takes (1 to 2 us)
// on top.  And where a test has a part of the kernel fall silent.
constexpr unsigned WAIT_US = 4000000, TILE_WAIT_US = 10, SILENT_WAIT_US = 20000;
constexpr int ITEMS = 2;                 // slots of work items: the one being computed, and the one whose tiles are fetched

// Shapes by the padded head width DP (64 or 128; the copies fill what a head
// lacks with zeros).  The products take DV of its columns (64; 96 or 128).
template <int DP>
struct Shape {
    static constexpr int HALF = 128 * 128;                 // bytes of 128 rows of 64 elements
    static constexpr int TILE = DP / 64 * HALF;
    static constexpr int STAGES = DP == 128 ? 5 : 8;       // key and value tiles in flight
    static constexpr int SMEM = 2 * TILE + STAGES * TILE + 1024 /* alignment */;
    static_assert(STAGES <= 2 * CUTS, "a cut tile's slot is taken again only once its stage was free");
};

struct PromptArgs {
    opattr_prompt a;
    // a sub-tile's rows are `pack` heads of one key head of `span` tokens, head by head; an item
    // has two of them, one behind the other, and heads_x items stand side by side
    int pack, span, heads_x;
    int tiles;                           // places of query tiles
    int q_mul, k_mul, v_mul;             // 0 where all heads read the same rows
    int wide;                            // 1: rows of the output are 32-byte aligned and DP wide
    unsigned *next;                      // items given out past each block's first; zero between launches
    // where blocks have equal runs of keys, else NULL
    const struct Item *plan;             // a block's items after those of the block before
    const int *start;                    // [grid + 1] where they begin
    float *parts;                        // [block][2][sub-tile] partial results, four columns of every row side by side; then the rows' maxima and sums
    uint32_t *tickets;                   // [block][sub-tile] arrivals
    unsigned limit_us;                   // of every wait
    int silent;                          // Serve::silent
};

// A work item: two sub-tiles of queries of one sequence, and keys of it.
struct Item {
    int q0, lq, k0, lk;                  // the sequence's queries; the keys taken here
    int t0, head0;                       // first query within it, and (first) head
    int ahead;                           // query i sees the keys up to i + ahead
    int first, piece, pieces;            // the first block that has some of its keys, which part this is, and how many there are
    int some;                            // 0: there are no more
};

struct Ctrl {
    uint64_t item_full[ITEMS], item_free[ITEMS], item_want, q_full, q_free, kv_full[8], kv_free[8];
    uint64_t s_full[2], p_half[2], p_full[2], o_full[2], o_free[2], v_full[CUTS], v_ready[CUTS], met[2], drain;
    uint32_t tmem;
    int stop;
    int poison[CUTS];
    int last[2];
    Item item[ITEMS];
};

// A place in a ring of N, and the parity of its barrier.
template <int N>
struct Place {
    int at = 0, ph = 0;
    __device__ __forceinline__ void step() {
        if (++at == N) at = 0, ph ^= 1;
    }
};

// What an item's sub-tiles have to do.  (Queries and keys may come near 2^31 in number, and
// places a tile past the last of them pass it: those are sums without a sign.)
struct Work {
    int base[2], tiles[2], clean[2];     // first query; key tiles; the first of them that a mask cuts
    int n, cut;                          // key tiles of either; the first that is looked over
    __device__ __forceinline__ Work(const Item &it, int span, int causal) {
        const int ahead = it.ahead;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            base[s] = (int)((unsigned)it.t0 + s * span);
            const int rows = min(span, (int)((unsigned)it.lq - base[s]));
            const int keys = rows <= 0 ? 0 : causal ? max(0, min(it.lk, base[s] + rows + ahead)) : it.lk;
            tiles[s] = ((unsigned)keys + KEYS - 1) / KEYS;
            clean[s] = (causal ? max(0, min(it.lk, (int)((unsigned)base[s] + 1 + ahead))) : it.lk) / KEYS;
        }
        n = max(tiles[0], tiles[1]);
        cut = tiles[1] > 0 ? min(clean[0], clean[1]) : clean[0];
    }
};

// Byte of column `col` in row r of a swizzled tile.
__device__ __forceinline__ uint32_t tile_at(int half_bytes, int r, int col) {
    return (uint32_t)((col >> 6) * half_bytes + r * 128 + (((col & 63) * 2) ^ ((r & 7) << 4)));
}

__device__ __forceinline__ uint32_t tm_ld1(uint32_t at) {
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(at));
    return r;
}

// 32 bytes of a thread in one store: whole sectors, where rows lie far apart.
__device__ __forceinline__ void store32(void *p, const uint32_t *r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

// The next item for a whole warp: numbers past the blocks' own, in order.  Every
// block draws until it is told that there are none, so `total` are drawn in all, and
// the last one puts the count back to zero.
__device__ __forceinline__ unsigned draw(unsigned *next, unsigned total) {
    unsigned k = 0;
    if (lane_id() == 0) {
        k = atomicAdd(next, 1u);
        if (k == total - 1) atomicExch(next, 0u);
    }
    return gridDim.x + __shfl_sync(0xffffffffu, k, 0);
}

// CUT: the items come from a plan, and may be parts of the keys that are joined.
template <typename T, int DP, int DV, bool CUT>
__global__ void __launch_bounds__(THREADS, 1)
k_prompt(const __grid_constant__ PromptArgs p, const __grid_constant__ CUtensorMap mq,
         const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, unsigned *err) {
    using S = Shape<DP>;
    constexpr bool BF = std::is_same<T, __nv_bfloat16>::value;
    // Weights stand at up to 2^(OFFSET + SLACK): the accumulator is rescaled only
    // when a row's maximum has grown by more than SLACK powers of two since the
    // last time.  Half's range ends at 2^16 above and loses bits below 2^-14,
    // so there the weights of a row's maximum start at 2^8.
    constexpr float OFFSET = BF ? 0.f : 8.f, SLACK = BF ? 8.f : 7.f;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Ctrl ctl;
    unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t sq = smem_addr(smem), skv = sq + 2 * S::TILE;
    const int warp = threadIdx.x >> 5;
    volatile int *stop = &ctl.stop;
    const opattr_prompt &a = p.a;
    const uint32_t bar_kv = smem_addr(&ctl.kv_full[0]), bar_free = smem_addr(&ctl.kv_free[0]);
    if (threadIdx.x == 0) {
        for (int i = 0; i < ITEMS; ++i) bar_init(smem_addr(&ctl.item_full[i]), 1), bar_init(smem_addr(&ctl.item_free[i]), 11);
        bar_init(smem_addr(&ctl.item_want), 1);
        bar_init(smem_addr(&ctl.q_full), 1), bar_init(smem_addr(&ctl.q_free), 1);
        for (int i = 0; i < S::STAGES; ++i) bar_init(bar_kv + 8 * i, 1), bar_init(bar_free + 8 * i, 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_addr(&ctl.s_full[i]), 1);
            bar_init(smem_addr(&ctl.p_half[i]), 4);
            bar_init(smem_addr(&ctl.p_full[i]), 4);
            bar_init(smem_addr(&ctl.o_full[i]), 1);
            bar_init(smem_addr(&ctl.o_free[i]), 4);
            bar_init(smem_addr(&ctl.met[i]), 4);
        }
        for (int i = 0; i < CUTS; ++i) bar_init(smem_addr(&ctl.v_full[i]), 1), bar_init(smem_addr(&ctl.v_ready[i]), 1);
        bar_init(smem_addr(&ctl.drain), 1);
        ctl.stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        map_prefetch(&mq), map_prefetch(&mk), map_prefetch(&mv);
    }
    if (warp == MMA_WARP) tm_alloc(smem_addr(&ctl.tmem), 512);
    tm_before();
    __syncthreads();
    tm_after();
    constexpr uint32_t tm = 0;                           // all of the tensor memory: its first column is column 0
    pdl_wait();

    // the next item, for a whole warp; its slot is given back by item_done
    Place<ITEMS> slot;
    auto item_next = [&](Item &it) {
        if (!warp_wait(smem_addr(&ctl.item_full[slot.at]), slot.ph, stop, p.limit_us)) return false;
        it = ctl.item[slot.at];
        __syncwarp();
        if (lane_id() == 0) bar_arrive(smem_addr(&ctl.item_free[slot.at]));
        slot.step();
        return it.some != 0;
    };

    if (warp < 8) {
        // ---- softmax: a warpgroup per sub-tile, a thread per query
        regs_more<REGS_SOFTMAX>();
        const int s = warp >> 2, r = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tm + s * 128 + lanes, to = tm + 256 + s * DP + lanes;
        const uint32_t b_s = smem_addr(&ctl.s_full[s]), b_half = smem_addr(&ctl.p_half[s]), b_p = smem_addr(&ctl.p_full[s]);
        // (a negative scale's sign is the products'; for none, the least that keeps -inf what it is)
        const float c = a.scale == 0.f ? __uint_as_float(1) : fabsf(a.scale) * LOG2E;
        const uint64_t c2 = pair(c, c);
        const int row_token = r / p.pack, row_head = r % p.pack;
        Place<1> turn_s, turn_o, turn_met;
        // the four warps of the sub-tile wait for one another
        auto meet = [&] {
            __syncwarp();
            if (lane_id() == 0) bar_arrive(smem_addr(&ctl.met[s]));
            const bool all = warp_wait(smem_addr(&ctl.met[s]), turn_met.ph, stop, p.limit_us);
            turn_met.step();
            return all;
        };
        Place<CUTS> over;                                // cut value tiles, of either sub-tile
        Place<S::STAGES> ring;                           // value tiles
        ring.step();
        Item it;
        bool ok = true;
        while (ok && item_next(it)) {
            const Work w(it, p.span, a.causal);
            const int n_tiles = s ? w.tiles[1] : w.tiles[0], clean = s ? w.clean[1] : w.clean[0];
            const int head = it.head0 + row_head, row = (int)((unsigned)(s ? w.base[1] : w.base[0]) + row_token);
            const int seen = a.causal ? min(it.lk, (int)((unsigned)row + 1 + it.ahead)) : it.lk;
            // (rows past the queries, or past the sub-tile's last whole token, are nobody's: what
            // is in them has no say in when the others are rescaled)
            const bool live = (unsigned)row < (unsigned)it.lq && row_token < p.span;
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < w.n; ++j) {
                if (j < n_tiles) {
                    if (!(ok = warp_wait(b_s, turn_s.ph, stop, p.limit_us))) break;
                    turn_s.step();
                    tm_after();
                    uint32_t x[KEYS];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tm_ld32(ts + 32 * q, x + 32 * q);
                    tm_wait_ld();
                    if (j >= clean) {
                        // of the 32s of keys that a mask cuts, most are seen by all of the warp's rows
                        const int left = (int)((unsigned)seen - j * KEYS);
#pragma unroll
                        for (int q = 0; q < KEYS; q += 32) {
                            if (__all_sync(0xffffffffu, left >= q + 32)) continue;
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[q + i] = i < left - q ? x[q + i] : 0xff800000u;
                        }
                    }
                    float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < KEYS; i += 8)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            t[q] = max3(t[q], __uint_as_float(x[i + 2 * q]), __uint_as_float(x[i + 2 * q + 1]));
                    const float top = fmaxf(max3(m, t[0], t[1]), fmaxf(t[2], t[3]));
                    if (__any_sync(0xffffffffu, live && (top - m) * c > SLACK)) {
                        const float keep = top == m ? 1.f : exp2_fast((m - top) * c);
                        m = top;
                        l *= keep;
                        if (j > 0) {
                            // (the scores are there, so the products before them are done)
                            const uint64_t keep2 = pair(keep, keep);
#pragma unroll 1
                            for (int d = 0; d < DP; d += 32) {
                                uint32_t o[32];
                                tm_ld32(to + d, o);
                                tm_wait_ld();
#pragma unroll
                                for (int i = 0; i < 32; i += 2) {
                                    const float2 y = unpair(mul2(pair(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), keep2));
                                    o[i] = __float_as_uint(y.x), o[i + 1] = __float_as_uint(y.y);
                                }
                                tm_st32(to + d, o);
                            }
                        }
                    }
                    const float from = m == -INFINITY ? OFFSET : __fmaf_rn(-m, c, OFFSET);
                    const uint64_t from2 = pair(from, from);
                    uint64_t sum[2] = {0, 0};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t y[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int e = 32 * q + 2 * i;
                            const float2 z = unpair(fma2(pair(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, from2));
                            const float lo = exp2_fast(z.x), hi = exp2_fast(z.y);
                            sum[i & 1] = add2(sum[i & 1], pair(lo, hi));
                            y[i] = Type2<T>::down(lo, hi);
                        }
                        tm_st16(ts + 16 * q, y);
                        if (q == 1) {
                            // the products with the first half of the keys may begin
                            tm_wait_st();
                            tm_before();
                            __syncwarp();
                            if (lane_id() == 0) bar_arrive(b_half);
                        }
                    }
                    const float2 z = unpair(add2(sum[0], sum[1]));
                    l += z.x + z.y;
                    tm_wait_st();
                }
                if (j >= w.cut) {
                    if (a.causal && j < n_tiles) {
                        // a value that is not finite times a weight of zero would reach the rows
                        // that do not see it: such a tile's products are made here, key by key
                        if (!(ok = warp_wait(smem_addr(&ctl.v_ready[over.at]), over.ph, stop, p.limit_us))) break;
                        if (seldom(*(volatile int *)&ctl.poison[over.at])) {
                            const unsigned char *v = smem + 2 * S::TILE + ring.at * S::TILE;
                            const int left = (int)((unsigned)seen - j * KEYS);
#pragma unroll 1
                            for (int d = 0; d < DP; d += 32) {
                                uint32_t o[32] = {};
                                if (j > 0) {
                                    tm_ld32(to + d, o);
                                    tm_wait_ld();
                                }
#pragma unroll 1
                                for (int i = 0; i < KEYS; ++i) {
                                    const uint32_t u2 = tm_ld1(ts + i / 2);
                                    tm_wait_ld();
                                    const float2 w2 = Type2<T>::up(u2);
                                    const float weight = i & 1 ? w2.y : w2.x;
#pragma unroll
                                    for (int e = 0; e < 32; e += 8) {
                                        const uint4 u = *reinterpret_cast<const uint4 *>(v + tile_at(S::HALF, i, d + e));
                                        const uint32_t uu[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                                        for (int q = 0; q < 4; ++q) {
                                            const float2 y = Type2<T>::up(uu[q]);
                                            uint32_t *z = o + e + 2 * q;
                                            if (i < left) {
                                                z[0] = __float_as_uint(__fmaf_rn(weight, y.x, __uint_as_float(z[0])));
                                                z[1] = __float_as_uint(__fmaf_rn(weight, y.y, __uint_as_float(z[1])));
                                            }
                                        }
                                    }
                                }
                                tm_st32(to + d, o);
                            }
                            tm_wait_st();
                        }
                    }
                    over.step();
                }
                ring.step(), ring.step();
                if (j < n_tiles) {
                    tm_before();
                    __syncwarp();
                    if (lane_id() == 0) bar_arrive(b_p);
                }
            }
            if (!ok) break;
            if (n_tiles > 0) {
                if (!(ok = warp_wait(smem_addr(&ctl.o_full[s]), turn_o.ph, stop, p.limit_us))) break;
                turn_o.step();
                tm_after();
            }
            const bool wide = p.wide;
            float ref = m == -INFINITY ? m : m * c;      // the row's sum counts in 2^(ref - OFFSET)
            bool mine = true, joined = false;
            const float *parts = nullptr;
            auto o_read = [&] {                          // the next item's products may go there
                tm_before();
                __syncwarp();
                if (lane_id() == 0) bar_arrive(smem_addr(&ctl.o_free[s]));
            };
            constexpr int PART = ROWS * (DP + 2);
            // a block's part of the item that it ends with is its second, of the one it begins with its first
            auto part_at = [&](int k) { return parts + ((long long)k * 2 + (k == 0)) * 2 * PART; };
            if (CUT && seldom(it.pieces > 1)) {
                // a part of the keys: the result so far goes to memory, and whoever brings the
                // last part of the tile puts them together, in order
                parts = p.parts + (long long)it.first * 4 * PART + s * PART;
                float *part = const_cast<float *>(part_at(it.piece));
#pragma unroll 1
                for (int d = 0; d < DP; d += 32) {
                    uint32_t o[32] = {};
                    if (n_tiles > 0) {
                        tm_ld32(to + d, o);
                        tm_wait_ld();
                        if (d + 32 == DP) o_read();
                    }
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            __stcg(reinterpret_cast<uint4 *>(part + (d + e) * ROWS + 4 * r), make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]));
                    }
                }
                if (live) *reinterpret_cast<float2 *>(part + ROWS * DP + 2 * r) = make_float2(ref, l);
                __threadfence();
                if (seldom(p.silent == SILENT_PARTS && (warp & 3) == 1)) break;
                if (!meet()) break;
                if (r == 0) {
                    __threadfence();
                    uint32_t *t = p.tickets + it.first * 2 + s;      // (a block ends with one item at most)
                    const bool all = atomicAdd(t, 1u) == (unsigned)it.pieces - 1;
                    if (all) atomicExch(t, 0u);
                    ctl.last[s] = all;
                }
                if (!meet()) break;
                mine = joined = *(volatile int *)&ctl.last[s];
                if (joined) {
                    __threadfence();
                    ref = -INFINITY;
#pragma unroll 4
                    for (int k = 0; k < it.pieces; ++k)
                        if (live) ref = fmaxf(ref, __ldcg(part_at(k) + ROWS * DP + 2 * r));
                    l = 0.f;
#pragma unroll 4
                    for (int k = 0; k < it.pieces; ++k) {
                        const float2 y = live ? __ldcg(reinterpret_cast<const float2 *>(part_at(k) + ROWS * DP + 2 * r)) : make_float2(ref, 0.f);
                        l = __fmaf_rn(y.y, y.x == ref ? 1.f : exp2_fast(y.x - ref), l);
                    }
                }
            }
            const float share = l == 0.f ? 0.f : 1.f / l;
            T *out = (T *)a.out.data + (int64_t)(it.q0 + row) * a.out.token_stride + head * a.out.head_stride;
            // (where no parts are joined this is short: in one piece 12,301 tokens take 810 us, in a loop 826)
#pragma unroll (CUT ? 1 : DP / 32)
            for (int d = 0; d < DP && mine; d += 32) {
                uint32_t o[32] = {};
                if (joined && live) {
#pragma unroll 4
                    for (int k = 0; k < it.pieces; ++k) {
                        const float *part = part_at(k);
                        const float y = __ldcg(part + ROWS * DP + 2 * r), f = y == ref ? 1.f : exp2_fast(y - ref);
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 z = __ldcg(reinterpret_cast<const float4 *>(part + (d + e) * ROWS + 4 * r));
                            o[e] = __float_as_uint(__fmaf_rn(z.x, f, __uint_as_float(o[e])));
                            o[e + 1] = __float_as_uint(__fmaf_rn(z.y, f, __uint_as_float(o[e + 1])));
                            o[e + 2] = __float_as_uint(__fmaf_rn(z.z, f, __uint_as_float(o[e + 2])));
                            o[e + 3] = __float_as_uint(__fmaf_rn(z.w, f, __uint_as_float(o[e + 3])));
                        }
                    }
                }
                if (n_tiles > 0 && !joined) {
                    tm_ld32(to + d, o);
                    tm_wait_ld();
                    if (d + 32 == DP) o_read();
                }
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    o[e] = l == 0.f ? 0u : Type2<T>::down(__uint_as_float(o[2 * e]) * share, __uint_as_float(o[2 * e + 1]) * share);
                if (live) {
                    if (wide) {
                        store32(out + d, o);
                        store32(out + d + 16, o + 8);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (d + 8 * e < a.head_dim) *reinterpret_cast<uint4 *>(out + d + 8 * e) = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                    }
                }
            }
            if (live && mine && a.lse)
                a.lse[(int64_t)(it.q0 + row) * a.q_heads + head] =
                    l == 0.f ? -INFINITY : ((ref == -INFINITY ? 0.f : ref) - OFFSET + log2f(l)) * LN2;
        }
    } else {
        regs_fewer<REGS_OTHERS>();
        if (warp == MMA_WARP) {
            // ---- products: one thread issues them, but the whole warp walks along, so that
            // descriptors stay in uniform registers (from one lane's branch each operand
            // would be moved there anew: 75 cycles a product instead of the 64 that it takes)
            const uint32_t DS = mma_desc(BF, ROWS, KEYS, false) | (a.scale < 0.f ? MMA_NEGATE : 0u);
            constexpr uint32_t DO = mma_desc(BF, ROWS, DV, true);
            const bool lead = elect();
            // descriptors count in 16 bytes: a tile's is its first one's and an offset
            const uint64_t qdesc = tile_desc(sq, 16), kdesc = tile_desc(skv, 16), vdesc = tile_desc(skv, S::HALF);
            Place<S::STAGES> keys, values;
            Place<CUTS> over;
            Place<1> q_turn, s_turn[2], o_turn[2];
            auto scores = [&](int s, int st) {
                const uint64_t qd = qdesc + s * (S::TILE >> 4), kd = kdesc + st * (S::TILE >> 4);
                if (lead) {
#pragma unroll
                    for (int k = 0; k < DV / 16; ++k) {
                        const int off = (k / 4) * (S::HALF >> 4) + (k % 4) * 2;
                        mma_ss(tm + s * 128, qd + off, kd + off, DS, k > 0);
                    }
                    mma_commit(smem_addr(&ctl.s_full[s]));
                }
            };
            auto full = [&](const Place<S::STAGES> &x) { return warp_wait(bar_kv + x.at * 8, x.ph, stop, p.limit_us); };
            auto release = [&](int st) {
                if (lead) mma_commit(bar_free + st * 8);
            };
            bool ok = true;
            Item it;
            while (ok && item_next(it)) {
                const Work w(it, p.span, a.causal);
                const int nt = uniform(w.n), nt0 = uniform(w.tiles[0]), nt1 = uniform(w.tiles[1]), from = uniform(w.cut);
                if (nt == 0) continue;
                bool by_hand = false;
                // values of tile j and keys of tile j + 1
                auto next = [&](int j) {
                    values = keys;
                    values.step();
                    keys = values;
                    keys.step();
                    if (!full(values) || (j + 1 < nt && !full(keys))) return false;
                    by_hand = false;
                    if (j >= from) {
                        if (!warp_wait(smem_addr(&ctl.v_ready[over.at]), over.ph, stop, p.limit_us)) return false;
                        by_hand = a.causal && uniform(*(volatile int *)&ctl.poison[over.at]);
                        over.step();
                    }
                    return true;
                };
                if (!(ok = warp_wait(smem_addr(&ctl.q_full), q_turn.ph, stop, p.limit_us) && full(keys))) break;
                q_turn.step();
                tm_after();
                if (nt0 > 0) scores(0, keys.at);
                if (nt1 > 0) scores(1, keys.at);
                release(keys.at);
                if (nt == 1 && lead) mma_commit(smem_addr(&ctl.q_free));
                if (!(ok = next(0))) break;
                for (int j = 0; ok && j < nt; ++j) {
                    const int vst = values.at, kst = keys.at;
                    const uint64_t vd = vdesc + vst * (S::TILE >> 4);
                    const bool hand = by_hand;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int mine = s ? nt1 : nt0;
                        if (j < mine) {
                            if (!(ok = warp_wait(smem_addr(&ctl.p_half[s]), s_turn[s].ph, stop, p.limit_us))) break;
                            if (j == 0) {
                                // the results before these have been read (a new barrier's parity 1 is over)
                                if (!(ok = warp_wait(smem_addr(&ctl.o_free[s]), o_turn[s].ph ^ 1, stop, p.limit_us))) break;
                                o_turn[s].step();
                            }
                            tm_after();
                            if (!hand && lead) {
#pragma unroll
                                for (int k = 0; k < KEYS / 32; ++k)
                                    mma_ts(tm + 256 + s * DP, tm + s * 128 + 8 * k, vd + k * 128, DO, k > 0 || j > 0);
                            }
                            if (!(ok = warp_wait(smem_addr(&ctl.p_full[s]), s_turn[s].ph, stop, p.limit_us))) break;
                            s_turn[s].step();
                            tm_after();
                            if (!hand && lead) {
#pragma unroll
                                for (int k = KEYS / 32; k < KEYS / 16; ++k)
                                    mma_ts(tm + 256 + s * DP, tm + s * 128 + 8 * k, vd + k * 128, DO, true);
                            }
                            if (j + 1 < mine) scores(s, kst);
                            else if (lead) mma_commit(smem_addr(&ctl.o_full[s]));
                        }
                        // while the tensor cores have the first sub-tile's products to do
                        if (s == 0 && j + 1 < nt && !(ok = next(j + 1))) break;
                    }
                    if (!ok) break;
                    release(vst);
                    if (j + 1 < nt) release(kst);
                    if (j + 2 == nt && lead) mma_commit(smem_addr(&ctl.q_free));
                }
                // (after the last tile `keys` is the place of the next item's first)
            }
            // nothing of this thread's is under way when the block ends
            if (lead) mma_commit(smem_addr(&ctl.drain));
            int last = 0;
            bar_wait(smem_addr(&ctl.drain), 0, &last, p.limit_us);
        } else if (warp == LOAD_WARP) {
            // ---- tile copies: one thread
            const bool lead = elect();
            const uint32_t bq = smem_addr(&ctl.q_full);
            Place<S::STAGES> ring;
            Place<CUTS> over;
            Place<1> q_turn;
            uint32_t bars[S::STAGES];                    // barrier of the last copy into each stage, and its parity
            int pars[S::STAGES];
            for (int i = 0; i < S::STAGES; ++i) bars[i] = 0;
            bool ok = true;
            int q_out = 0, out = 0;
            Item it;
            while (ok && item_next(it)) {
                const Work w(it, p.span, a.causal);
                // A block draws its next item when no more than SHORT of this one's tiles are left to
                // fetch, which hides the lookup: drawn three ahead, the last items went to the blocks
                // that asked first (8,192 causal tokens, 8 heads of 128: 133 us, so 103).
                const int ask = max(0, 2 * (w.n - SHORT));
                if (lead && w.n == 0) bar_arrive(smem_addr(&ctl.item_want));
                const int g = it.head0 / (a.q_heads / a.kv_heads), subs = w.tiles[1] > 0 ? 2 : 1;
                // the queries as soon as those before them are done with; until then the first keys
                // and values go ahead, as far as the item before this one leaves stages free
                bool q_due = true;
                for (int load = 0; load < 2 * w.n; ++load) {
                    if (seldom(++out == p.silent)) {
                        ok = false;
                        break;
                    }
                    if (lead && load == ask) bar_arrive(smem_addr(&ctl.item_want));
                    if (q_due && (load == S::STAGES - 2 || load == 2 * w.n - 1 ||
                                  __all_sync(0xffffffffu, bar_is_done(smem_addr(&ctl.q_free), q_turn.ph ^ 1)))) {
                        if (!(ok = warp_wait(smem_addr(&ctl.q_free), q_turn.ph ^ 1, stop, p.limit_us))) break;
                        q_turn.step();
                        q_due = false;
                        if (lead) {
                            bar_expect(bq, subs * p.pack * p.span * DP * 2);
                            for (int s = 0; s < subs; ++s)
                                for (int d = 0; d < DP / 64; ++d)
                                    tile_load(sq + s * S::TILE + d * S::HALF, &mq, 64 * d, it.head0 * p.q_mul,
                                              it.q0 + (s ? w.base[1] : w.base[0]), bq);
                        }
                        q_out = 1;
                    }
                    if (!(ok = warp_wait(bar_free + 8 * ring.at, ring.ph ^ 1, stop, p.limit_us))) break;
                    // K0, V0, K1, V1, ..; values that are looked over have a barrier of their own: the
                    // stage's may have gone round several times before the tail's warp sees it
                    const bool keys = load % 2 == 0, cut = !keys && load / 2 >= w.cut;
                    const uint32_t bar = cut ? smem_addr(&ctl.v_full[over.at]) : bar_kv + 8 * ring.at;
                    if (lead) {
                        bar_expect(bar, S::TILE);
                        for (int d = 0; d < DP / 64; ++d)
                            tile_load(skv + ring.at * S::TILE + d * S::HALF, keys ? &mk : &mv, 64 * d, g * (keys ? p.k_mul : p.v_mul),
                                      it.k0 + load / 2 * KEYS, bar);
                        if (cut) bar_arrive(bar_kv + 8 * ring.at);
                    }
                    bars[ring.at] = bar;
                    pars[ring.at] = cut ? over.ph : ring.ph;
                    if (cut) over.step();
                    ring.step();
                }
            }
            // the block ends with no copy under way: where a wait gave up, nobody else waits for them
            int last = 0;
            for (int i = 0; i < S::STAGES; ++i)
                if (bars[i]) bar_wait(bars[i], pars[i], &last, p.limit_us);
            if (q_out) bar_wait(bq, q_turn.ph ^ 1, &last, p.limit_us);
        } else if (warp == TAIL_WARP) {
            // ---- value tiles that a mask cuts: rows past the sequence's keys become zeros, and,
            // causal, the others are looked over for values that are not finite
            constexpr unsigned INF = BF ? 0x7f80u : 0x7c00u;
            Place<CUTS> over;
            Place<S::STAGES> ring;
            ring.step();
            bool ok = true;
            Item it;
            while (ok && item_next(it)) {
                const Work w(it, p.span, a.causal);
                for (int j = 0; j < w.n; ++j, ring.step(), ring.step()) {
                    if (j < w.cut) continue;
                    if (!(ok = warp_wait(smem_addr(&ctl.v_full[over.at]), over.ph, stop, p.limit_us))) break;
                    uint4 *v = reinterpret_cast<uint4 *>(smem + 2 * S::TILE + ring.at * S::TILE);
                    const int keys = min(KEYS, it.lk - j * KEYS);
                    unsigned most = 0;
                    for (int d = 0; d < DP / 64; ++d) {
                        if (a.causal) {
#pragma unroll 8
                            for (int i = lane_id(); i < keys * 8; i += 32) {
                                const uint4 y = v[d * (S::HALF / 16) + i];
                                most = __vmaxu2(most, __vmaxu2(__vmaxu2(y.x & 0x7fff7fffu, y.y & 0x7fff7fffu),
                                                               __vmaxu2(y.z & 0x7fff7fffu, y.w & 0x7fff7fffu)));
                            }
                        }
                        for (int i = keys * 8 + lane_id(); i < S::HALF / 16; i += 32) v[d * (S::HALF / 16) + i] = make_uint4(0, 0, 0, 0);
                    }
                    const bool found = __any_sync(0xffffffffu, (most >> 16) >= INF || (most & 0xffffu) >= INF);
                    fence_smem_async();
                    __syncwarp();
                    if (lane_id() == 0) {
                        ctl.poison[over.at] = found;
                        bar_arrive(smem_addr(&ctl.v_ready[over.at]));
                    }
                    over.step();
                }
            }
        } else {
            // ---- work items, the longest of a causal sequence first: query tiles count from the
            // last one.  Up to 32 sequences' tiles are numbered as they are, from what each lane
            // keeps of one of them.  Of more, sequence b has the places from q_offsets[b] / per + b
            // on, enough for its tiles whatever comes before it; those it does not need are passed
            // over.  A block's first item is its number, others are drawn.
            const int per = 2 * p.span;                  // tokens of an item
            const bool few = !CUT && a.n_seqs <= 32;
            // after a wait that gave up nothing more is begun
            const unsigned gave_up = *(volatile unsigned *)err & SERVE_TIMEOUT;
            int vq0 = 0, vq1 = 0, vk0 = 0, vk1 = 0;
            auto fetch = [&](int b) {
                vq0 = a.q_offsets[b], vq1 = a.q_offsets[b + 1], vk0 = a.k_offsets[b], vk1 = a.k_offsets[b + 1];
            };
            auto good = [&] {
                return vq0 >= 0 && vq1 >= vq0 && vq1 <= a.q_tokens && vk0 >= 0 && vk1 >= vk0 && vk1 <= a.k_tokens;
            };
            int mine = 0, upto = 0, tiles = p.tiles;
            if (few) {
                fetch(min((int)lane_id(), a.n_seqs - 1));
                mine = (int)lane_id() < a.n_seqs && good() ? ((unsigned)(vq1 - vq0) + per - 1) / per : 0;
                upto = warp_inclusive_scan(mine);
                tiles = min(tiles, __shfl_sync(0xffffffffu, upto, 31));
            }
            const unsigned heads_x = p.heads_x, total = CUT ? (unsigned)p.start[blockIdx.x + 1] : heads_x * (unsigned)tiles;
            const bool none = uniform(gave_up) != 0;
            Place<1> wanted;
            unsigned i = CUT ? (unsigned)p.start[blockIdx.x] : blockIdx.x;
            for (bool more = true; more;) {
                Item it{};
                while (i < total && !none) {
                    if (CUT) {
                        it = p.plan[i];
                        break;
                    }
                    const unsigned back = i / heads_x;
                    const int head0 = (int)(i - back * heads_x) * p.pack;
                    const int x = tiles - 1 - (int)back;
                    int k, t0;
                    if (few) {
                        k = max(0, __ffs(__ballot_sync(0xffffffffu, upto > x)) - 1);
                        t0 = (int)((unsigned)(x - __shfl_sync(0xffffffffu, upto - mine, k)) * per);
                    } else {
                        // the last sequence whose places begin at x or before it, 32 at a time
                        int lo = 0, n = a.n_seqs;
                        while (n > 32) {
                            const int step = (n + 31) / 32, b = lo + step * (int)lane_id();
                            const bool le = step * (int)lane_id() < n && a.q_offsets[b] / per + b <= x;
                            const int at = max(0, 31 - __clz(__ballot_sync(0xffffffffu, le)));
                            lo += at * step;
                            n = min(step, n - at * step);
                        }
                        const int b = lo + min((int)lane_id(), n - 1);
                        fetch(b);
                        k = max(0, 31 - __clz(__ballot_sync(0xffffffffu, (int)lane_id() < n && vq0 / per + b <= x)));
                        t0 = (int)((unsigned)(x - __shfl_sync(0xffffffffu, vq0, k) / per - (lo + k)) * per);
                    }
                    const int q0 = __shfl_sync(0xffffffffu, vq0, k), lq = __shfl_sync(0xffffffffu, vq1, k) - q0;
                    const int k0 = __shfl_sync(0xffffffffu, vk0, k), lk = __shfl_sync(0xffffffffu, vk1, k) - k0;
                    if (__shfl_sync(0xffffffffu, (int)good(), k) && t0 >= 0 && t0 < lq) {
                        it = Item{q0, lq, k0, lk, t0, head0, lk - lq, 0, 0, 1, 1};
                        break;
                    }
                    i = draw(p.next, total);
                }
                more = it.some != 0;
                if (!warp_wait(smem_addr(&ctl.item_free[slot.at]), slot.ph ^ 1, stop, p.limit_us)) break;
                if (lane_id() == 0) {
                    ctl.item[slot.at] = it;
                    bar_arrive(smem_addr(&ctl.item_full[slot.at]));
                }
                slot.step();
                if (more) {
                    if (!warp_wait(smem_addr(&ctl.item_want), wanted.ph, stop, p.limit_us)) break;
                    wanted.step();
                    i = CUT ? i + 1 : draw(p.next, total);
                }
            }
            if (blockIdx.x == 0) {
                bool bad = lane_id() == 0 && (a.q_offsets[0] != 0 || a.q_offsets[a.n_seqs] != a.q_tokens ||
                                              a.k_offsets[0] != 0 || a.k_offsets[a.n_seqs] != a.k_tokens);
                for (int b = lane_id(); b < a.n_seqs; b += 32)
                    bad = bad || a.q_offsets[b + 1] < a.q_offsets[b] || a.k_offsets[b + 1] < a.k_offsets[b];
                if (bad) atomicOr(err, SERVE_INVALID);
            }
        }
    }
    tm_before();
    __syncthreads();
    if (threadIdx.x == 0 && *stop) atomicOr(err, SERVE_TIMEOUT);
    __syncwarp();
    if (warp == MMA_WARP) tm_free(ctl.tmem, 512);
}

// ---------------------------------------------------------------- the plan of equal runs
// All items' key tiles are laid end to end, an item's after ITEM_COST places for what it
// costs to begin and to end it, and cut into equal runs, one per block, of at least the
// square root of the longest item's tiles (a part that has to be joined costs about what
// a tile does).  One block.
constexpr int PLACES = 2048, ITEM_COST = 2;

__global__ void __launch_bounds__(1024) k_prompt_plan(PromptArgs p, int blocks, Item *plan, int *start) {
    __shared__ long long at[PLACES + 1];                 // where a place's items begin
    __shared__ long long wide_buf[33];
    __shared__ int seq_of[PLACES], warp_buf[33], longest;
    pdl_wait();
    const opattr_prompt &a = p.a;
    const int per = 2 * p.span;
    auto item_of = [&](int x, int b) {                   // of place x, which is sequence b's
        const int q0 = a.q_offsets[b], q1 = a.q_offsets[b + 1], k0 = a.k_offsets[b], k1 = a.k_offsets[b + 1];
        const int t0 = (int)((unsigned)(x - q0 / per - b) * per);
        if (q0 < 0 || q1 < q0 || q1 > a.q_tokens || k0 < 0 || k1 < k0 || k1 > a.k_tokens || t0 < 0 || t0 >= q1 - q0) return Item{};
        return Item{q0, q1 - q0, k0, k1 - k0, t0, 0, (k1 - k0) - (q1 - q0), 0, 0, 1, 1};
    };
    if (threadIdx.x == 0) longest = 0;
    long long total = 0;
    for (int x0 = 0; x0 < p.tiles; x0 += 1024) {
        const int x = x0 + (int)threadIdx.x;
        int n = 0, lo = 0;
        if (x < p.tiles) {
            for (int hi = a.n_seqs; hi - lo > 1;) {
                const int mid = (lo + hi) >> 1;
                if (a.q_offsets[mid] / per + mid <= x) lo = mid;
                else hi = mid;
            }
            const Item it = item_of(x, lo);
            if (it.some) n = max(1, Work(it, p.span, a.causal).n);
        }
        long long sum;
        const long long before = block_exclusive_scan(n ? (long long)(n + ITEM_COST) * p.heads_x : 0ll, wide_buf, &sum);
        if (x < p.tiles) at[x] = total + before, seq_of[x] = lo;
        total += sum;
        n = __reduce_max_sync(0xffffffffu, n);
        if (lane_id() == 0) atomicMax(&longest, n);
    }
    if (threadIdx.x == 0) at[p.tiles] = total;
    __syncthreads();
    const long long runs = min((long long)blocks, total / (ITEM_COST + (int)ceilf(sqrtf((float)longest))));
    const long long S = max(1ll, runs), b = threadIdx.x;
    // every part of run b, in order: its place, head, first step of the item, and from and to of its tiles
    auto walk = [&](auto &&part) {
        if (b >= S || total == 0) return;
        const long long s0 = b * total / S, s1 = (b + 1) * total / S;
        int x = 0;
        for (int hi = p.tiles; hi - x > 1;) {            // (the last place that begins there has items)
            const int mid = (x + hi) >> 1;
            if (at[mid] <= s0) x = mid;
            else hi = mid;
        }
        int cost = (int)((at[x + 1] - at[x]) / p.heads_x), hx = (int)((s0 - at[x]) / cost);
        for (long long item = at[x] + (long long)hx * cost; item < s1; item += cost, ++hx) {
            if (hx == p.heads_x) {
                hx = 0;
                while (at[++x + 1] == item);             // (s1 is no more than the total: there is one)
                cost = (int)((at[x + 1] - at[x]) / p.heads_x);
            }
            const long long first = item + ITEM_COST;
            const int n = cost - ITEM_COST, from = (int)max(0ll, s0 - first), to = (int)min((long long)n, s1 - first);
            if (from < to) part(x, hx, first, n, from, to);
        }
    };
    int mine = 0, sum;
    walk([&](int, int, long long, int, int, int) { ++mine; });
    int place = block_exclusive_scan(mine, warp_buf, &sum);
    if (b < blocks) start[b] = place;
    if (b == 0) start[blocks] = sum;
    walk([&](int x, int hx, long long first, int n, int from, int to) {
        Item it = item_of(x, seq_of[x]);
        const int block1 = (int)(((first + 1) * S - 1) / total), block2 = (int)(((first + n) * S - 1) / total);
        it.head0 = hx * p.pack;
        it.k0 += from * KEYS;
        // the last part has what is left of the keys, and with them the masks
        it.lk = (to == n ? it.lk : to * KEYS) - from * KEYS;
        it.ahead -= from * KEYS;
        it.first = block1, it.piece = (int)b - block1, it.pieces = block2 - block1 + 1;
        plan[place++] = it;
    });
}

// ---------------------------------------------------------------- host
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

template <typename T, int DP, int DV, bool CUT>
static opattr_status launch_prompt(Ctx &c, Serve &s, const PromptArgs &p, const CUtensorMap *m, unsigned grid) {
    constexpr unsigned bit = 1u << (2 * ((std::is_same<T, __half>::value ? 3 : 0) + (DP == 64 ? 0 : DV == 96 ? 1 : 2)) + CUT);
    if (!(s.prompt_room & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(k_prompt<T, DP, DV, CUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP>::SMEM);
        if (e != cudaSuccess) return cuda_status(c, e);
        s.prompt_room |= bit;
    }
    launch(c, "prompt", k_prompt<T, DP, DV, CUT>, dim3(grid), dim3(THREADS), Shape<DP>::SMEM, p, m[0], m[1], m[2], s.err);
    return cuda_status(c, c.last_error);
}
template <typename T, int DP, int DV>
static opattr_status run_prompt(Ctx &c, Serve &s, PromptArgs &p, const CUtensorMap *m) {
    const opattr_prompt &a = p.a;
    const int64_t items = (int64_t)p.heads_x * p.tiles;
    const int sms = sm_count(c);
    // Equal runs of keys where whole items would leave SMs idle for longer than 14 tiles take,
    // which is what a plan and joined parts cost.  What whole items take, in key tiles: the
    // longest where each SM has one at most, else an SM's share and what the last round leaves idle
    // (of the least item: causal prompts' items come longest first, so that the last ones are short).
    // Whole items, then runs, us: 1 query over 100,000 keys, 8 heads of 128: 926, 100; 4 over
    // 20,000 for each of 20, 32 heads on 8: 413, 266; 512 over 8,192: 107, 67; 4,096 causal, 8 heads:
    // 58, 49; and on the other side 4,096 not causal: 58, 69; 8,192 causal: 108, 121; 64 x 512, 8
    // heads of 64: 54, 79.
    const double per = 2. * p.span, q_each = (double)a.q_tokens / a.n_seqs, keys = (double)a.k_tokens / a.n_seqs / KEYS;
    const double queries = a.causal ? std::min(q_each / KEYS, keys) : 0., mean = keys - queries / 2, least = keys - queries;
    const double each = std::max(1., q_each / per + .5) * a.n_seqs * p.heads_x / sms;        // items of an SM
    const double whole = each <= 1 ? keys : std::max(keys, each * mean + (std::ceil(each) - each) * least);
    if (p.tiles <= PLACES && whole > each * mean + 14) {
        const int64_t parts = (int64_t)sms * 4 * ROWS * (DP + 2), most = items + sms;
        const opattr_status st = ensure_lasting_arena(c, Need().add<int>(sms + 1).add<Item>(most).add<float>(parts).bytes);
        if (st) return st;
        Arena ar(c);
        int *start = ar.take<int>(sms + 1);
        Item *plan = ar.take<Item>(most);
        p.start = start;
        p.plan = plan;
        p.parts = ar.take<float>(parts);
        p.tickets = s.tickets;
        launch(c, "prompt_plan", k_prompt_plan, dim3(1), dim3(1024), 0, p, sms, plan, start);
    }
    return p.plan ? launch_prompt<T, DP, DV, true>(c, s, p, m, (unsigned)sms)
                  : launch_prompt<T, DP, DV, false>(c, s, p, m, (unsigned)std::min<int64_t>(items, sms));
}

template <typename T>
static opattr_status prompt_of(Ctx &c, Serve &s, PromptArgs &p, const CUtensorMap *m) {
    if (p.a.head_dim <= 64) return run_prompt<T, 64, 64>(c, s, p, m);
    return p.a.head_dim <= 96 ? run_prompt<T, 128, 96>(c, s, p, m) : run_prompt<T, 128, 128>(c, s, p, m);
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
    CUtensorMap m[3];
    const opattr_rows &k = a->k_tokens ? a->k : a->q, &v = a->k_tokens ? a->v : a->q;
    const int64_t keys = a->k_tokens ? a->k_tokens : 1;
    if (!row_map(&m[0], a->dtype, a->q, a->q_tokens, a->q_heads, a->head_dim, p.pack, p.span) ||
        !row_map(&m[1], a->dtype, k, keys, a->kv_heads, a->head_dim, 1, KEYS) ||
        !row_map(&m[2], a->dtype, v, keys, a->kv_heads, a->head_dim, 1, KEYS))
        return OPATTR_E_INVALID_ARG;
    return a->dtype == OPATTR_BF16 ? prompt_of<__nv_bfloat16>(c, s, p, m) : prompt_of<__half>(c, s, p, m);
}

}  // namespace opattr
