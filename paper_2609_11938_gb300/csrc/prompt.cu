// prompt.cu -- attention over whole prompts: packed sequences of any lengths,
// grouped heads, causal or not (opattr_attention).
//
//   s_ij = scale * q_i . k_j,  j seen by i: j < Lk and, causal, j <= i + Lk - Lq
//   o_i = sum_j exp(s_ij - m_i) v_j / sum_j exp(s_ij - m_i),  lse_i = m_i + log of that sum
// A row that sees no key gets o = 0 and lse = -inf.
#include <math.h>

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
constexpr int ROWS = 128;                // queries of a sub-tile: one thread and one lane of tensor memory each
constexpr int THREADS = 384;             // two warpgroups for the softmax of two sub-tiles, one for the rest
constexpr int MMA_WARP = 8, LOAD_WARP = 9, TAIL_WARP = 10;
// registers: 384 x 168 at launch = 256 x 208 + 128 x 88
constexpr int REGS_SOFTMAX = 208, REGS_OTHERS = 88;
constexpr int MOST_MASKED = 4;           // key tiles that an item's masks cut: three at most (256 queries)

// Shapes by the padded head width DP (64 or 128; the copies fill what a head
// lacks with zeros).
template <int DP>
struct Shape {
    static constexpr int HALF = 128 * 128;                 // bytes of 128 rows of 64 elements
    static constexpr int TILE = DP / 64 * HALF;
    static constexpr int STAGES = DP == 128 ? 5 : 8;       // key and value tiles in flight
    static constexpr int SMEM = 2 * TILE + STAGES * TILE + 1024 /* alignment */;
};

struct PromptArgs {
    opattr_prompt a;
    int heads_x;                         // work items side by side: pairs of heads, or heads
    int pair;                            // 1: an item's sub-tiles are two heads of one key head; 0: 256 queries of one
    int tiles;                           // upper bound of query tiles over the sequences
    int q_mul, k_mul, v_mul;             // 0 where all heads read the same rows
};

struct Ctrl {
    uint64_t q_full, kv_full[8], kv_empty[8], s_full[2], p_full[2], o_full[2], v_full[MOST_MASKED], v_ready[MOST_MASKED], drain;
    uint32_t tmem;
    int stop;
    int poison[MOST_MASKED];
    int item[4];                         // sequence, tile, -1: none
    int scan[33];
};

// 16-bit value i of a swizzled tile's row r, columns 32 * at .. + 32, four to a register pair.
__device__ __forceinline__ uint32_t tile_at(int half_bytes, int r, int col) {
    return (uint32_t)((col >> 6) * half_bytes + r * 128 + (((col & 63) * 2) ^ ((r & 7) << 4)));
}

__device__ __forceinline__ uint32_t tm_ld1(uint32_t at) {
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(at));
    return r;
}

template <typename T, int DP>
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
    if (threadIdx.x == 0) {
        bar_init(smem_addr(&ctl.q_full), 1);
        for (int i = 0; i < S::STAGES; ++i) bar_init(smem_addr(&ctl.kv_full[i]), 1), bar_init(smem_addr(&ctl.kv_empty[i]), 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_addr(&ctl.s_full[i]), 1);
            bar_init(smem_addr(&ctl.p_full[i]), 4);
            bar_init(smem_addr(&ctl.o_full[i]), 1);
        }
        for (int i = 0; i < MOST_MASKED; ++i)
            bar_init(smem_addr(&ctl.v_full[i]), 1), bar_init(smem_addr(&ctl.v_ready[i]), 2), ctl.poison[i] = 0;
        bar_init(smem_addr(&ctl.drain), 1);
        ctl.stop = 0;
        ctl.item[0] = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        map_prefetch(&mq), map_prefetch(&mk), map_prefetch(&mv);
    }
    if (warp == MMA_WARP) tm_alloc(smem_addr(&ctl.tmem), 512);
    pdl_wait();

    // ---- the item: query tiles run from the last one to the first, so that the
    // longest of a causal sequence come first; heads side by side share keys in L2
    const opattr_prompt &a = p.a;
    const int per = p.pair ? ROWS : 2 * ROWS;
    const int hx = blockIdx.x % p.heads_x;
    {
        const int want = p.tiles - 1 - (int)(blockIdx.x / p.heads_x);
        int before = 0;
        bool bad = threadIdx.x == 0 && (a.q_offsets[0] != 0 || a.q_offsets[a.n_seqs] != a.q_tokens || a.k_offsets[0] != 0 ||
                                        a.k_offsets[a.n_seqs] != a.k_tokens);
        for (int b0 = 0; b0 < a.n_seqs; b0 += THREADS) {
            const int b = b0 + threadIdx.x;
            int mine = 0;
            if (b < a.n_seqs) {
                const int q0 = a.q_offsets[b], q1 = a.q_offsets[b + 1], k0 = a.k_offsets[b], k1 = a.k_offsets[b + 1];
                if (q0 < 0 || q1 < q0 || q1 > a.q_tokens || k0 < 0 || k1 < k0 || k1 > a.k_tokens) bad = true;
                else mine = (q1 - q0 + per - 1) / per;
            }
            int sum;
            const int at = before + block_exclusive_scan(mine, ctl.scan, &sum);
            if (want >= at && want < at + mine) ctl.item[0] = b, ctl.item[1] = want - at;
            before += sum;
            if (before > p.tiles) break;                 // only where an offset is wrong
        }
        if (bad) atomicOr(err, SERVE_INVALID);
        // after a wait that gave up nothing more is begun
        if (threadIdx.x == 0 && (*(volatile unsigned *)err & SERVE_TIMEOUT)) ctl.stop = 2;
    }
    tm_before();
    __syncthreads();
    tm_after();
    const uint32_t tm = ctl.tmem;
    const int b = ctl.item[0];
    if (b >= 0 && *stop == 0) {
    const int q0 = a.q_offsets[b], lq = a.q_offsets[b + 1] - q0, k0 = a.k_offsets[b], lk = a.k_offsets[b + 1] - k0;
    const int t0 = ctl.item[1] * per, ahead = lk - lq;   // query i sees the keys up to i + ahead
    const int head0 = p.pair ? 2 * hx : hx, g = head0 / (a.q_heads / a.kv_heads);
    // each sub-tile: its first query, its key tiles, and the first of them that a mask cuts
    int base[2], n_tiles[2], clean[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        base[s] = p.pair ? t0 : t0 + s * ROWS;
        const int rows = min(ROWS, lq - base[s]);
        const int keys = rows <= 0 ? 0 : a.causal ? max(0, min(lk, base[s] + rows + ahead)) : lk;
        n_tiles[s] = (keys + KEYS - 1) / KEYS;
        clean[s] = (a.causal ? max(0, min(lk, base[s] + 1 + ahead)) : lk) / KEYS;
    }
    const int n = max(n_tiles[0], n_tiles[1]);
    const int cut = n_tiles[1] > 0 ? min(clean[0], clean[1]) : clean[0];     // tiles from here on are looked over
    const uint32_t bar_kv = smem_addr(&ctl.kv_full[0]), bar_free = smem_addr(&ctl.kv_empty[0]);

    if (warp < 8) {
        regs_more<REGS_SOFTMAX>();
        // ---- softmax: a warpgroup per sub-tile, a thread per query
        const int s = warp >> 2, r = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tm + s * 128 + lanes, to = tm + 256 + s * DP + lanes;
        const float c = a.scale == 0.f ? 1.f : fabsf(a.scale) * LOG2E;
        const float sign = a.scale < 0.f ? -1.f : 0.f;
        const bool turn = !(a.scale > 0.f);
        const int head = p.pair ? head0 + s : head0, row = base[s] + r;
        const int seen = a.causal ? min(lk, row + 1 + ahead) : lk;
        const uint64_t c2 = pair(c, c);
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < n_tiles[s]; ++j) {
            if (!(ok = warp_wait(smem_addr(&ctl.s_full[s]), j & 1, stop))) break;
            tm_after();
            uint32_t x[KEYS];
#pragma unroll
            for (int q = 0; q < 4; ++q) tm_ld32(ts + 32 * q, x + 32 * q);
            tm_wait_ld();
            if (turn) {
#pragma unroll
                for (int i = 0; i < KEYS; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * sign);
            }
            if (j >= clean[s]) {
                const int left = seen - j * KEYS;
#pragma unroll
                for (int i = 0; i < KEYS; ++i) x[i] = i < left ? x[i] : 0xff800000u;
            }
            float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < KEYS; i += 8)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    t[q] = fmaxf(t[q], fmaxf(__uint_as_float(x[i + 2 * q]), __uint_as_float(x[i + 2 * q + 1])));
            const float top = fmaxf(m, fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])));
            if (__any_sync(0xffffffffu, (top - m) * c > SLACK)) {
                const float keep = top == m ? 1.f : exp2_fast((m - top) * c);
                m = top;
                l *= keep;
                if (j > 0) {
                    const uint64_t keep2 = pair(keep, keep);
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
            }
            const float2 z = unpair(add2(sum[0], sum[1]));
            l += z.x + z.y;
            tm_wait_st();
            if (a.causal && j >= cut) {
                // a value that is not finite times a weight of zero would reach the rows
                // that do not see it: such a tile's products are made here, key by key
                if (!(ok = warp_wait(smem_addr(&ctl.v_ready[j - cut]), 0, stop))) break;
                if (*(volatile int *)&ctl.poison[j - cut]) {
                    const unsigned char *v = smem + 2 * S::TILE + (2 * j + 1) % S::STAGES * S::TILE;
                    const int left = seen - j * KEYS;
                    for (int d = 0; d < DP; d += 32) {
                        uint32_t o[32] = {};
                        if (j > 0) {
                            tm_ld32(to + d, o);
                            tm_wait_ld();
                        }
                        for (int i = 0; i < KEYS; ++i) {
                            const uint32_t w = tm_ld1(ts + i / 2);
                            tm_wait_ld();
                            const float2 w2 = Type2<T>::up(w);
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
            tm_before();
            __syncwarp();
            if (lane_id() == 0) bar_arrive(smem_addr(&ctl.p_full[s]));
        }
        if (n_tiles[s] > 0 && ok) ok = warp_wait(smem_addr(&ctl.o_full[s]), 0, stop);
        tm_after();
        if (ok) {
            const bool live = row < lq;
            const float share = l == 0.f ? 0.f : 1.f / l;
            T *out = (T *)a.out.data + (int64_t)(q0 + row) * a.out.token_stride + head * a.out.head_stride;
            for (int d = 0; d < DP; d += 32) {
                uint32_t o[32] = {};
                if (n_tiles[s] > 0) {
                    tm_ld32(to + d, o);
                    tm_wait_ld();
                }
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint4 y;
                    uint32_t *yy = reinterpret_cast<uint32_t *>(&y);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float lo = __uint_as_float(o[e + 2 * q]) * share, hi = __uint_as_float(o[e + 2 * q + 1]) * share;
                        yy[q] = l == 0.f ? 0u : Type2<T>::down(lo, hi);
                    }
                    if (live && d + e < a.head_dim) *reinterpret_cast<uint4 *>(out + d + e) = y;
                }
            }
            if (live && a.lse)
                a.lse[(int64_t)(q0 + row) * a.q_heads + head] =
                    l == 0.f ? -INFINITY : (__fmaf_rn(m == -INFINITY ? 0.f : m, c, -OFFSET) + log2f(l)) * LN2;
        }
    } else {
    regs_fewer<REGS_OTHERS>();
    if (warp == MMA_WARP) {
        // ---- products: one thread
        if (lane_id() == 0 && n > 0) {
            constexpr uint32_t DS = mma_desc(BF, ROWS, KEYS, false), DO = mma_desc(BF, ROWS, DP, true);
            auto scores = [&](int s, int j) {
                const uint32_t qa = sq + s * S::TILE, ka = skv + (j == 0 ? 0 : 2 * j) % S::STAGES * S::TILE;
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t off = (k / 4) * S::HALF + (k % 4) * 32;
                    mma_ss(tm + s * 128, tile_desc(qa + off, 16), tile_desc(ka + off, 16), DS, k > 0);
                }
                mma_commit(smem_addr(&ctl.s_full[s]));
            };
            auto full = [&](int load) { return bar_wait(bar_kv + load % S::STAGES * 8, load / S::STAGES & 1, stop); };
            auto release = [&](int load) { mma_commit(bar_free + load % S::STAGES * 8); };
            bool ok = bar_wait(smem_addr(&ctl.q_full), 0, stop) && full(0);
            if (ok) {
                tm_after();
                for (int s = 0; s < 2; ++s)
                    if (n_tiles[s] > 0) scores(s, 0);
                release(0);
            }
            for (int j = 0; ok && j < n; ++j) {
                const bool more = j + 1 < n;
                if (!(ok = full(2 * j + 1))) break;
                if (j >= cut && !(ok = bar_wait(smem_addr(&ctl.v_ready[j - cut]), 0, stop))) break;
                if (more && !(ok = full(2 * j + 2))) break;
                const bool by_hand = a.causal && j >= cut && *(volatile int *)&ctl.poison[j - cut];
                const uint32_t va = skv + (2 * j + 1) % S::STAGES * S::TILE;
                for (int s = 0; s < 2; ++s) {
                    if (j >= n_tiles[s]) continue;
                    if (!(ok = bar_wait(smem_addr(&ctl.p_full[s]), j & 1, stop))) break;
                    tm_after();
                    if (!by_hand) {
#pragma unroll
                        for (int k = 0; k < KEYS / 16; ++k)
                            mma_ts(tm + 256 + s * DP, tm + s * 128 + 8 * k, tile_desc(va + k * 2048, S::HALF), DO, j > 0 || k > 0);
                    }
                    if (j + 1 < n_tiles[s]) scores(s, j + 1);
                    else mma_commit(smem_addr(&ctl.o_full[s]));
                }
                if (!ok) break;
                release(2 * j + 1);
                if (more) release(2 * j + 2);
            }
            // nothing of this thread's is under way when the block ends
            mma_commit(smem_addr(&ctl.drain));
            int never = 0;
            bar_wait(smem_addr(&ctl.drain), 0, &never);
        }
    } else if (warp == LOAD_WARP) {
        // ---- tile copies: one thread
        if (lane_id() == 0 && n > 0) {
            const uint32_t bq = smem_addr(&ctl.q_full);
            const int subs = n_tiles[1] > 0 ? 2 : 1;
            bar_expect(bq, subs * S::TILE);
            for (int s = 0; s < subs; ++s)
                for (int d = 0; d < DP / 64; ++d)
                    tile_load(sq + s * S::TILE + d * S::HALF, &mq, 64 * d, (p.pair ? head0 + s : head0) * p.q_mul, q0 + base[s], bq);
            int load = 0;
            for (; load < 2 * n; ++load) {
                const int st = load % S::STAGES;
                if (load >= S::STAGES && !bar_wait(bar_free + 8 * st, (load / S::STAGES - 1) & 1, stop)) break;
                // K0, V0, K1, V1, ..
                const bool keys = load % 2 == 0;
                const int j = load / 2;
                // values that are looked over have a barrier of their own: the stage's may
                // have gone round several times before the tail's warps see it
                const bool over = !keys && j >= cut;
                const uint32_t bar = over ? smem_addr(&ctl.v_full[j - cut]) : bar_kv + 8 * st;
                bar_expect(bar, S::TILE);
                for (int d = 0; d < DP / 64; ++d)
                    tile_load(skv + st * S::TILE + d * S::HALF, keys ? &mk : &mv, 64 * d, keys ? g * p.k_mul : g * p.v_mul,
                              k0 + j * KEYS, bar);
                if (over) bar_arrive(bar_kv + 8 * st);
            }
            // copies that nobody waited for any more
            int never = 0;
            if (*stop)
                for (int i = max(0, load - S::STAGES); i < load; ++i) {
                    const bool over = i % 2 && i / 2 >= cut;
                    bar_wait(over ? smem_addr(&ctl.v_full[i / 2 - cut]) : bar_kv + i % S::STAGES * 8, over ? 0 : i / S::STAGES & 1,
                             &never);
                }
            if (*stop) bar_wait(bq, 0, &never);
        }
    } else {
        // ---- tiles that a mask cuts, two warps: rows past the sequence's keys become
        // zeros, and, causal, the others are looked over for values that are not finite
        const int w = threadIdx.x - 32 * TAIL_WARP;
        for (int j = cut; j < n; ++j) {
            const int load = 2 * j + 1, keys = min(KEYS, lk - j * KEYS);
            if (!warp_wait(smem_addr(&ctl.v_full[j - cut]), 0, stop)) break;
            unsigned char *v = smem + 2 * S::TILE + load % S::STAGES * S::TILE;
            unsigned most = 0;
            for (int i = w; i < S::TILE / 16; i += 64) {
                uint4 *u = reinterpret_cast<uint4 *>(v) + i;
                if ((i * 16 % S::HALF) / 128 >= keys) *u = make_uint4(0, 0, 0, 0);
                else if (a.causal) {
                    const uint4 y = *u;
                    most = __vmaxu2(most, __vmaxu2(__vmaxu2(y.x & 0x7fff7fffu, y.y & 0x7fff7fffu),
                                                   __vmaxu2(y.z & 0x7fff7fffu, y.w & 0x7fff7fffu)));
                }
            }
            constexpr unsigned INF = BF ? 0x7f80u : 0x7c00u;
            if ((most >> 16) >= INF || (most & 0xffffu) >= INF) ctl.poison[j - cut] = 1;
            fence_smem_async();
            __syncwarp();
            if (lane_id() == 0) bar_arrive(smem_addr(&ctl.v_ready[j - cut]));
        }
    }
    }
    }
    tm_before();
    __syncthreads();
    if (threadIdx.x == 0 && *stop == 1) atomicOr(err, SERVE_TIMEOUT);
    __syncwarp();
    if (warp == MMA_WARP) tm_free(tm, 512);
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

// Boxes of 128 rows of 64 elements of one head; past a head's width or the last row: zeros.
static bool row_map(CUtensorMap *m, int dtype, const opattr_rows &r, int64_t tokens, int heads, int dim) {
    const bool one = heads == 1 || r.head_stride == 0;
    const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)(one ? 1 : heads), (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {2 * (cuuint64_t)(one ? dim : r.head_stride),
                                   2 * (cuuint64_t)(tokens == 1 ? dim : r.token_stride)};
    const cuuint32_t box[3] = {64, 1, 128}, step[3] = {1, 1, 1};
    return encode_tiled()(m, dtype == OPATTR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                          r.data, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DP>
static opattr_status run_prompt(Ctx &c, Serve &s, const PromptArgs &p, const CUtensorMap *m) {
    using S = Shape<DP>;
    const cudaError_t e = cudaFuncSetAttribute(k_prompt<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    if (e != cudaSuccess) return cuda_status(c, e);
    launch(c, "prompt", k_prompt<T, DP>, dim3((unsigned)((int64_t)p.heads_x * p.tiles)), dim3(THREADS), S::SMEM, p, m[0], m[1],
           m[2], s.err);
    return cuda_status(c, c.last_error);
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
    PromptArgs p{};
    p.a = *a;
    const int group = a->q_heads / a->kv_heads;
    p.pair = group % 2 == 0;
    p.heads_x = p.pair ? a->q_heads / 2 : a->q_heads;
    const int64_t tiles = a->q_tokens / (p.pair ? ROWS : 2 * ROWS) + a->n_seqs;
    if (tiles * p.heads_x > INT32_MAX) return OPATTR_E_INVALID_ARG;
    p.tiles = (int)tiles;
    p.q_mul = a->q_heads > 1 && a->q.head_stride != 0;
    p.k_mul = a->kv_heads > 1 && a->k.head_stride != 0;
    p.v_mul = a->kv_heads > 1 && a->v.head_stride != 0;
    if (!encode_tiled()) return OPATTR_E_CUDA;
    // without keys there is nothing to copy, and any rows stand in for them
    CUtensorMap m[3];
    if (!row_map(&m[0], a->dtype, a->q, a->q_tokens, a->q_heads, a->head_dim) ||
        !row_map(&m[1], a->dtype, a->k_tokens ? a->k : a->q, a->k_tokens ? a->k_tokens : 1, a->kv_heads, a->head_dim) ||
        !row_map(&m[2], a->dtype, a->k_tokens ? a->v : a->q, a->k_tokens ? a->k_tokens : 1, a->kv_heads, a->head_dim))
        return OPATTR_E_INVALID_ARG;
    if (a->dtype == OPATTR_BF16)
        return a->head_dim <= 64 ? run_prompt<__nv_bfloat16, 64>(c, s, p, m) : run_prompt<__nv_bfloat16, 128>(c, s, p, m);
    return a->head_dim <= 64 ? run_prompt<__half, 64>(c, s, p, m) : run_prompt<__half, 128>(c, s, p, m);
}

}  // namespace opattr
