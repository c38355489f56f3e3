// Attention over the 8-bit paged cache for many query rows per KV head (a prompt's chunk, cross attention): tcgen05 products with the
// scores, the weights and the sums in tensor memory.
#include <algorithm>
#include <type_traits>

#include "eosq_kv8.cuh"
#include "eosq_sm100.cuh"

namespace eosq {

using namespace sm100;

namespace {

// A CTA takes a run of units (Kv8Tiles): 256 query rows, in two halves of 128, against tiles of 128 tokens.
//   warps 0-3, 4-7   the halves' weights, a row per thread: scores out of tensor memory, weights back into it (in the scores' place, as the
//                    A operand of the second product), maximum and sum in registers; results out
//   warps 8-11       turn codes into fp16 operands
//   warp 12          issues the products; while one half's weights are made, the other half's products run
//   warp 13          walks through the run, tells the others about each tile, and fetches codes, a tile ahead, and scales
//   warps 14, 15     bring the next row tile's queries in as soon as this one's last scores have been made
// A half's chain is what bounds it: products of 128 x 128 x d twice (some 1500 cycles, shared memory feeding them), then the weights of a row per thread (some 2500, of
// which the special function units need 1024, or 2048 where the halves meet); the halves overlap, so a tile takes some 4800 cycles: four prompts
// of 2048 queries on 12000 tokens run at 998 TFLOP/s (1717 for a library product), four of 500 to 2048 on 2048 to 12000, with their diagonal and their
// last row tiles, at 888 (1004 and 893 while a turn was made again instead of looking at what is left of a tile, which did not end on some scores beyond 2^27).  Half the weights' 2^x by a polynomial
// instead was slower, so were scores of 64 tokens with the next 64 beside them, and twice the warps for the codes.
constexpr int ROWS = 256, HALF = 128, KEYS = KV8_KEYS, GROUP = KV8_GROUP, GROUPS = KV8_GROUPS;
constexpr int LOADER = 8, ISSUER = 12, FETCHER = 13, THREADS = 32 * 16, STAGES = 2, INFOS = 4;
// A row tile's beginning and end (queries in, a first tile looked at twice, results out, nothing of one half beside the other's) take as long as five tiles with bf16
// queries, as three and a half with fp16: four prompts of 500 to 2048 queries, bf16 / fp16, 623 / 499 us counted as two, 550 / 465 as four, 544 / 463 as five, 539 / 465 as six.
constexpr int COST = 5;
static_assert(COST <= KV8_COST_BOUND, "the bound on a call's units");
using Tiles = Kv8Tiles<ROWS, KEYS, COST>;

struct TileInfo {
    int end;                // 1: some of the tokens may be behind the sequence's last; -1: the run has ended, there is no tile
    int first, last;        // of the CTA's run within one row tile
    int tok0;               // the tile's first position
    int q0, len, m, r, h;   // the entry's queries, its length; row tile, KV head
    int slot;               // -1: the whole row tile is this CTA's, else the slot of its partial result
    float ks[GROUPS], vlog[GROUPS], vinv[GROUPS];   // per 16 tokens: key scale, log2 of the value scale (-infinity: not there) and its inverse
};

constexpr size_t operand_bytes(int d) { return static_cast<size_t>(HALF) * d * 2; }   // 128 rows of fp16
constexpr size_t smem_bytes(int d) { return 1024 + (2 + 2 * STAGES) * operand_bytes(d) + 2 * static_cast<size_t>(KEYS) * d; }
static_assert(smem_bytes(128) + 1700 <= 232448, "shared memory of a CTA, with the barriers and scales");
static_assert(2 * STAGES * operand_bytes(64) >= sizeof(int) * EOSQ_KV8_MAX_SEQS, "units of every entry");

__device__ __forceinline__ uint64_t desc_of(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}

template <int DIM, int FMT, bool BF16>
__global__ void __launch_bounds__(THREADS, 1) kv8_tiles_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                                  const Kv8Attend a) {
    extern __shared__ uint8_t tiles_smem[];
    __shared__ __align__(8) uint64_t q_full[2], q_free[2], s_full[2], p_full[2], o_done[2], k_full[STAGES], v_full[STAGES], k_free[STAGES], v_free[STAGES], info_full[INFOS],
        info_free[INFOS], code_full[2], code_free[2], drain_bar;
    __shared__ TileInfo info[INFOS];
    __shared__ int8_t q_exp[2][ROWS];   // by row tile in turn: the power of two that its queries were divided by
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile int abort_flag;
    __shared__ uint32_t fills[2];   // of keys, of values
    constexpr uint32_t OPERAND = HALF * DIM * 2, PANEL = HALF * 128;   // an operand: panels of 64 channels, 128 rows of 128 bytes each
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(tiles_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t *q_smem = smem, *k_smem = smem + 2 * OPERAND, *v_smem = k_smem + STAGES * OPERAND, *codes = v_smem + STAGES * OPERAND;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = tid & 31;
    const Kv8 &c = a.c;
    if (tid == 0) {
        tma_prefetch_desc(&kmap);
        tma_prefetch_desc(&vmap);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&code_full[i], 1);
            mbar_init(&code_free[i], 4);
            mbar_init(&q_full[i], 2);
            mbar_init(&q_free[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
            mbar_init(&o_done[i], 1);
        }
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&k_full[i], 4);
            mbar_init(&v_full[i], 4);
            mbar_init(&k_free[i], 1);
            mbar_init(&v_free[i], 1);
        }
        for (int i = 0; i < INFOS; ++i) {
            mbar_init(&info_full[i], 1);
            mbar_init(&info_free[i], ISSUER + 1);   // the warps that read them
        }
        mbar_init(&drain_bar, 1);
        abort_flag = 0;
        fills[0] = fills[1] = 0;
        fence_mbar_init();
    }
    if (warp == ISSUER) {
        tmem_alloc(&tmem_base_s, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    pdl_wait();
    const Kv8Run run = kv8_run<Tiles, THREADS>(a, reinterpret_cast<int *>(k_smem));
    tc_fence_after_sync();
    fence_proxy_async_smem();   // the entries' units have been read; from here on operands and copies are there
    __syncthreads();
    const uint32_t tmem = warp_uniform(tmem_base_s);

    if (warp < LOADER) {
        // ---- weights ------------------------------------------------------------------------
        const int half = warp >> 2, row_in = (warp & 3) * 32 + lane;
        const uint32_t s_at = tmem + half * KEYS + (static_cast<uint32_t>((warp & 3) * 32) << 16), o_at = s_at - half * KEYS + 256 + half * DIM;
        const float scale = fabsf(a.scale_log2);
        uint32_t tiles_done = 0, items_done = 0, items = 0;   // tiles and row tiles of this half, row tiles in all
        int lo = 0, hi = 0;
        bool ok = true, active = false, live = false;   // (active: some row of this half is a query)
        float m = -INFINITY, l = 0.0f, kscale = scale;
        for (uint32_t it = 0;; ++it) {
            const int slot = it % INFOS;
            ok = mbar_wait_warp(&info_full[slot], (it / INFOS) & 1u, &abort_flag);
            if (!ok) break;
            const TileInfo &ti = info[slot];
            if (ti.end < 0) break;
            const bool first = ti.first != 0, last = ti.last != 0;
            if (first) {
                const int row0 = ti.r * ROWS + half * HALF, rows = ti.m * a.G;
                active = row0 < rows;
                live = row0 + row_in < rows;
                lo = 0;
                hi = 1 << 30;   // (rows that are no query see everything: that they saw nothing would hold up the others)
                if (live) {
                    const int t = (row0 + row_in) / a.G;
                    Tiles::span(a, Kv8Seq{0, ti.len, ti.m, 0}, t, t, lo, hi);
                }
                m = -INFINITY;
                l = 0.0f;
            }
            if (active) {
                const int tok0 = ti.tok0;
                const bool edge = __any_sync(0xffffffffu, live && (tok0 < lo || tok0 + KEYS > hi));
                ok = mbar_wait_warp(&s_full[half], tiles_done & 1u, &abort_flag);
                if (!ok) break;
                tiles_done += 1;
                tc_fence_after_sync();
                if (BF16 && first) kscale = scale * __uint_as_float(static_cast<uint32_t>(127 + q_exp[items & 1][half * HALF + row_in]) << 23);
                // A row's base-2 logarithms are s * ks + vlog, with a key and a value scale for every 16 tokens.  (ks is kept above zero, so that masked scores stay
                // -infinity under a scale of zero.)
                auto ks_of = [&](int g) { return fmaxf(ti.ks[g] * kscale, 1e-37f); };
                uint32_t x[GROUP];
                auto read = [&](int g) {
                    tmem_ld16(s_at + GROUP * g, x);
                    tmem_ld_wait(x);
                };
                auto hide = [&](int g) {
                    const int at = tok0 + GROUP * g;
#pragma unroll
                    for (int e = 0; e < GROUP; ++e)
                        if (at + e < lo || at + e >= hi) x[e] = 0xff800000u;   // -infinity
                };
                // The largest logarithm of the 16 tokens in x ...
                auto largest = [&](int g) {
                    float t0 = __uint_as_float(x[0]), t1 = __uint_as_float(x[1]);
#pragma unroll
                    for (int e = 2; e < GROUP; e += 2) {
                        t0 = fmaxf(t0, __uint_as_float(x[e]));
                        t1 = fmaxf(t1, __uint_as_float(x[e + 1]));
                    }
                    return fmaf(fmaxf(t0, t1), ks_of(g), ti.vlog[g]);
                };
                // ... their weights, as 2^(x * kf + cf), and the sum of those.
                uint32_t p[GROUP / 2];
                auto weights = [&](const uint32_t (&x)[GROUP], uint32_t (&p)[GROUP / 2], float kf, float cf) {
                    const uint64_t k2 = pair_of(kf, kf), c2 = pair_of(cf, cf);
                    uint64_t sum = 0;
#pragma unroll
                    for (int e = 0; e < GROUP; e += 2) {
                        float y0, y1;
                        unpair(fma_pair(pair_of(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), k2, c2), y0, y1);
                        y0 = exp2_fast(y0);
                        y1 = exp2_fast(y1);
                        sum = add_pair(sum, pair_of(y0, y1));
                        p[e >> 1] = half2_bits(y0, y1);
                    }
                    float s0, s1;
                    unpair(sum, s0, s1);
                    return s0 + s1;
                };
                // A new maximum, for the sum and for the sums of values (the products that made them have ended: the scores came behind them).
                auto move = [&](float top) {
                    const float to = kv8_moved(m, top), by = (to == -INFINITY) ? 1.0f : exp2_fast(m - to);
                    m = to;
                    l *= by;
                    if (!first) {
#pragma unroll 1
                        for (int k = 0; k < DIM / 16; ++k) {
                            tmem_ld16(o_at + 16 * k, x);
                            tmem_ld_wait(x);
#pragma unroll
                            for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * by);
                            tmem_st16(o_at + 16 * k, x);
                        }
                    }
                    return by;
                };
                // Short loops: the warps of a quarter of an SM all run different parts of this kernel through one small instruction cache.  And one pass over the scores
                // where it can be.  Four prompts of 500 to 2048 queries on up to 12000 tokens, and four of 2048 on 12000: two passes in loops of 32 tokens, twice unrolled,
                // 745 and 1879 us; of 16 tokens 635 and 1687; one pass of 16 tokens 638 and 1662, of 32 634 and 1524, of 64 629 and 1458.
                constexpr int TURN = 4;   // in sixteens
                const bool look = first || edge || __any_sync(0xffffffffu, m == -INFINITY || kv8_far(m));
                int done = 0;   // sixteens whose weights have been made
                if (!look) {
                    // Under the maximum so far.  Where the weights of a turn add up to no more than 2^14 none is beyond fp16's range, nor is the maximum more than KV8_SLACK behind; else, which
                    // is rare, this turn and what is left of the tile is looked at first.
#pragma unroll 1
                    for (; done < GROUPS; done += TURN) {
                        uint32_t y[TURN][GROUP], q[TURN][GROUP / 2];
#pragma unroll
                        for (int i = 0; i < TURN; ++i) tmem_ld16(s_at + GROUP * (done + i), y[i]);
                        float sum = 0.0f, add = 0.0f;
#pragma unroll
                        for (int i = 0; i < TURN; ++i) {
                            const float kf = ks_of(done + i), cf = ti.vlog[done + i] + KV8_SHIFT;
                            tmem_ld_wait(y[i]);
                            const float s16 = weights(y[i], q[i], kf, cf - m);
                            sum += s16;
                            add = fmaf(s16, ti.vinv[done + i], add);
                        }
                        if (__any_sync(0xffffffffu, sum > 16384.0f)) break;   // (not for a NaN, which stays one)
                        l += add;
#pragma unroll
                        for (int i = 0; i < TURN; ++i) tmem_st8(s_at + GROUP / 2 * (done + i), q[i]);   // in the place of scores that have been read
                    }
                }
                if (done < GROUPS) {
                    // With a look at all scores that are left before the next weight: a row tile's first tile, masks, rows that have seen nothing yet; a turn whose weights were too
                    // large; and logarithms beyond kv8_far's bound.  Whatever the scores are, each is looked at once and then weighed once.
                    float top = -INFINITY;
#pragma unroll 1
                    for (int g = done; g < GROUPS; ++g) {
                        read(g);
                        if (edge) hide(g);
                        top = fmaxf(top, largest(g));
                    }
                    if (__any_sync(0xffffffffu, top - m > (look ? KV8_SLACK : 0.0f))) {
                        if (done) tmem_st_wait();   // weights that are read again below have been stored: nothing else orders a load behind a store to tensor memory
                        const __half2 by = __float2half2_rn(move(top));
#pragma unroll 1
                        for (int i = 0; i < done; ++i) {   // the weights before these
                            tmem_ld8(s_at + GROUP / 2 * i, p);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < GROUP / 2; ++e) {
                                const __half2 v = __hmul2(*reinterpret_cast<const __half2 *>(&p[e]), by);
                                p[e] = *reinterpret_cast<const uint32_t *>(&v);
                            }
                            tmem_st8(s_at + GROUP / 2 * i, p);
                        }
                    }
                    const bool mine_far = kv8_far(m), far = __any_sync(0xffffffffu, mine_far);   // (a row's arithmetic goes by its own maximum)
                    const float m0 = (m == -INFINITY) ? 0.0f : m, b = KV8_SHIFT - m0;
#pragma unroll 1
                    for (int g = done; g < GROUPS; ++g) {
                        read(g);
                        if (edge) hide(g);
                        float kf = ks_of(g), cf = ti.vlog[g] + b;
                        if (far) {
#pragma unroll
                            for (int e = 0; e < GROUP; ++e)
                                if (mine_far) x[e] = __float_as_uint(fmaf(__uint_as_float(x[e]), kf, ti.vlog[g]) - m0);
                            kf = mine_far ? 1.0f : kf;
                            cf = mine_far ? KV8_SHIFT : cf;
                        }
                        l = fmaf(weights(x, p, kf, cf), ti.vinv[g], l);
                        tmem_st8(s_at + GROUP / 2 * g, p);   // in the place of scores that have been read
                    }
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[half]);
            }
            if (last) items += 1;
            if (last && active) {
                const int row = ti.r * ROWS + half * HALF + row_in, place = ti.slot;
                const int t_of = row / a.G, hq = ti.h * a.G + row - t_of * a.G;
                const long long tq = ti.q0 + static_cast<long long>(t_of);
                __syncwarp();
                if (lane == 0) mbar_arrive(&info_free[slot]);
                ok = mbar_wait_warp(&o_done[half], items_done & 1u, &abort_flag);
                items_done += 1;
                if (!ok) break;
                tc_fence_after_sync();
                const float inv = (place >= 0) ? 1.0f : (m == -INFINITY ? 0.0f : 1.0f / l);
                const Kv8Parts<ROWS> parts(a, gridDim.x);
                const size_t pr = static_cast<size_t>(2 * blockIdx.x + max(place, 0)) * ROWS + half * HALF + row_in;
#pragma unroll 1
                for (int k = 0; k < DIM / 32; ++k) {
                    uint32_t o[32];
                    float v[32];
                    tmem_ld32(o_at + 32 * k, o);
                    tmem_ld_wait(o);
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(o[e]) * inv;
                    if (live) {
                        if (place < 0) {
                            store_row<BF16, 32>(static_cast<__half *>(a.out) + tq * a.o_tok + hq * a.o_head + 32 * k, v);
                        } else {
#pragma unroll
                            for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4 *>(parts.four(2 * blockIdx.x + place, half * HALF + row_in, 32 * k + e)) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                        }
                    }
                }
                if (live) {
                    if (place >= 0) {
                        parts.m[pr] = m;
                        parts.l[pr] = l;
                    } else if (a.lse) {
                        a.lse[tq * (c.heads * a.G) + hq] = row_lse(m, l);
                    }
                }
                tc_fence_before_sync();
            } else {
                __syncwarp();
                if (lane == 0) mbar_arrive(&info_free[slot]);
            }
        }
    } else if (warp < ISSUER) {
        // ---- keys and values ----------------------------------------------------------------
        constexpr int PER = DIM / 16, TOKS = 128 / PER, LOADS = KEYS / TOKS;   // threads of a token, tokens of a round, rounds
        const int part = (tid & 127) % PER, tok_in = (tid & 127) / PER;
        const int swap = (DIM == 128 && part >= 4) ? 1 : 0;   // which of a thread's two chunks is written first: all banks at once
        bool ok = true;
        for (uint32_t it = 0; ok; ++it) {
            const int st = it % STAGES, slot = it % INFOS;
            const uint32_t free_parity = ((it / STAGES) & 1u) ^ 1u;
            ok = mbar_wait_warp(&info_full[slot], (it / INFOS) & 1u, &abort_flag);
            if (!ok) break;
            const int end = info[slot].end;
            __syncwarp();
            if (lane == 0) mbar_arrive(&info_free[slot]);
            if (end < 0) break;
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
                ok = mbar_wait_warp(&code_full[kv], it & 1u, &abort_flag);
                if (!ok) break;
                ok = mbar_wait_warp(kv ? &v_free[st] : &k_free[st], free_parity, &abort_flag);
                if (!ok) break;
                const uint8_t *src = codes + kv * (KEYS * DIM);
                uint8_t *dst = (kv ? v_smem : k_smem) + st * OPERAND + (part >> 2) * PANEL;
                auto read = [&](int row) {
                    const int chunk = (DIM == 128) ? part ^ (row & 7) : part ^ ((row >> 1) & 3);
                    return *reinterpret_cast<const uint4 *>(src + row * DIM + chunk * 16);
                };
                uint4 x = read(tok_in);
#pragma unroll 1
                for (int k = 0; k < LOADS; ++k) {   // (short code: the warps of an SM's quarter all run different parts of this kernel, through one small instruction cache)
                    const int row = k * TOKS + tok_in;
                    const uint32_t y[4] = {x.x, x.y, x.z, x.w};
                    if (k + 1 < LOADS) x = read(row + TOKS);
                    uint32_t z[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) codes_to_half<FMT>(y[e], z[2 * e], z[2 * e + 1]);
                    if (end) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = no_nan<FMT>(z[e]);
                    }
                    uint8_t *line = dst + row * 128;
                    const int c0 = (part & 3) * 2;
                    const uint4 u = make_uint4(z[0], z[1], z[2], z[3]), v = make_uint4(z[4], z[5], z[6], z[7]);
                    *reinterpret_cast<uint4 *>(line + (((c0 + swap) ^ (row & 7)) << 4)) = swap ? v : u;
                    *reinterpret_cast<uint4 *>(line + (((c0 + 1 - swap) ^ (row & 7)) << 4)) = swap ? u : v;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&code_free[kv]);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(kv ? &v_full[st] : &k_full[st]);
            }
        }
    } else if (warp == ISSUER) {
        // ---- products -----------------------------------------------------------------------
        constexpr uint32_t idesc_s = umma_idesc_f16(HALF, KEYS, false, false), idesc_o = umma_idesc_f16(HALF, DIM, false, true);
        const bool issuer = elect_one();
        uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0};   // row tiles, tiles of each half
        bool ok = true;
        // An operand's descriptor: its lower word counts addresses in 16 bytes, so that a step along the operand is an addition there; the upper one is the same for all.
        const uint64_t any_desc = umma_desc_sw128(0, 0, 1024);
        const uint32_t hi_desc = static_cast<uint32_t>(any_desc >> 32);
        const uint32_t q_desc = smem_u32(q_smem) >> 4, k_desc = smem_u32(k_smem) >> 4, v_desc = (smem_u32(v_smem) >> 4) | ((PANEL >> 4) << 16);
        auto scores = [&](int half, int st) {
            const uint32_t q = q_desc + half * (OPERAND >> 4), kd = k_desc + st * (OPERAND >> 4), to = tmem + half * KEYS;
            if (issuer) {
#pragma unroll 2
                for (int k = 0; k < DIM / 16; ++k) {
                    constexpr uint32_t panel = PANEL >> 4;
                    umma_f16(to, desc_of(q + (k >> 2) * panel + (k & 3) * 2, hi_desc), desc_of(kd + (k >> 2) * panel + (k & 3) * 2, hi_desc), idesc_s, k ? 1u : 0u);
                }
                umma_commit(&s_full[half]);
            }
            __syncwarp();
        };
        auto values = [&](int half, int st, bool first) {
            const uint32_t vd = v_desc + st * (OPERAND >> 4), of = tmem + half * KEYS, to = tmem + 256 + half * DIM;
            const uint32_t more = first ? 0u : 1u;
            if (issuer) {
#pragma unroll 2
                for (int k = 0; k < KEYS / 16; ++k) umma_f16_ts(to, of + 8 * k, desc_of(vd + k * 128, hi_desc), idesc_o, k ? 1u : more);
            }
            __syncwarp();
        };
        auto commit = [&](uint64_t *bar) {
            if (issuer) umma_commit(bar);
            __syncwarp();
        };
        int halves = 0, first = 0, last = 0;
        auto read = [&](uint32_t it) {   // tile `it`: how many halves have queries (0: the run has ended)
            const int slot = it % INFOS;
            ok = mbar_wait_warp(&info_full[slot], (it / INFOS) & 1u, &abort_flag);
            if (!ok) return 0;
            const TileInfo &ti = info[slot];
            const int n = ti.end < 0 ? 0 : (ti.r * ROWS + HALF < ti.m * a.G ? 2 : 1);
            first = ti.first;
            last = ti.last;
            __syncwarp();
            if (lane == 0) mbar_arrive(&info_free[slot]);
            return n;
        };
        halves = read(0);
        // The values of tile it - 1, then the scores of tile it, one half after the other.  A row tile's first scores do not wait for the results of
        // the one before to be out, which are elsewhere in tensor memory; they come behind both halves' values, since their queries may not be there yet.
        int before = 0;
        bool started = false;   // tile it - 1 was a row tile's first: its values begin the sums
        for (uint32_t it = 0; ok && (halves || before); ++it) {
            const bool begins = halves && first, ends = last != 0;
            const int st = it % STAGES, sv = (it + STAGES - 1) % STAGES;
            if (halves && !begins) ok = mbar_wait_warp(&k_full[st], (it / STAGES) & 1u, &abort_flag);
            if (ok && before) ok = mbar_wait_warp(&v_full[sv], ((it - 1) / STAGES) & 1u, &abort_flag);
#pragma unroll 1
            for (int half = 0; half < before; ++half) {
                ok = mbar_wait_warp(&p_full[half], p_phase[half] & 1u, &abort_flag);
                if (!ok) break;
                p_phase[half] += 1;
                tc_fence_after_sync();
                values(half, sv, started);
                if (half == before - 1) commit(&v_free[sv]);
                if (halves && !begins) {
                    scores(half, st);
                    if (half == halves - 1) commit(&k_free[st]);
                    if (ends) commit(&q_free[half]);
                } else {
                    commit(&o_done[half]);
                }
            }
            if (!ok) break;
            started = false;
            if (begins) {
                ok = mbar_wait_warp(&k_full[st], (it / STAGES) & 1u, &abort_flag);
#pragma unroll 1
                for (int half = 0; half < halves && ok; ++half) {
                    ok = mbar_wait_warp(&q_full[half], q_phase[half] & 1u, &abort_flag);
                    if (!ok) break;
                    q_phase[half] += 1;
                    tc_fence_after_sync();
                    scores(half, st);
                    if (ends) commit(&q_free[half]);
                }
                if (!ok) break;
                commit(&k_free[st]);
                started = true;
            }
            before = halves;
            if (halves) halves = read(it + 1);
        }
    } else if (warp > FETCHER) {
        // ---- queries ------------------------------------------------------------------------
        // 64 rows of each half for a warp, copied as they are (all under way together); then, where bf16 rows have to be brought to fp16's range (as query_row
        // does) or the scale is negative, whose sign goes with them, worked over in place.
        constexpr int LANES = DIM / 8, PER = 32 / LANES, LOADS = HALF / 2 / PER;   // lanes of a row, rows of an instruction, instructions
        const int part = lane % LANES, row_lane = (warp - FETCHER - 1) * (HALF / 2) + lane / LANES;
        const uint32_t flip = (a.scale_log2 < 0.0f) ? 0x80008000u : 0u;
        const int step_t = PER / a.G, step_g = PER - step_t * a.G;
        uint32_t uses[2] = {0, 0}, items = 0;
        bool ok = true;
        Kv8Walk<Tiles> w(a, run.entry, run.skip, run.u1 - run.u0);   // (of their own: the first queries come beside the first pages, scales and codes)
        while (ok && w.next()) {
            const int rows = w.s.m * a.G;
            for (int half = 0; half < 2 && ok; ++half) {
                const int row0 = w.r * ROWS + half * HALF;
                if (row0 >= rows) break;
                ok = mbar_wait_warp(&q_free[half], (uses[half] & 1u) ^ 1u, &abort_flag);
                if (!ok) break;
                uses[half] += 1;
                auto place = [&](int at) { return q_smem + half * OPERAND + (part >> 3) * PANEL + at * 128 + (((part & 7) ^ (at & 7)) << 4); };
                int t = (row0 + row_lane) / a.G, g = row0 + row_lane - t * a.G;
#pragma unroll 4
                for (int k = 0; k < LOADS; ++k) {
                    const int at = row_lane + k * PER;
                    const bool there = row0 + at < rows;
                    const long long from = there ? (w.s.q0 + static_cast<long long>(t)) * a.q_tok + (w.h * a.G + g) * a.q_head + part * 8 : 0;
                    cp_async16(place(at), static_cast<const __half *>(a.q) + from, there);
                    t += step_t;
                    g += step_g;
                    if (g >= a.G) {
                        g -= a.G;
                        t += 1;
                    }
                }
                cp_async_wait_all();
                __syncwarp();
                if (BF16 || flip) {   // four lanes to a row
                    constexpr int MINE = DIM / 32;   // 16-byte pieces of a lane
#pragma unroll 1
                    for (int k = 0; k < HALF / 2 / 8; ++k) {
                        const int at = (warp - FETCHER - 1) * (HALF / 2) + 8 * k + (lane >> 2);
                        uint4 *q[MINE], v[MINE];
#pragma unroll
                        for (int j = 0; j < MINE; ++j) {
                            const int piece = (lane & 3) + 4 * j;   // (of 8 in a panel)
                            q[j] = reinterpret_cast<uint4 *>(q_smem + half * OPERAND + (piece >> 3) * PANEL + at * 128 + (((piece & 7) ^ (at & 7)) << 4));
                            v[j] = *q[j];
                        }
                        float g = 1.0f;
                        if constexpr (BF16) {
                            // the largest magnitude: bf16 magnitudes order as their bits do, two at a time
                            uint32_t top = 0;
#pragma unroll
                            for (int j = 0; j < MINE; ++j) {
                                top = __vmaxu2(top, __vmaxu2(v[j].x & 0x7fff7fffu, v[j].y & 0x7fff7fffu));
                                top = __vmaxu2(top, __vmaxu2(v[j].z & 0x7fff7fffu, v[j].w & 0x7fff7fffu));
                            }
                            top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
                            top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
                            const int e2 = min(max(static_cast<int>(max(top >> 16, top & 0xffffu) >> 7) - 127 - 14, KV8_EXP_MIN), KV8_EXP_MAX);
                            g = __uint_as_float(static_cast<uint32_t>(127 - e2) << 23);
                            if ((lane & 3) == 0) q_exp[items & 1][half * HALF + at] = static_cast<int8_t>(e2);
                        }
#pragma unroll
                        for (int j = 0; j < MINE; ++j) {
                            uint32_t x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if constexpr (BF16) x[e] = half2_bits(__uint_as_float(x[e] << 16) * g, __uint_as_float(x[e] & 0xffff0000u) * g);
                                x[e] ^= flip;
                            }
                            *q[j] = make_uint4(x[0], x[1], x[2], x[3]);
                        }
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[half]);
            }
            items += 1;
        }
    } else if (warp == FETCHER) {
        // ---- codes and scales ----------------------------------------------------------------
        Kv8Fetch<Tiles, ROWS> fetch(a, run, lane);
        uint32_t it = 0;
        bool ok = true;
        Kv8Batch now = fetch.next();
        if (now.tiles) fetch.scales(now);
        Kv8Batch next = fetch.next();
        while (ok && now.tiles) {
            Kv8Batch after = next;
            const float vs = fminf(fmaxf(now.vs, KV8_SCALE_MIN), KV8_SCALE_MAX);
            const float vlog = now.page >= 0 ? log2f(vs) : -INFINITY, vinv = 1.0f / vs;
            int row;
            const bool leader = fetch.leads(now, row);
            const unsigned leaders = __ballot_sync(0xffffffffu, leader);
            for (int t = 0; t < now.tiles; ++t, ++it) {
                const int slot = it % INFOS;
                ok = mbar_wait_warp(&info_free[slot], ((it / INFOS) & 1u) ^ 1u, &abort_flag);
                if (!ok) break;
                const bool mine = lane / GROUPS == t;
                if (mine) {
                    info[slot].ks[lane % GROUPS] = now.ks;
                    info[slot].vlog[lane % GROUPS] = vlog;
                    info[slot].vinv[lane % GROUPS] = vinv;
                }
                // (the end, pages that are missing, and what is before a window: tiles of which some codes are not there)
                const unsigned there = __ballot_sync(0xffffffffu, now.page >= 0);
                if (lane == 0) {
                    info[slot].first = now.first && t == 0;
                    info[slot].last = now.last && t == now.tiles - 1;
                    info[slot].tok0 = now.tok0 + t * KEYS;
                    info[slot].q0 = now.q0;
                    info[slot].len = now.len;
                    info[slot].m = now.m;
                    info[slot].r = now.r;
                    info[slot].h = now.h;
                    info[slot].slot = now.slot;
                }
                if (lane == 0) info[slot].end = (now.tok0 + (t + 1) * KEYS > now.hi || ((there >> (t * GROUPS)) & 0xffu) != 0xffu) ? 1 : 0;
                __syncwarp();
                if (lane == 0) mbar_arrive(&info_full[slot]);
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    ok = mbar_wait_warp(&code_free[kv], (it & 1u) ^ 1u, &abort_flag);
                    if (!ok) break;
                    if (lane == 0) {
                        fills[kv] = it + 1;
                        mbar_arrive_expect_tx(&code_full[kv], __popc((leaders >> (t * GROUPS)) & 0xffu) * fetch.box * DIM);
                    }
                    __syncwarp();
                    if (mine && leader) tma_load_2d(codes + kv * (KEYS * DIM) + (lane % GROUPS) * (GROUP * DIM), kv ? &vmap : &kmap, &code_full[kv], 0, row);
                    __syncwarp();
                }
                if (!ok) break;
                if (t == 0 && next.tiles) {   // (behind this batch's first copies, which need not wait for the next one's pages)
                    fetch.scales(next);
                    after = fetch.next();
                }
            }
            now = next;
            next = after;
        }
        if (ok) {
            const int slot = it % INFOS;
            ok = mbar_wait_warp(&info_free[slot], ((it / INFOS) & 1u) ^ 1u, &abort_flag);
            if (ok && lane == 0) {
                info[slot].end = -1;
                mbar_arrive(&info_full[slot]);
            }
        }
        if (lane == 0 && run.u0 < run.u1) kv8_cut(fetch.w, run.total, run.u1, run.ctas);
        __syncwarp();
    }
    __syncthreads();
    if (abort_flag) {
        if (tid == 0) {
            atomicOr(a.err, KV8_ERR_ATTEND_TIMEOUT);
            // copies that are still in flight land before the shared memory is given back
            volatile int scratch = 0;
            for (int kv = 0; kv < 2; ++kv)
                if (fills[kv]) mbar_wait(&code_full[kv], (fills[kv] - 1u) & 1u, &scratch);
        }
        if (warp == ISSUER) {
            volatile int scratch = 0;
            if (elect_one()) umma_commit(&drain_bar);
            __syncwarp();
            mbar_wait(&drain_bar, 0, &scratch);
        }
        __syncthreads();
    }
    if (warp == ISSUER) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

int ctas_of(int sm_count) { return std::min(sm_count, KV8_MAX_CTAS / 2); }

template <int DIM, int FMT, bool BF16>
bool launch_tiles(const Kv8Attend &a, int sm_count, cudaStream_t s) {
    const Kv8 &c = a.c;
    CUtensorMap km, vm;
    const long long rows = (static_cast<long long>(c.num_pages) * c.heads) << c.ps_shift;
    if (!make_code_tensor_map(c.code[0], rows, DIM, c.page_size(), &km) || !make_code_tensor_map(c.code[1], rows, DIM, c.page_size(), &vm)) return false;
    auto kernel = kv8_tiles_kernel<DIM, FMT, BF16>;
    if (!ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), smem_bytes(DIM))) return false;
    launch_dependent(kernel, dim3(static_cast<unsigned>(ctas_of(sm_count))), THREADS, smem_bytes(DIM), s, km, vm, a);
    return true;
}

}  // namespace

size_t kv8_tiles_scratch(int d) { return sizeof(float) * KV8_MAX_CTAS * ROWS * (static_cast<size_t>(d) + 2); }

int launch_kv8_tiles(const Kv8Attend &a, int fmt, int dtype, int sm_count, cudaStream_t s) {
    const bool bf = dtype == EOSQ_BF16, i8 = fmt == EOSQ_KV_INT8;
    bool ok;
    if (a.c.d_shift == 7) {
        if (i8) ok = bf ? launch_tiles<128, EOSQ_KV_INT8, true>(a, sm_count, s) : launch_tiles<128, EOSQ_KV_INT8, false>(a, sm_count, s);
        else ok = bf ? launch_tiles<128, EOSQ_KV_E4M3, true>(a, sm_count, s) : launch_tiles<128, EOSQ_KV_E4M3, false>(a, sm_count, s);
    } else {
        if (i8) ok = bf ? launch_tiles<64, EOSQ_KV_INT8, true>(a, sm_count, s) : launch_tiles<64, EOSQ_KV_INT8, false>(a, sm_count, s);
        else ok = bf ? launch_tiles<64, EOSQ_KV_E4M3, true>(a, sm_count, s) : launch_tiles<64, EOSQ_KV_E4M3, false>(a, sm_count, s);
    }
    return ok ? EOSQ_OK : EOSQ_ERR_CUDA;
}

void launch_kv8_tiles_join(const Kv8Attend &a, int dtype, int sm_count, cudaStream_t s) { launch_join<ROWS>(a, dtype, ctas_of(sm_count), s); }

}  // namespace eosq
