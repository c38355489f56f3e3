// Attention over the 8-bit paged cache for many query rows per KV head (a prompt's chunk, cross attention): tcgen05 products with the
// scores, the weights and the sums in tensor memory.
#include <algorithm>

#include "eosq_kv8.cuh"
#include "eosq_sm100.cuh"

namespace eosq {

using namespace sm100;

namespace {

// A CTA takes a run of units (Kv8Tiles): 256 query rows, in two halves of 128, against tiles of 128 tokens.
//   warps 0-3, 4-7   the halves' weights, a row per thread: scores out of tensor memory, weights back into it (in the scores' place, as the
//                    A operand of the second product), maximum and sum in registers; queries in, results out
//   warps 8-11       turn codes into fp16 operands
//   warp 12          issues the products; while one half's weights are made, the other half's products run
//   warp 13          fetches codes, a tile ahead, and the scales
// The weights are the bottleneck: 2^x of 128 x 256 scores is 2048 cycles of an SM's special function units, as many as the two products take.
constexpr int ROWS = 256, HALF = 128, KEYS = KV8_KEYS, GROUP = KV8_GROUP, GROUPS = KV8_GROUPS;
constexpr int LOADER = 8, ISSUER = 12, FETCHER = 13, THREADS = 32 * 14, STAGES = 2, INFOS = 4;
constexpr int COST = 2;
using Tiles = Kv8Tiles<ROWS, KEYS, COST>;

struct TileInfo {
    int end;   // 1: some of the tokens may be behind the sequence's last; -1: the run has ended, there is no tile
    float ks[GROUPS], vlog[GROUPS], vinv[GROUPS];   // per 16 tokens: key scale, log2 of the value scale (-infinity: not there) and its inverse
};

constexpr size_t operand_bytes(int d) { return static_cast<size_t>(HALF) * d * 2; }   // 128 rows of fp16
constexpr size_t smem_bytes(int d) { return 1024 + (2 + 2 * STAGES) * operand_bytes(d) + 2 * static_cast<size_t>(KEYS) * d; }
static_assert(smem_bytes(128) + 1400 <= 232448, "shared memory of a CTA, with the barriers and scales");
static_assert(2 * STAGES * operand_bytes(64) >= sizeof(int) * EOSQ_KV8_MAX_SEQS, "units of every entry");

__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <int DIM, int FMT, bool BF16>
__global__ void __launch_bounds__(THREADS, 1) kv8_tiles_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                                  const Kv8Attend a) {
    extern __shared__ uint8_t tiles_smem[];
    __shared__ __align__(8) uint64_t q_full[2], s_full[2], p_full[2], o_done[2], k_full[STAGES], v_full[STAGES], k_free[STAGES], v_free[STAGES], info_full[INFOS],
        info_free[INFOS], code_full[2], code_free[2], drain_bar;
    __shared__ TileInfo info[INFOS];
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
            mbar_init(&q_full[i], 4);
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
            mbar_init(&info_free[i], 12);
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
        uint8_t *q_mine = q_smem + half * OPERAND + row_in * 128;
        Kv8Walk<Tiles> w(a, run.entry, run.skip, run.u1 - run.u0);
        uint32_t it = 0, s_phase = 0, o_phase = 0;
        bool ok = true;
        while (ok && w.next()) {
            const int row = w.r * ROWS + half * HALF + row_in, rows = w.s.m * a.G;
            const bool active = w.r * ROWS + half * HALF < rows, live = row < rows;   // (active: some row of this half)
            const int t_of = live ? row / a.G : 0, hq = w.h * a.G + (live ? row % a.G : 0);
            int lo = 0, hi = 0;
            float f = 1.0f;
            if (active) {
                // The queries: this row's, as fp16; bf16 rows brought to its range (query_row does the same for a quarter of a row).  The scale's sign goes with them.
                const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const __half *>(a.q) + (w.s.q0 + static_cast<long long>(t_of)) * a.q_tok + hq * a.q_head);
                float g = 1.0f;
                if constexpr (BF16) {
                    float top = 0.0f;
                    if (live) {
#pragma unroll 4
                        for (int k = 0; k < DIM / 8; ++k) {
                            const uint4 v = src[k];
                            const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(x[e] << 16)), fabsf(__uint_as_float(x[e] & 0xffff0000u))));
                        }
                    }
                    const int e2 = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127 - 14, -100), 100);
                    g = __uint_as_float(static_cast<uint32_t>(127 - e2) << 23);
                    f = __uint_as_float(static_cast<uint32_t>(127 + e2) << 23);
                }
                const uint32_t flip = (a.scale_log2 < 0.0f) ? 0x80008000u : 0u;
#pragma unroll 4
                for (int k = 0; k < DIM / 8; ++k) {
                    const uint4 v = live ? src[k] : make_uint4(0, 0, 0, 0);
                    uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (BF16) x[e] = half2_bits(__uint_as_float(x[e] << 16) * g, __uint_as_float(x[e] & 0xffff0000u) * g);
                        x[e] ^= flip;
                    }
                    *reinterpret_cast<uint4 *>(q_mine + (k >> 3) * PANEL + (((k & 7) ^ (row_in & 7)) << 4)) = make_uint4(x[0], x[1], x[2], x[3]);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[half]);
                if (live) Tiles::span(a, w.s, t_of, t_of, lo, hi);
            }
            float m = -INFINITY, l = 0.0f;
            const float kscale = scale * f;
            for (int t = 0; t < w.take; ++t, ++it) {
                const int slot = it % INFOS;
                ok = mbar_wait_warp(&info_full[slot], (it / INFOS) & 1u, &abort_flag);
                if (!ok) break;
                if (active) {
                    const TileInfo &ti = info[slot];
                    ok = mbar_wait_warp(&s_full[half], s_phase & 1u, &abort_flag);
                    if (!ok) break;
                    s_phase += 1;
                    tc_fence_after_sync();
                    const int tok0 = (w.tile0 + w.from + t) * KEYS;
                    const bool edge = __any_sync(0xffffffffu, live && (tok0 < lo || tok0 + KEYS > hi));
                    // A row's base-2 logarithms are s * ks + vlog, with a key and a value scale for every 16 tokens.  (ks is kept above
                    // zero, so that masked scores stay -infinity under a scale of zero.)  The scores are read twice, 32 at a time: first the largest, ...
                    auto masked = [&](uint32_t (&x)[32], int at) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (at + e < lo || at + e >= hi) x[e] = 0xff800000u;   // -infinity
                    };
                    auto ks_of = [&](int g) { return fmaxf(ti.ks[g] * kscale, 1e-37f); };
                    float top = -INFINITY;
                    auto largest = [&](uint32_t (&x)[32], int k) {
                        if (edge) masked(x, tok0 + 32 * k);
#pragma unroll
                        for (int gg = 0; gg < 2; ++gg) {
                            float t0 = __uint_as_float(x[16 * gg]), t1 = __uint_as_float(x[16 * gg + 1]);
#pragma unroll
                            for (int e = 2; e < GROUP; e += 2) {
                                t0 = fmaxf(t0, __uint_as_float(x[16 * gg + e]));
                                t1 = fmaxf(t1, __uint_as_float(x[16 * gg + e + 1]));
                            }
                            const int g = 2 * k + gg;
                            top = fmaxf(top, fmaf(fmaxf(t0, t1), ks_of(g), ti.vlog[g]));
                        }
                    };
                    uint32_t x[32], y[32];
                    tmem_ld32(s_at, x);
                    tmem_ld_wait(x);
#pragma unroll 1
                    for (int k = 0; k < KEYS / 32; k += 2) {
                        tmem_ld32(s_at + 32 * (k + 1), y);
                        largest(x, k);
                        tmem_ld_wait(y);
                        tmem_ld32(s_at + 32 * ((k + 2) % (KEYS / 32)), x);   // (at the end the first ones again)
                        largest(y, k + 1);
                        tmem_ld_wait(x);
                    }
                    if (__any_sync(0xffffffffu, top > m + KV8_SLACK)) {
                        const float n = fmaxf(m, top), by = (n == -INFINITY) ? 1.0f : exp2_fast(m - n);
                        m = n;
                        l *= by;
                        if (t > 0) {   // the products before have completed: the issuer's scores of this tile came behind them
#pragma unroll 1
                            for (int k = 0; k < DIM / 32; ++k) {
                                uint32_t o[32];
                                tmem_ld32(o_at + 32 * k, o);
                                tmem_ld_wait(o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                                tmem_st32(o_at + 32 * k, o);
                            }
                        }
                    }
                    const float b = (m == -INFINITY) ? 0.0f : KV8_SHIFT - m;
                    // Below, s * ks + (vlog - m + shift) is rounded once, m before: of logarithms beyond 2^22 the difference could pass fp16's range.  There
                    // every logarithm is rounded as m was.
                    const bool far = __any_sync(0xffffffffu, fabsf(m) > 4194304.0f && m != -INFINITY);
                    // ... then the weights, 32 of them into the place of 16 scores that have been read.
                    auto weights = [&](uint32_t (&x)[32], int k) {
                        if (edge) masked(x, tok0 + 32 * k);
                        uint32_t p[16];
#pragma unroll
                        for (int gg = 0; gg < 2; ++gg) {
                            const int g = 2 * k + gg;
                            float kf = ks_of(g), cf = ti.vlog[g] + b;
                            if (far) {
#pragma unroll
                                for (int e = 0; e < GROUP; ++e) x[16 * gg + e] = __float_as_uint(fmaf(__uint_as_float(x[16 * gg + e]), kf, ti.vlog[g]));
                                kf = 1.0f;
                                cf = b;
                            }
                            const uint64_t k2 = pair_of(kf, kf), c2 = pair_of(cf, cf);
                            uint64_t sum = 0;
#pragma unroll
                            for (int e = 0; e < GROUP; e += 2) {
                                float y0, y1;
                                unpair(fma_pair(pair_of(__uint_as_float(x[16 * gg + e]), __uint_as_float(x[16 * gg + e + 1])), k2, c2), y0, y1);
                                y0 = exp2_fast(y0);
                                y1 = exp2_fast(y1);
                                sum = add_pair(sum, pair_of(y0, y1));
                                p[8 * gg + (e >> 1)] = half2_bits(y0, y1);
                            }
                            float s0, s1;
                            unpair(sum, s0, s1);
                            l = fmaf(s0 + s1, ti.vinv[g], l);
                        }
                        tmem_st16(s_at + 16 * k, p);
                    };
#pragma unroll 1
                    for (int k = 0; k < KEYS / 32; k += 2) {
                        tmem_ld32(s_at + 32 * (k + 1), y);
                        weights(x, k);
                        tmem_ld_wait(y);
                        if (k + 2 < KEYS / 32) tmem_ld32(s_at + 32 * (k + 2), x);
                        weights(y, k + 1);
                        tmem_ld_wait(x);
                    }
                    tmem_st_wait();
                    tc_fence_before_sync();
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&info_free[slot]);
                    if (active) mbar_arrive(&p_full[half]);
                }
            }
            if (!ok) break;
            if (!active) continue;
            ok = mbar_wait_warp(&o_done[half], o_phase & 1u, &abort_flag);
            if (!ok) break;
            o_phase += 1;
            tc_fence_after_sync();
            const int slot = w.slot();
            const float inv = (slot >= 0) ? 1.0f : (m == -INFINITY ? 0.0f : 1.0f / l);
            const long long tq = w.s.q0 + static_cast<long long>(t_of);
            const Kv8Parts<ROWS> parts(a, gridDim.x);
            const size_t pr = static_cast<size_t>(2 * blockIdx.x + max(slot, 0)) * ROWS + half * HALF + row_in;
#pragma unroll 1
            for (int k = 0; k < DIM / 32; ++k) {
                uint32_t o[32];
                float v[32];
                tmem_ld32(o_at + 32 * k, o);
                tmem_ld_wait(o);
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(o[e]) * inv;
                if (live) {
                    if (slot < 0) {
                        store_row<BF16, 32>(static_cast<__half *>(a.out) + tq * a.o_tok + hq * a.o_head + 32 * k, v);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4 *>(parts.o + pr * DIM + 32 * k + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                    }
                }
            }
            if (live) {
                if (slot >= 0) {
                    parts.m[pr] = m;
                    parts.l[pr] = l;
                } else if (a.lse) {
                    a.lse[tq * (c.heads * a.G) + hq] = row_lse(m, l);
                }
            }
            tc_fence_before_sync();
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
                uint4 x[LOADS];
#pragma unroll
                for (int k = 0; k < LOADS; ++k) {
                    const int row = k * TOKS + tok_in;
                    const int chunk = (DIM == 128) ? part ^ (row & 7) : part ^ ((row >> 1) & 3);
                    x[k] = *reinterpret_cast<const uint4 *>(codes + kv * (KEYS * DIM) + row * DIM + chunk * 16);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&code_free[kv]);
                ok = mbar_wait_warp(kv ? &v_free[st] : &k_free[st], free_parity, &abort_flag);
                if (!ok) break;
                uint8_t *dst = (kv ? v_smem : k_smem) + st * OPERAND + (part >> 2) * PANEL;
#pragma unroll
                for (int k = 0; k < LOADS; ++k) {
                    const int row = k * TOKS + tok_in;
                    const uint32_t y[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
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
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(kv ? &v_full[st] : &k_full[st]);
            }
        }
    } else if (warp == ISSUER) {
        // ---- products -----------------------------------------------------------------------
        {
            constexpr uint32_t idesc_s = umma_idesc_f16(HALF, KEYS, false, false), idesc_o = umma_idesc_f16(HALF, DIM, false, true);
            const bool issuer = elect_one();
            Kv8Walk<Tiles> w(a, run.entry, run.skip, run.u1 - run.u0);
            uint32_t it = 0, q_phase = 0, p_phase[2] = {0, 0};
            uint32_t q_phases[2] = {0, 0};
            bool ok = true;
            (void)q_phase;
            const uint32_t q_addr = smem_u32(q_smem), k_addr = smem_u32(k_smem), v_addr = smem_u32(v_smem);
            // Scores of one half against the keys of stage st.
            auto scores = [&](int half, int st) {
                if (issuer) {
#pragma unroll
                    for (int k = 0; k < DIM / 16; ++k) {
                        const uint32_t off = (k >> 2) * PANEL + (k & 3) * 32;
                        umma_f16(tmem + half * KEYS, umma_desc_sw128(q_addr + half * OPERAND + off, 16, 1024), umma_desc_sw128(k_addr + st * OPERAND + off, 16, 1024), idesc_s,
                                 k ? 1u : 0u);
                    }
                    umma_commit(&s_full[half]);
                }
                __syncwarp();
            };
            auto values = [&](int half, int st, bool first) {
                if (issuer) {
#pragma unroll
                    for (int k = 0; k < KEYS / 16; ++k)
                        umma_f16_ts(tmem + 256 + half * DIM, tmem + half * KEYS + 8 * k, umma_desc_sw128(v_addr + st * OPERAND + k * 2048, PANEL, 1024), idesc_o,
                                    (first && k == 0) ? 0u : 1u);
                }
                __syncwarp();
            };
            auto commit = [&](uint64_t *bar) {
                if (issuer) umma_commit(bar);
                __syncwarp();
            };
            while (ok && w.next()) {
                const bool two = w.r * ROWS + HALF < w.s.m * a.G;
                const int halves = two ? 2 : 1;
                for (int t = -1; t < w.take && ok; ++t) {
                    // the values of tile t, then the scores of tile t + 1, one half after the other
                    const bool more = t + 1 < w.take;
                    const uint32_t kt = it + t + 1, vt = it + t;
                    if (more) ok = mbar_wait_warp(&k_full[kt % STAGES], (kt / STAGES) & 1u, &abort_flag);
                    if (ok && t >= 0) ok = mbar_wait_warp(&v_full[vt % STAGES], (vt / STAGES) & 1u, &abort_flag);
                    for (int half = 0; half < halves && ok; ++half) {
                        if (t < 0) {
                            ok = mbar_wait_warp(&q_full[half], q_phases[half] & 1u, &abort_flag);
                            q_phases[half] += 1;
                        } else {
                            ok = mbar_wait_warp(&p_full[half], p_phase[half] & 1u, &abort_flag);
                            p_phase[half] += 1;
                        }
                        if (!ok) break;
                        tc_fence_after_sync();
                        if (t >= 0) values(half, vt % STAGES, t == 0);
                        if (t >= 0 && half == halves - 1) commit(&v_free[vt % STAGES]);
                        if (more) {
                            scores(half, kt % STAGES);
                            if (half == halves - 1) commit(&k_free[kt % STAGES]);
                        } else {
                            commit(&o_done[half]);
                        }
                    }
                }
                it += w.take;
            }
        }
    } else {
        // ---- codes and scales ----------------------------------------------------------------
        Kv8Fetch<Tiles, ROWS> fetch(a, run, lane);
        uint32_t it = 0;
        bool ok = true;
        Kv8Batch now = fetch.next();
        if (now.tiles) fetch.scales(now);
        Kv8Batch next = fetch.next();
        while (ok && now.tiles) {
            if (next.tiles) fetch.scales(next);
            const Kv8Batch after = next.tiles ? fetch.next() : next;
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
