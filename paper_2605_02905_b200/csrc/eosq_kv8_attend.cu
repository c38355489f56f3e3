// Attention over the 8-bit paged cache for few query rows per KV head (a decoding step: one token, a handful of grouped heads), and the
// kernel that joins partial results.
#include <algorithm>

#include <cuda_bf16.h>

#include "eosq_kv8.cuh"
#include "eosq_sm100.cuh"

namespace eosq {

using namespace sm100;

namespace {

// A CTA takes a run of units (Kv8Tiles): one warp fetches tiles of 64 tokens, keys and values, into a ring in shared memory; four
// warps work on 16 tokens of every tile each, with statistics and sums of their own, which meet at the end of a row tile.
constexpr int ROWS = 16, KEYS = 64, GROUP = 16;         // query rows; tokens of a tile; tokens of a warp's share, all in one page
constexpr int WORKERS = KEYS / GROUP, THREADS = 32 * (WORKERS + 1);
constexpr int STAGES = 4, CTAS_PER_SM = 2;
using Tiles = Kv8Tiles<ROWS, KEYS>;

struct TileInfo {
    int first, last;        // of the CTA's run within one row tile
    int tok0;               // the tile's first position
    int q0, len, m, r, h;   // the entry's queries, its length; row tile, KV head
    int slot;               // -1: the whole row tile is this CTA's, else the slot of its partial result
    float ks[WORKERS], vlog[WORKERS], vinv[WORKERS];   // per 16 tokens: key scale, log2 of the value scale and its inverse
};

constexpr size_t SUM_BYTES = sizeof(float) * WORKERS * ROWS * (128 + 4);   // the workers' sums; before that the units of every entry
static_assert(SUM_BYTES >= sizeof(int) * EOSQ_KV8_MAX_SEQS, "units of every entry");
constexpr size_t smem_bytes(int d) { return 1024 + static_cast<size_t>(STAGES) * KEYS * d * 2 + SUM_BYTES; }

__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// NQ query values of a row, as fp16.  bf16 values are first multiplied by a power of two that brings the row's largest to 2^14 .. 2^15:
// fp16 then holds all that are at least 2^-28 of it exactly, and smaller ones to 2^-39 of it.  Its inverse goes with the scale.
template <bool BF16, int NQ>
__device__ __forceinline__ float query_row(const void *p, uint32_t (&v)[NQ / 2], bool live) {
    if (!live) {
#pragma unroll
        for (int i = 0; i < NQ / 2; ++i) v[i] = 0u;
    } else {
#pragma unroll
        for (int i = 0; i < NQ / 8; ++i) {
            const uint4 w = reinterpret_cast<const uint4 *>(p)[i];
            v[4 * i] = w.x;
            v[4 * i + 1] = w.y;
            v[4 * i + 2] = w.z;
            v[4 * i + 3] = w.w;
        }
    }
    if constexpr (!BF16) return 1.0f;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < NQ / 2; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(v[i] << 16)), fabsf(__uint_as_float(v[i] & 0xffff0000u))));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127 - 14, -100), 100);
    const float f = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
    for (int i = 0; i < NQ / 2; ++i) v[i] = half2_bits(__uint_as_float(v[i] << 16) * f, __uint_as_float(v[i] & 0xffff0000u) * f);
    return __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
}

template <int DIM, int FMT, bool BF16>
__global__ void __launch_bounds__(THREADS, CTAS_PER_SM) kv8_rows_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                                          const Kv8Attend a) {
    extern __shared__ uint8_t rows_smem[];
    __shared__ __align__(8) uint64_t full_bar[STAGES], empty_bar[STAGES], join_bar;
    __shared__ TileInfo info[STAGES];
    __shared__ volatile int abort_flag;
    __shared__ uint32_t fills[STAGES];
    __shared__ float top_s[WORKERS][ROWS], sum_s[WORKERS][ROWS];
    constexpr int TILE = KEYS * DIM;   // bytes of a tile's keys, or values
    uint8_t *stages = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(rows_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    float *sums = reinterpret_cast<float *>(stages + STAGES * TILE * 2);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Kv8 &c = a.c;
    if (tid == 0) {
        tma_prefetch_desc(&kmap);
        tma_prefetch_desc(&vmap);
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], WORKERS);
            fills[s] = 0;
        }
        mbar_init(&join_bar, WORKERS);
        abort_flag = 0;
        fence_mbar_init();
    }
    pdl_wait();
    const Kv8Run run = kv8_run<Tiles, THREADS>(a, reinterpret_cast<int *>(sums));

    if (warp == WORKERS) {
        uint32_t it = 0;
        bool ok = true;
        Kv8Walk<Tiles> w(a, run.entry, run.skip, run.u1 - run.u0);
        const int box = min(c.page_size(), KEYS);   // what one page gives to a tile
        while (ok && w.next()) {
            const Kv8Seq &s = w.s;
            const int32_t *pages = c.table + static_cast<size_t>(s.row) * c.max_pages;
            int lo, hi;
            Tiles::span(a, s, w.r * ROWS / a.G, min(s.m - 1, (w.r * ROWS + ROWS - 1) / a.G), lo, hi);
            for (int t = 0; t < w.take; ++t, ++it) {
                const int st = it % STAGES;
                const int tok0 = (w.tile0 + w.from + t) * KEYS;
                // the page of each 16 tokens, and its scales
                float ks = 0.0f, vs = 1.0f, vlog = -INFINITY;
                int page = -1;
                const int tok = tok0 + lane * GROUP, box0 = tok & ~(box - 1);
                if (lane < WORKERS && box0 < hi && box0 + box > lo) {
                    page = pages[tok >> c.ps_shift];
                    if (page < 0 || page >= c.num_pages) {
                        raise(c, EOSQ_KV8_BAD_PAGE);
                        page = -1;
                    } else {
                        const size_t slot = static_cast<size_t>(page) * c.heads + w.h;
                        ks = c.scale[0][slot] * (Kv8Unit<FMT>::value * a.scale_log2);
                        vs = fminf(fmaxf(c.scale[1][slot], KV8_SCALE_MIN), KV8_SCALE_MAX) * Kv8Unit<FMT>::value;
                        vlog = log2f(vs);
                    }
                }
                ok = mbar_wait_warp(&empty_bar[st], ((it / STAGES) & 1u) ^ 1u, &abort_flag);
                if (!ok) break;
                const bool leader = page >= 0 && (tok & (box - 1)) == 0;
                const unsigned boxes = __popc(__ballot_sync(0xffffffffu, leader));
                if (lane < WORKERS) {
                    info[st].ks[lane] = ks;
                    info[st].vlog[lane] = vlog;
                    info[st].vinv[lane] = 1.0f / vs;
                }
                if (lane == 0) {
                    info[st].first = t == 0;
                    info[st].last = t == w.take - 1;
                    info[st].tok0 = tok0;
                    info[st].q0 = s.q0;
                    info[st].len = s.len;
                    info[st].m = s.m;
                    info[st].r = w.r;
                    info[st].h = w.h;
                    info[st].slot = w.slot();
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_expect_tx(&full_bar[st], boxes * box * DIM * 2);
                    fills[st] += 1;
                }
                __syncwarp();
                if (leader) {
                    uint8_t *dst = stages + st * TILE * 2 + (tok - tok0) * DIM;
                    const int row = ((page * c.heads + w.h) << c.ps_shift) + (tok & (c.page_size() - 1));
                    tma_load_2d(dst, &kmap, &full_bar[st], 0, row);
                    tma_load_2d(dst + TILE, &vmap, &full_bar[st], 0, row);
                }
                __syncwarp();
            }
        }
        if (lane == 0 && run.u0 < run.u1) kv8_cut(w, run.total, run.u1, run.ctas);
    } else {
        constexpr int STEPS = DIM / 16, WORDS = DIM / 32, OWN = DIM / 4;   // MMA steps over d; words of a token's values per lane; a lane's share of a row
        const int g = lane >> 2, q = lane & 3;                              // (g: row or token; q: which part of it)
        uint32_t qa[STEPS][4];
        float o[4 * WORDS][4], m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f, f0 = 1.0f, f1 = 1.0f;
        int lo0 = 0, hi0 = 0, lo1 = 0, hi1 = 0, lo_all = 0, hi_all = 0, lo_max = 0, hi_min = 0;
        uint32_t joins = 0;
        bool ok = true;
        for (uint32_t it = 0; it < static_cast<uint32_t>(run.u1 - run.u0); ++it) {
            const int st = it % STAGES;
            ok = mbar_wait_warp(&full_bar[st], (it / STAGES) & 1u, &abort_flag);
            if (!ok) break;
            const TileInfo &ti = info[st];
            const int m = ti.m, r = ti.r, h = ti.h, rows = m * a.G, slot = ti.slot, q0 = ti.q0;
            const bool last = ti.last != 0;
            if (ti.first) {
                const int len = ti.len;
                auto row_span = [&](int row, int &lo, int &hi) {
                    lo = hi = 0;
                    if (row < rows) Tiles::span(a, Kv8Seq{0, len, m, 0}, row / a.G, row / a.G, lo, hi);
                };
                const int ra = r * ROWS + g, rb = ra + 8, end = min(rows, r * ROWS + ROWS) - 1;
                row_span(ra, lo0, hi0);
                row_span(rb, lo1, hi1);
                Tiles::span(a, Kv8Seq{0, len, m, 0}, r * ROWS / a.G, end / a.G, lo_all, hi_all);
                int unused;
                row_span(r * ROWS, unused, hi_min);
                row_span(end, lo_max, unused);
                const __half *base = static_cast<const __half *>(a.q);   // (or bf16: two bytes each)
                auto row_at = [&](int row) { return base + (q0 + static_cast<long long>(row / a.G)) * a.q_tok + (h * a.G + row % a.G) * a.q_head + q * OWN; };
                uint32_t v[OWN / 2];
                f0 = query_row<BF16, OWN>(row_at(ra), v, ra < rows);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    qa[s][0] = v[2 * s];
                    qa[s][2] = v[2 * s + 1];
                }
                f1 = query_row<BF16, OWN>(row_at(rb), v, rb < rows);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    qa[s][1] = v[2 * s];
                    qa[s][3] = v[2 * s + 1];
                }
                m0 = m1 = -INFINITY;
                l0 = l1 = 0.0f;
#pragma unroll
                for (int b = 0; b < 4 * WORDS; ++b) o[b][0] = o[b][1] = o[b][2] = o[b][3] = 0.0f;
            }
            const int tok = ti.tok0 + warp * GROUP;
            const float vlog = ti.vlog[warp];
            if (tok < hi_all && tok + GROUP > lo_all && vlog != -INFINITY) {
                const float ks = ti.ks[warp], vinv = ti.vinv[warp];
                const uint8_t *kt = stages + st * TILE * 2 + warp * GROUP * DIM, *vt = kt + TILE;
                // Scores: rows x 16 tokens.  A lane holds a quarter of a token's row, contiguous: which channels an MMA step takes is free as long as
                // queries and keys agree.
                float sc[2][4];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int t = 8 * b + g;
                    uint32_t w[DIM / 16];
                    if constexpr (DIM == 128) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(kt + t * 128 + (((2 * q) ^ (t & 7)) << 4));
                        const uint4 y = *reinterpret_cast<const uint4 *>(kt + t * 128 + (((2 * q + 1) ^ (t & 7)) << 4));
                        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
                        w[4] = y.x; w[5] = y.y; w[6] = y.z; w[7] = y.w;
                    } else {
                        const uint4 x = *reinterpret_cast<const uint4 *>(kt + t * 64 + ((q ^ ((t >> 1) & 3)) << 4));
                        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
                    }
                    sc[b][0] = sc[b][1] = sc[b][2] = sc[b][3] = 0.0f;
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        uint32_t b0, b1;
                        codes_to_half<FMT>(w[s], b0, b1);
                        mma_16816(sc[b], qa[s], b0, b1);
                    }
                }
                // Base-2 logarithms of the weights, value scale included.
                const float k0 = ks * f0, k1 = ks * f1;
                const bool edge = tok < lo_max || tok + GROUP > hi_min;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x0 = fmaf(sc[b][e], k0, vlog), x1 = fmaf(sc[b][2 + e], k1, vlog);
                        if (edge) {
                            const int t = tok + 8 * b + 2 * q + e;
                            if (t < lo0 || t >= hi0) x0 = -INFINITY;
                            if (t < lo1 || t >= hi1) x1 = -INFINITY;
                        }
                        sc[b][e] = x0;
                        sc[b][2 + e] = x1;
                    }
                float t0 = fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[1][0], sc[1][1]));
                float t1 = fmaxf(fmaxf(sc[0][2], sc[0][3]), fmaxf(sc[1][2], sc[1][3]));
                t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, 1));
                t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, 1));
                t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, 2));
                t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, 2));
                if (__any_sync(0xffffffffu, t0 > m0 + KV8_SLACK || t1 > m1 + KV8_SLACK)) {
                    const float n0 = fmaxf(m0, t0), n1 = fmaxf(m1, t1);
                    const float a0 = (n0 == -INFINITY) ? 1.0f : exp2_fast(m0 - n0), a1 = (n1 == -INFINITY) ? 1.0f : exp2_fast(m1 - n1);
                    m0 = n0;
                    m1 = n1;
                    l0 *= a0;
                    l1 *= a1;
#pragma unroll
                    for (int b = 0; b < 4 * WORDS; ++b) {
                        o[b][0] *= a0;
                        o[b][1] *= a0;
                        o[b][2] *= a1;
                        o[b][3] *= a1;
                    }
                }
                const float b0 = (m0 == -INFINITY) ? 0.0f : KV8_SHIFT - m0, b1 = (m1 == -INFINITY) ? 0.0f : KV8_SHIFT - m1;
                float s0 = 0.0f, s1 = 0.0f;
                uint32_t pa[4];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const float p0 = exp2_fast(sc[b][0] + b0), p1 = exp2_fast(sc[b][1] + b0);
                    const float p2 = exp2_fast(sc[b][2] + b1), p3 = exp2_fast(sc[b][3] + b1);
                    s0 += p0 + p1;
                    s1 += p2 + p3;
                    pa[2 * b] = half2_bits(p0, p1);
                    pa[2 * b + 1] = half2_bits(p2, p3);
                }
                l0 = fmaf(s0, vinv, l0);
                l1 = fmaf(s1, vinv, l1);
                // Values: a lane takes the same DIM / 8 channels of the four tokens whose weights it has; bytes of two tokens are interleaved into pairs.
                uint32_t w[4][WORDS];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = 2 * q + (k & 1) + 8 * (k >> 1);
                    if constexpr (DIM == 128) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(vt + t * 128 + ((g ^ (t & 7)) << 4));
                        w[k][0] = x.x; w[k][1] = x.y; w[k][2] = x.z; w[k][3] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(vt + t * 64 + (((g >> 1) ^ ((t >> 1) & 3)) << 4) + (g & 1) * 8);
                        w[k][0] = x.x; w[k][1] = x.y;
                    }
                }
#pragma unroll
                for (int j = 0; j < WORDS; ++j) {
                    uint32_t v0[4], v1[4];
                    codes_to_half<FMT>(__byte_perm(w[0][j], w[1][j], 0x5140), v0[0], v0[1]);
                    codes_to_half<FMT>(__byte_perm(w[0][j], w[1][j], 0x7362), v0[2], v0[3]);
                    codes_to_half<FMT>(__byte_perm(w[2][j], w[3][j], 0x5140), v1[0], v1[1]);
                    codes_to_half<FMT>(__byte_perm(w[2][j], w[3][j], 0x7362), v1[2], v1[3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) mma_16816(o[4 * j + e], pa, v0[e], v1[e]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty_bar[st]);
            if (!last) continue;

            // The row tile's end: the workers' sums, under one maximum, are added up.
            auto together = [&]() {
                __syncwarp();
                if (lane == 0) mbar_arrive(&join_bar);
                ok = mbar_wait_warp(&join_bar, joins & 1u, &abort_flag);
                joins += 1;
                return ok;
            };
            l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
            l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
            l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
            l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
            if (q == 0) {
                top_s[warp][g] = m0;
                top_s[warp][g + 8] = m1;
                sum_s[warp][g] = l0;
                sum_s[warp][g + 8] = l1;
            }
            if (!together()) break;
            auto top_of = [&](int row) {
                float t = top_s[0][row];
#pragma unroll
                for (int w = 1; w < WORKERS; ++w) t = fmaxf(t, top_s[w][row]);
                return t;
            };
            const float n0 = top_of(g), n1 = top_of(g + 8);
            const float a0 = (m0 == -INFINITY) ? 0.0f : exp2_fast(m0 - n0), a1 = (m1 == -INFINITY) ? 0.0f : exp2_fast(m1 - n1);
            constexpr int PITCH = DIM + 4, PART = DIM / 8;   // lane's channels (2 q + e) * PART + 4 j + i are o[4 j + i][e]
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < WORDS; ++j) {
                        const float f = half ? a1 : a0;
                        float4 v;
                        v.x = o[4 * j][2 * half + e] * f;
                        v.y = o[4 * j + 1][2 * half + e] * f;
                        v.z = o[4 * j + 2][2 * half + e] * f;
                        v.w = o[4 * j + 3][2 * half + e] * f;
                        *reinterpret_cast<float4 *>(sums + (warp * ROWS + g + 8 * half) * PITCH + (2 * q + e) * PART + 4 * j) = v;
                    }
            if (!together()) break;
            const int row = tid >> 3, part = tid & 7, at = r * ROWS + row;
            if (at < rows) {
                const float top = top_of(row);
                float l = 0.0f, v[PART];
#pragma unroll
                for (int k = 0; k < PART; ++k) v[k] = 0.0f;
#pragma unroll
                for (int w = 0; w < WORKERS; ++w) {
                    const float mw = top_s[w][row];
                    l = fmaf(sum_s[w][row], (mw == -INFINITY) ? 0.0f : exp2_fast(mw - top), l);
#pragma unroll
                    for (int k = 0; k < PART; k += 4) {
                        const float4 x = *reinterpret_cast<const float4 *>(sums + (w * ROWS + row) * PITCH + part * PART + k);
                        v[k] += x.x;
                        v[k + 1] += x.y;
                        v[k + 2] += x.z;
                        v[k + 3] += x.w;
                    }
                }
                if (slot < 0) {
                    const float inv = (top == -INFINITY) ? 0.0f : 1.0f / l;
#pragma unroll
                    for (int k = 0; k < PART; ++k) v[k] *= inv;
                    const long long tq = q0 + at / a.G;
                    const int hq = h * a.G + at % a.G;
                    store_row<BF16, PART>(static_cast<__half *>(a.out) + tq * a.o_tok + hq * a.o_head + part * PART, v);
                    if (a.lse && part == 0) a.lse[tq * (c.heads * a.G) + hq] = row_lse(top, l);
                } else {
                    const Kv8Parts<ROWS> parts(a, gridDim.x);
                    const size_t pr = static_cast<size_t>(2 * blockIdx.x + slot) * ROWS + row;
#pragma unroll
                    for (int k = 0; k < PART; k += 4)
                        *reinterpret_cast<float4 *>(parts.o + pr * DIM + part * PART + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
                    if (part == 0) {
                        parts.m[pr] = top;
                        parts.l[pr] = l;
                    }
                }
            }
            if (!together()) break;
        }
    }
    __syncthreads();
    if (abort_flag && tid == 0) {
        atomicOr(a.err, KV8_ERR_ATTEND_TIMEOUT);
        // loads that are still in flight land before the shared memory is given back
        volatile int scratch = 0;
        for (int s = 0; s < STAGES; ++s)
            if (fills[s]) mbar_wait(&full_bar[s], (fills[s] - 1u) & 1u, &scratch);
    }
}

int ctas_of(int sm_count) { return std::min(CTAS_PER_SM * sm_count, KV8_MAX_CTAS); }

template <int DIM, int FMT, bool BF16>
bool launch_rows(const CUtensorMap &km, const CUtensorMap &vm, const Kv8Attend &a, int sm_count, cudaStream_t s) {
    auto kernel = kv8_rows_kernel<DIM, FMT, BF16>;
    if (!ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), smem_bytes(DIM))) return false;
    launch_dependent(kernel, dim3(static_cast<unsigned>(ctas_of(sm_count))), THREADS, smem_bytes(DIM), s, km, vm, a);
    return true;
}

}  // namespace

size_t kv8_rows_scratch(int d) { return sizeof(float) * 2 * KV8_MAX_CTAS * ROWS * (static_cast<size_t>(d) + 2); }

int launch_kv8_rows(const Kv8Attend &a, int fmt, int dtype, int sm_count, cudaStream_t s) {
    const Kv8 &c = a.c;
    CUtensorMap km, vm;
    const long long rows = (static_cast<long long>(c.num_pages) * c.heads) << c.ps_shift;
    const int d = 1 << c.d_shift, box = std::min(c.page_size(), KEYS);
    if (!make_code_tensor_map(c.code[0], rows, d, box, &km) || !make_code_tensor_map(c.code[1], rows, d, box, &vm)) return EOSQ_ERR_CUDA;
    const bool bf = dtype == EOSQ_BF16, i8 = fmt == EOSQ_KV_INT8;
    bool ok;
    if (d == 128) {
        if (i8) ok = bf ? launch_rows<128, EOSQ_KV_INT8, true>(km, vm, a, sm_count, s) : launch_rows<128, EOSQ_KV_INT8, false>(km, vm, a, sm_count, s);
        else ok = bf ? launch_rows<128, EOSQ_KV_E4M3, true>(km, vm, a, sm_count, s) : launch_rows<128, EOSQ_KV_E4M3, false>(km, vm, a, sm_count, s);
    } else {
        if (i8) ok = bf ? launch_rows<64, EOSQ_KV_INT8, true>(km, vm, a, sm_count, s) : launch_rows<64, EOSQ_KV_INT8, false>(km, vm, a, sm_count, s);
        else ok = bf ? launch_rows<64, EOSQ_KV_E4M3, true>(km, vm, a, sm_count, s) : launch_rows<64, EOSQ_KV_E4M3, false>(km, vm, a, sm_count, s);
    }
    return ok ? EOSQ_OK : EOSQ_ERR_CUDA;
}

void launch_kv8_rows_join(const Kv8Attend &a, int dtype, int sm_count, cudaStream_t s) { launch_join<ROWS>(a, dtype, ctas_of(sm_count), s); }

}  // namespace eosq
