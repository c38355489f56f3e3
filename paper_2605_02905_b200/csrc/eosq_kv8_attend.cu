// Attention over the 8-bit paged cache for few query rows per KV head (a decoding step: one token, a handful of grouped heads), and the
// kernel that joins partial results.
#include <algorithm>

#include <cuda_bf16.h>

#include "eosq_kv8.cuh"
#include "eosq_sm100.cuh"

namespace eosq {

using namespace sm100;

namespace {

// A CTA takes a run of units (Kv8Tiles): one warp fetches tiles of 128 tokens, keys and values, into a ring in shared memory; four
// warps work on 32 tokens of every tile each, with statistics and sums of their own, which meet at the end of a row tile.
// Both products have the tokens' side as the MMA's larger one: scores are (16 tokens) x (8 query rows), the sums (16 channels) x (8 rows).
// A product of queries by keys (16 rows, half of them empty with up to 8 heads to a group) would take twice the MMAs, weights and registers: it was
// 573 instructions for 16 tokens and 286 us for 16 x 32768 tokens.
// What bounds it is the memory: those tokens, 8 heads of 128 with four queries each, take 168 us in a graph, 6.4 TB/s of codes (a copy reaches 6.46), with half the issue
// slots in use.  Short of that it is the way to the first tile: 1.4 us (48 entries: 2.4) until a CTA knows its run, 1.3 for a page's number, as much for its scales, 2
// for the codes, 2 for the queries, which wait behind other CTAs' codes; then 1 us a tile until the code has been fetched.  48 x 64 .. 8192 tokens: 40 us, 26.5 at a copy's rate.
// Queries brought by the fetching warp with the codes gained 2 % there and lost 3 % at d = 64 and on one short sequence; codes asked for before
// their scales are known gained nothing.
constexpr int KEYS = KV8_KEYS, GROUP = KV8_GROUP, GROUPS = KV8_GROUPS;
constexpr int WORKERS = 4, SHARE = KEYS / WORKERS / GROUP, THREADS = 32 * (WORKERS + 1);
constexpr int CTAS_PER_SM = 2, COST = 2;   // (one unit or three for a row tile: 43.5 and 41.4 us for those 48 sequences, 39.8 so)

struct TileInfo {
    int first, last;        // of the CTA's run within one row tile; first = -1: the run has ended, there is no tile
    int tok0;               // the tile's first position
    int q0, len, m, r, h;   // the entry's queries, its length; row tile, KV head
    int slot;               // -1: the whole row tile is this CTA's, else the slot of its partial result
    float ks[GROUPS], vlog[GROUPS], vinv[GROUPS];   // per 16 tokens: key scale, log2 of the value scale and its inverse
};

constexpr int stages_of(int d, int nb) { return (nb == 1 ? 3 : 2) * (128 / d); }
constexpr size_t sums_bytes(int d, int nb) { return sizeof(float) * WORKERS * (WORKERS - 1) * (d / 4) * 8 * nb; }
constexpr size_t smem_bytes(int d, int nb) { return 1024 + static_cast<size_t>(stages_of(d, nb)) * KEYS * d * 2 + sums_bytes(d, nb); }
static_assert(2 * 2 * KEYS * 128 >= sizeof(int) * EOSQ_KV8_MAX_SEQS, "units of every entry, where the tiles will be");

// The transpose of an 8 x 8 matrix of fp16, a row's pair to a lane.
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
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
    const int e = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127 - 14, KV8_EXP_MIN), KV8_EXP_MAX);
    const float f = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
    for (int i = 0; i < NQ / 2; ++i) v[i] = half2_bits(__uint_as_float(v[i] << 16) * f, __uint_as_float(v[i] & 0xffff0000u) * f);
    return __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
}

// NB: query rows of a row tile, in eights.
template <int DIM, int FMT, bool BF16, int NB>
__global__ void __launch_bounds__(THREADS, CTAS_PER_SM) kv8_rows_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                                                                          const Kv8Attend a) {
    constexpr int ROWS = 8 * NB, STAGES = stages_of(DIM, NB);
    using Tiles = Kv8Tiles<ROWS, KEYS, COST>;
    extern __shared__ uint8_t rows_smem[];
    __shared__ __align__(8) uint64_t full_bar[STAGES], empty_bar[STAGES], put_bar, got_bar;
    __shared__ TileInfo info[STAGES];
    __shared__ volatile int abort_flag;
    __shared__ uint32_t fills[STAGES];
    __shared__ float top_s[2][WORKERS][ROWS], sum_s[2][WORKERS][ROWS];
    constexpr int TILE = KEYS * DIM;   // bytes of a tile's keys, or values
    uint8_t *stages = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(rows_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    float4 *sums = reinterpret_cast<float4 *>(stages + STAGES * TILE * 2);
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
        mbar_init(&put_bar, WORKERS);
        mbar_init(&got_bar, WORKERS);
        abort_flag = 0;
        fence_mbar_init();
    }
    pdl_wait();
    const Kv8Run run = kv8_run<Tiles, THREADS>(a, reinterpret_cast<int *>(stages));
    fence_proxy_async_smem();   // the entries' units have been read; from here on copies write there
    __syncthreads();

    if (warp == WORKERS) {
        // The pages of the batch after next and the scales of the next one are on their way while this one's codes are being fetched.
        Kv8Fetch<Tiles, ROWS> fetch(a, run, lane);
        uint32_t it = 0;
        bool ok = true;
        Kv8Batch now = fetch.next();
        if (now.tiles) fetch.scales(now);
        Kv8Batch next = fetch.next();
        while (ok && now.tiles) {
            Kv8Batch after = next;
            const float ks = BF16 ? now.ks : now.ks * a.scale_log2;   // (with bf16 the scale goes with the row's power of two first, which it may well cancel)
            const float vs = fminf(fmaxf(now.vs, KV8_SCALE_MIN), KV8_SCALE_MAX);
            const float vlog = now.page >= 0 ? log2f(vs) : -INFINITY, vinv = 1.0f / vs;
            int row;
            const bool leader = fetch.leads(now, row);
            const unsigned leaders = __ballot_sync(0xffffffffu, leader);
            for (int t = 0; t < now.tiles; ++t, ++it) {
                const int st = it % STAGES;
                ok = mbar_wait_warp(&empty_bar[st], ((it / STAGES) & 1u) ^ 1u, &abort_flag);
                if (!ok) break;
                const bool mine = lane / GROUPS == t;
                if (mine) {
                    info[st].ks[lane % GROUPS] = ks;
                    info[st].vlog[lane % GROUPS] = vlog;
                    info[st].vinv[lane % GROUPS] = vinv;
                }
                if (lane == 0) {
                    info[st].first = now.first && t == 0;
                    info[st].last = now.last && t == now.tiles - 1;
                    info[st].tok0 = now.tok0 + t * KEYS;
                    info[st].q0 = now.q0;
                    info[st].len = now.len;
                    info[st].m = now.m;
                    info[st].r = now.r;
                    info[st].h = now.h;
                    info[st].slot = now.slot;
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_expect_tx(&full_bar[st], __popc((leaders >> (t * GROUPS)) & ((1u << GROUPS) - 1u)) * fetch.box * DIM * 2);
                    fills[st] += 1;
                }
                __syncwarp();
                if (mine && leader) {
                    uint8_t *dst = stages + st * TILE * 2 + (lane % GROUPS) * (GROUP * DIM);
                    tma_load_2d(dst, &kmap, &full_bar[st], 0, row);
                    tma_load_2d(dst + TILE, &vmap, &full_bar[st], 0, row);
                }
                __syncwarp();
                if (t == 0 && next.tiles) {   // (behind this batch's first copies, which need not wait for the next one's pages)
                    fetch.scales(next);
                    after = fetch.next();
                }
            }
            now = next;
            next = after;
        }
        if (ok) {
            const int st = it % STAGES;
            ok = mbar_wait_warp(&empty_bar[st], ((it / STAGES) & 1u) ^ 1u, &abort_flag);
            if (ok && lane == 0) {
                info[st].first = -1;
                mbar_arrive(&full_bar[st]);
                fills[st] += 1;
            }
        }
        if (lane == 0 && run.u0 < run.u1) kv8_cut(fetch.w, run.total, run.u1, run.ctas);
    } else {
        constexpr int STEPS = DIM / 16, WORDS = DIM / 32, OWN = DIM / 4;   // MMA steps over d; words of a token's values per lane; a lane's share of a row
        const int g = lane >> 2, q = lane & 3;                              // g: token, channel or, of the queries, row; q: which part, or which two rows
        uint32_t qb[NB][STEPS][2];
        float o[NB][2 * WORDS][4], m[NB][2], l[NB][2], f[NB][2];            // o: channels (8 by 8, two of a word each) x rows 2 q, 2 q + 1
        int lo[NB][2], hi[NB][2], lo_all = 0, hi_all = 0, lo_max = 0, hi_min = 0;
        // Rows of the row tile `tile_of`: query and head (row - query * G) of the one that this lane loads, and of the two that it holds weights of.
        int tile_of = -1, t_load[NB], h_load[NB], t_row[NB][2], h_row[NB][2];
        uint32_t items = 0;
        bool ok = true, far = false;   // far: some row's maximum is (kv8_far)
        for (uint32_t it = 0;; ++it) {
            const int st = it % STAGES;
            ok = mbar_wait_warp(&full_bar[st], (it / STAGES) & 1u, &abort_flag);
            if (!ok) break;
            const TileInfo &ti = info[st];
            if (ti.first < 0) break;
            const int mq = ti.m, h = ti.h, slot = ti.slot, q0 = ti.q0;
            const bool last = ti.last != 0;
            if (ti.first) {
                const Kv8Seq sq{0, ti.len, mq, 0};
                const int r = ti.r;
                far = false;
                if (r != tile_of) {
                    tile_of = r;
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        t_load[n] = (r * ROWS + 8 * n + g) / a.G;
                        h_load[n] = r * ROWS + 8 * n + g - t_load[n] * a.G;
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            t_row[n][e] = (r * ROWS + 8 * n + 2 * q + e) / a.G;
                            h_row[n][e] = r * ROWS + 8 * n + 2 * q + e - t_row[n][e] * a.G;
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const __half *base = static_cast<const __half *>(a.q);   // (or bf16: two bytes each)
                    uint32_t v[OWN / 2];
                    const float mine =
                        query_row<BF16, OWN>(base + (q0 + static_cast<long long>(t_load[n])) * a.q_tok + (h * a.G + h_load[n]) * a.q_head + q * OWN, v, t_load[n] < mq);
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        qb[n][s][0] = v[2 * s];
                        qb[n][s][1] = v[2 * s + 1];
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        f[n][e] = BF16 ? __shfl_sync(0xffffffffu, mine, (2 * q + e) * 4) * a.scale_log2 : 1.0f;
                        lo[n][e] = hi[n][e] = 0;
                        if (t_row[n][e] < mq) Tiles::span(a, sq, t_row[n][e], t_row[n][e], lo[n][e], hi[n][e]);
                        m[n][e] = -INFINITY;
                        l[n][e] = 0.0f;
                    }
#pragma unroll
                    for (int b = 0; b < 2 * WORDS; ++b) o[n][b][0] = o[n][b][1] = o[n][b][2] = o[n][b][3] = 0.0f;
                }
                const int t_first = __shfl_sync(0xffffffffu, t_load[0], 0), t_last = min(__shfl_sync(0xffffffffu, t_load[NB - 1], 28), mq - 1);   // (of row 8 NB - 1)
                Tiles::span(a, sq, t_first, t_last, lo_all, hi_all);
                int unused;
                Tiles::span(a, sq, t_first, t_first, unused, hi_min);
                Tiles::span(a, sq, t_last, t_last, lo_max, unused);
            }
            const int tok = ti.tok0 + warp * SHARE * GROUP;
            if (tok < hi_all && tok + SHARE * GROUP > lo_all) {
                const uint8_t *kt = stages + st * TILE * 2 + warp * SHARE * GROUP * DIM, *vt = kt + TILE;
                // Scores.  A lane holds a quarter of a token's row, contiguous: which channels an MMA step takes is free as long as queries and keys agree.
                float sc[SHARE][NB][4];   // rows 2 q, 2 q + 1 of token g, then of token g + 8
#pragma unroll
                for (int p = 0; p < SHARE; ++p) {
                    uint32_t w[2][DIM / 16];
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int t = 16 * p + 8 * b + g;
                        if constexpr (DIM == 128) {
                            const uint4 x = *reinterpret_cast<const uint4 *>(kt + t * 128 + (((2 * q) ^ (t & 7)) << 4));
                            const uint4 y = *reinterpret_cast<const uint4 *>(kt + t * 128 + (((2 * q + 1) ^ (t & 7)) << 4));
                            w[b][0] = x.x; w[b][1] = x.y; w[b][2] = x.z; w[b][3] = x.w;
                            w[b][4] = y.x; w[b][5] = y.y; w[b][6] = y.z; w[b][7] = y.w;
                        } else {
                            const uint4 x = *reinterpret_cast<const uint4 *>(kt + t * 64 + ((q ^ ((t >> 1) & 3)) << 4));
                            w[b][0] = x.x; w[b][1] = x.y; w[b][2] = x.z; w[b][3] = x.w;
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NB; ++n) sc[p][n][0] = sc[p][n][1] = sc[p][n][2] = sc[p][n][3] = 0.0f;
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        uint32_t ka[4];
                        codes_to_half<FMT>(w[0][s], ka[0], ka[2]);
                        codes_to_half<FMT>(w[1][s], ka[1], ka[3]);
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma_16816(sc[p][n], ka, qb[n][s][0], qb[n][s][1]);
                    }
                }
                // Base-2 logarithms of the weights, value scale included; a row's largest.
                float top[NB][2];
                bool edge = tok < lo_max || tok + SHARE * GROUP > hi_min;   // some token may be hidden from some row, or not there
#pragma unroll
                for (int p = 0; p < SHARE; ++p) edge |= ti.vlog[warp * SHARE + p] == -INFINITY;
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        top[n][e] = -INFINITY;
#pragma unroll
                        for (int p = 0; p < SHARE; ++p) {
                            const float k = ti.ks[warp * SHARE + p] * f[n][e], v = ti.vlog[warp * SHARE + p];
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                float x = fmaf(sc[p][n][2 * b + e], k, v);
                                if (edge) {
                                    const int t = tok + 16 * p + 8 * b + g;
                                    if (t < lo[n][e] || t >= hi[n][e] || v == -INFINITY) x = -INFINITY;
                                }
                                sc[p][n][2 * b + e] = x;
                                top[n][e] = fmaxf(top[n][e], x);
                            }
                        }
                    }
                bool moved = false;
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) moved |= top[n][e] - m[n][e] > KV8_SLACK;   // (of two minus infinities: no)
                if (__any_sync(0xffffffffu, moved)) {
                    bool mine_far = false;
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float t = top[n][e];
                            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
                            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
                            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
                            const float to = fmaxf(m[n][e], t), by = (to == -INFINITY) ? 1.0f : exp2_fast(m[n][e] - to);
                            m[n][e] = to;
                            mine_far |= kv8_far(to);
                            l[n][e] *= by;
#pragma unroll
                            for (int b = 0; b < 2 * WORDS; ++b) {
                                o[n][b][e] *= by;
                                o[n][b][2 + e] *= by;
                            }
                        }
                    }
                    far = __any_sync(0xffffffffu, mine_far);
                }
                uint32_t pb[SHARE][NB][2];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    float b[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) b[e] = (m[n][e] == -INFINITY) ? 0.0f : KV8_SHIFT - m[n][e];
                    if (far) {   // (a row's arithmetic goes by its own maximum)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (kv8_far(m[n][e])) {
#pragma unroll
                                for (int p = 0; p < SHARE; ++p) {
                                    sc[p][n][e] -= m[n][e];
                                    sc[p][n][2 + e] -= m[n][e];
                                }
                                b[e] = KV8_SHIFT;
                            }
                    }
#pragma unroll
                    for (int p = 0; p < SHARE; ++p) {
                        const float p0 = exp2_fast(sc[p][n][0] + b[0]), p1 = exp2_fast(sc[p][n][1] + b[1]);
                        const float p2 = exp2_fast(sc[p][n][2] + b[0]), p3 = exp2_fast(sc[p][n][3] + b[1]);
                        const float vinv = ti.vinv[warp * SHARE + p];
                        l[n][0] = fmaf(p0 + p2, vinv, l[n][0]);
                        l[n][1] = fmaf(p1 + p3, vinv, l[n][1]);
                        pb[p][n][0] = transposed(half2_bits(p0, p1));
                        pb[p][n][1] = transposed(half2_bits(p2, p3));
                    }
                }
                // Values: a lane takes the same DIM / 8 channels of the four tokens whose weights it has; bytes of two tokens are interleaved into pairs.
#pragma unroll
                for (int p = 0; p < SHARE; ++p) {
                    uint32_t w[4][WORDS];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int t = 16 * p + 2 * q + (k & 1) + 8 * (k >> 1);
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
                        uint32_t va[2][4];   // channels 4 j, 4 j + 1 of the lane's, then 4 j + 2, 4 j + 3
                        codes_to_half<FMT>(__byte_perm(w[0][j], w[1][j], 0x5140), va[0][0], va[0][1]);
                        codes_to_half<FMT>(__byte_perm(w[2][j], w[3][j], 0x5140), va[0][2], va[0][3]);
                        codes_to_half<FMT>(__byte_perm(w[0][j], w[1][j], 0x7362), va[1][0], va[1][1]);
                        codes_to_half<FMT>(__byte_perm(w[2][j], w[3][j], 0x7362), va[1][2], va[1][3]);
                        if (edge) {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                va[0][k] = no_nan<FMT>(va[0][k]);
                                va[1][k] = no_nan<FMT>(va[1][k]);
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            mma_16816(o[n][2 * j], va[0], pb[p][n][0], pb[p][n][1]);
                            mma_16816(o[n][2 * j + 1], va[1], pb[p][n][0], pb[p][n][1]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty_bar[st]);
            if (!last) continue;

            // The row tile's end: the workers' sums, under one maximum, are added up, a quarter of the channels by each worker (of every lane's: word
            // by word; at d = 64, half a word).  They are put down once all have read those of the row tile before, and read once all have been put down.
            const int set = items & 1;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 4);
                    l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 8);
                    l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 16);
                    if (g == 0) {
                        top_s[set][warp][8 * n + 2 * q + e] = m[n][e];
                        sum_s[set][warp][8 * n + 2 * q + e] = l[n][e];
                    }
                }
            constexpr int QUARTER = 2 * WORDS / 4;   // MMA tiles of 16 channels that a worker adds up
            // [reader][writer, the reader left out][row eight][tile][lane]
            auto place = [&](int reader, int writer, int n, int b) {
                return sums + (((reader * (WORKERS - 1) + (writer - (writer > reader ? 1 : 0))) * NB + n) * QUARTER + b) * 32 + lane;
            };
            static_assert(sums_bytes(DIM, NB) == sizeof(float4) * WORKERS * (WORKERS - 1) * NB * QUARTER * 32, "the place of the sums");
            if (items > 0) {
                ok = mbar_wait_warp(&got_bar, (items - 1) & 1u, &abort_flag);
                if (!ok) break;
            }
#pragma unroll
            for (int reader = 0; reader < WORKERS; ++reader)
                if (reader != warp) {
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int b = 0; b < QUARTER; ++b) {
                            const float(&x)[4] = o[n][reader * QUARTER + b];
                            *place(reader, warp, n, b) = make_float4(x[0], x[1], x[2], x[3]);
                        }
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(&put_bar);
            ok = mbar_wait_warp(&put_bar, items & 1u, &abort_flag);
            if (!ok) break;
            float total[NB][2], top[NB][2];
            float x[NB][QUARTER][4];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float by[WORKERS][2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = 8 * n + 2 * q + e;
                    float t = top_s[set][0][row];
#pragma unroll
                    for (int w = 1; w < WORKERS; ++w) t = fmaxf(t, top_s[set][w][row]);
                    float sum = 0.0f;
#pragma unroll
                    for (int w = 0; w < WORKERS; ++w) {
                        const float mw = top_s[set][w][row];
                        by[w][e] = (mw == -INFINITY) ? 0.0f : exp2_fast(mw - t);
                        sum = fmaf(sum_s[set][w][row], by[w][e], sum);
                    }
                    top[n][e] = t;
                    total[n][e] = sum;
                }
#pragma unroll
                for (int b = 0; b < QUARTER; ++b) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[n][b][k] = 0.0f;
#pragma unroll
                    for (int w = 0; w < WORKERS; ++w) {
                        float4 y = make_float4(o[n][w * QUARTER + b][0], o[n][w * QUARTER + b][1], o[n][w * QUARTER + b][2], o[n][w * QUARTER + b][3]);
                        if (w != warp) y = *place(warp, w, n, b);
                        x[n][b][0] = fmaf(y.x, by[w][0], x[n][b][0]);
                        x[n][b][1] = fmaf(y.y, by[w][1], x[n][b][1]);
                        x[n][b][2] = fmaf(y.z, by[w][0], x[n][b][2]);
                        x[n][b][3] = fmaf(y.w, by[w][1], x[n][b][3]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&got_bar);
            items += 1;
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                // tile b of worker w: channels g * (DIM / 8) + 2 (w QUARTER + b), + 1
                const int ch = g * (DIM / 8) + 2 * QUARTER * warp;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = 8 * n + 2 * q + e;
                    if (t_row[n][e] >= mq) continue;
                    if (slot < 0) {
                        const float inv = (top[n][e] == -INFINITY) ? 0.0f : 1.0f / total[n][e];
                        const long long tq = q0 + t_row[n][e];
                        const int hq = h * a.G + h_row[n][e];
                        uint32_t *dst = reinterpret_cast<uint32_t *>(static_cast<__half *>(a.out) + tq * a.o_tok + hq * a.o_head + ch);
                        uint32_t y[QUARTER];
#pragma unroll
                        for (int b = 0; b < QUARTER; ++b) y[b] = pair_bits<BF16>(x[n][b][e] * inv, x[n][b][2 + e] * inv);
                        if constexpr (QUARTER == 2) *reinterpret_cast<uint2 *>(dst) = make_uint2(y[0], y[1]);
                        else dst[0] = y[0];
                        if (a.lse && warp == 0 && g == 0) a.lse[tq * (c.heads * a.G) + hq] = row_lse(top[n][e], total[n][e]);
                    } else {
                        const Kv8Parts<ROWS> parts(a, gridDim.x);
                        const size_t pr = static_cast<size_t>(2 * blockIdx.x + slot) * ROWS + row;
#pragma unroll
                        for (int b = 0; b < QUARTER; ++b) *reinterpret_cast<float2 *>(parts.four(2 * blockIdx.x + slot, row, (ch + 2 * b) & ~3) + ((ch + 2 * b) & 3)) = make_float2(x[n][b][e], x[n][b][2 + e]);
                        if (warp == 0 && g == 0) {
                            parts.m[pr] = top[n][e];
                            parts.l[pr] = total[n][e];
                        }
                    }
                }
            }
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

template <int DIM, int FMT, bool BF16, int NB>
bool launch_rows(const Kv8Attend &a, int sm_count, cudaStream_t s) {
    const Kv8 &c = a.c;
    CUtensorMap km, vm;
    const long long rows = (static_cast<long long>(c.num_pages) * c.heads) << c.ps_shift;
    if (!make_code_tensor_map(c.code[0], rows, DIM, c.page_size(), &km) || !make_code_tensor_map(c.code[1], rows, DIM, c.page_size(), &vm)) return false;
    auto kernel = kv8_rows_kernel<DIM, FMT, BF16, NB>;
    if (!ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), smem_bytes(DIM, NB))) return false;
    launch_dependent(kernel, dim3(static_cast<unsigned>(ctas_of(sm_count))), THREADS, smem_bytes(DIM, NB), s, km, vm, a);
    return true;
}
template <int DIM, int NB>
bool launch_rows(const Kv8Attend &a, bool i8, bool bf, int sm_count, cudaStream_t s) {
    if (i8) return bf ? launch_rows<DIM, EOSQ_KV_INT8, true, NB>(a, sm_count, s) : launch_rows<DIM, EOSQ_KV_INT8, false, NB>(a, sm_count, s);
    return bf ? launch_rows<DIM, EOSQ_KV_E4M3, true, NB>(a, sm_count, s) : launch_rows<DIM, EOSQ_KV_E4M3, false, NB>(a, sm_count, s);
}

}  // namespace

size_t kv8_rows_scratch(int d) { return sizeof(float) * 2 * KV8_MAX_CTAS * 16 * (static_cast<size_t>(d) + 2); }

int launch_kv8_rows(const Kv8Attend &a, int fmt, int dtype, int sm_count, cudaStream_t s) {
    const bool bf = dtype == EOSQ_BF16, i8 = fmt == EOSQ_KV_INT8, eight = a.rows_max <= 8;
    bool ok;
    if (a.c.d_shift == 7) ok = eight ? launch_rows<128, 1>(a, i8, bf, sm_count, s) : launch_rows<128, 2>(a, i8, bf, sm_count, s);
    else ok = eight ? launch_rows<64, 1>(a, i8, bf, sm_count, s) : launch_rows<64, 2>(a, i8, bf, sm_count, s);
    return ok ? EOSQ_OK : EOSQ_ERR_CUDA;
}

void launch_kv8_rows_join(const Kv8Attend &a, int dtype, int sm_count, cudaStream_t s) {
    if (a.rows_max <= 8) launch_join<8>(a, dtype, ctas_of(sm_count), s);
    else launch_join<16>(a, dtype, ctas_of(sm_count), s);
}

}  // namespace eosq
