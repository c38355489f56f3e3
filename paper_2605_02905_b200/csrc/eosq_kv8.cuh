// The 8-bit paged cache: what its kernels share -- the view of a cache, codes and scales, a call's sequences, and how
// attention's work is dealt out.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "eosq_common.cuh"

namespace eosq {

constexpr int KV8_ERR_ATTEND_TIMEOUT = 64;   // device-side error word

// A cache as the kernels see it: eosq_kv8_t with a layer's arrays, sizes as shifts where they are powers of two.
struct Kv8 {
    uint8_t *code[2];    // keys, values
    float *scale[2];
    int32_t *table, *lengths, *refs;
    unsigned *flags;
    int layers, num_pages, heads, ps_shift, d_shift, max_seqs, max_pages;
    __host__ __device__ int page_size() const { return 1 << ps_shift; }
    __host__ __device__ size_t page_bytes() const { return static_cast<size_t>(heads) << (ps_shift + d_shift); }   // of keys, or of values
};

// ---- two numbers in an instruction ----------------------------------------------------------------
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

// ---- codes ------------------------------------------------------------------------------------
constexpr float KV8_SCALE_MIN = 5.421010862427522e-20f;   // 2^-64
constexpr float KV8_SCALE_MAX = 1.8446744073709552e19f;   // 2^64

// Four codes as fp16, in pairs, exactly.  int8: 1024 + 128 + c has c + 128 in its low mantissa bits, so the byte c ^ 0x80 under the
// exponent byte of 1024 is that number, and one subtraction makes it c.  e4m3: an instruction for two (moving sign, exponent and mantissa bits to
// fp16's places takes eight for four: 231 us for 16 x 32768 tokens, 173 so).  A page behind its last token holds whatever it held: bytes of every
// kind, among them e4m3's NaNs, whose product with a weight of 0 would be NaN.  Where that can be, no_nan() makes 448 of them.
__device__ __forceinline__ uint32_t half2_minus(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int FMT>
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (FMT == EOSQ_KV_INT8) {
        w ^= 0x80808080u;
        lo = half2_minus(__byte_perm(w, 0x64646464u, 0x4140), 0x64806480u);
        hi = half2_minus(__byte_perm(w, 0x64646464u, 0x4342), 0x64806480u);
    } else {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
    }
}
template <int FMT>
__device__ __forceinline__ uint32_t no_nan(uint32_t h) {
    if constexpr (FMT == EOSQ_KV_E4M3) asm("min.f16x2 %0, %1, %2;" : "=r"(h) : "r"(h), "r"(0x5f005f00u));   // (448: of a number and NaN the number)
    return h;
}

// ---- a call's sequences -------------------------------------------------------------------------
struct Kv8Seq {
    int row, len, m, q0;   // row of the table, tokens, this call's tokens or queries and the first one's row; m = 0: nothing to do
};
__device__ __forceinline__ void raise(const Kv8 &c, unsigned bits) { atomicOr(c.flags, bits); }
// Entry i of a list with offsets `cu` into `total` rows, none longer than `most`.
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8 &c, const int32_t *seqs, const int32_t *cu, int i, long long total, int most) {
    Kv8Seq s{seqs[i], 0, 0, 0};
    if (s.row == -1) return s;
    const int c0 = cu[i], c1 = cu[i + 1];
    if (s.row < 0 || s.row >= c.max_seqs || c0 < 0 || c1 < c0 || c1 > total || c1 - c0 > most) {
        raise(c, EOSQ_KV8_BAD_SEQ);
        return s;
    }
    s.len = c.lengths[s.row];
    if (s.len < 0 || s.len > (static_cast<long long>(c.max_pages) << c.ps_shift)) {
        raise(c, EOSQ_KV8_BAD_SEQ);
        return s;
    }
    s.q0 = c0;
    s.m = c1 - c0;
    return s;
}

// ---- attention ----------------------------------------------------------------------------------
// A row tile that begins in one CTA and ends in another (last_cta; -1: there is none).
struct Kv8Cut {
    int last_cta, q0, m, r, h, unused[3];
};
constexpr int KV8_MAX_CTAS = 320;
struct Kv8Attend {
    Kv8 c;
    const int32_t *seqs, *cu;
    int n, max_q, G, causal, window;
    int rows_min, rows_max;                    // entries of fewer or more rows than this are another launch's (or nobody's)
    int whole;                                 // row tiles are not shared between CTAs: a unit is one of them with a head
    long long total;
    const void *q;
    void *out;
    float *lse;
    long long q_tok, q_head, o_tok, o_head;   // strides in elements
    float scale_log2;                          // scale * log2(e)
    Kv8Cut *cuts;                       // [KV8_MAX_CTAS] scratch: row tiles that go on in the next CTA
    float *part;                               // scratch: partial results, two slots per CTA
    int *err;
};

// The work of one call: every entry's query rows (query t, head g of a KV head: row t * G + g) cut into tiles of RT, the keys that
// a row tile sees cut into tiles of KT.  A unit is one key tile of one row tile and KV head, or one of COST that stand for a row tile's beginning and
// end; units are numbered entry by entry, row tile by row tile, head by head, first those COST, then key tile by key tile.  CTAs take equal runs of
// them.
template <int RT, int KT, int COST_>
struct Kv8Tiles {
    static constexpr int COST = COST_;
    // Positions [lo, hi) that queries t0 .. t1 of the entry see between them.
    static __device__ __forceinline__ void span(const Kv8Attend &a, const Kv8Seq &s, int t0, int t1, int &lo, int &hi) {
        hi = a.causal ? max(min(s.len, s.len - s.m + t1 + 1), 0) : s.len;
        lo = a.window > 0 ? max(s.len - s.m + t0 - a.window + 1, 0) : 0;
    }
    static __device__ __forceinline__ int row_tiles(const Kv8Attend &a, const Kv8Seq &s) {
        const int rows = s.m * a.G;
        return (rows < a.rows_min || rows > a.rows_max) ? 0 : (rows + RT - 1) / RT;
    }
    // Units of a row tile of so many key tiles and a head.
    static __device__ __forceinline__ int units(const Kv8Attend &a, int tiles) { return a.whole ? 1 : tiles + COST; }
    // First key tile of row tile r, and how many: at least one, so that rows which see nothing are written too.
    static __device__ __forceinline__ int key_tiles(const Kv8Attend &a, const Kv8Seq &s, int r, int &first) {
        int lo, hi;
        span(a, s, r * RT / a.G, min(s.m - 1, (r * RT + RT - 1) / a.G), lo, hi);
        first = 0;
        if (hi <= lo) return 1;
        first = lo / KT;
        return (hi + KT - 1) / KT - first;
    }
};
// Of min(ctas, units) CTAs, `cta` takes units [unit_of(cta), unit_of(cta + 1)): at least one.
__device__ __forceinline__ int unit_of(int units, int cta, int ctas) { return static_cast<int>(static_cast<long long>(units) * cta / ctas); }
__device__ __forceinline__ int cta_of(int units, int unit, int ctas) {
    return static_cast<int>(((static_cast<long long>(unit) + 1) * ctas - 1) / units);
}
// The row tiles and heads of a run of units, one after another; the same in every thread of a warp.
template <typename T>
struct Kv8Walk {
    const Kv8Attend &a;
    int i, at, left;                                 // entry; units of it that come before; units to go
    Kv8Seq s;
    int row_tiles, r, h, tile0, tiles, from, take;   // now: row tile, head, its key tiles [tile0, tile0 + tiles), of which `take` from `from` on are the run's
    int reached;                                     // units of the row tile and head up to the run's last
    bool fresh;
    __device__ __forceinline__ Kv8Walk(const Kv8Attend &a_, int entry, int skip, int units)
        : a(a_), i(entry), at(skip), left(units), s{-1, 0, 0, 0}, r(0), h(0), tile0(0), tiles(1), from(0), take(0), reached(0), fresh(true) {
        if (left > 0) enter();
    }
    __device__ __forceinline__ void enter() {
        s = kv8_seq(a.c, a.seqs, a.cu, i, a.total, a.max_q);
        row_tiles = (s.m > 0) ? T::row_tiles(a, s) : 0;
        r = 0;
    }
    __device__ __forceinline__ bool next() {
        while (left > 0) {
            if (fresh || ++h >= a.c.heads) {
                if (!fresh) ++r;
                fresh = false;
                h = 0;
                while (true) {
                    if (r >= row_tiles) {
                        if (++i >= a.n) {   // (the units say that there is more; unless memory changes under the call)
                            left = take = 0;
                            return false;
                        }
                        enter();
                        continue;
                    }
                    tiles = T::key_tiles(a, s, r, tile0);
                    const int all = T::units(a, tiles) * a.c.heads;
                    if (at < all) break;
                    at -= all;
                    ++r;
                }
                h = at / T::units(a, tiles);
                at -= h * T::units(a, tiles);
            }
            reached = at + min(T::units(a, tiles) - at, left);
            left -= reached - at;
            from = a.whole ? 0 : max(at - T::COST, 0);
            take = a.whole ? tiles : max(reached - T::COST, 0) - from;
            at = 0;
            if (take > 0) return true;
        }
        return false;
    }
    // -1: the whole row tile is in the run, else the slot of its partial result: 1 for the run's last, 0 for one that began before.
    __device__ __forceinline__ int slot() const { return (take == tiles) ? -1 : (from == 0 ? 1 : 0); }
};
// A CTA's run of units: first entry, units of it that come before, [u0, u1) of `total`, the runs that there are.
struct Kv8Run {
    int entry, skip, u0, u1, total, ctas;
};

// What a fetching warp asks for ahead of the copies: up to four tiles of 128 tokens of a row tile at a time, a lane for 16 of their tokens (which are in one
// page): first the page, with the batch after it the scales.
constexpr int KV8_KEYS = 128, KV8_GROUP = 16, KV8_GROUPS = KV8_KEYS / KV8_GROUP;   // tokens of a tile; tokens of a lane; lanes of a tile
struct Kv8Batch {
    int tiles, tok0, first, last, q0, len, m, r, h, slot, hi;   // uniform; first, last: whether the run's part of a row tile begins, ends here; hi: end of what is seen
    int page;                                                // of this lane's 16 tokens, -1: none
    bool wanted;                                             // whether it should have one
    float ks, vs;
};
template <typename T, int RT>
struct Kv8Fetch {
    Kv8Walk<T> w;
    int done, all;   // tiles of the walk's row tile that are in batches already, and how many it has
    const int lane, box;
    __device__ __forceinline__ Kv8Fetch(const Kv8Attend &a, const Kv8Run &run, int lane_)
        : w(a, run.entry, run.skip, run.u1 - run.u0), done(0), all(0), lane(lane_), box(min(a.c.page_size(), KV8_KEYS)) {}
    __device__ __forceinline__ Kv8Batch next() {
        const Kv8 &c = w.a.c;
        Kv8Batch b;
        b.tiles = 0;
        b.page = -1;
        b.wanted = false;
        if (done == all) {
            if (!w.next()) return b;
            done = 0;
            all = w.take;
        }
        b.tiles = min(all - done, 32 / KV8_GROUPS);
        b.tok0 = (w.tile0 + w.from + done) * KV8_KEYS;
        b.first = done == 0;
        done += b.tiles;
        b.last = done == all;
        b.q0 = w.s.q0;
        b.len = w.s.len;
        b.m = w.s.m;
        b.r = w.r;
        b.h = w.h;
        b.slot = w.slot();
        int lo;
        T::span(w.a, w.s, w.r * RT / w.a.G, min(w.s.m - 1, (w.r * RT + RT - 1) / w.a.G), lo, b.hi);
        const int tok = b.tok0 + lane * KV8_GROUP, box0 = tok & ~(box - 1);   // a box: what one page gives to a tile
        b.wanted = lane < b.tiles * KV8_GROUPS && box0 < b.hi && box0 + box > lo;
        if (b.wanted) b.page = c.table[static_cast<size_t>(w.s.row) * c.max_pages + (tok >> c.ps_shift)];
        return b;
    }
    __device__ __forceinline__ void scales(Kv8Batch &b) {
        const Kv8 &c = w.a.c;
        b.ks = 0.0f;
        b.vs = 1.0f;
        if (b.page >= 0 && b.page < c.num_pages) {
            const size_t slot = static_cast<size_t>(b.page) * c.heads + b.h;
            b.ks = c.scale[0][slot];
            b.vs = c.scale[1][slot];
        } else {
            if (b.wanted) raise(c, EOSQ_KV8_BAD_PAGE);
            b.page = -1;
        }
    }
    // Whether this lane's page begins a box, and the row of the codes where it does.
    __device__ __forceinline__ bool leads(const Kv8Batch &b, int &row) const {
        const Kv8 &c = w.a.c;
        const int tok = b.tok0 + lane * KV8_GROUP;
        const bool yes = b.page >= 0 && (tok & (box - 1)) == 0;
        row = yes ? ((b.page * c.heads + b.h) << c.ps_shift) + (tok & (c.page_size() - 1)) : 0;
        return yes;
    }
};

// A bf16 row is divided by 2^e, which brings its largest value to 2^14 .. 2^15 (a row of less than 2^-112: to less).  These are all exponents that finite rows can have
// there; 2^e and 2^-e are normal numbers.
constexpr int KV8_EXP_MIN = -126, KV8_EXP_MAX = 113;

// Scores are base-2 logarithms; a weight is 2^(x - m + KV8_SHIFT), m being a running maximum that is only moved when a score passes
// it by more than KV8_SLACK.  So weights are at most 2^14, inside fp16, and those of fp16's smallest normal numbers are 2^-20 of
// the largest when m is exact.  They are rounded to fp16 because the second product takes fp16 operands, which hold the codes of both formats exactly: half a step of 2^-11 each,
// independent of one another, while their sum is of the weights before that, in fp32.  x contains log2 of the page's value scale, so that the product with the codes of the values needs no
// scaling; the sum of the weights takes it out again.
constexpr float KV8_SHIFT = 6.0f, KV8_SLACK = 8.0f;
// Base-2 logarithms beyond 2^22 are so far apart in fp32 that SHIFT - m, or a bound on them under one rounding, is off by whole powers of two of a weight: where a
// maximum is that large, exponents are (x - m) + SHIFT, with x rounded as m was.  x - m is then exact where it matters, and no more than KV8_SLACK.
__host__ __device__ __forceinline__ bool kv8_far(float m) { return fabsf(m) > 4194304.0f && m != -INFINITY; }
// A maximum that only moves up, by whole powers of two, so that what has been rounded already is rescaled exactly.  (Where fp32 holds no fractions, the
// sum may round to less than `top`, which is then itself a whole number away from m, or so far that nothing is left of what was there.)
__host__ __device__ __forceinline__ float kv8_moved(float m, float top) {
    return (m == -INFINITY) ? top : fmaxf(m + ceilf(fmaxf(top - m, 0.0f)), top);
}
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Exclusive prefix sums of units[0 .. n) in place, by one warp; the total, or KV8_TOO_MANY where it is as much or more (the sums are of no use then).
constexpr int KV8_TOO_MANY = 0x7fffffff;
__device__ __forceinline__ int sum_of(int a, int b) { return static_cast<int>(min(static_cast<unsigned>(a) + static_cast<unsigned>(b), static_cast<unsigned>(KV8_TOO_MANY))); }
__device__ __forceinline__ int warp_prefix(int *units, int n) {
    const int lane = threadIdx.x & 31;
    int total = 0;
    for (int base = 0; base < n; base += 32) {
        const int v = (base + lane < n) ? units[base + lane] : 0;
        int x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x = sum_of(x, y);
        }
        if (base + lane < n) units[base + lane] = sum_of(total, x - v);
        total = sum_of(total, __shfl_sync(0xffffffffu, x, 31));
    }
    return total;
}

template <bool BF16>
__device__ __forceinline__ uint32_t pair_bits(float lo, float hi) {
    if constexpr (BF16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&b);
    } else {
        return half2_bits(lo, hi);
    }
}
template <bool BF16, int N>
__device__ __forceinline__ void store_row(void *p, const float (&v)[N]) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = pair_bits<BF16>(v[2 * i], v[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) reinterpret_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

// Every thread of the CTA (of THREADS) takes part; `units` is shared memory for every entry's units, which may be used otherwise once this has returned.
template <typename T, int THREADS>
__device__ __forceinline__ Kv8Run kv8_run(const Kv8Attend &a, int *units) {
    __shared__ int total_units;
    const int tid = threadIdx.x;
    for (int i = tid; i < a.n; i += THREADS) {
        const Kv8Seq s = kv8_seq(a.c, a.seqs, a.cu, i, a.total, a.max_q);
        int u = 0;
        if (s.m > 0) {
            const int tiles = T::row_tiles(a, s);
            int first;
            for (int r = 0; r < tiles; ++r) u += T::units(a, T::key_tiles(a, s, r, first));
        }
        units[i] = u * a.c.heads;
    }
    __syncthreads();
    if (tid < 32) {
        int t = warp_prefix(units, a.n);
        if (t == KV8_TOO_MANY) {   // more than all rows can have (the entry point's bound): offsets go back, and rows are counted many times over
            t = 0;
            if (tid == 0) raise(a.c, EOSQ_KV8_BAD_SEQ);
        }
        if (tid == 0) total_units = t;
    }
    __syncthreads();
    Kv8Run run{0, 0, 0, 0, total_units, min(static_cast<int>(gridDim.x), total_units)};
    const int cta = blockIdx.x;
    if (cta < run.ctas) {
        run.u0 = unit_of(run.total, cta, run.ctas);
        run.u1 = unit_of(run.total, cta + 1, run.ctas);
        int lo = 0, hi = a.n;   // the last entry that begins at or before u0 (those behind with the same beginning have no units)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (units[mid] <= run.u0) lo = mid;
            else hi = mid;
        }
        run.entry = lo;
        run.skip = run.u0 - units[lo];
    } else if (tid == 0) {
        a.cuts[cta].last_cta = -1;
    }
    __syncthreads();
    return run;
}

// log sum exp of a row from its maximum and the sum of its weights (both as the kernels hold them): -infinity for a row that saw nothing, whose maximum is
// -infinity and whose sum is 0; NaN for one with a NaN among its scores, whose sum is that.
__device__ __forceinline__ float row_lse(float m, float l) {
    return (m - KV8_SHIFT + log2f(l)) * 0.6931471805599453f;
}

// Partial results: sums as [slots][d / 4][RT][4], so that neighbouring rows' go side by side, then [slots][RT] maxima, then sums of weights.
template <int RT>
struct Kv8Parts {
    float *o, *m, *l;
    int d_shift;
    __device__ __forceinline__ Kv8Parts(const Kv8Attend &a, int ctas) : d_shift(a.c.d_shift) {
        const size_t rows = static_cast<size_t>(2) * ctas * RT;
        o = a.part;
        m = o + (rows << d_shift);
        l = m + rows;
    }
    // Four channels from `ch` on (a multiple of four).
    __device__ __forceinline__ float *four(int slot, int row, int ch) const { return o + (((static_cast<size_t>(slot) << (d_shift - 2)) + (ch >> 2)) * RT + row) * 4; }
};

// What a CTA says about its last row tile: whether it goes on behind the run [.., u1) of `ctas` runs.
template <typename T>
__device__ __forceinline__ void kv8_cut(const Kv8Walk<T> &w, int total, int u1, int ctas) {
    Kv8Cut cut{-1, w.s.q0, w.s.m, w.r, w.h, {0, 0, 0}};
    if (w.from == 0 && w.take > 0 && w.take < w.tiles) cut.last_cta = min(cta_of(total, u1 - w.reached + T::COST + w.tiles - 1, ctas), ctas - 1);
    w.a.cuts[blockIdx.x] = cut;
}

// Row tiles that several CTAs worked on: their partial results under one maximum, in the order of the keys.  A CTA of this kernel per 16 rows (or 8) and
// CTA of the other, which a row tile may begin in and not end; a thread per 8 channels of a row.  It is a launch behind the last CTA's end and a chain of loads,
// so those of four partial results are under way together (one after another, and the maxima first: 128 queries on 32768 tokens, ten partial results each, 99.5 us, so 90.6).
constexpr int KV8_JOIN_PART = 8;
template <int RT, int DIM>
constexpr int join_threads = (RT < 16 ? RT : 16) * (DIM / KV8_JOIN_PART);
template <int RT, int DIM, bool BF16>
__global__ void __launch_bounds__(join_threads<RT, DIM>) kv8_join_kernel(const Kv8Attend a, int ctas) {
    pdl_wait();
    constexpr int JOIN = RT < 16 ? RT : 16, PER = RT / JOIN, PART = KV8_JOIN_PART, AHEAD = 4;
    const int ca = blockIdx.x / PER, row0 = (blockIdx.x % PER) * JOIN;
    const Kv8Cut cut = a.cuts[ca];
    const int rows = cut.m * a.G, row = row0 + threadIdx.x % JOIN, at = cut.r * RT + row, part = threadIdx.x / JOIN;
    if (cut.last_cta < 0 || at >= rows) return;
    const Kv8Parts<RT> parts(a, ctas);
    float top = -INFINITY, l = 0.0f, v[PART];
#pragma unroll
    for (int e = 0; e < PART; ++e) v[e] = 0.0f;
    for (int k0 = ca; k0 <= cut.last_cta; k0 += AHEAD) {
        float mk[AHEAD], lk[AHEAD];
        float4 x[AHEAD], y[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int k = k0 + j;
            mk[j] = -INFINITY;
            if (k <= cut.last_cta) {
                const int slot = 2 * k + (k == ca);
                mk[j] = parts.m[static_cast<size_t>(slot) * RT + row];
                lk[j] = parts.l[static_cast<size_t>(slot) * RT + row];
                x[j] = *reinterpret_cast<const float4 *>(parts.four(slot, row, part * PART));
                y[j] = *reinterpret_cast<const float4 *>(parts.four(slot, row, part * PART + 4));
            }
        }
        float to = top;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) to = fmaxf(to, mk[j]);
        const float by = (top == -INFINITY) ? 0.0f : exp2_fast(top - to);
        top = to;
        l *= by;
#pragma unroll
        for (int e = 0; e < PART; ++e) v[e] *= by;
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (k0 + j > cut.last_cta) continue;
            const float f = (mk[j] == -INFINITY) ? 0.0f : exp2_fast(mk[j] - top);
            l = fmaf(lk[j], f, l);
            v[0] = fmaf(x[j].x, f, v[0]); v[1] = fmaf(x[j].y, f, v[1]); v[2] = fmaf(x[j].z, f, v[2]); v[3] = fmaf(x[j].w, f, v[3]);
            v[4] = fmaf(y[j].x, f, v[4]); v[5] = fmaf(y[j].y, f, v[5]); v[6] = fmaf(y[j].z, f, v[6]); v[7] = fmaf(y[j].w, f, v[7]);
        }
    }
    const float inv = (top == -INFINITY) ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < PART; ++e) v[e] *= inv;
    const long long tq = cut.q0 + at / a.G;
    const int hq = cut.h * a.G + at % a.G;
    store_row<BF16, PART>(static_cast<__half *>(a.out) + tq * a.o_tok + hq * a.o_head + part * PART, v);
    if (a.lse && part == 0) a.lse[tq * (a.c.heads * a.G) + hq] = row_lse(top, l);
}

template <int RT>
void launch_join(const Kv8Attend &a, int dtype, int ctas, cudaStream_t s) {
    const dim3 grid(static_cast<unsigned>(ctas) * (RT < 16 ? 1 : RT / 16));
    const bool bf = dtype == EOSQ_BF16;
    if (a.c.d_shift == 7) {
        if (bf) launch_dependent(kv8_join_kernel<RT, 128, true>, grid, join_threads<RT, 128>, 0, s, a, ctas);
        else launch_dependent(kv8_join_kernel<RT, 128, false>, grid, join_threads<RT, 128>, 0, s, a, ctas);
    } else {
        if (bf) launch_dependent(kv8_join_kernel<RT, 64, true>, grid, join_threads<RT, 64>, 0, s, a, ctas);
        else launch_dependent(kv8_join_kernel<RT, 64, false>, grid, join_threads<RT, 64>, 0, s, a, ctas);
    }
}

// Which kernel a call goes through: the one for few rows (eosq_kv8_attend.cu), which takes row tiles of 16 one after another, or the one that works on tiles of 256 rows
// (eosq_kv8_attend_tc.cu).  most: rows (queries times heads of a group) of the longest entry, rows: of all n entries, per KV head.  With equal entries the first
// is ahead up to 32 rows at d = 128 (8 heads, 32768 tokens: 41 us, the other 50; 48 rows: 56 and 50) and up to 48 at d = 64, where its codes take half the work
// (38 and 42; 64 rows: 46 and 42); what counts is the mean, since its time goes by row tiles of 16 and the other's by entries (24 of 1 to 60 rows, d = 64: 23
// and 36).
inline bool kv8_few_rows(long long most, long long rows, int n, int d) { return most <= 16 || rows <= static_cast<long long>(n) * (d == 128 ? 36 : 52); }
// Both, where a prompt's chunk comes with sequences that get a token each: entries of up to so many rows through the first and then the others through the second; 0: one
// of them takes all.  8 heads, G = 4, d = 128, through one kernel / both: 63 single tokens on 4096 each and a chunk of 512 queries 347 / 168 us, with a chunk of 128
// 179 / 139; 31 on 2000 and a chunk of 512 on 16000 231 / 201; 63 on 500 with one of 128 44 / 48, two more launches; 7 on 1000 with one of 128 51 / 54.
// Chunks of fewer rows than that go through one kernel, mostly the first, by the mean.  On short contexts that is ahead, on long ones it is not: a call as it is / two calls,
// of the single tokens and of the chunk, for a chunk of 16 and of 127 queries among 7 single tokens on 500 each 15 / 32 and 26 / 39 us, on 4096 33 / 44 and 60 / 59, on 32768 164 / 147
// and 309 / 191; among 31 on 32768 485 / 377 and 862 / 421; among 63 on 4096 142 / 129 and 190 / 139.
inline int kv8_split(long long most, long long rows, int n, int G) {
    if (most < 512 || rows > n * (most / 4) || G > 16) return 0;
    return G <= 8 ? 8 : 16;
}
constexpr int KV8_COST_BOUND = 5;   // no kernel counts a row tile's beginning and end as more units

// ---- launchers ------------------------------------------------------------------------------------
void launch_kv8_store(const Kv8 &c, int fmt, const void *const (&x)[2], int dtype, long long total, const long long (&tok)[2],
                      const long long (&head)[2], const int32_t *seqs, const int32_t *first, const int32_t *cu, int n, int max_new, int sm_count, cudaStream_t s);
bool launch_kv8_reserve(const Kv8 &c, const int32_t *seqs, const int32_t *add, int n, int32_t *first, cudaStream_t s);
bool launch_kv8_fork(const Kv8 &c, const int32_t *src, const int32_t *dst, int n, int2 *plan, cudaStream_t s);
void launch_kv8_fork_copy(const Kv8 &c, const int32_t *src, const int32_t *dst, int n, const int2 *plan, cudaStream_t s);
void launch_kv8_free(const Kv8 &c, const int32_t *seqs, int n, cudaStream_t s);
void launch_kv8_compact_plan(const Kv8 &c, int32_t *remap, int32_t *moves, cudaStream_t s);
void launch_kv8_compact_move(const Kv8 &c, const int32_t *remap, const int32_t *moves, int sm_count, cudaStream_t s);
void launch_kv8_copy(const Kv8 &from, const Kv8 &to, const int32_t *src, const int32_t *dst, int n, cudaStream_t s);
// Attention: scratch for a call's partial results, the kernel (EOSQ_OK, EOSQ_ERR_UNSUPPORTED or EOSQ_ERR_CUDA; nothing enqueued unless OK), and the one that
// joins what CTAs share between them.
size_t kv8_rows_scratch(int d);
size_t kv8_tiles_scratch(int d);
int launch_kv8_rows(const Kv8Attend &a, int fmt, int dtype, int sm_count, cudaStream_t s);
int launch_kv8_tiles(const Kv8Attend &a, int fmt, int dtype, int sm_count, cudaStream_t s);
void launch_kv8_rows_join(const Kv8Attend &a, int dtype, int sm_count, cudaStream_t s);
void launch_kv8_tiles_join(const Kv8Attend &a, int dtype, int sm_count, cudaStream_t s);
// Tensor map over the codes of a layer's keys or values, [rows][d] bytes, in boxes of box_rows rows with a swizzle as wide as a row (eosq_tc.cu).
bool make_code_tensor_map(const void *codes, long long rows, int d, int box_rows, CUtensorMap *out);

}  // namespace eosq
