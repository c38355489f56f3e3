// The 8-bit paged cache: what its kernels share -- the view of a cache, codes and scales, a call's sequences, and how
// attention's work is dealt out.
#pragma once

#include <cuda.h>
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

// ---- codes ------------------------------------------------------------------------------------
constexpr float KV8_SCALE_MIN = 5.421010862427522e-20f;   // 2^-64
constexpr float KV8_SCALE_MAX = 1.8446744073709552e19f;   // 2^64

// Four codes as fp16, in pairs.  int8: 1024 + 128 + c has c + 128 in its low mantissa bits, so the byte c ^ 0x80 under the
// exponent byte of 1024 is that number, and one subtraction makes it c, exactly.  e4m3: sign, exponent and mantissa bits
// moved to fp16's places are 2^-8 of the number (fp16's exponent bias is larger by 8), subnormal numbers included; the
// factor KV8_UNIT goes with the scale.  (Every byte is then a finite number: what a page holds behind its last token cannot turn a masked weight
// of 0 into a NaN.)
template <int FMT> struct Kv8Unit { static constexpr float value = (FMT == EOSQ_KV_E4M3) ? 256.0f : 1.0f; };
__device__ __forceinline__ uint32_t half2_minus(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The two codes in the upper bytes of w's halves (lower bytes 0).
__device__ __forceinline__ uint32_t e4m3_halves(uint32_t w) { return (w & 0x80008000u) | ((w & 0x7f007f00u) >> 1); }
template <int FMT>
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (FMT == EOSQ_KV_INT8) {
        w ^= 0x80808080u;
        lo = half2_minus(__byte_perm(w, 0x64646464u, 0x4140), 0x64806480u);
        hi = half2_minus(__byte_perm(w, 0x64646464u, 0x4342), 0x64806480u);
    } else {
        lo = e4m3_halves(__byte_perm(w, 0u, 0x1404));
        hi = e4m3_halves(__byte_perm(w, 0u, 0x3424));
    }
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
struct Kv8Attend {
    Kv8 c;
    const int32_t *seqs, *cu;
    int n, max_q, G, causal, window;
    long long total;
    const void *q;
    void *out;
    float *lse;
    long long q_tok, q_head, o_tok, o_head;   // strides in elements
    float scale_log2;                          // scale * log2(e)
    int32_t *first_unit;                       // [n + 1] scratch: units before each entry
    float *part;                               // scratch: partial results, two slots per CTA
    int *err;
};

// The work of one call: every entry's query rows (query t, head g of a KV head: row t * G + g) cut into tiles of RT, the keys that
// a row tile sees cut into tiles of KT.  A unit is one key tile of one row tile and KV head; units are numbered entry by
// entry, row tile by row tile, head by head, key tile by key tile.  CTAs take equal runs of them.
template <int RT, int KT>
struct Kv8Tiles {
    // Positions [lo, hi) that queries t0 .. t1 of the entry see between them.
    static __device__ __forceinline__ void span(const Kv8Attend &a, const Kv8Seq &s, int t0, int t1, int &lo, int &hi) {
        hi = a.causal ? max(min(s.len, s.len - s.m + t1 + 1), 0) : s.len;
        lo = a.window > 0 ? max(s.len - s.m + t0 - a.window + 1, 0) : 0;
    }
    static __device__ __forceinline__ int row_tiles(const Kv8Attend &a, const Kv8Seq &s) { return (s.m * a.G + RT - 1) / RT; }
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
// Scores are base-2 logarithms; a weight is 2^(x - m + KV8_SHIFT), m being a running maximum that is only moved when a score passes
// it by more than KV8_SLACK.  So weights are at most 2^14, inside fp16, and those of fp16's smallest normal numbers are 2^-20 of
// the largest when m is exact.  x contains log2 of the page's value scale, so that the product with the codes of the values needs no
// scaling; the sum of the weights takes it out again.
constexpr float KV8_SHIFT = 6.0f, KV8_SLACK = 8.0f;
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// ---- launchers ------------------------------------------------------------------------------------
void launch_kv8_store(const Kv8 &c, int fmt, const void *const (&x)[2], int dtype, long long total, const long long (&tok)[2],
                      const long long (&head)[2], const int32_t *seqs, const int32_t *first, const int32_t *cu, int n, int max_new, cudaStream_t s);
bool launch_kv8_reserve(const Kv8 &c, const int32_t *seqs, const int32_t *add, int n, int32_t *first, cudaStream_t s);
bool launch_kv8_fork(const Kv8 &c, const int32_t *src, const int32_t *dst, int n, int2 *plan, cudaStream_t s);
void launch_kv8_fork_copy(const Kv8 &c, const int32_t *src, const int32_t *dst, int n, const int2 *plan, cudaStream_t s);
void launch_kv8_free(const Kv8 &c, const int32_t *seqs, int n, cudaStream_t s);
void launch_kv8_compact_plan(const Kv8 &c, int32_t *remap, int32_t *moves, cudaStream_t s);
void launch_kv8_compact_move(const Kv8 &c, const int32_t *remap, const int32_t *moves, int sm_count, cudaStream_t s);
void launch_kv8_copy(const Kv8 &from, const Kv8 &to, const int32_t *src, const int32_t *dst, int n, cudaStream_t s);
// Attention: scratch for a call's partial results, the kernel (EOSQ_OK, EOSQ_ERR_UNSUPPORTED or EOSQ_ERR_CUDA; nothing enqueued unless OK), and the one that
// joins what CTAs share between them.
size_t kv8_attend_scratch(int query_rows, int d);
int launch_kv8_attend(const Kv8Attend &a, int fmt, int dtype, int sm_count, cudaStream_t s);
void launch_kv8_join(const Kv8Attend &a, int dtype, int sm_count, cudaStream_t s);
// Tensor map over the codes of a layer's keys or values, [rows][d] bytes, in boxes of box_rows rows with a swizzle as wide as a row (eosq_tc.cu).
bool make_code_tensor_map(const void *codes, long long rows, int d, int box_rows, CUtensorMap *out);

}  // namespace eosq
