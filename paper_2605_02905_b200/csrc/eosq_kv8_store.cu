// Writing into the 8-bit paged cache: scale of a page and head, codes of its new tokens, codes of its older tokens brought to a larger scale.
#include <algorithm>

#include <cuda_bf16.h>

#include "eosq_kv8.cuh"

namespace eosq {
namespace {

struct StoreArgs {
    Kv8 c;
    const void *x[2];
    long long tok[2], head[2];   // strides in elements
    const int32_t *seqs, *first, *cu;
    long long total;
    int slots, max_new;          // pages that an entry may touch
};

template <typename T> struct Chunk8;   // eight neighbouring channels of a token as they are read
template <> struct Chunk8<__half> {
    static constexpr uint32_t INF = 0x7c00u;   // bits of infinity: magnitudes order as their bits do
    uint4 v;
    __device__ __forceinline__ uint32_t top(uint32_t t) const {   // the larger of t and the magnitudes' bits, in two halves
        t = __vmaxu2(t, __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu));
        return __vmaxu2(t, __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    }
    static __device__ __forceinline__ uint32_t one(uint32_t t) { return max(t >> 16, t & 0xffffu); }
    static __device__ __forceinline__ float value(uint32_t t) { return __half2float(__ushort_as_half(static_cast<unsigned short>(t))); }
    __device__ __forceinline__ void load(const __half *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void floats(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            f[2 * i] = t.x;
            f[2 * i + 1] = t.y;
        }
    }
};
template <> struct Chunk8<__nv_bfloat16> {
    static constexpr uint32_t INF = 0x7f80u;
    uint4 v;
    __device__ __forceinline__ uint32_t top(uint32_t t) const {
        t = __vmaxu2(t, __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu));
        return __vmaxu2(t, __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    }
    static __device__ __forceinline__ uint32_t one(uint32_t t) { return max(t >> 16, t & 0xffffu); }
    static __device__ __forceinline__ float value(uint32_t t) { return __uint_as_float(t << 16); }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void floats(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
template <> struct Chunk8<float> {
    static constexpr uint32_t INF = 0x7f800000u;
    float4 a, b;
    __device__ __forceinline__ uint32_t top(uint32_t t) const {
        float f[8];
        floats(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) t = max(t, __float_as_uint(f[e]) & 0x7fffffffu);
        return t;
    }
    static __device__ __forceinline__ uint32_t one(uint32_t t) { return t; }
    static __device__ __forceinline__ float value(uint32_t t) { return __uint_as_float(t); }
    __device__ __forceinline__ void load(const float *p) {
        a = *reinterpret_cast<const float4 *>(p);
        b = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void floats(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
};

__device__ __forceinline__ float clamp_scale(float s) { return fminf(fmaxf(s, KV8_SCALE_MIN), KV8_SCALE_MAX); }

template <int FMT>
__device__ __forceinline__ float scale_of(float a) {
    if constexpr (FMT == EOSQ_KV_INT8) {
        return clamp_scale(__fdiv_rn(a, 127.0f));
    } else {
        // 448 = 1.75 * 2^8: the exponent of a less 8, or less 7 for a mantissa above 1.75.
        const uint32_t bits = __float_as_uint(a);
        const int e = static_cast<int>(bits >> 23) - 127 - (((bits & 0x7fffffu) > 0x600000u) ? 7 : 8);
        return __uint_as_float(static_cast<uint32_t>(min(max(e, -64), 64) + 127) << 23);
    }
}

// round(x / s) to a whole number, half to even, held to +-127, as if the quotient were exact; 0 for NaN.  x * (1 / s) is off by less than 2^-22 of itself, so the
// whole number next to it is the right one or a neighbour; what is left over, x - c s, is exact in fp32 (a multiple of 2^-24 of s's binade
// that is no larger than s), and says which.
__device__ __forceinline__ int code_int8(float x, float s, float inv) {
    if (!(x == x)) return 0;
    float c = rintf(fminf(fmaxf(x * inv, -128.0f), 128.0f));
    const float r = fmaf(-c, s, x), half = 0.5f * s;
    if (fabsf(r) >= half && fabsf(c) < 128.0f) {
        const bool odd = (static_cast<int>(c) & 1) != 0;
        if (r > half || (r == half && odd)) c += 1.0f;
        if (r < -half || (r == -half && odd)) c -= 1.0f;
    }
    return static_cast<int>(fminf(fmaxf(c, -127.0f), 127.0f));
}
template <int FMT>
__device__ __forceinline__ uint2 codes8(const float (&f)[8], float s, float inv) {   // any values
    uint2 r;
    if constexpr (FMT == EOSQ_KV_INT8) {
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = static_cast<uint32_t>(code_int8(f[i], s, inv)) & 0xffu;
        r.x = b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
        r.y = b[4] | (b[5] << 8) | (b[6] << 16) | (b[7] << 24);
    } else {
        // s is a power of two, so f * inv is exact and the conversion rounds once
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = (f[2 * i] == f[2 * i]) ? f[2 * i] * inv : 0.0f, hi = (f[2 * i + 1] == f[2 * i + 1]) ? f[2 * i + 1] * inv : 0.0f;
            h[i] = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
        }
        r.x = h[0] | (h[1] << 16);
        r.y = h[2] | (h[3] << 16);
    }
    return r;
}
// The same for finite values that s does not saturate.  int8: adding 1.5 * 2^23 rounds the quotient's estimate to a whole number, whose lowest byte is then the
// code; only where what is left over says that the estimate was on a border's wrong side, or on the border, is it looked at again.
template <int FMT>
__device__ __forceinline__ uint2 codes8_plain(const float (&f)[8], float s, float inv) {
    if constexpr (FMT == EOSQ_KV_INT8) {
        const uint64_t round = pair_of(12582912.0f, 12582912.0f), back = pair_of(-12582912.0f, -12582912.0f), by = pair_of(inv, inv), less = pair_of(-s, -s);
        uint32_t t[8];
        float off = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const uint64_t y = pair_of(f[i], f[i + 1]), x = fma_pair(y, by, round);
            float lo, hi;
            unpair(fma_pair(add_pair(x, back), less, y), lo, hi);
            off = fmaxf(off, fmaxf(fabsf(lo), fabsf(hi)));
            unpair(x, lo, hi);
            t[i] = __float_as_uint(lo);
            t[i + 1] = __float_as_uint(hi);
        }
        if (off >= 0.5f * s) return codes8<FMT>(f, s, inv);
        uint2 r;
        r.x = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
        r.y = __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410);
        return r;
    } else {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * i] * inv, f[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
    }
}
// An old code under a larger scale.  int8: the product has 31 bits and the quotient is at least 2^-25 of itself away from any border it is not on,
// so a division in 64 bits decides as the exact one does.
template <int FMT>
__device__ __forceinline__ uint32_t recode(uint32_t code, float s0, float s1) {
    if constexpr (FMT == EOSQ_KV_INT8) {
        const double q = static_cast<double>(static_cast<int8_t>(code)) * static_cast<double>(s0) / static_cast<double>(s1);
        return static_cast<uint32_t>(__double2int_rn(fmin(fmax(q, -127.0), 127.0))) & 0xffu;
    } else {
        const __half_raw h = __nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(code), __NV_E4M3);
        const float v = __half2float(__half(h)) * __fdiv_rn(s0, s1);
        return __nv_cvt_float_to_fp8((v == v) ? v : 0.0f, __NV_SATFINITE, __NV_E4M3);
    }
}

// A CTA takes a page of an entry, and of its heads' keys and values one after another every gridDim.y-th: the new tokens are read once and stay in
// registers (up to CHUNKS * 8 values a thread) between the largest magnitude and the codes, and the next ones are on their way meanwhile.  (A CTA per head and
// keys or values spent most of its time finding out where: 50.4 us for 27800 tokens, this 34.9, 171 MB in and out at 4.9 TB/s; a copy's rate would be
// 26.5.  More CTAs to an SM by fewer registers: 36.0.)
template <typename T, int FMT, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS) kv8_store_kernel(const StoreArgs a) {
    pdl_wait();
    const Kv8 &c = a.c;
    const int j = blockIdx.x % a.slots, i = blockIdx.x / a.slots;
    const int tid = threadIdx.x;
    const Kv8Seq sq = kv8_seq(c, a.seqs, a.cu, i, a.total, a.max_new);
    if (sq.m == 0) return;
    const int pos0 = a.first[i];
    if (pos0 < 0) return;
    if (pos0 > sq.len - sq.m) {
        if (tid == 0) raise(c, EOSQ_KV8_BAD_SEQ);
        return;
    }
    const int ps = c.page_size();
    const int col = (pos0 >> c.ps_shift) + j;
    const int begin = max(pos0, col << c.ps_shift), end = min(pos0 + sq.m, (col + 1) << c.ps_shift);
    if (begin >= end) return;
    const int page = c.table[static_cast<size_t>(sq.row) * c.max_pages + col];
    if (page < 0 || page >= c.num_pages) {
        if (tid == 0) raise(c, EOSQ_KV8_BAD_PAGE);
        return;
    }
    const int m = end - begin, t0 = begin & (ps - 1), per = c.d_shift - 3;   // tokens, the first one's place in the page, log2 of chunks per token
    const long long row0 = sq.q0 + static_cast<long long>(begin - pos0);
    __shared__ uint32_t tops[2][THREADS / 32];
    int turn = 0;
    auto ask = [&](int item, Chunk8<T> (&x)[CHUNKS], float &s0) {
        const int kv = item & 1, h = item >> 1;
        if (t0 > 0) s0 = c.scale[kv][static_cast<size_t>(page) * c.heads + h];   // (a page that begins here has none yet)
        const T *src = static_cast<const T *>(a.x[kv]) + row0 * a.tok[kv] + h * a.head[kv];
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const int q = tid + THREADS * k;
            x[k].zero();
            if (q < (m << per)) x[k].load(src + (q >> per) * a.tok[kv] + ((q & ((1 << per) - 1)) << 3));
        }
    };
    auto put = [&](int item, const Chunk8<T> (&x)[CHUNKS], float s0) {
        const int kv = item & 1, h = item >> 1;
        const size_t slot = static_cast<size_t>(page) * c.heads + h;
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) bits = x[k].top(bits);
        bits = Chunk8<T>::one(bits);
        auto over_all = [&](uint32_t v) {
            v = __reduce_max_sync(0xffffffffu, v);
            if constexpr (THREADS > 32) {
                uint32_t *at = tops[turn ^= 1];   // (two in turn: a barrier is between a write and the reads before it)
                if ((tid & 31) == 0) at[tid >> 5] = v;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < THREADS / 32; ++w) v = max(v, at[w]);
            }
            return v;
        };
        bits = over_all(bits);
        const bool finite = bits < Chunk8<T>::INF;
        float top = Chunk8<T>::value(bits);
        if (!finite) {   // again, without those that are not
            top = 0.0f;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                float f[8];
                x[k].floats(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, (fabsf(f[e]) <= 3.402823466e38f) ? fabsf(f[e]) : 0.0f);
            }
            top = __uint_as_float(over_all(__float_as_uint(top)));
        }
        float s1 = scale_of<FMT>(top);
        if (t0 > 0) s1 = fmaxf(s1, clamp_scale(s0));
        uint8_t *dst = c.code[kv] + (slot << (c.ps_shift + c.d_shift));
        if (t0 > 0 && s1 > s0) {
            uint32_t *old = reinterpret_cast<uint32_t *>(dst);
            for (int w = tid; w < (t0 << (c.d_shift - 2)); w += THREADS) {
                const uint32_t v = old[w];
                uint32_t r = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b) r |= recode<FMT>((v >> (8 * b)) & 0xffu, s0, s1) << (8 * b);
                old[w] = r;
            }
        }
        const float inv = __fdiv_rn(1.0f, s1);
        const bool plain = finite && s1 < KV8_SCALE_MAX;
        uint2 *out = reinterpret_cast<uint2 *>(dst + (static_cast<size_t>(t0) << c.d_shift));
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            const int q = tid + THREADS * k;
            if (q < (m << per)) {
                float f[8];
                x[k].floats(f);
                out[q] = plain ? codes8_plain<FMT>(f, s1, inv) : codes8<FMT>(f, s1, inv);
            }
        }
        if (tid == 0) c.scale[kv][slot] = s1;   // (every thread has its s0: the reduction has been between)
    };
    const int items = 2 * c.heads, step = gridDim.y;
    Chunk8<T> x[CHUNKS], y[CHUNKS];
    float sx = 0.0f, sy = 0.0f;
    ask(blockIdx.y, x, sx);
    for (int item = blockIdx.y; item < items; item += 2 * step) {
        if (item + step < items) ask(item + step, y, sy);
        put(item, x, sx);
        if (item + step >= items) break;
        if (item + 2 * step < items) ask(item + 2 * step, x, sx);
        put(item + step, y, sy);
    }
}

template <typename T, int FMT>
void launch_store(const StoreArgs &a, dim3 grid, int chunks, cudaStream_t s) {
    if (chunks <= 32) launch_dependent(kv8_store_kernel<T, FMT, 32, 1>, grid, 32, 0, s, a);
    else if (chunks <= 256) launch_dependent(kv8_store_kernel<T, FMT, 128, 2>, grid, 128, 0, s, a);
    else if (chunks <= 512) launch_dependent(kv8_store_kernel<T, FMT, 128, 4>, grid, 128, 0, s, a);
    else if (chunks <= 1024) launch_dependent(kv8_store_kernel<T, FMT, 256, 4>, grid, 256, 0, s, a);
    else launch_dependent(kv8_store_kernel<T, FMT, 512, 4>, grid, 512, 0, s, a);
}

}  // namespace

void launch_kv8_store(const Kv8 &c, int fmt, const void *const (&x)[2], int dtype, long long total, const long long (&tok)[2],
                      const long long (&head)[2], const int32_t *seqs, const int32_t *first, const int32_t *cu, int n, int max_new, int sm_count, cudaStream_t s) {
    StoreArgs a;
    a.c = c;
    for (int kv = 0; kv < 2; ++kv) {
        a.x[kv] = x[kv];
        a.tok[kv] = tok[kv];
        a.head[kv] = head[kv];
    }
    a.seqs = seqs;
    a.first = first;
    a.cu = cu;
    a.total = total;
    a.max_new = max_new;
    a.slots = (max_new + c.page_size() - 2) / c.page_size() + 1;
    // Of a page's heads, keys and values, so many CTAs' shares that there are eight CTAs per SM, if there are pages for fewer.
    const long long pages = static_cast<long long>(n) * a.slots, wanted = (8ll * sm_count + pages - 1) / pages;
    const dim3 grid(static_cast<unsigned>(pages), static_cast<unsigned>(std::min<long long>(2ll * c.heads, std::max(wanted, 2ll))));
    const int chunks = std::min(max_new, c.page_size()) << (c.d_shift - 3);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (fmt == EOSQ_KV_INT8) launch_store<T, EOSQ_KV_INT8>(a, grid, chunks, s);
        else launch_store<T, EOSQ_KV_E4M3>(a, grid, chunks, s);
    };
    if (dtype == EOSQ_F16) go(__half());
    else if (dtype == EOSQ_BF16) go(__nv_bfloat16());
    else go(0.0f);
}

}  // namespace eosq
