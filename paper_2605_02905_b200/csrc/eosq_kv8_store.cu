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
    uint4 v;
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
    uint4 v;
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
    float4 a, b;
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
__device__ __forceinline__ uint2 codes8(const float (&f)[8], float s, float inv) {
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

// A CTA per page, head and keys or values: the new tokens of the page are read once and stay in registers (up to CHUNKS * 8 values a thread) between
// the largest magnitude and the codes.
template <typename T, int FMT, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS) kv8_store_kernel(const StoreArgs a) {
    pdl_wait();
    const Kv8 &c = a.c;
    const int kv = blockIdx.x & 1;
    const int h = (blockIdx.x >> 1) % c.heads, rest = (blockIdx.x >> 1) / c.heads;
    const int j = rest % a.slots, i = rest / a.slots;
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
    const T *src = static_cast<const T *>(a.x[kv]) + (sq.q0 + static_cast<long long>(begin - pos0)) * a.tok[kv] + h * a.head[kv];
    Chunk8<T> x[CHUNKS];
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const int q = tid + THREADS * k;
        x[k].zero();
        if (q < (m << per)) x[k].load(src + (q >> per) * a.tok[kv] + ((q & ((1 << per) - 1)) << 3));
    }
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        float f[8];
        x[k].floats(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = fabsf(f[e]);
            top = fmaxf(top, (v <= 3.402823466e38f) ? v : 0.0f);
        }
    }
    const size_t slot = static_cast<size_t>(page) * c.heads + h;
    float *scale_at = c.scale[kv] + slot;
    const float s0 = *scale_at;
    uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));   // magnitudes order as their bits do
    if constexpr (THREADS > 32) {
        __shared__ uint32_t tops[THREADS / 32];
        if ((tid & 31) == 0) tops[tid >> 5] = bits;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) bits = max(bits, tops[w]);
    }
    float s1 = scale_of<FMT>(__uint_as_float(bits));
    if (t0 > 0) s1 = fmaxf(s1, clamp_scale(s0));
    __syncwarp();
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
    uint2 *out = reinterpret_cast<uint2 *>(dst + (static_cast<size_t>(t0) << c.d_shift));
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        const int q = tid + THREADS * k;
        if (q < (m << per)) {
            float f[8];
            x[k].floats(f);
            out[q] = codes8<FMT>(f, s1, inv);
        }
    }
    if (tid == 0 && s1 != s0) *scale_at = s1;   // (every thread has read s0: the barrier, or the warp, is between)
}

template <typename T, int FMT>
void launch_store(const StoreArgs &a, long long ctas, int chunks, cudaStream_t s) {
    const dim3 grid(static_cast<unsigned>(ctas));
    if (chunks <= 32) launch_dependent(kv8_store_kernel<T, FMT, 32, 1>, grid, 32, 0, s, a);
    else if (chunks <= 256) launch_dependent(kv8_store_kernel<T, FMT, 128, 2>, grid, 128, 0, s, a);
    else if (chunks <= 1024) launch_dependent(kv8_store_kernel<T, FMT, 256, 4>, grid, 256, 0, s, a);
    else launch_dependent(kv8_store_kernel<T, FMT, 256, 8>, grid, 256, 0, s, a);
}

}  // namespace

void launch_kv8_store(const Kv8 &c, int fmt, const void *const (&x)[2], int dtype, long long total, const long long (&tok)[2],
                      const long long (&head)[2], const int32_t *seqs, const int32_t *first, const int32_t *cu, int n, int max_new, cudaStream_t s) {
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
    const long long ctas = 2ll * n * a.slots * c.heads;
    const int chunks = std::min(max_new, c.page_size()) << (c.d_shift - 3);
    auto go = [&](auto t) {
        using T = decltype(t);
        if (fmt == EOSQ_KV_INT8) launch_store<T, EOSQ_KV_INT8>(a, ctas, chunks, s);
        else launch_store<T, EOSQ_KV_E4M3>(a, ctas, chunks, s);
    };
    if (dtype == EOSQ_F16) go(__half());
    else if (dtype == EOSQ_BF16) go(__nv_bfloat16());
    else go(0.0f);
}

}  // namespace eosq
