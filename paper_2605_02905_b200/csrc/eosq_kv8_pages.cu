// Pages of the 8-bit cache: taking them, sharing them between sequences, giving them back, moving the used ones together.  The
// decisions (which page goes where) are one CTA's: prefix sums over the list and over the pool, so that the lowest free page is always taken
// next and a call's result does not depend on how its threads run.  The bytes are moved by a kernel behind it.
#include <climits>

#include "eosq_kv8.cuh"

namespace eosq {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PAGES_PER_LANE = 8;   // pages that a thread looks at per step: 8192 a step, their loads under way together
constexpr int PAGES_PER_STEP = PLAN_THREADS * PAGES_PER_LANE;
constexpr int FOUND = 4096;         // pages that a list may need before they are looked for a second time
constexpr size_t PLAN_SMEM = sizeof(int) * (2 * EOSQ_KV8_MAX_SEQS + 1 + FOUND);

// Exclusive prefix sum of v over the CTA, and the total.
__device__ __forceinline__ int block_prefix(int v, int &total) {
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();   // sums of the call before have been read
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    int w = (lane < PLAN_THREADS / 32) ? sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return x - v + (warp ? before : 0);
}

// Calls found(rank, page) for every page with wanted(page, refs), in ascending order, ranks from 0; stops once `most` have been found.  Every
// thread of the CTA takes part.  Returns how many there were up to there.
template <typename W, typename F>
__device__ __forceinline__ int each_page(const Kv8 &c, int most, W &&wanted, F &&found) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int rank = 0;
    for (long long base = 0; base < c.num_pages && rank < most; base += PAGES_PER_STEP) {
        const long long p0 = base + warp * 32 * PAGES_PER_LANE + lane;
        int refs[PAGES_PER_LANE];
#pragma unroll
        for (int k = 0; k < PAGES_PER_LANE; ++k) refs[k] = (p0 + 32 * k < c.num_pages) ? c.refs[p0 + 32 * k] : 0;
        unsigned mask[PAGES_PER_LANE];
        int mine = 0;
#pragma unroll
        for (int k = 0; k < PAGES_PER_LANE; ++k) {
            mask[k] = __ballot_sync(0xffffffffu, p0 + 32 * k < c.num_pages && wanted(static_cast<int>(p0 + 32 * k), refs[k]));
            mine += __popc(mask[k]);
        }
        int total;
        int r = rank + __shfl_sync(0xffffffffu, block_prefix(lane == 0 ? mine : 0, total), 0);
#pragma unroll
        for (int k = 0; k < PAGES_PER_LANE; ++k) {
            if ((mask[k] >> lane) & 1u) found(r + __popc(mask[k] & ((1u << lane) - 1u)), static_cast<int>(p0 + 32 * k));
            r += __popc(mask[k]);
        }
        rank += total;
    }
    return rank;
}

// An entry's length before, what it will be, and the pages that it needs; need < 0: refused.  Padding has need = -1 and raises nothing.
struct Entry {
    int row, from, len, need;
};

struct ReserveList {
    const int32_t *seqs, *add;
    __device__ __forceinline__ int key(int i) const { return seqs[i]; }
    __device__ __forceinline__ Entry get(const Kv8 &c, int i, const int *seen, unsigned &flags) const {
        Entry e{seqs[i], 0, 0, -1};
        if (e.row == -1) return e;
        if (e.row < 0 || e.row >= c.max_seqs || seen[e.row] != i || add[i] < 0 || c.lengths[e.row] < 0) {
            flags |= EOSQ_KV8_BAD_SEQ;
            return e;
        }
        e.from = c.lengths[e.row];
        const long long after = static_cast<long long>(e.from) + add[i], room = static_cast<long long>(c.max_pages) << c.ps_shift;
        if (after > room) {
            flags |= EOSQ_KV8_TOO_LONG;
            return e;
        }
        e.len = static_cast<int>(after);
        const int ps = c.page_size();
        e.need = ((e.len + ps - 1) >> c.ps_shift) - ((e.from + ps - 1) >> c.ps_shift);
        return e;
    }
};
struct ForkList {
    const int32_t *src, *dst;
    __device__ __forceinline__ int key(int i) const { return src[i] == -1 ? -1 : dst[i]; }
    __device__ __forceinline__ Entry get(const Kv8 &c, int i, const int *seen, unsigned &flags) const {
        Entry e{dst[i], 0, 0, -1};
        if (src[i] == -1 || e.row == -1) return e;
        const long long room = static_cast<long long>(c.max_pages) << c.ps_shift;
        if (e.row < 0 || e.row >= c.max_seqs || seen[e.row] != i || src[i] < 0 || src[i] >= c.max_seqs || c.lengths[e.row] != 0 ||
            c.lengths[src[i]] < 0 || c.lengths[src[i]] > room) {
            flags |= EOSQ_KV8_BAD_SEQ;
            return e;
        }
        e.from = e.len = c.lengths[src[i]];
        e.need = (e.len & (c.page_size() - 1)) ? 1 : 0;
        return e;
    }
};

// Which entries of a list get their pages, and which pages: entries in order, pages in ascending order.  take(i, entry, k, page) is called for an entry's
// k-th page, done(i, entry, ok) for every entry.
template <typename L, typename T, typename D>
__device__ __forceinline__ void deal_pages(const Kv8 &c, const L &list, int n, T &&take, D &&done) {
    extern __shared__ int plan_smem[];
    // [max_seqs] first entry that lists a sequence; [n + 1] pages needed before an entry; [FOUND] free pages
    int *seen = plan_smem, *before = plan_smem + c.max_seqs, *pages = before + n + 1;
    const int tid = threadIdx.x;
    unsigned flags = 0;
    for (int s = tid; s < c.max_seqs; s += PLAN_THREADS) seen[s] = INT_MAX;
    __syncthreads();
    for (int i = tid; i < n; i += PLAN_THREADS) {
        const int s = list.key(i);
        if (s >= 0 && s < c.max_seqs) atomicMin(&seen[s], i);
    }
    __syncthreads();
    int wanted = 0;
    Entry mine{-1, 0, 0, -1};   // of the first PLAN_THREADS entries: this thread's
    for (int base = 0; base < n; base += PLAN_THREADS) {
        const int i = base + tid;
        // (a step adds at most 1024 * (2^20 + 1): pools have at most 2^20 pages)
        int need = 0;
        if (i < n) {
            const Entry e = list.get(c, i, seen, flags);
            if (base == 0) mine = e;
            need = min(max(e.need, 0), c.num_pages + 1);
        }
        int total;
        const int p = block_prefix(need, total);
        if (i < n) before[i] = wanted + p;
        wanted = min(wanted + total, 1 << 29);
    }
    if (tid == 0) before[n] = wanted;
    __syncthreads();
    auto is_free = [](int, int refs) { return refs == 0; };
    const int have = min(each_page(c, wanted, is_free, [&](int rank, int page) { if (rank < FOUND) pages[rank] = page; }), wanted);
    auto give = [&](int rank, int page) {
        if (rank >= have) return;
        int lo = 0, hi = n;   // the last entry with before[i] <= rank
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (before[mid] <= rank) lo = mid;
            else hi = mid;
        }
        if (before[lo + 1] > have) return;   // refused
        unsigned unused = 0;
        take(lo, list.get(c, lo, seen, unused), rank - before[lo], page);
        c.refs[page] = 1;
    };
    __syncthreads();
    if (have <= FOUND) {
        for (int r = tid; r < have; r += PLAN_THREADS) give(r, pages[r]);
    } else {
        each_page(c, have, is_free, give);
    }
    __syncthreads();
    for (int i = tid; i < n; i += PLAN_THREADS) {
        unsigned again = 0;   // (raised before)
        const Entry e = i < PLAN_THREADS ? mine : list.get(c, i, seen, again);
        const bool ok = e.need == 0 || (e.need > 0 && before[i] + e.need <= have);
        if (e.need > 0 && !ok) flags |= EOSQ_KV8_NO_PAGE;
        done(i, e, ok);
    }
    flags = __reduce_or_sync(0xffffffffu, flags);
    if ((tid & 31) == 0 && flags) raise(c, flags);
}

__global__ void __launch_bounds__(PLAN_THREADS) kv8_reserve_kernel(const Kv8 c, const int32_t *seqs, const int32_t *add, int n, int32_t *first) {
    pdl_wait();
    deal_pages(
        c, ReserveList{seqs, add}, n,
        [&](int, const Entry &e, int k, int page) {
            c.table[static_cast<size_t>(e.row) * c.max_pages + ((e.from + c.page_size() - 1) >> c.ps_shift) + k] = page;
        },
        [&](int i, const Entry &e, bool ok) {
            first[i] = ok ? e.from : -1;
            if (ok) c.lengths[e.row] = e.len;
        });
}

// plan[i]: tokens of the new sequence (-1: refused) and the page for its last, partly filled one.
__global__ void __launch_bounds__(PLAN_THREADS) kv8_fork_kernel(const Kv8 c, const int32_t *src, const int32_t *dst, int n, int2 *plan) {
    pdl_wait();
    pdl_trigger();   // the copying kernel's CTAs find their places meanwhile
    deal_pages(
        c, ForkList{src, dst}, n, [&](int i, const Entry &, int, int page) { plan[i].y = page; },
        [&](int i, const Entry &e, bool ok) { plan[i].x = ok ? e.len : -1; });
}

// ---- moving pages ------------------------------------------------------------------------------
// A page of one layer's keys or values is contiguous; it moves in pieces of 16 KB, a CTA each, 64 bytes a thread under way.  HBM bounds it: 378 MB read and written
// in 67 us, 5.6 TB/s (a copy 6.5).  Few pages: the plan's chain of loads and barriers, 5 us, and two launches.
constexpr int COPY_THREADS = 256, COPY_LOADS = 4;
constexpr size_t PIECE = COPY_THREADS * COPY_LOADS * 16;

__host__ __device__ __forceinline__ int pieces_of(const Kv8 &c) { return static_cast<int>((c.page_bytes() + PIECE - 1) / PIECE); }

__device__ __forceinline__ void copy_piece(const Kv8 &from, const Kv8 &to, int src, int dst, int layer, int kv, int piece) {
    const size_t bytes = from.page_bytes();
    const size_t a = (static_cast<size_t>(layer) * from.num_pages + src), b = (static_cast<size_t>(layer) * to.num_pages + dst);
    const uint4 *x = reinterpret_cast<const uint4 *>(from.code[kv] + a * bytes);
    uint4 *y = reinterpret_cast<uint4 *>(to.code[kv] + b * bytes);
    const size_t end = bytes / 16, q0 = static_cast<size_t>(piece) * (PIECE / 16) + threadIdx.x;
    uint4 v[COPY_LOADS];
#pragma unroll
    for (int k = 0; k < COPY_LOADS; ++k)
        if (q0 + k * COPY_THREADS < end) v[k] = x[q0 + k * COPY_THREADS];
#pragma unroll
    for (int k = 0; k < COPY_LOADS; ++k)
        if (q0 + k * COPY_THREADS < end) y[q0 + k * COPY_THREADS] = v[k];
    if (piece == 0)
        for (int h = threadIdx.x; h < from.heads; h += COPY_THREADS) to.scale[kv][b * to.heads + h] = from.scale[kv][a * from.heads + h];
}

__global__ void __launch_bounds__(COPY_THREADS) kv8_fork_copy_kernel(const Kv8 c, const int32_t *src, const int32_t *dst, const int2 *plan, int pieces) {
    pdl_wait();
    const int per = c.layers * 2 * pieces, i = blockIdx.x / per, q = blockIdx.x % per;
    const int len = plan[i].x;
    if (len <= 0) return;
    const int full = len >> c.ps_shift;
    const bool tail = (len & (c.page_size() - 1)) != 0;
    const int32_t *from = c.table + static_cast<size_t>(src[i]) * c.max_pages;
    int32_t *to = c.table + static_cast<size_t>(dst[i]) * c.max_pages;
    if (q == 0) {
        for (int col = threadIdx.x; col < full; col += COPY_THREADS) {
            const int p = from[col];
            if (p < 0 || p >= c.num_pages) {
                raise(c, EOSQ_KV8_BAD_PAGE);
                continue;
            }
            to[col] = p;
            atomicAdd(&c.refs[p], 1);
        }
        if (threadIdx.x == 0) c.lengths[dst[i]] = len;
    }
    if (!tail) return;
    const int p = from[full];
    const bool there = p >= 0 && p < c.num_pages;
    if (q == 0 && threadIdx.x == 0) {
        if (there) {
            to[full] = plan[i].y;
        } else {   // nothing to copy: the page that was taken for it is free again, and the copy's entry is none, as its other ones outside the pool are
            c.refs[plan[i].y] = 0;
            raise(c, EOSQ_KV8_BAD_PAGE);
        }
    }
    if (!there) return;
    copy_piece(c, c, p, plan[i].y, q / (2 * pieces), (q / pieces) & 1, q % pieces);
}

__global__ void __launch_bounds__(COPY_THREADS) kv8_copy_kernel(const Kv8 from, const Kv8 to, const int32_t *src, const int32_t *dst, int pieces) {
    pdl_wait();
    const int per = from.layers * 2 * pieces, i = blockIdx.x / per, q = blockIdx.x % per;
    const int a = src[i], b = dst[i];
    if (a < 0 || a >= from.num_pages || b < 0 || b >= to.num_pages) {
        if (threadIdx.x == 0) raise(to, EOSQ_KV8_BAD_PAGE);
        return;
    }
    copy_piece(from, to, a, b, q / (2 * pieces), (q / pieces) & 1, q % pieces);
}

// ---- giving back ---------------------------------------------------------------------------------
__global__ void __launch_bounds__(128) kv8_free_kernel(const Kv8 c, const int32_t *seqs) {
    pdl_wait();
    const int i = blockIdx.x, s = seqs[i];
    if (s == -1) return;
    bool again = s < 0 || s >= c.max_seqs;
    for (int j = threadIdx.x; j < i; j += 128) again |= seqs[j] == s;
    if (__syncthreads_or(again)) {
        if (threadIdx.x == 0) raise(c, EOSQ_KV8_BAD_SEQ);
        return;
    }
    int32_t *row = c.table + static_cast<size_t>(s) * c.max_pages;
    for (int col = threadIdx.x; col < c.max_pages; col += 128) {
        const int p = row[col];
        if (p == -1) continue;
        row[col] = -1;
        if (p < 0 || p >= c.num_pages || atomicSub(&c.refs[p], 1) <= 0) {
            if (p >= 0 && p < c.num_pages) atomicAdd(&c.refs[p], 1);   // it was free already: the table and the counts disagree
            raise(c, EOSQ_KV8_BAD_PAGE);
        }
    }
    if (threadIdx.x == 0) c.lengths[s] = 0;
}

// ---- compaction ----------------------------------------------------------------------------------
// moves: [0] how many, from [64] on the free pages below L, then the used ones from L on, both ascending.
constexpr int MOVES_AT = 64;
__global__ void __launch_bounds__(PLAN_THREADS) kv8_compact_kernel(const Kv8 c, int32_t *remap, int32_t *moves) {
    pdl_wait();
    pdl_trigger();
    const int used = each_page(c, INT_MAX, [](int, int refs) { return refs != 0; }, [](int, int) {});
    int32_t *list = moves + MOVES_AT;
    const int both = each_page(
        c, INT_MAX,
        [&](int p, int refs) {
            remap[p] = refs != 0 ? p : -1;
            return (p < used) != (refs != 0);
        },
        [&](int rank, int page) { list[rank] = page; });
    __syncthreads();
    const int n = both / 2;
    for (int r = threadIdx.x; r < n; r += PLAN_THREADS) {
        const int to = list[r], of = list[n + r];
        remap[of] = to;
        c.refs[to] = c.refs[of];
        c.refs[of] = 0;
    }
    if (threadIdx.x == 0) moves[0] = n;
}

__global__ void __launch_bounds__(COPY_THREADS) kv8_move_kernel(const Kv8 c, const int32_t *remap, const int32_t *moves, int pieces) {
    pdl_wait();
    const int n = moves[0];
    const long long per = static_cast<long long>(c.layers) * 2 * pieces, all = per * n;
    for (long long u = blockIdx.x; u < all; u += gridDim.x) {
        const int r = static_cast<int>(u / per), q = static_cast<int>(u % per);
        copy_piece(c, c, moves[MOVES_AT + n + r], moves[MOVES_AT + r], q / (2 * pieces), (q / pieces) & 1, q % pieces);
    }
    const long long entries = static_cast<long long>(c.max_seqs) * c.max_pages;
    for (long long e = static_cast<long long>(blockIdx.x) * COPY_THREADS + threadIdx.x; e < entries; e += static_cast<long long>(gridDim.x) * COPY_THREADS) {
        const int p = c.table[e];
        if (p == -1) continue;
        const int to = (p >= 0 && p < c.num_pages) ? remap[p] : -1;
        if (to < 0) raise(c, EOSQ_KV8_BAD_PAGE);
        else if (to != p) c.table[e] = to;
    }
}

}  // namespace

bool launch_kv8_reserve(const Kv8 &c, const int32_t *seqs, const int32_t *add, int n, int32_t *first, cudaStream_t s) {
    if (!ensure_dynamic_smem(reinterpret_cast<const void *>(kv8_reserve_kernel), PLAN_SMEM)) return false;
    launch_dependent(kv8_reserve_kernel, dim3(1), PLAN_THREADS, sizeof(int) * (c.max_seqs + n + 1 + FOUND), s, c, seqs, add, n, first);
    return true;
}
bool launch_kv8_fork(const Kv8 &c, const int32_t *src, const int32_t *dst, int n, int2 *plan, cudaStream_t s) {
    if (!ensure_dynamic_smem(reinterpret_cast<const void *>(kv8_fork_kernel), PLAN_SMEM)) return false;
    launch_dependent(kv8_fork_kernel, dim3(1), PLAN_THREADS, sizeof(int) * (c.max_seqs + n + 1 + FOUND), s, c, src, dst, n, plan);
    return true;
}
void launch_kv8_fork_copy(const Kv8 &c, const int32_t *src, const int32_t *dst, int n, const int2 *plan, cudaStream_t s) {
    const int pieces = pieces_of(c);
    launch_dependent(kv8_fork_copy_kernel, dim3(static_cast<unsigned>(n * c.layers * 2 * pieces)), COPY_THREADS, 0, s, c, src, dst, plan, pieces);
}
void launch_kv8_free(const Kv8 &c, const int32_t *seqs, int n, cudaStream_t s) {
    launch_dependent(kv8_free_kernel, dim3(static_cast<unsigned>(n)), 128, 0, s, c, seqs);
}
void launch_kv8_compact_plan(const Kv8 &c, int32_t *remap, int32_t *moves, cudaStream_t s) {
    launch_dependent(kv8_compact_kernel, dim3(1), PLAN_THREADS, 0, s, c, remap, moves);
}
void launch_kv8_compact_move(const Kv8 &c, const int32_t *remap, const int32_t *moves, int sm_count, cudaStream_t s) {
    launch_dependent(kv8_move_kernel, dim3(static_cast<unsigned>(8 * sm_count)), COPY_THREADS, 0, s, c, remap, moves, pieces_of(c));
}
void launch_kv8_copy(const Kv8 &from, const Kv8 &to, const int32_t *src, const int32_t *dst, int n, cudaStream_t s) {
    const int pieces = pieces_of(from);
    launch_dependent(kv8_copy_kernel, dim3(static_cast<unsigned>(n * from.layers * 2 * pieces)), COPY_THREADS, 0, s, from, to, src, dst, pieces);
}

}  // namespace eosq
