// C-ABI entry points of the 8-bit paged cache: argument checks, scratch and the launch sequence of each call.
#include <algorithm>
#include <cmath>

#include "eosq_kv8.cuh"

using namespace eosq;

namespace {

constexpr int MAX_POOL = 1 << 20;      // pages: prefix sums over needs stay in 32 bits
constexpr int MAX_TOKENS = 1 << 30;    // of a sequence: positions and windows add up in 32 bits
constexpr int MAX_ROWS_PER_HEAD = 1 << 30;

int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

// EOSQ_OK and the kernels' view of `layer`, or what is wrong with the cache.
int view_of(const eosq_kv8_t *c, int layer, Kv8 *out) {
    if (!c || c->layers <= 0 || c->num_pages <= 0 || c->kv_heads <= 0 || c->max_seqs <= 0 || c->max_pages <= 0 || layer < 0 || layer >= c->layers)
        return EOSQ_ERR_INVALID_ARG;
    const int ps = c->page_size;
    if ((ps != 16 && ps != 32 && ps != 64 && ps != 128) || (c->d != 64 && c->d != 128) || (c->format != EOSQ_KV_INT8 && c->format != EOSQ_KV_E4M3) ||
        c->num_pages > MAX_POOL || c->max_seqs > EOSQ_KV8_MAX_SEQS || static_cast<int64_t>(c->max_pages) * ps > MAX_TOKENS ||
        static_cast<int64_t>(c->num_pages) * c->kv_heads * ps >= (int64_t(1) << 31))
        return EOSQ_ERR_UNSUPPORTED;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->table || !c->lengths || !c->refs || !c->flags) return EOSQ_ERR_INVALID_ARG;
    auto off = [](const void *p, uintptr_t mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; };
    if (off(c->k, 15) || off(c->v, 15) || off(c->k_scale, 3) || off(c->v_scale, 3) || off(c->table, 3) || off(c->lengths, 3) || off(c->refs, 3) || off(c->flags, 3))
        return EOSQ_ERR_INVALID_ARG;
    if (!out) return EOSQ_OK;
    Kv8 v;
    v.layers = c->layers;
    v.num_pages = c->num_pages;
    v.heads = c->kv_heads;
    v.ps_shift = log2_of(ps);
    v.d_shift = log2_of(c->d);
    v.max_seqs = c->max_seqs;
    v.max_pages = c->max_pages;
    const size_t pages = static_cast<size_t>(layer) * c->num_pages;
    v.code[0] = c->k + pages * v.page_bytes();
    v.code[1] = c->v + pages * v.page_bytes();
    v.scale[0] = c->k_scale + pages * c->kv_heads;
    v.scale[1] = c->v_scale + pages * c->kv_heads;
    v.table = c->table;
    v.lengths = c->lengths;
    v.refs = c->refs;
    v.flags = reinterpret_cast<unsigned *>(c->flags);
    *out = v;
    return EOSQ_OK;
}

bool misaligned(const void *p, uintptr_t mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }
// Rows of d contiguous elements that vector loads can read: base and strides multiples of 16 bytes.
bool rows_ok(const void *p, int64_t tok, int64_t head, int esize) {
    return p && !misaligned(p, 15) && tok >= 0 && head >= 0 && (tok * esize) % 16 == 0 && (head * esize) % 16 == 0 && tok < (int64_t(1) << 40) && head < (int64_t(1) << 40);
}
bool list_ok(const void *p) { return p && !misaligned(p, 3); }

// No exception leaves a C entry point.
template <typename F>
int entry(F &&f) {
    try {
        return f();
    } catch (...) {
        return EOSQ_ERR_CUDA;
    }
}

// A fork's plan (lists with padding may be longer than the cache has sequences), a compaction's moves.
size_t pages_scratch(const eosq_kv8_t *c) {
    return std::max(sizeof(int2) * static_cast<size_t>(EOSQ_KV8_MAX_SEQS), sizeof(int32_t) * (64 + static_cast<size_t>(c->num_pages)));
}
size_t kv8_attend_scratch(int64_t most, int d) { return most <= 16 ? kv8_rows_scratch(d) : std::max(kv8_rows_scratch(d), kv8_tiles_scratch(d)); }
size_t cuts_scratch() { return align_up(sizeof(Kv8Cut) * KV8_MAX_CTAS, 256); }

int set_up_failed(eosq_ctx *ctx, const char *what) {
    ctx->last_error = what;
    return EOSQ_ERR_CUDA;
}

}  // namespace

extern "C" size_t eosq_kv8_workspace_bytes(const eosq_kv8_t *cache, int query_rows) {
    if (query_rows < 0 || view_of(cache, 0, nullptr) == EOSQ_ERR_UNSUPPORTED || !cache || cache->max_seqs <= 0 || cache->num_pages <= 0) return 0;
    size_t bytes = pages_scratch(cache);
    if (query_rows > 0) bytes = std::max(bytes, cuts_scratch() + kv8_attend_scratch(query_rows, cache->d));
    return align_up(bytes, 256);
}

extern "C" int eosq_kv8_reserve(eosq_ctx *ctx, const eosq_kv8_t *cache, const int32_t *seqs, const int32_t *add, int n, int32_t *first,
                                void *cuda_stream) {
    return entry([&]() -> int {
        Kv8 c;
        if (!ctx || n < 0) return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(cache, 0, &c)) return rc;
        if (n > EOSQ_KV8_MAX_SEQS) return EOSQ_ERR_UNSUPPORTED;
        if (n == 0) return EOSQ_OK;
        if (!list_ok(seqs) || !list_ok(add) || !list_ok(first) || !on_ctx_device(ctx)) return EOSQ_ERR_INVALID_ARG;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        bool ok = true;
        run_stage(ctx, ST_OTHER, s, [&] { ok = launch_kv8_reserve(c, seqs, add, n, first, s); });
        if (!ok) return set_up_failed(ctx, "eosq_kv8_reserve: launch set-up failed");
        return record_cuda(ctx, cudaGetLastError(), "eosq_kv8_reserve launch") ? EOSQ_ERR_CUDA : EOSQ_OK;
    });
}

extern "C" int eosq_kv8_store(eosq_ctx *ctx, const eosq_kv8_t *cache, int layer, const void *k, const void *v, int dtype, int64_t total,
                              int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                              const int32_t *seqs, const int32_t *first, const int32_t *cu, int n, int max_new, void *cuda_stream) {
    return entry([&]() -> int {
        Kv8 c;
        if (!ctx || n < 0 || total < 0 || max_new < 0 || (dtype != EOSQ_F16 && dtype != EOSQ_F32 && dtype != EOSQ_BF16)) return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(cache, layer, &c)) return rc;
        if (n > EOSQ_KV8_MAX_SEQS || total >= (int64_t(1) << 31) || max_new > MAX_TOKENS) return EOSQ_ERR_UNSUPPORTED;
        if (n == 0 || total == 0 || max_new == 0) return EOSQ_OK;
        const int esize = dtype == EOSQ_F32 ? 4 : 2;
        if (!rows_ok(k, k_token_stride, k_head_stride, esize) || !rows_ok(v, v_token_stride, v_head_stride, esize) || !list_ok(seqs) || !list_ok(first) ||
            !list_ok(cu) || !on_ctx_device(ctx))
            return EOSQ_ERR_INVALID_ARG;
        const int most = static_cast<int>(std::min<int64_t>(max_new, total));
        const int64_t slots = (most + c.page_size() - 2) / c.page_size() + 1;
        if (2 * slots * n * c.heads >= (int64_t(1) << 31)) return EOSQ_ERR_UNSUPPORTED;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        run_stage(ctx, ST_OTHER, s, [&] {
            launch_kv8_store(c, cache->format, {k, v}, dtype, total, {k_token_stride, v_token_stride}, {k_head_stride, v_head_stride}, seqs, first, cu, n,
                             most, ctx->sm_count, s);
        });
        return record_cuda(ctx, cudaGetLastError(), "eosq_kv8_store launch") ? EOSQ_ERR_CUDA : EOSQ_OK;
    });
}

extern "C" int eosq_kv8_attend(eosq_ctx *ctx, const eosq_kv8_t *cache, int layer, const void *q, int dtype, int64_t total,
                               int64_t q_token_stride, int64_t q_head_stride, const int32_t *seqs, const int32_t *cu, int n, int max_q, int G,
                               float scale, int causal, int window, void *out, int64_t out_token_stride, int64_t out_head_stride, float *lse,
                               void *workspace, size_t workspace_bytes, void *cuda_stream) {
    return entry([&]() -> int {
        Kv8Attend a;
        if (!ctx || n < 0 || total < 0 || max_q < 0 || G < 1 || window < 0 || (window > 0 && !causal) || !std::isfinite(scale) ||
            (dtype != EOSQ_F16 && dtype != EOSQ_BF16))
            return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(cache, layer, &a.c)) return rc;
        if (n > EOSQ_KV8_MAX_SEQS || total >= (int64_t(1) << 31) || static_cast<int64_t>(max_q) * G > MAX_ROWS_PER_HEAD || window > MAX_TOKENS)
            return EOSQ_ERR_UNSUPPORTED;
        if (n == 0 || total == 0 || max_q == 0) return EOSQ_OK;
        if (!rows_ok(q, q_token_stride, q_head_stride, 2) || !rows_ok(out, out_token_stride, out_head_stride, 2) || !list_ok(seqs) || !list_ok(cu) ||
            misaligned(lse, 3) || !workspace || misaligned(workspace, 255))
            return EOSQ_ERR_INVALID_ARG;
        const int most = static_cast<int>(std::min<int64_t>(max_q, total));
        // Units (key tiles of row tiles and heads) are counted in 32 bits: there are at most total * G / row tile + n row tiles, over as many keys as a row of the table has room for.
        const int64_t most_rows = static_cast<int64_t>(most) * G;
        const int split = kv8_split(most_rows, total * G, n, G);
        const bool few = !split && kv8_few_rows(most_rows, total * G, n, cache->d);
        const double row_tiles = static_cast<double>(total) * G / (few ? (most_rows <= 8 ? 8 : 16) : 256) + n;
        const double key_tiles = static_cast<double>(cache->max_pages) * cache->page_size / KV8_KEYS + 2.0 + KV8_COST_BOUND;
        if (row_tiles * key_tiles * cache->kv_heads >= 2147483648.0) return EOSQ_ERR_UNSUPPORTED;
        if (workspace_bytes < cuts_scratch() + kv8_attend_scratch(static_cast<int64_t>(most) * G, cache->d)) return EOSQ_ERR_BUFFER_TOO_SMALL;
        if (!on_ctx_device(ctx)) return EOSQ_ERR_INVALID_ARG;
        a.seqs = seqs;
        a.cu = cu;
        a.n = n;
        a.max_q = most;
        a.G = G;
        a.causal = causal != 0;
        a.window = window;
        // Rows of the table that hold few tokens: what CTAs could share of a row tile is less than joining it would cost, and the second kernel is not needed.
        // Shared and joined / whole, one query a sequence, 8 heads: 10.6 / 9.0 us at one sequence of 300 tokens, 15.3 / 11.8 at 19 of 440, 20.2 / 17.2 at 64
        // of 300, 16.7 / 16.8 at 64 of 1 to 500; 22.1 / 23.9 at 100 queries on 300 tokens and 25.6 / 22.4 at 300 queries.  With many row tiles to a CTA
        // what is saved falls (52.6 / 48.2 at 256) and runs of long sequences would make some CTAs late.  (The sequences' lengths are in device memory: what is asked for here is the
        // table's width, so short sequences in a wide table are shared out like long ones.)
        a.whole = static_cast<int64_t>(cache->max_pages) * cache->page_size <= 4 * KV8_KEYS && row_tiles * cache->kv_heads <= 8.0 * ctx->sm_count;
        a.total = total;
        a.q = q;
        a.out = out;
        a.lse = lse;
        a.q_tok = q_token_stride;
        a.q_head = q_head_stride;
        a.o_tok = out_token_stride;
        a.o_head = out_head_stride;
        a.scale_log2 = scale * 1.4426950408889634f;
        char *p = static_cast<char *>(workspace);
        a.cuts = reinterpret_cast<Kv8Cut *>(p);
        a.part = reinterpret_cast<float *>(p + cuts_scratch());
        a.err = ctx->dev_err;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        for (const bool rows : {true, false}) {
            if (!split && rows != few) continue;
            a.rows_min = (split && !rows) ? split + 1 : 1;
            a.rows_max = (split && rows) ? split : static_cast<int>(most_rows);
            int why = 0;
            run_stage(ctx, ST_OTHER, s, [&] {
                why = rows ? launch_kv8_rows(a, cache->format, dtype, ctx->sm_count, s) : launch_kv8_tiles(a, cache->format, dtype, ctx->sm_count, s);
            });
            if (why) return set_up_failed(ctx, "eosq_kv8_attend: tensor map or launch set-up failed");
            if (!a.whole) run_stage(ctx, ST_OTHER, s, [&] {
                if (rows) launch_kv8_rows_join(a, dtype, ctx->sm_count, s);
                else launch_kv8_tiles_join(a, dtype, ctx->sm_count, s);
            });
        }
        return record_cuda(ctx, cudaGetLastError(), "eosq_kv8_attend launch") ? EOSQ_ERR_CUDA : EOSQ_OK;
    });
}

extern "C" int eosq_kv8_fork(eosq_ctx *ctx, const eosq_kv8_t *cache, const int32_t *src, const int32_t *dst, int n, void *workspace,
                             size_t workspace_bytes, void *cuda_stream) {
    return entry([&]() -> int {
        Kv8 c;
        if (!ctx || n < 0) return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(cache, 0, &c)) return rc;
        if (n > EOSQ_KV8_MAX_SEQS || static_cast<int64_t>(n) * c.layers * 2 * ((c.page_bytes() >> 14) + 1) >= (int64_t(1) << 31)) return EOSQ_ERR_UNSUPPORTED;
        if (n == 0) return EOSQ_OK;
        if (!list_ok(src) || !list_ok(dst) || !workspace || misaligned(workspace, 255)) return EOSQ_ERR_INVALID_ARG;
        if (workspace_bytes < pages_scratch(cache)) return EOSQ_ERR_BUFFER_TOO_SMALL;
        if (!on_ctx_device(ctx)) return EOSQ_ERR_INVALID_ARG;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        int2 *plan = static_cast<int2 *>(workspace);
        bool ok = true;
        run_stage(ctx, ST_OTHER, s, [&] { ok = launch_kv8_fork(c, src, dst, n, plan, s); });
        if (!ok) return set_up_failed(ctx, "eosq_kv8_fork: launch set-up failed");
        run_stage(ctx, ST_OTHER, s, [&] { launch_kv8_fork_copy(c, src, dst, n, plan, s); });
        return record_cuda(ctx, cudaGetLastError(), "eosq_kv8_fork launch") ? EOSQ_ERR_CUDA : EOSQ_OK;
    });
}

extern "C" int eosq_kv8_free(eosq_ctx *ctx, const eosq_kv8_t *cache, const int32_t *seqs, int n, void *cuda_stream) {
    return entry([&]() -> int {
        Kv8 c;
        if (!ctx || n < 0) return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(cache, 0, &c)) return rc;
        if (n > EOSQ_KV8_MAX_SEQS) return EOSQ_ERR_UNSUPPORTED;
        if (n == 0) return EOSQ_OK;
        if (!list_ok(seqs) || !on_ctx_device(ctx)) return EOSQ_ERR_INVALID_ARG;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        run_stage(ctx, ST_OTHER, s, [&] { launch_kv8_free(c, seqs, n, s); });
        return record_cuda(ctx, cudaGetLastError(), "eosq_kv8_free launch") ? EOSQ_ERR_CUDA : EOSQ_OK;
    });
}

extern "C" int eosq_kv8_compact(eosq_ctx *ctx, const eosq_kv8_t *cache, int32_t *remap, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    return entry([&]() -> int {
        Kv8 c;
        if (!ctx) return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(cache, 0, &c)) return rc;
        if (!list_ok(remap) || !workspace || misaligned(workspace, 255)) return EOSQ_ERR_INVALID_ARG;
        if (workspace_bytes < pages_scratch(cache)) return EOSQ_ERR_BUFFER_TOO_SMALL;
        if (!on_ctx_device(ctx)) return EOSQ_ERR_INVALID_ARG;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        int32_t *moves = static_cast<int32_t *>(workspace);
        run_stage(ctx, ST_OTHER, s, [&] { launch_kv8_compact_plan(c, remap, moves, s); });
        run_stage(ctx, ST_OTHER, s, [&] { launch_kv8_compact_move(c, remap, moves, ctx->sm_count, s); });
        return record_cuda(ctx, cudaGetLastError(), "eosq_kv8_compact launch") ? EOSQ_ERR_CUDA : EOSQ_OK;
    });
}

extern "C" int eosq_kv8_copy_pages(eosq_ctx *ctx, const eosq_kv8_t *from, const eosq_kv8_t *to, const int32_t *src_pages, const int32_t *dst_pages,
                                   int n, void *cuda_stream) {
    return entry([&]() -> int {
        Kv8 a, b;
        if (!ctx || n < 0) return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(from, 0, &a)) return rc;
        if (int rc = view_of(to, 0, &b)) return rc;
        if (from->layers != to->layers || from->kv_heads != to->kv_heads || from->page_size != to->page_size || from->d != to->d || from->format != to->format)
            return EOSQ_ERR_INVALID_ARG;
        if (n > MAX_POOL || static_cast<int64_t>(n) * a.layers * 2 * ((a.page_bytes() >> 14) + 1) >= (int64_t(1) << 31)) return EOSQ_ERR_UNSUPPORTED;
        if (n == 0) return EOSQ_OK;
        if (!list_ok(src_pages) || !list_ok(dst_pages) || !on_ctx_device(ctx)) return EOSQ_ERR_INVALID_ARG;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        run_stage(ctx, ST_OTHER, s, [&] { launch_kv8_copy(a, b, src_pages, dst_pages, n, s); });
        return record_cuda(ctx, cudaGetLastError(), "eosq_kv8_copy_pages launch") ? EOSQ_ERR_CUDA : EOSQ_OK;
    });
}

extern "C" int eosq_kv8_check(eosq_ctx *ctx, const eosq_kv8_t *cache, uint32_t *flags, void *cuda_stream) {
    return entry([&]() -> int {
        Kv8 c;
        if (!ctx) return EOSQ_ERR_INVALID_ARG;
        if (int rc = view_of(cache, 0, &c)) return rc;
        if (!on_ctx_device(ctx)) return EOSQ_ERR_INVALID_ARG;
        cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        uint32_t got = 0;
        if (record_cuda(ctx, cudaMemcpyAsync(&got, c.flags, sizeof(got), cudaMemcpyDeviceToHost, s), "flags copy") ||
            record_cuda(ctx, cudaMemsetAsync(c.flags, 0, sizeof(got), s), "flags reset"))
            return EOSQ_ERR_CUDA;
        const int rc = eosq_check_status(ctx, nullptr, 0, nullptr, cuda_stream);   // synchronises
        if (flags) *flags = got;
        if (rc != EOSQ_OK) return rc;
        return got ? EOSQ_WARN_BLOCK_STATUS : EOSQ_OK;
    });
}
