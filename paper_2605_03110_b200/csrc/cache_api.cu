// C ABI of the paged key / value cache: argument checks, views, which kernel a call takes.
#include <float.h>
#include <math.h>

#include "api_util.h"
#include "cache_args.h"
#include "cache_dev.cuh"

using namespace ada;

namespace {

// the checks that every call makes, and what its kernels get
ada_status open_cache(const ada_ctx* ctx, const ada_kv_cache* kv, int64_t B, const int32_t* off, const int32_t* len,
                      int64_t N, ada_dtype dt, CacheView* c, Ragged* r) {
    if (ctx == nullptr) return ADA_ERR_INVALID_ARG;
    const ada_status st = check_cache(kv, B, off, len, N, dt);
    if (st != ADA_OK) return st;
    if (!gram_tc_available()) return ADA_ERR_UNSUPPORTED;
    c->k = static_cast<__nv_bfloat16*>(kv->k); c->v = static_cast<__nv_bfloat16*>(kv->v);
    c->kmin = static_cast<__nv_bfloat16*>(kv->kmin); c->kmax = static_cast<__nv_bfloat16*>(kv->kmax);
    c->table = kv->table; c->table_ld = kv->table_ld; c->page_stride = kv->page_stride;
    c->n_pages = (int)kv->n_pages; c->max_pages = (int)kv->max_pages; c->shift = page_shift(kv->page_size);
    c->h_kv = (int)kv->h_kv; c->d = (int)kv->d_h;
    r->off = off; r->len = len; r->B = (int)B; r->N = (int)N;
    return ADA_OK;
}

// Partial results and their counters: of one size per device, so that they are allocated once and a captured
// graph keeps a valid pointer whatever is called later.
cudaError_t ensure_cache_ws(ada_ctx* ctx, cudaStream_t s) {
    if (ctx->cache_ws != nullptr) return cudaSuccess;
    // While a graph is captured the counters would be cleared by the graph's first replay, not now.
    cudaStreamCaptureStatus capture;
    cudaError_t e = cudaStreamIsCapturing(s, &capture);
    if (e != cudaSuccess) return e;
    if (capture != cudaStreamCaptureStatusNone) return cudaErrorStreamCaptureUnsupported;
    const size_t part = 2 * (size_t)ctx->sm_count * cache_part_floats() * 4, ctr = 8 * (size_t)ctx->sm_count * 4;
    char* p = nullptr;
    if ((e = cudaMalloc(&p, part + ctr)) != cudaSuccess) return e;
    e = cudaMemsetAsync(p + part, 0, ctr, s);
    if (e != cudaSuccess) { cudaFree(p); return e; }
    ctx->cache_ws = p;
    ctx->cache_part = reinterpret_cast<float*>(p);
    ctx->cache_ctr = reinterpret_cast<unsigned*>(p + part);
    ctx->cache_ctr_bytes = ctr;
    return cudaSuccess;
}

// scale of the scores, times log2(e).  Not 0 where fp32 has nothing smaller: 0 times a masked score, -inf, is NaN.
// (2^-149 times the largest product of fp32 is 5e-7: equal weights either way.)
float score_scale(double scale, int64_t d) {
    const float f = (float)((scale == 0.0 ? 1.0 / sqrt((double)d) : scale) * 1.4426950408889634);
    return f == 0.f ? FLT_TRUE_MIN : f;
}

}  // namespace

extern "C" {

ada_status ada_cache_append(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off, const int32_t* len,
                            int32_t* len_out, int64_t N, const void* K, int64_t ldk, const void* V, int64_t ldv,
                            ada_dtype dt, const void* Q, int64_t h, int64_t ldq, void* q_out, int64_t ldqo,
                            const void* q_norm, const void* k_norm, double eps, const double* inv_freq, int64_t rot,
                            const int32_t* pos0, const int32_t* rep_idx, const int32_t* rep_cnt, uint32_t flags,
                            void* stream) {
    CacheView c;
    Ragged r;
    ada_status st = open_cache(ctx, cache, B, off, len, N, dt, &c, &r);
    if (st != ADA_OK) return st;
    if ((st = check_append(cache, B, off, len, N, len_out, pos0, K, ldk, V, ldv, Q, h, ldq, q_out, ldqo, q_norm, k_norm, eps, inv_freq, rot,
                           rep_idx, rep_cnt, flags)) != ADA_OK)
        return st;
    AppendJob j;
    j.Q = static_cast<const __nv_bfloat16*>(Q); j.K = static_cast<const __nv_bfloat16*>(K);
    j.V = static_cast<const __nv_bfloat16*>(V);
    j.ldq = ldq; j.ldk = ldk; j.ldv = ldv;
    j.q_out = static_cast<__nv_bfloat16*>(q_out); j.ldqo = ldqo; j.h = Q != nullptr ? (int)h : 0;
    j.q_norm = static_cast<const __nv_bfloat16*>(q_norm); j.k_norm = static_cast<const __nv_bfloat16*>(k_norm);
    j.eps = (float)eps;
    j.inv_freq = inv_freq; j.rot = inv_freq != nullptr ? (int)rot : 0; j.pairs = (flags & ADA_ROPE_PAIRS) ? 1 : 0;
    j.pos0 = pos0; j.rep_idx = rep_idx; j.rep_cnt = rep_cnt; j.len_out = len_out;
    DeviceGuard guard(ctx->device);
    CU(launch_cache_append(ctx, c, r, j, static_cast<cudaStream_t>(stream)));
    return ADA_OK;
}

ada_status ada_attention_cached(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off,
                                const int32_t* len, int64_t N, int64_t max_new, const void* Q, int64_t h, int64_t ldq,
                                ada_dtype dt, double scale, void* out, int64_t ldo, uint32_t flags, void* stream) {
    CacheView c;
    Ragged r;
    ada_status st = open_cache(ctx, cache, B, off, len, N, dt, &c, &r);
    if (st != ADA_OK || (st = check_heads(cache, h)) != ADA_OK) return st;
    if ((st = check_rows(Q, h, c.d, ldq)) != ADA_OK || (st = check_rows(out, h, c.d, ldo)) != ADA_OK ||
        (st = check_out(Q, ldq, out, ldo)) != ADA_OK)
        return st;
    if ((flags & ~ADA_ATTN_CAUSAL) != 0 || max_new < 1 || !scale_ok(scale)) return ADA_ERR_INVALID_ARG;
    AttendJob j;
    j.scale = score_scale(scale, c.d);
    j.Q = static_cast<const __nv_bfloat16*>(Q); j.ldq = ldq;
    j.out = static_cast<__nv_bfloat16*>(out); j.ldo = ldo;
    j.h = (int)h; j.max_new = (int)(max_new < N ? max_new : N); j.causal = (flags & ADA_ATTN_CAUSAL) ? 1 : 0;
    j.blk_idx = j.blk_cnt = nullptr; j.k = 0; j.few = 0;
    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    CU(ensure_cache_ws(ctx, s));
    // Up to as many rows of a key head as one 16-row tile of mma.sync holds, or tiles of 128 rows; several sequences may be
    // mixed.  Both kernels, 32 heads on 8, us with 4, 8 and 16 rows, d_h 128: 16 sequences of 8192 91, 95, 104 (tiles of 128
    // rows: 114, 118, 120), one of 8192 15, 21, 32 (32 each), one of 131072 96, 102, 119 (135 to 141); d_h 64: 51, 52, 58 (98), 11,
    // 14, 20 (26), 55, 59, 69 (110).  17 to 128 rows take what 16 take there: 123 to 131, 32 to 34, 135 to 140; 107, 26, 111.
    const int few = 16 / (j.h / c.h_kv);
    if (j.max_new <= few) {
        CU(launch_cache_step(ctx, c, r, j, s));
        return ADA_OK;
    }
    if (r.B > 1 && few > 0) {
        j.few = few;
        AttendJob step = j;
        step.max_new = few;
        CU(launch_cache_step(ctx, c, r, step, s));
    }
    CU(launch_cache_chunk(ctx, c, r, j, s));
    return ADA_OK;
}

ada_status ada_select_blocks(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off, const int32_t* len,
                             int64_t N, const void* Q, int64_t h, int64_t ldq, ada_dtype dt, int64_t k, int64_t n_first,
                             int64_t n_last, int32_t* blk_idx, int32_t* blk_cnt, uint32_t flags, void* stream) {
    CacheView c;
    Ragged r;
    ada_status st = open_cache(ctx, cache, B, off, len, N, dt, &c, &r);
    if (st != ADA_OK || (st = check_heads(cache, h)) != ADA_OK) return st;
    if ((st = check_rows(Q, h, c.d, ldq)) != ADA_OK) return st;
    if ((st = check_select(cache, k, n_first, n_last, blk_idx, blk_cnt, flags)) != ADA_OK) return st;
    SelectJob j;
    j.Q = static_cast<const __nv_bfloat16*>(Q); j.ldq = ldq; j.h = (int)h;
    j.causal = (flags & ADA_ATTN_CAUSAL) ? 1 : 0;
    j.k = (int)k; j.n_first = (int)n_first; j.n_last = (int)n_last;
    j.blk_idx = blk_idx; j.blk_cnt = blk_cnt;
    DeviceGuard guard(ctx->device);
    CU(launch_cache_select(ctx, c, r, j, static_cast<cudaStream_t>(stream)));
    return ADA_OK;
}

ada_status ada_attention_blocks(ada_ctx* ctx, const ada_kv_cache* cache, int64_t B, const int32_t* off,
                                const int32_t* len, int64_t N, const void* Q, int64_t h, int64_t ldq, ada_dtype dt,
                                const int32_t* blk_idx, const int32_t* blk_cnt, int64_t k, double scale, void* out,
                                int64_t ldo, uint32_t flags, void* stream) {
    CacheView c;
    Ragged r;
    ada_status st = open_cache(ctx, cache, B, off, len, N, dt, &c, &r);
    if (st != ADA_OK || (st = check_heads(cache, h)) != ADA_OK) return st;
    if ((st = check_rows(Q, h, c.d, ldq)) != ADA_OK || (st = check_rows(out, h, c.d, ldo)) != ADA_OK ||
        (st = check_out(Q, ldq, out, ldo)) != ADA_OK)
        return st;
    if (blk_idx == nullptr || blk_cnt == nullptr || (flags & ~ADA_ATTN_CAUSAL) != 0 || k < 1 || !scale_ok(scale))
        return ADA_ERR_INVALID_ARG;
    if (k > SELECT_MAX_PAGES) return ADA_ERR_UNSUPPORTED;
    AttendJob j;
    j.scale = score_scale(scale, c.d);
    j.Q = static_cast<const __nv_bfloat16*>(Q); j.ldq = ldq;
    j.out = static_cast<__nv_bfloat16*>(out); j.ldo = ldo;
    j.h = (int)h; j.max_new = 1; j.causal = (flags & ADA_ATTN_CAUSAL) ? 1 : 0;
    j.blk_idx = blk_idx; j.blk_cnt = blk_cnt; j.k = (int)k; j.few = 0;
    DeviceGuard guard(ctx->device);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    CU(ensure_cache_ws(ctx, s));
    CU(launch_cache_step(ctx, c, r, j, s));
    return ADA_OK;
}

}  // extern "C"
