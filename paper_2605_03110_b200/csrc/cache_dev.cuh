// Paged key / value cache: what the kernels that write and read it share.
//
// Pages of `ps` = 2^shift slots, head-major inside a page, so that the keys (values) of one head and page are one
// contiguous block of ps x d_h elements: what a single TMA box of the attention kernels fetches.
#pragma once

#include "cache_args.h"
#include "common.cuh"

namespace ada {

struct CacheView {
    __nv_bfloat16 *k, *v;       // element (page, head, slot, e) at page * page_stride + (head * ps + slot) * d + e
    __nv_bfloat16 *kmin, *kmax; // [n_pages][h_kv][d], or NULL
    const int32_t* table;       // [B][table_ld]: page of slots (p ps) .. (p ps + ps - 1) of sequence b
    int64_t table_ld, page_stride;
    int n_pages, max_pages, shift, h_kv, d;
};

// New tokens of all sequences stand one after the other: sequence b has rows off[b] .. off[b + 1].
struct Ragged {
    const int32_t* off;         // [B + 1]
    const int32_t* len;         // [B] tokens in the cache
    int B, N;                   // sequences, rows
};

#ifdef __CUDACC__
// off[b + 1] - off[b] where both lie in [0, N] and do not descend, else 0 (and off0 = 0): whatever the arrays hold,
// rows off0 .. off0 + n are rows of the call
static __device__ __forceinline__ int seq_rows(const Ragged& r, int b, int& off0) {
    const int o0 = r.off[b], o1 = r.off[b + 1];
    const bool ok = o0 >= 0 && o1 >= o0 && o1 <= r.N;
    off0 = ok ? o0 : 0;
    return ok ? o1 - o0 : 0;
}
// tokens of sequence b in the cache, at most what its page table has room for
static __device__ __forceinline__ int seq_len(const Ragged& r, const CacheView& c, int b) {
    return min(max(r.len[b], 0), c.max_pages << c.shift);
}
// The sequence of row i, by all lanes of a warp together: the last b with off[b] <= i.  -1 if the row is no
// sequence's (behind the last one, or the offsets are out of order).  A call with no more rows than sequences is mostly
// one token each: looked at first, it saves two dependent loads.
static __device__ __forceinline__ int seq_of_row(const Ragged& r, int i) {
    const int lane = threadIdx.x & 31;
    if (r.N <= r.B && r.off[i] == i && r.off[i + 1] == i + 1) return i;
    int lo = 0, n = r.B;                         // the answer, if any, is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) >> 5, at = lane * step;
        const bool le = at < n && r.off[lo + at] <= i;
        const unsigned m = __ballot_sync(0xffffffffu, le);
        if (m == 0u) return -1;
        const int j = 31 - __clz(m);
        lo += j * step;
        n = min(step, n - j * step);
    }
    int o;
    const int rows = seq_rows(r, lo, o);
    return i >= o && i < o + rows ? lo : -1;
}
// Faults of the arrays that describe the sequences, found by the threads first, first + 1 .. of `step` of one block: offsets that descend or leave [0, N],
// lengths outside [0, capacity].
static __device__ __forceinline__ void check_ragged(const Ragged& r, const CacheView& c, unsigned* status, int first,
                                                    int step) {
    for (int b = first; b < r.B; b += step) {
        const int o0 = r.off[b], o1 = r.off[b + 1], n = r.len[b];
        unsigned bad = 0u;
        if (o0 < 0 || o1 < o0 || o1 > r.N || (b == 0 && o0 != 0)) bad |= ST_BAD_INDEX;
        if (n < 0 || n > c.max_pages << c.shift) bad |= ST_BAD_COUNT;
        if (bad != 0u) atomicOr(status, bad);
    }
}
// page of the p-th page of sequence b, -1 (and a status bit) if the table names none
static __device__ __forceinline__ int page_of(const CacheView& c, int b, int p, unsigned* status) {
    const int page = c.table[(int64_t)b * c.table_ld + p];
    if (page >= 0 && page < c.n_pages) return page;
    atomicOr(status, ST_BAD_INDEX);
    return -1;
}
// Units [first, first + n) of a job dealt out in runs of `per`, seen from CTA `c`, whose run has some of them: the first CTA
// with any of them and the last one.  (32-bit divisions: n is a few thousand, `per` may be anything.)
static __device__ __forceinline__ void shares_of(int64_t first, int n, int64_t per, int c, int& c0, int& c1) {
    const unsigned p32 = per > 0x7fffffff ? 0x7fffffffu : (unsigned)per;
    const int64_t mine = per * c;
    const int before = (int)(first < mine ? mine - first : 0);              // of them in front of the run, behind it
    const int64_t end = first + n - (mine + per);
    const int after = (int)(end > 0 ? end : 0);
    c0 = c - (int)(((unsigned)before + p32 - 1u) / p32);
    c1 = c + (int)(((unsigned)after + p32 - 1u) / p32);
}
static __device__ __forceinline__ unsigned ld_acquire(const unsigned* p) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
static __device__ __forceinline__ int64_t slot_at(const CacheView& c, int page, int head, int slot) {
    return (int64_t)page * c.page_stride + ((int64_t)(head << c.shift) + slot) * c.d;
}
#endif

// Dynamic shared memory above 48 KB has to be allowed for a kernel, once per device: `bit` says which kernel it is.
template <typename K>
inline cudaError_t allow_smem(ada_ctx* ctx, int bit, K kernel, int bytes) {
    if (ctx->cache_attr >> bit & 1u) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) ctx->cache_attr |= 1u << bit;
    return e;
}

// launchers -------------------------------------------------------------------------------------
struct AppendJob {
    const __nv_bfloat16 *Q, *K, *V;     // Q may be NULL
    int64_t ldq, ldk, ldv;              // row strides in elements
    __nv_bfloat16* q_out;
    int64_t ldqo;
    int h;                              // query heads
    const __nv_bfloat16 *q_norm, *k_norm;
    float eps;
    const double* inv_freq;             // [rot / 2], or NULL
    int rot, pairs;                     // rotated elements of a head; neighbouring elements form the pairs
    const int32_t* pos0;                // [B] position of a sequence's first new token; NULL: its length
    const int32_t *rep_idx, *rep_cnt;   // NULL: every token goes to the cache
    int32_t* len_out;
};
cudaError_t launch_cache_append(ada_ctx* ctx, const CacheView& c, const Ragged& r, const AppendJob& j, cudaStream_t s);

struct AttendJob {
    const __nv_bfloat16* Q;
    int64_t ldq;
    __nv_bfloat16* out;
    int64_t ldo;
    int h, max_new, causal;
    int few;                            // > 0: sequences of up to `few` new tokens are cache_step's, the others
                                        // cache_chunk's; 0: all of them are whose kernel is called
    float scale;                        // of the scores, times log2(e)
    const int32_t *blk_idx, *blk_cnt;   // [N][h_kv][k], [N][h_kv]; NULL: every page
    int k;
};
// single tokens and few rows (mma.sync), or the listed pages
cudaError_t launch_cache_step(ada_ctx* ctx, const CacheView& c, const Ragged& r, const AttendJob& j, cudaStream_t s);
// chunks of new tokens (tcgen05)
size_t cache_part_floats();             // of one place for partial results; two per SM
cudaError_t launch_cache_chunk(ada_ctx* ctx, const CacheView& c, const Ragged& r, const AttendJob& j, cudaStream_t s);

struct SelectJob {
    const __nv_bfloat16* Q;
    int64_t ldq;
    int h, causal, k, n_first, n_last;
    int32_t *blk_idx, *blk_cnt;
};
cudaError_t launch_cache_select(ada_ctx* ctx, const CacheView& c, const Ragged& r, const SelectJob& j, cudaStream_t s);

}  // namespace ada
