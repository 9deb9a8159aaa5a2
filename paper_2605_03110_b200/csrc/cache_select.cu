// Choice of pages (ada_select_blocks): for every new token and key head the k pages whose keys can matter most.
//
//   s(p) = sum_g sum_e max(q_ge kmax_pe, q_ge kmin_pe)  >=  sum_g q_g . key   for every key of page p
// g runs over the heads that share the key head.  max(q a, q b) with a >= b is q a for q > 0 and q b for q < 0, so with
// the sums of the positive and of the negative parts, P_e = sum_g max(q_ge, 0) and M_e = sum_g min(q_ge, 0),
//   s(p) = sum_e P_e kmax_pe + M_e kmin_pe:
// one dot product of 2 d_h elements, whatever the number of heads.
#include "cache_dev.cuh"

namespace ada {

namespace {

constexpr int SEL_THREADS = 256;

__device__ __forceinline__ unsigned long long sort_key(double x) {
    if (!(x == x)) return 0ull;                                  // NaN: behind everything
    x += 0.0;                                                    // -0 is 0
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}

__global__ void __launch_bounds__(SEL_THREADS)
k_cache_select(const CacheView c, const Ragged r, const SelectJob j, unsigned* __restrict__ status) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ double qp[128], qm[128];
    __shared__ int cnt_w[SEL_THREADS / 32], tie_w[SEL_THREADS / 32];
    unsigned long long* key = reinterpret_cast<unsigned long long*>(smem);
    grid_dep_wait();
    grid_dep_launch_next();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row = blockIdx.x, head = blockIdx.y, G = j.h / c.h_kv;
    if (row == 0 && head == 0) check_ragged(r, c, status, tid, SEL_THREADS);
    const int b = seq_of_row(r, row);
    if (b < 0) return;
    int o;
    const int n = seq_rows(r, b, o), len = seq_len(r, c, b);
    const int lim = j.causal ? max(len - n + (row - o) + 1, 0) : len;
    const int nb = (lim + (1 << c.shift) - 1) >> c.shift;
    int32_t* idx = j.blk_idx + ((int64_t)row * c.h_kv + head) * j.k;
    const int take = min(nb, j.k);
    if (tid == 0) j.blk_cnt[(int64_t)row * c.h_kv + head] = take;
    if (nb <= j.k) {
        for (int i = tid; i < j.k; i += SEL_THREADS) idx[i] = i < nb ? i : -1;
        return;
    }
    for (int e = tid; e < c.d; e += SEL_THREADS) {
        double p = 0.0, m = 0.0;
        for (int g = 0; g < G; ++g) {
            const double x = (double)__bfloat162float(j.Q[(int64_t)row * j.ldq + ((int64_t)head * G + g) * c.d + e]);
            p += x > 0.0 ? x : 0.0;
            m += x > 0.0 ? 0.0 : x;
        }
        qp[e] = p; qm[e] = m;
    }
    __syncthreads();
    for (int p = tid; p < nb; p += SEL_THREADS) {
        unsigned long long k = ~0ull;
        if (p >= j.n_first && p < nb - j.n_last) {
            const int page = page_of(c, b, p, status);
            double s = 0.0;
            if (page >= 0) {
                const int64_t at = ((int64_t)page * c.h_kv + head) * c.d;
                for (int e = 0; e < c.d; e += 8) {
                    const uint4 a = *reinterpret_cast<const uint4*>(c.kmax + at + e), z = *reinterpret_cast<const uint4*>(c.kmin + at + e);
                    const __nv_bfloat16 *pa = reinterpret_cast<const __nv_bfloat16*>(&a), *pz = reinterpret_cast<const __nv_bfloat16*>(&z);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        s = fma(qp[e + q], (double)__bfloat162float(pa[q]), fma(qm[e + q], (double)__bfloat162float(pz[q]), s));
                }
            }
            k = page >= 0 ? sort_key(s) : 0ull;
        }
        key[p] = k;
    }
    __syncthreads();
    // the take-th largest key, bit by bit
    auto count = [&](unsigned long long t) {
        int n_ge = 0;
        for (int p = tid; p < nb; p += SEL_THREADS) n_ge += key[p] >= t;
        n_ge = __reduce_add_sync(0xffffffffu, n_ge);
        __syncthreads();
        if (lane == 0) cnt_w[warp] = n_ge;
        __syncthreads();
        int s = 0;
#pragma unroll
        for (int w = 0; w < SEL_THREADS / 32; ++w) s += cnt_w[w];
        return s;
    };
    unsigned long long thr = 0ull;
    for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long t = thr | 1ull << bit;
        if (count(t) >= take) thr = t;
    }
    int ties = take - (thr == ~0ull ? 0 : count(thr + 1ull));    // of the pages with that key, the lowest
    int out = 0;
    for (int p0 = 0; p0 < nb; p0 += SEL_THREADS) {
        const int p = p0 + tid;
        const unsigned long long k = p < nb ? key[p] : 0ull;
        const bool eq = p < nb && k == thr, gt = p < nb && k > thr;
        const unsigned me = __ballot_sync(0xffffffffu, eq);
        __syncthreads();
        if (lane == 0) tie_w[warp] = __popc(me);
        __syncthreads();
        int before = __popc(me & ((1u << lane) - 1u)), all = 0;
#pragma unroll
        for (int w = 0; w < SEL_THREADS / 32; ++w) { if (w < warp) before += tie_w[w]; all += tie_w[w]; }
        const bool in = gt || (eq && before < ties);
        ties -= min(ties, all);
        const unsigned mi = __ballot_sync(0xffffffffu, in);
        if (lane == 0) cnt_w[warp] = __popc(mi);
        __syncthreads();
        int at = out + __popc(mi & ((1u << lane) - 1u));
#pragma unroll
        for (int w = 0; w < SEL_THREADS / 32; ++w) { if (w < warp) at += cnt_w[w]; out += cnt_w[w]; }
        if (in) idx[at] = p;
    }
}

}  // namespace

cudaError_t launch_cache_select(ada_ctx* ctx, const CacheView& c, const Ragged& r, const SelectJob& j, cudaStream_t s) {
    const int smem = c.max_pages * 8;
    cudaError_t e = cudaFuncSetAttribute(k_cache_select, cudaFuncAttributeMaxDynamicSharedMemorySize, SELECT_MAX_PAGES * 8);
    if (e != cudaSuccess) return e;
    return launch_k(ctx, k_cache_select, dim3(r.N, c.h_kv), dim3(SEL_THREADS), smem, s, c, r, j, ctx->status);
}

}  // namespace ada
