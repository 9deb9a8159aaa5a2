// Appending to the paged cache (ada_cache_append): per-head RMS norm of queries and keys, rotation, queries written
// out, keys and values written behind the tokens that the sequence has, and the bounds of every page written.
//
//   x'_e = w_e x_e / sqrt(mean(x^2) + eps)                          (fp32; the weights are bf16)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t),   t = pos * inv_freq_i
// The angle is formed in 64 bits and reduced to a fraction of a turn there (pos * inv_freq passes 2^24 radians for
// far positions, where an fp32 product knows nothing of the angle any more); sine and cosine of the fraction are fp32.
// One rounding to bf16, at the store.
//
// Bound by memory (2 bytes in, 2 out per element), for single tokens by latency.  A group of 16 (d_h <= 64: 8) lanes
// holds one head's row, 8 elements a lane, so that norm and rotation are shuffles inside the group; a token's
// sines and cosines are made once per block and shared by all of its heads.
#include "cache_dev.cuh"

namespace ada {

namespace {

constexpr int APP_THREADS = 256;
constexpr int APP_ROWS = 4;              // rows of a group in flight
constexpr int APP_TOK = 4;               // most tokens per block
constexpr int MAX_HALF = 64;             // rot / 2 <= 64

struct TokInfo {
    int page, slot, src, bad;            // page -1: nothing is kept of this row
};

// bf16 pairs with an exponent of all ones
__device__ __forceinline__ bool nonfinite2(unsigned w) {
    return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ bool nonfinite8(const uint4& v) {
    return nonfinite2(v.x) || nonfinite2(v.y) || nonfinite2(v.z) || nonfinite2(v.w);
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const unsigned*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// grid (token tiles of `tok` rows, shares of a token's head rows)
template <int LG>
__global__ void __launch_bounds__(APP_THREADS)
k_cache_append(const CacheView c, const Ragged r, const AppendJob j, int tok, unsigned* __restrict__ status) {
    __shared__ TokInfo info[APP_TOK];
    __shared__ int pos_q[APP_TOK], pos_k[APP_TOK];
    __shared__ float2 ang[2][APP_TOK][MAX_HALF];     // (cos, sin) at the token's own position; at the kept row's
    grid_dep_wait();
    grid_dep_launch_next();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int i0 = blockIdx.x * tok;
    const int n_tok = min(tok, r.N - i0);
    if (warp < n_tok) {
        const int i = i0 + warp, b = seq_of_row(r, i);
        TokInfo t = {-1, 0, 0, 0};
        int pq = 0, pk = 0;
        if (b >= 0) {
            int o;
            const int n = seq_rows(r, b, o), old = seq_len(r, c, b), li = i - o;
            const int p0 = j.pos0 != nullptr ? j.pos0[b] : old;
            int kept = n, at = li;
            if (j.rep_cnt != nullptr) {
                kept = j.rep_cnt[b];
                if (kept < 0 || kept > n) { t.bad |= ST_BAD_COUNT; kept = min(max(kept, 0), n); }
                if (li < kept) {
                    at = j.rep_idx[i];
                    if (at < 0 || at >= n || (li > 0 && j.rep_idx[i - 1] >= at)) { t.bad |= ST_BAD_INDEX; kept = 0; }
                }
            }
            pq = p0 + li;
            if (li < kept) {
                const int64_t slot = (int64_t)old + li;
                pk = p0 + at;
                t.src = o + at;
                if (slot >= (int64_t)c.max_pages << c.shift) {
                    t.bad |= ST_BAD_COUNT;
                } else {
                    const int page = c.table[(int64_t)b * c.table_ld + (slot >> c.shift)];
                    if (page < 0 || page >= c.n_pages) t.bad |= ST_BAD_INDEX;
                    else { t.page = page; t.slot = (int)slot & ((1 << c.shift) - 1); }
                }
            }
        }
        if (lane == 0) {
            // row i's queries are its own; its keys come from row src (itself without a list)
            info[warp] = t;
            pos_q[warp] = b >= 0 ? pq : INT_MIN;
            pos_k[warp] = pk;
            if (t.bad != 0 && blockIdx.y == 0) atomicOr(status, (unsigned)t.bad);
        }
    }
    __syncthreads();
    const int half = j.inv_freq != nullptr ? j.rot >> 1 : 0;
    const int sets = j.rep_idx != nullptr ? 2 : 1;
    for (int q = threadIdx.x; q < sets * n_tok * half; q += APP_THREADS) {
        const int i = q % half, t = q / half % n_tok, s = q / (half * n_tok);
        const double turns = (double)(s == 0 ? pos_q[t] : pos_k[t]) * j.inv_freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
        float sn, cs;
        sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
        ang[s][t][i] = make_float2(cs, sn);
    }
    __syncthreads();

    const int nvec = c.d >> 3, hv = half >> 3, h_q = j.Q != nullptr ? j.h : 0;
    const int per_tok = h_q + 2 * c.h_kv;
    constexpr int GROUPS = APP_THREADS / LG;
    const int group = threadIdx.x / LG, v = threadIdx.x % LG;
    const bool on = v < nvec;
    const int total = n_tok * per_tok;
    bool bad = false;
    for (int base = blockIdx.y * GROUPS + group; base < total; base += gridDim.y * GROUPS * APP_ROWS) {
        uint4 in[APP_ROWS];
        __nv_bfloat16* dst[APP_ROWS];
        int kind[APP_ROWS], at[APP_ROWS];
#pragma unroll
        for (int u = 0; u < APP_ROWS; ++u) {
            const int row = base + u * gridDim.y * GROUPS;
            in[u] = make_uint4(0u, 0u, 0u, 0u);
            dst[u] = nullptr;
            kind[u] = 3; at[u] = 0;
            if (row < total) {
                const int t = row / per_tok, x = row - t * per_tok;
                at[u] = t;
                const __nv_bfloat16* src = nullptr;
                if (x < h_q) {
                    kind[u] = 0;
                    if (pos_q[t] != INT_MIN) {
                        src = j.Q + (int64_t)(i0 + t) * j.ldq + (int64_t)x * c.d;
                        dst[u] = j.q_out + (int64_t)(i0 + t) * j.ldqo + (int64_t)x * c.d;
                    }
                } else if (info[t].page >= 0) {
                    const bool is_v = x - h_q >= c.h_kv;
                    const int head = x - h_q - (is_v ? c.h_kv : 0);
                    kind[u] = is_v ? 2 : 1;
                    src = is_v ? j.V + (int64_t)info[t].src * j.ldv : j.K + (int64_t)info[t].src * j.ldk;
                    src += (int64_t)head * c.d;
                    dst[u] = (is_v ? c.v : c.k) + slot_at(c, info[t].page, head, info[t].slot);
                }
                if (on && src != nullptr) in[u] = *reinterpret_cast<const uint4*>(src + v * 8);
            }
        }
#pragma unroll
        for (int u = 0; u < APP_ROWS; ++u) {
            bad = bad || nonfinite8(in[u]);
            uint4 o = in[u];
            const __nv_bfloat16* w = kind[u] == 0 ? j.q_norm : j.k_norm;
            // (the branches are the same for all lanes of a group, not of a warp: the shuffles name the group's lanes)
            const unsigned mask = LG == 16 ? 0xffffu << (threadIdx.x & 16) : 0xffu << (threadIdx.x & 24);
            if (kind[u] < 2 && (w != nullptr || half != 0)) {
                float x[8];
                unpack8(in[u], x);
                if (w != nullptr) {
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
#pragma unroll
                    for (int m = LG / 2; m > 0; m >>= 1) s += __shfl_xor_sync(mask, s, m, LG);
                    const float f = rsqrtf(s / (float)c.d + j.eps);
                    float g[8];
                    unpack8(on ? *reinterpret_cast<const uint4*>(w + v * 8) : make_uint4(0u, 0u, 0u, 0u), g);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * f * g[e];
                }
                if (half != 0) {
                    const float2* a = ang[kind[u] == 1 && sets == 2 ? 1 : 0][at[u]];
                    if (j.pairs) {
                        if (v * 8 < j.rot) {
#pragma unroll
                            for (int e = 0; e < 8; e += 2) {
                                const float2 cs = a[v * 4 + (e >> 1)];
                                const float p = x[e], q = x[e + 1];
                                x[e] = p * cs.x - q * cs.y;
                                x[e + 1] = q * cs.x + p * cs.y;
                            }
                        }
                    } else {
                        const bool low = v < hv, in_rot = v < 2 * hv;
                        const int other = low ? v + hv : in_rot ? v - hv : v;
                        float y[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = __shfl_sync(mask, x[e], other, LG);
                        if (in_rot) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float2 cs = a[(low ? v : v - hv) * 8 + e];
                                x[e] = low ? x[e] * cs.x - y[e] * cs.y : x[e] * cs.x + y[e] * cs.y;
                            }
                        }
                    }
                }
                o = pack8(x);
            }
            if (on && dst[u] != nullptr) *reinterpret_cast<uint4*>(dst[u] + v * 8) = o;
        }
    }
    if (bad) atomicOr(status, ST_NONFINITE);
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        check_ragged(r, c, status, threadIdx.x, APP_THREADS);
        if (j.len_out != nullptr)
            for (int b = threadIdx.x; b < r.B; b += APP_THREADS) {
                int o;
                int n = seq_rows(r, b, o);
                if (j.rep_cnt != nullptr) n = min(max(j.rep_cnt[b], 0), n);
                j.len_out[b] = (int)min((int64_t)seq_len(r, c, b) + n, (int64_t)c.max_pages << c.shift);
            }
    }
}

// Elementwise minimum and maximum of a page's keys, over the slots below the sequence's new length, from the page
// itself: what a page held before (another sequence, tokens taken back) has no part in them.  Block (x, y):
// the x-th page that the call wrote to, head y.  Exact, whatever the order.
constexpr int BND_THREADS = 128;
__global__ void __launch_bounds__(BND_THREADS)
k_cache_bounds(const CacheView c, const Ragged r, const int32_t* __restrict__ rep_cnt) {
    __shared__ uint4 part[2][BND_THREADS];
    grid_dep_wait();
    grid_dep_launch_next();
    const int lane = threadIdx.x & 31, head = blockIdx.y;
    int left = blockIdx.x, page = -1, live = 0;
    for (int b0 = 0; b0 < r.B; b0 += 32) {
        int n = 0, old = 0, o;
        if (b0 + lane < r.B) {
            n = seq_rows(r, b0 + lane, o);
            if (rep_cnt != nullptr) n = min(max(rep_cnt[b0 + lane], 0), n);
            old = seq_len(r, c, b0 + lane);
            n = (int)min((int64_t)n, ((int64_t)c.max_pages << c.shift) - old);
        }
        const int first = old >> c.shift, pages = n > 0 ? ((old + n - 1) >> c.shift) - first + 1 : 0;
        int sum = pages;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, m);
            if (lane >= m) sum += y;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, left < sum);
        if (hit != 0u) {
            const int l = __ffs(hit) - 1;
            const int p = __shfl_sync(0xffffffffu, first + left - (sum - pages), l);
            live = __shfl_sync(0xffffffffu, old + n, l) - (p << c.shift);
            page = c.table[(int64_t)(b0 + l) * c.table_ld + p];
            break;
        }
        left -= __shfl_sync(0xffffffffu, sum, 31);
    }
    if (page < 0 || page >= c.n_pages) return;      // (the append has flagged a page that the table does not name)
    const int ps = 1 << c.shift, nvec = c.d >> 3;
    live = min(live, ps);
    const int lanes = nvec <= 8 ? 8 : 16, rows = BND_THREADS / lanes;
    const int v = threadIdx.x % lanes, row = threadIdx.x / lanes;
    uint4 lo = make_uint4(0x7f807f80u, 0x7f807f80u, 0x7f807f80u, 0x7f807f80u), hi = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
    auto take = [](uint4& l, uint4& h, const uint4& a, const uint4& b) {
        __nv_bfloat162 *pl = reinterpret_cast<__nv_bfloat162*>(&l), *ph = reinterpret_cast<__nv_bfloat162*>(&h);
        const __nv_bfloat162 *pa = reinterpret_cast<const __nv_bfloat162*>(&a), *pb = reinterpret_cast<const __nv_bfloat162*>(&b);
#pragma unroll
        for (int i = 0; i < 4; ++i) { pl[i] = __hmin2(pl[i], pa[i]); ph[i] = __hmax2(ph[i], pb[i]); }
    };
    if (v < nvec) {
        const __nv_bfloat16* src = c.k + slot_at(c, page, head, 0) + v * 8;
#pragma unroll 4
        for (int s = row; s < live; s += rows) {
            const uint4 x = *reinterpret_cast<const uint4*>(src + (int64_t)s * c.d);
            take(lo, hi, x, x);
        }
    }
    part[0][threadIdx.x] = lo;
    part[1][threadIdx.x] = hi;
    __syncthreads();
    if (row == 0 && v < nvec) {
        for (int q = 1; q < rows; ++q) take(lo, hi, part[0][q * lanes + v], part[1][q * lanes + v]);
        const int64_t at = ((int64_t)page * c.h_kv + head) * c.d + v * 8;
        *reinterpret_cast<uint4*>(c.kmin + at) = lo;
        *reinterpret_cast<uint4*>(c.kmax + at) = hi;
    }
}

}  // namespace

cudaError_t launch_cache_append(ada_ctx* ctx, const CacheView& c, const Ragged& r, const AppendJob& j, cudaStream_t s) {
    const int lg = c.d <= 64 ? 8 : 16, groups = APP_THREADS / lg;
    const int per_tok = (j.Q != nullptr ? j.h : 0) + 2 * c.h_kv;
    // one token per block, its rows spread over as many blocks as are needed for one round each, while the tokens
    // alone do not fill the GPU; else several tokens per block
    const int tok = r.N >= 8 * ctx->sm_count ? APP_TOK : 1;
    const int tiles = (r.N + tok - 1) / tok;
    int shares = 1;
    if (tok == 1) {
        const int want = (per_tok + groups - 1) / groups, room = (4 * ctx->sm_count + tiles - 1) / tiles;
        shares = want < room ? want : room;
    }
    auto kernel = lg == 8 ? k_cache_append<8> : k_cache_append<16>;
    cudaError_t e = launch_k(ctx, kernel, dim3(tiles, shares), dim3(APP_THREADS), 0, s, c, r, j, tok, ctx->status);
    if (e != cudaSuccess) return e;
    if (c.kmin != nullptr) {
        // a sequence of n new tokens writes to at most n and at most (n - 1) / ps + 2 pages
        const int64_t most = (int64_t)(r.N >> c.shift) + 2 * (int64_t)r.B;
        const int pages = (int)(most < r.N ? most : r.N);
        e = launch_k(ctx, k_cache_bounds, dim3(pages, c.h_kv), dim3(BND_THREADS), 0, s, c, r, j.rep_cnt);
    }
    return e;
}

}  // namespace ada
