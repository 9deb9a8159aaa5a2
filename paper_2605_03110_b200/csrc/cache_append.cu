// Appending to the paged cache (ada_cache_append): per-head RMS norm of queries and keys, rotation, queries written
// out, keys and values written behind the tokens that the sequence has, and the bounds of every page written.
//
//   x'_e = w_e x_e / sqrt(mean(x^2) + eps)                          (fp32; the weights are bf16)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t),   t = pos * inv_freq_i
// The angle is formed in 64 bits and reduced to a fraction of a turn there (pos * inv_freq passes 2^24 radians for
// far positions, where an fp32 product knows nothing of the angle any more); sine and cosine of the fraction are fp32.
// One rounding to bf16, at the store.
//
// Bound by memory (2 bytes in, 2 out per element), for single tokens by latency.  A warp has one token (or a share of its
// heads), half a warp (d_h <= 64: a quarter) one head's row at a time.  A lane holds two pieces of four elements that the
// rotation pairs with each other, so that it needs nobody else's elements, and keeps the four sines and cosines of
// its pairs, and the norm's weights, in registers for all heads of the token.  (With a lane holding eight neighbouring
// elements, partners by shuffle and the sines in shared memory, 6660 tokens of 3 x 32 heads of 128 took 102 us, bound by
// issue; now 70, of them 57 at 5.8 TB/s here and 12 for the bounds.)
//
// The bounds of a page need all of its keys.  Calls of several tokens each form them in a second kernel, from the pages (12
// of 70 us for 6660 tokens of 3 x 32 heads of 128; a kernel that took the keys page by page and kept the bounds on the way was
// slower, 76: a page's tokens are too few warps).  Where
// there are no more tokens than sequences (a decoding step) the second launch would take as long as the first: there a
// warp of its own takes each key head of a token and reads the page's older keys beside the new one; should several new
// tokens lie in a page, the last one's warp forms the others' keys once more.  (64 tokens of 32 + 8 + 8 heads of 128, pages of
// 64: 10.4 -> 6.4 us, a chain of five dependent loads.)
#include "cache_dev.cuh"

namespace ada {

namespace {

constexpr int APP_THREADS = 128;
constexpr int APP_WARPS = APP_THREADS / 32;
constexpr int APP_ROWS = 4;              // rows of a group in flight

// bf16 pairs with an exponent of all ones
__device__ __forceinline__ bool nonfinite2(unsigned w) {
    return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ bool nonfinite4(const uint2& v) { return nonfinite2(v.x) || nonfinite2(v.y); }
__device__ __forceinline__ void unpack4(const uint2& v, float* x) {
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ uint2 pack4(const float* x) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    return make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
}

// What a lane does to its eight elements of every row: elements at e0 .. e0 + 3 and e1 .. e1 + 3 of the head.
struct Lane {
    int e0, e1;
    bool on, turns;                      // has elements; they are rotated
};

// cosines and sines of the lane's four pairs at position p0 + i (which may be behind the largest int32)
__device__ __forceinline__ void angles(const AppendJob& j, const Lane& ln, int v, int p0, int i, float (&cs)[4], float (&sn)[4]) {
    const double pos = (double)p0 + (double)i;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        cs[q] = 1.f; sn[q] = 0.f;
        if (ln.turns) {
            const double turns = pos * j.inv_freq[4 * v + q] * 0.15915494309189533577;   // 1 / (2 pi)
            sincospif(2.0f * (float)(turns - rint(turns)), &sn[q], &cs[q]);
        }
    }
}

// A head's row in a lane's registers, normed (g: the lane's weights) and rotated
template <int LG, bool PAIRS>
__device__ __forceinline__ void transform(uint2& a, uint2& b, bool norm, const float (&g)[8], float eps, int d, const float (&cs)[4],
                                          const float (&sn)[4], unsigned mask) {
    float x[8];
    unpack4(a, x);
    unpack4(b, x + 4);
    if (norm) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
#pragma unroll
        for (int m = LG / 2; m > 0; m >>= 1) s += __shfl_xor_sync(mask, s, m, LG);
        const float f = rsqrtf(s / (float)d + eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= f * g[e];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {                                // (an unrotated lane has cosine 1, sine 0)
        const int p = PAIRS ? 2 * i : i, q = PAIRS ? 2 * i + 1 : 4 + i;
        const float y = x[p], z = x[q];
        x[p] = y * cs[i] - z * sn[i];
        x[q] = z * cs[i] + y * sn[i];
    }
    a = pack4(x);
    b = pack4(x + 4);
}
__device__ __forceinline__ void weights(const __nv_bfloat16* w, const Lane& ln, float (&g)[8]) {
    if (w == nullptr) return;
    unpack4(ln.on ? *reinterpret_cast<const uint2*>(w + ln.e0) : make_uint2(0u, 0u), g);
    unpack4(ln.on ? *reinterpret_cast<const uint2*>(w + ln.e1) : make_uint2(0u, 0u), g + 4);
}

// Rows first, first + step, .. < count of one token, `src` to `dst`, head x at x * d (src) and x * dst_step (dst):
// normed by the lane's weights w (NULL: not), rotated.
template <int LG, bool PAIRS>
__device__ __forceinline__ void move_rows(const __nv_bfloat16* src, __nv_bfloat16* dst, int64_t dst_step, int first, int step,
                                          int count, int d, const Lane& ln, const __nv_bfloat16* w, float eps, bool rotate,
                                          const float (&cs)[4], const float (&sn)[4], unsigned mask, bool& bad) {
    float g[8];
    weights(w, ln, g);
    for (int x0 = first; x0 < count; x0 += APP_ROWS * step) {
        uint2 a[APP_ROWS], b[APP_ROWS];
#pragma unroll
        for (int u = 0; u < APP_ROWS; ++u) {
            a[u] = b[u] = make_uint2(0u, 0u);
            if (x0 + u * step < count && ln.on) {
                const __nv_bfloat16* p = src + (x0 + u * step) * d;
                a[u] = *reinterpret_cast<const uint2*>(p + ln.e0);
                b[u] = *reinterpret_cast<const uint2*>(p + ln.e1);
            }
        }
#pragma unroll
        for (int u = 0; u < APP_ROWS; ++u) {
            if (x0 + u * step >= count) break;                   // (the same for all lanes of the group)
            bad = bad || nonfinite4(a[u]) || nonfinite4(b[u]);
            if (w != nullptr || rotate) transform<LG, PAIRS>(a[u], b[u], w != nullptr, g, eps, d, cs, sn, mask);
            if (ln.on) {
                __nv_bfloat16* p = dst + (x0 + u * step) * dst_step;
                *reinterpret_cast<uint2*>(p + ln.e0) = a[u];
                *reinterpret_cast<uint2*>(p + ln.e1) = b[u];
            }
        }
    }
}

__device__ __forceinline__ void widen(uint2& lo, uint2& hi, const uint2& a, const uint2& b) {
    __nv_bfloat162 *l = reinterpret_cast<__nv_bfloat162*>(&lo), *h = reinterpret_cast<__nv_bfloat162*>(&hi);
    const __nv_bfloat162 *x = reinterpret_cast<const __nv_bfloat162*>(&a), *y = reinterpret_cast<const __nv_bfloat162*>(&b);
#pragma unroll
    for (int i = 0; i < 2; ++i) { l[i] = __hmin2(l[i], x[i]); h[i] = __hmax2(h[i], y[i]); }
}

// A warp: one token, or one of `shares` parts of its heads.  LG lanes have a head's row.  STEP: after the queries' shares every
// key head of the token has a warp of its own, which also forms the page's bounds.
template <int LG, bool PAIRS, bool STEP>
__global__ void __launch_bounds__(APP_THREADS, 6)
k_cache_append(const CacheView c, const Ragged r, const AppendJob j, int shares, unsigned* __restrict__ status) {
    grid_dep_wait();
    grid_dep_launch_next();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int item = blockIdx.x * APP_WARPS + warp;
    const int parts = STEP ? shares + c.h_kv : shares;
    const int i = item / parts, share = item - i * parts;
    if (blockIdx.x == 0) {
        check_ragged(r, c, status, threadIdx.x, APP_THREADS);
        if (j.len_out != nullptr)
            for (int b = threadIdx.x; b < r.B; b += APP_THREADS) {
                int o;
                int n = seq_rows(r, b, o);
                if (j.rep_cnt != nullptr) n = min(max(j.rep_cnt[b], 0), n);
                j.len_out[b] = (int)min((int64_t)seq_len(r, c, b) + n, (int64_t)c.max_pages << c.shift);
            }
    }
    if (i >= r.N) return;
    const int b = seq_of_row(r, i);
    if (b < 0) return;
    int o;
    const int n = seq_rows(r, b, o), old = seq_len(r, c, b), li = i - o;
    const int p0 = j.pos0 != nullptr ? j.pos0[b] : old;
    // row i's queries are its own; the keys and values that go to slot old + li are those of token `at`
    unsigned faults = 0u;
    int kept = n, at = li, page = -1, slot = 0;
    if (j.rep_cnt != nullptr) {
        kept = j.rep_cnt[b];
        if (kept < 0 || kept > n) { faults |= ST_BAD_COUNT; kept = min(max(kept, 0), n); }
        if (li < kept) {
            at = j.rep_idx[i];
            if (at < 0 || at >= n || (li > 0 && j.rep_idx[i - 1] >= at)) { faults |= ST_BAD_INDEX; kept = 0; }
        }
    }
    if (li < kept) {
        const int64_t s = (int64_t)old + li;
        if (s >= (int64_t)c.max_pages << c.shift) {
            faults |= ST_BAD_COUNT;
        } else {
            page = c.table[(int64_t)b * c.table_ld + (s >> c.shift)];
            if (page < 0 || page >= c.n_pages) { faults |= ST_BAD_INDEX; page = -1; }
            slot = (int)s & ((1 << c.shift) - 1);
        }
    }
    if (faults != 0u && lane == 0) atomicOr(status, faults);

    constexpr int PER = 32 / LG;                                 // rows of a warp at a time
    const int v = lane % LG, first = share * PER + lane / LG, step = shares * PER;
    const unsigned mask = LG == 16 ? 0xffffu << (lane & 16) : 0xffu << (lane & 24);
    const bool rotate = j.inv_freq != nullptr;
    // lanes below rot / 8 have four pairs each; the elements behind `rot` are the other lanes', eight in a row
    const int nvec = c.d >> 3, nrot = rotate ? j.rot >> 3 : 0;
    Lane ln;
    ln.on = v < nvec;
    ln.turns = v < nrot;
    ln.e0 = !PAIRS && ln.turns ? 4 * v : 8 * v;
    ln.e1 = !PAIRS && ln.turns ? 4 * v + (j.rot >> 1) : 8 * v + 4;
    float cs[4], sn[4];
    angles(j, ln, v, p0, li, cs, sn);
    bool bad = false;
    if (j.Q != nullptr && (!STEP || share < shares))
        move_rows<LG, PAIRS>(j.Q + (int64_t)i * j.ldq, j.q_out + (int64_t)i * j.ldqo, c.d, first, step, j.h, c.d, ln, j.q_norm,
                             j.eps, rotate, cs, sn, mask, bad);
    if (STEP) {
        const int head = share - shares;
        if (head >= 0 && page >= 0) {
            const unsigned full = 0xffffffffu;
            const int64_t at0 = slot_at(c, page, head, 0);
            const bool own = lane < LG;                          // (one group of lanes writes)
            // the page's slots [0, s0) are older, [s0, slot] come from this call
            const bool last = c.kmin != nullptr && (li + 1 == kept || slot == (1 << c.shift) - 1);
            const int s0 = max(slot - li, 0);
            uint2 lo[2], hi[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) { lo[u] = make_uint2(0x7f807f80u, 0x7f807f80u); hi[u] = make_uint2(0xff80ff80u, 0xff80ff80u); }
            float g[8];
            weights(j.k_norm, ln, g);
            int turned = li;                                     // whose angles the lane has
            for (int t = last ? li - (slot - s0) : li; t <= li; ++t) {      // this token, or all new ones of the page
                const int tok = j.rep_idx != nullptr ? min(max(j.rep_idx[o + t], 0), n - 1) : t;
                if (tok != turned) angles(j, ln, v, p0, tok, cs, sn);
                turned = tok;
                uint2 a = make_uint2(0u, 0u), b2 = a;
                if (ln.on) {
                    const __nv_bfloat16* p = j.K + (int64_t)(o + tok) * j.ldk + (int64_t)head * c.d;
                    a = *reinterpret_cast<const uint2*>(p + ln.e0);
                    b2 = *reinterpret_cast<const uint2*>(p + ln.e1);
                }
                if (t == li) bad = bad || nonfinite4(a) || nonfinite4(b2);
                if (j.k_norm != nullptr || rotate) transform<LG, PAIRS>(a, b2, j.k_norm != nullptr, g, j.eps, c.d, cs, sn, mask);
                if (t == li && own && ln.on) {
                    *reinterpret_cast<uint2*>(c.k + at0 + (int64_t)slot * c.d + ln.e0) = a;
                    *reinterpret_cast<uint2*>(c.k + at0 + (int64_t)slot * c.d + ln.e1) = b2;
                }
                widen(lo[0], hi[0], a, a);
                widen(lo[1], hi[1], b2, b2);
            }
            if (own && ln.on) {
                const __nv_bfloat16* p = j.V + (int64_t)(o + at) * j.ldv + (int64_t)head * c.d;
                const uint2 a = *reinterpret_cast<const uint2*>(p + ln.e0), b2 = *reinterpret_cast<const uint2*>(p + ln.e1);
                bad = bad || nonfinite4(a) || nonfinite4(b2);
                *reinterpret_cast<uint2*>(c.v + at0 + (int64_t)slot * c.d + ln.e0) = a;
                *reinterpret_cast<uint2*>(c.v + at0 + (int64_t)slot * c.d + ln.e1) = b2;
            }
            if (last) {
                if (ln.on) {                                     // the groups of lanes take turns at the older keys
                    const __nv_bfloat16* p = c.k + at0;
#pragma unroll 8
                    for (int q = lane / LG; q < s0; q += PER) {
                        const uint2 a = *reinterpret_cast<const uint2*>(p + (int64_t)q * c.d + ln.e0);
                        const uint2 b2 = *reinterpret_cast<const uint2*>(p + (int64_t)q * c.d + ln.e1);
                        widen(lo[0], hi[0], a, a);
                        widen(lo[1], hi[1], b2, b2);
                    }
                }
#pragma unroll
                for (int m = LG; m < 32; m <<= 1)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const uint2 a = make_uint2(__shfl_xor_sync(full, lo[u].x, m), __shfl_xor_sync(full, lo[u].y, m));
                        const uint2 b2 = make_uint2(__shfl_xor_sync(full, hi[u].x, m), __shfl_xor_sync(full, hi[u].y, m));
                        widen(lo[u], hi[u], a, b2);
                    }
                if (own && ln.on) {
                    const int64_t to = ((int64_t)page * c.h_kv + head) * c.d;
                    *reinterpret_cast<uint2*>(c.kmin + to + ln.e0) = lo[0];
                    *reinterpret_cast<uint2*>(c.kmin + to + ln.e1) = lo[1];
                    *reinterpret_cast<uint2*>(c.kmax + to + ln.e0) = hi[0];
                    *reinterpret_cast<uint2*>(c.kmax + to + ln.e1) = hi[1];
                }
            }
        }
    } else if (page >= 0) {
        const int64_t at0 = slot_at(c, page, 0, slot), head_step = (int64_t)c.d << c.shift;
        if (at != li) angles(j, ln, v, p0, at, cs, sn);
        move_rows<LG, PAIRS>(j.K + (int64_t)(o + at) * j.ldk, c.k + at0, head_step, first, step, c.h_kv, c.d, ln, j.k_norm, j.eps,
                             rotate, cs, sn, mask, bad);
        move_rows<LG, PAIRS>(j.V + (int64_t)(o + at) * j.ldv, c.v + at0, head_step, first, step, c.h_kv, c.d, ln, nullptr, 0.f,
                             false, cs, sn, mask, bad);
    }
    if (bad) atomicOr(status, ST_NONFINITE);
}

// Elementwise minimum and maximum of a page's keys, over the slots below the sequence's new length, from the page
// itself: what a page held before (another sequence, tokens taken back) has no part in them.  Block (x, y):
// the x-th page that the call wrote to, head y.  Exact, whatever the order.
constexpr int BND_THREADS = 128;
__global__ void __launch_bounds__(BND_THREADS)
k_cache_bounds(const CacheView c, const Ragged r, const int32_t* __restrict__ rep_cnt) {
    __shared__ uint4 part[2][BND_THREADS];
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
    // which page it is, is written in what was there before the append began; its keys are the append's
    grid_dep_wait();
    grid_dep_launch_next();
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
#pragma unroll 8
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
    // a token's heads are dealt to several warps while the tokens alone do not fill the GPU: as many as leave a warp
    // one round of rows of the larger of queries and keys
    const int per = c.d <= 64 ? 4 : 2;
    const bool step = r.N <= r.B && (int64_t)r.N * (c.h_kv + j.h) < (int64_t)1 << 30;
    const int heads = step ? j.h : j.h > c.h_kv ? j.h : c.h_kv;
    const int want = (heads + per * APP_ROWS - 1) / (per * APP_ROWS), room = 16 * ctx->sm_count / r.N;
    const int shares = room < 1 ? (heads > 0 ? 1 : 0) : want < room ? want : room;
    const int64_t items = (int64_t)r.N * (step ? shares + c.h_kv : shares);
    auto kernel = step ? (c.d <= 64 ? (j.pairs ? k_cache_append<8, true, true> : k_cache_append<8, false, true>)
                                    : (j.pairs ? k_cache_append<16, true, true> : k_cache_append<16, false, true>))
                       : (c.d <= 64 ? (j.pairs ? k_cache_append<8, true, false> : k_cache_append<8, false, false>)
                                    : (j.pairs ? k_cache_append<16, true, false> : k_cache_append<16, false, false>));
    prof_begin(ctx, K_CACHE_APPEND, s);
    cudaError_t e = launch_k(ctx, kernel, dim3((unsigned)((items + APP_WARPS - 1) / APP_WARPS)), dim3(APP_THREADS), 0, s, c, r, j,
                             shares, ctx->status);
    prof_end(ctx, s);
    if (e != cudaSuccess) return e;
    if (c.kmin != nullptr && !step) {
        // a sequence of n new tokens writes to at most n and at most (n - 1) / ps + 2 pages
        const int64_t most = (int64_t)(r.N >> c.shift) + 2 * (int64_t)r.B;
        const int pages = (int)(most < r.N ? most : r.N);
        prof_begin(ctx, K_CACHE_BOUNDS, s);
        e = launch_k(ctx, k_cache_bounds, dim3(pages, c.h_kv), dim3(BND_THREADS), 0, s, c, r, j.rep_cnt);
        prof_end(ctx, s);
    }
    return e;
}

}  // namespace ada
