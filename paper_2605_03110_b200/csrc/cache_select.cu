// Choice of pages (ada_select_blocks): for every new token and key head the k pages whose keys can matter most.
//
//   s(p) = sum_g sum_e max(q_ge kmax_pe, q_ge kmin_pe)  >=  sum_g q_g . key   for every key of page p
// g runs over the heads that share the key head.  max(q a, q b) with a >= b is q a for q > 0 and q b for q < 0, so with
// the sums of the positive and of the negative parts, P_e = sum_g max(q_ge, 0) and M_e = sum_g min(q_ge, 0),
//   s(p) = sum_e P_e kmax_pe + M_e kmin_pe:
// one dot product of 2 d_h elements, whatever the number of heads.
//
// The choice is that of scores in 64 bits, but few of them are ever formed.  fp32 scores whose error is bounded (E below)
// come first: a page whose score is more than 2 E above (below) the k-th largest is certainly in (out); the few in between
// are scored again in 64 bits by the warps that have the row.  Rows with more such pages than lanes (equal scores,
// infinities) are done in 64 bits throughout, by the whole block.
//
// Single tokens are bound by reading the bounds of all pages from HBM: a block per (token, key head), a warp takes
// eight pages at a time, 16 bytes a lane, straight into registers, the next eight under way.  Of several tokens of a sequence
// a block scores 16 against the same pages on mma.sync, P and M as two bf16 terms each (products exact, fp32
// sums); the bounds then come from L2 through a ring of four half stages.
//
// Measured (32 heads on 8 key heads of 128): 32 tokens over 512 pages each 17 us, 67 MB = 3.9 TB/s (loads 13 us, the choice 3);
// 1000 tokens over 257 pages 47 us: a block 3 for the tokens' sums, 9 for the scores, 6 for the choice, 1.7 blocks for
// every place.  How many tokens share a block goes by the width of the table, which the host knows, not by the lengths, which it
// does not: the same 1000 tokens with a table of 1024 entries take 97 us, of 4096 342, of 16384 376 (single tokens 17 up to
// 8192, 25 with 16384).  A call should pass the part of the table that its longest sequence needs.
// Without leaving pages aside first, every guess at the k-th score counting all of them: 21 and 54 us; all
// scores in 64 bits: 47 and 454.
#include "cache_tma.cuh"

namespace ada {

namespace {

constexpr int SEL_THREADS = 256;
constexpr int SEL_WARPS = SEL_THREADS / 32;
constexpr int SEL_PAGES = 64;            // pages per stage: eight for every warp
constexpr int SEL_ROWS = 16;             // tokens of a tile
constexpr int SEL_RING = 4;              // half stages (the maxima or the minima of SEL_PAGES pages) in shared memory
constexpr int SEL_SPAN = 512;            // scores of a row that one warp counts alone
constexpr int SEL_LEFT = 64;             // of them left to choose from, room for
constexpr float SEL_NONE = -3.402823466e38f;   // of pages that do not compete
// |fp32 score - s(p)| <= (error + (G - 1) 2^-24) sum_e (P_e + |M_e|) a_e, a_e the largest |bound| of element e in any
// page; P is an fp32 sum over G heads, (G - 1) 2^-24.
// mma.sync: two bf16 terms leave 2^-16 of P; d_h / 16 <= 8 matrix instructions for either sign add 16 products and the
// running sum, each of the 17 addends cut at 2^-24 of the largest: 2.4e-5; the sums of either sign and of the second
// terms, a few roundings more, are in the reserve.  Direct: 8 fused multiply-adds and 5 additions, each rounded: 13 x 2^-24.
constexpr float SEL_ERR_MMA = 2.7e-5f, SEL_ERR_ONE = 9e-7f;

__device__ __forceinline__ unsigned long long sort_key(double x) {
    if (!(x == x)) return 0ull;                                  // NaN: behind everything
    x += 0.0;                                                    // -0 is 0
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ unsigned sort_key(float x) {
    const unsigned b = __float_as_uint(x + 0.0f);
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k); }

__device__ __forceinline__ void cp16(unsigned dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldsm2(unsigned addr, unsigned (&r)[2]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}

struct SelShared {
    double qp[128], qm[128];                       // of a row that is done in 64 bits throughout
    unsigned col[128];                             // mma.sync: largest |bound| of every element (bits)
    unsigned reach[SEL_WARPS];                     // direct: sum_e (P_e + |M_e|) a_e, a_e over the warp's pages (bits)
    int n_hard, hard[SEL_ROWS];
    int cnt[2][SEL_WARPS], tie[SEL_WARPS];
    unsigned word[2][SEL_WARPS];
    int list[SEL_WARPS][32];
    unsigned long long key[SEL_WARPS][32];
};

// bytes of a row of d elements in shared memory: an odd number of 16-byte pieces, so that ldmatrix has no bank conflict
__host__ __device__ __forceinline__ int sel_row(int d) { return d * 2 + 16; }
__host__ __device__ __forceinline__ int sel_half(int d) { return SEL_PAGES * sel_row(d); }

// grid (tiles of `rows` tokens of one sequence, key heads).  ONE: one token per block; shared memory holds its scores.  Else:
// the ring of half stages | the tile's P and M as bf16 terms | scores [rows][stride].  A row done in 64 bits
// throughout has its keys at the start of it.
template <bool ONE>
__global__ void __launch_bounds__(SEL_THREADS, 2)
k_cache_select(const CacheView c, const Ragged r, const SelectJob j, int rows, int stride, int ring_room,
               unsigned* __restrict__ status) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ SelShared sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int head = blockIdx.y, G = j.h / c.h_kv;
    const int rb = sel_row(c.d);
    unsigned char* a_tile = smem + ring_room;                   // [P hi, P lo, M hi, M lo][16][rb]
    float* score = reinterpret_cast<float*>(ONE ? smem : a_tile + 4 * SEL_ROWS * rb);
    const int left_at = ONE ? stride * 4 : 0;                   // what is left of a row: behind the scores, over the ring
    grid_dep_wait();
    grid_dep_launch_next();
    if (blockIdx.x == 0 && head == 0) check_ragged(r, c, status, tid, SEL_THREADS);

    // ---- the tile: the sequence and its first token, by every warp for itself
    int b = -1, t0 = 0;
    if (ONE) {
        int o;
        b = seq_of_row(r, blockIdx.x);
        if (b >= 0) { seq_rows(r, b, o); t0 = (int)blockIdx.x - o; }
    } else {
        int left = blockIdx.x;
        for (int b0 = 0; b0 < r.B; b0 += 32) {
            int o;
            const int tiles = b0 + lane < r.B ? (seq_rows(r, b0 + lane, o) + rows - 1) / rows : 0;
            int sum = tiles;
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, sum, m);
                if (lane >= m) sum += y;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, left < sum);
            if (hit != 0u) {
                const int l = __ffs(hit) - 1;
                b = b0 + l;
                t0 = (left - __shfl_sync(0xffffffffu, sum - tiles, l)) * rows;
                break;
            }
            left -= __shfl_sync(0xffffffffu, sum, 31);
        }
    }
    if (b < 0) return;
    int o;
    const int n = seq_rows(r, b, o), len = seq_len(r, c, b);
    const int n_tok = min(rows, n - t0), row0 = o + t0;
    auto limit = [&](int t) { return j.causal ? max(len - n + t0 + t + 1, 0) : len; };
    auto pages_of = [&](int t) { return (limit(t) + (1 << c.shift) - 1) >> c.shift; };
    const int nb_all = pages_of(n_tok - 1);                     // the last token sees the most
    const int v = lane & 15, lower = lane >> 4, nvec = c.d >> 3;
    if (nb_all > j.k) {
        if (tid == 0) sh.n_hard = 0;
        if (ONE) {
            // ---- lanes 0..15 have P and the maxima, 16..31 M and the minima, eight elements each
            const __nv_bfloat16* bounds = (lower ? c.kmin : c.kmax) + (int64_t)head * c.d + v * 8;
            int id = -1;                                        // lane q: the table's entry for page q of the next eight
            auto fetch_ids = [&](int p0) {
                const int p = p0 + warp * 8 + lane;
                id = lane < 8 && p < nb_all ? page_of(c, b, p, status) : -1;
            };
            auto fetch = [&](uint4 (&x)[8]) {
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int page = __shfl_sync(0xffffffffu, id, q);
                    x[q] = make_uint4(0u, 0u, 0u, 0u);
                    if (page >= 0 && v < nvec) x[q] = __ldg(reinterpret_cast<const uint4*>(bounds + (int64_t)page * c.h_kv * c.d));
                }
            };
            uint4 cur[8], nxt[8];
            fetch_ids(0);
            fetch(cur);
            fetch_ids(SEL_PAGES);
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = 0.f;
            if (v < nvec) {
                const __nv_bfloat16* q = j.Q + (int64_t)row0 * j.ldq + (int64_t)head * G * c.d + v * 8;
#pragma unroll 4
                for (int g = 0; g < G; ++g) {
                    const uint4 u = *reinterpret_cast<const uint4*>(q + (int64_t)g * c.d);
                    const unsigned uu[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = __uint_as_float((e & 1) ? uu[e >> 1] & 0xffff0000u : uu[e >> 1] << 16);
                        w[e] += x != x ? x : lower ? fminf(x, 0.f) : fmaxf(x, 0.f);
                    }
                }
            }
            __nv_bfloat162 most[4];                              // largest |bound| of the lane's elements (NaN stays)
#pragma unroll
            for (int u = 0; u < 4; ++u) most[u] = __float2bfloat162_rn(0.f);
            for (int p0 = 0; p0 < nb_all; p0 += SEL_PAGES) {
                if (p0 + SEL_PAGES < nb_all) {
                    fetch(nxt);
                    fetch_ids(p0 + 2 * SEL_PAGES);
                }
                float a[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const unsigned uu[4] = {cur[q].x, cur[q].y, cur[q].z, cur[q].w};
                    a[q] = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        a[q] = fmaf(w[e], __uint_as_float((e & 1) ? uu[e >> 1] & 0xffff0000u : uu[e >> 1] << 16), a[q]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) most[u] = __hmax2_nan(most[u], __habs2(*reinterpret_cast<const __nv_bfloat162*>(&uu[u])));
                }
                // sums of eight pages over the lanes: halves of the pages change places with halves of the lanes
#pragma unroll
                for (int m = 4; m > 0; m >>= 1) {
                    const bool up = lane & (4 * m);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q < m) {
                            const float send = up ? a[q] : a[q + m], keep = up ? a[q + m] : a[q];
                            a[q] = keep + __shfl_xor_sync(0xffffffffu, send, 4 * m);
                        }
                }
                a[0] += __shfl_xor_sync(0xffffffffu, a[0], 2);
                a[0] += __shfl_xor_sync(0xffffffffu, a[0], 1);
                const int p = p0 + warp * 8 + (lane >> 2);       // (bits 4, 3, 2 of the lane: bits 2, 1, 0 of the page)
                if ((lane & 3) == 0 && p < nb_all) score[p] = a[0];
#pragma unroll
                for (int q = 0; q < 8; ++q) cur[q] = nxt[q];
            }
            float A = 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) A += fabsf(w[2 * u]) * __low2float(most[u]) + fabsf(w[2 * u + 1]) * __high2float(most[u]);
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) A += __shfl_xor_sync(0xffffffffu, A, m);
            if (lane == 0) sh.reach[warp] = __float_as_uint(A) & 0x7fffffffu;   // (a NaN's bits are larger than any number's)
            __syncthreads();
        } else {
            const int nhalf = 2 * ((nb_all + SEL_PAGES - 1) / SEL_PAGES);
            // half stage i: the maxima (i even) or minima (odd) of pages 64 (i / 2) ..; a warp's half has a page, 16 bytes a lane
            int id = -1, id_next = -1;                           // lane q: the table's entry for the warp's q-th page
            auto fetch_ids = [&](int p0) {
                const int p = p0 + warp * 8 + lane;
                id_next = lane < 8 && p < nb_all ? page_of(c, b, p, status) : -1;
            };
            fetch_ids(0);
            auto load_half = [&](int i) {
                if (i < nhalf) {
                    if ((i & 1) == 0) {
                        id = id_next;
                        fetch_ids(((i >> 1) + 1) * SEL_PAGES);
                    }
                    const __nv_bfloat16* bounds = ((i & 1) ? c.kmin : c.kmax) + (int64_t)head * c.d + v * 8;
                    const unsigned at = tc::smem_u32(smem + (i & (SEL_RING - 1)) * sel_half(c.d)) + (warp * 8) * rb + v * 16;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int page = __shfl_sync(0xffffffffu, id, 2 * q + lower);
                        if (v < nvec) cp16(at + (2 * q + lower) * rb, bounds + (int64_t)max(page, 0) * c.h_kv * c.d, page >= 0);
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            if (tid < 128) sh.col[tid] = 0u;
#pragma unroll 1
            for (int i = 0; i < SEL_RING - 1; ++i) load_half(i);
            // ---- P and M of the tile's tokens, eight elements a thread
            if (tid < SEL_ROWS * nvec) {
                const int t = tid / nvec, e0 = (tid - t * nvec) * 8;
                float p[8], m[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = m[e] = 0.f;
                if (t < n_tok) {
                    const __nv_bfloat16* q = j.Q + (int64_t)(row0 + t) * j.ldq + (int64_t)head * G * c.d + e0;
#pragma unroll 4
                    for (int g = 0; g < G; ++g) {
                        const uint4 u = *reinterpret_cast<const uint4*>(q + (int64_t)g * c.d);
                        const unsigned uu[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float x = __uint_as_float((e & 1) ? uu[e >> 1] & 0xffff0000u : uu[e >> 1] << 16);
                            p[e] += x != x ? x : fmaxf(x, 0.f);
                            m[e] += fminf(x, 0.f);
                        }
                    }
                }
                uint4 o4[4];
                unsigned* w = reinterpret_cast<unsigned*>(o4);
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const __nv_bfloat162 ph = __floats2bfloat162_rn(p[e], p[e + 1]), mh = __floats2bfloat162_rn(m[e], m[e + 1]);
                    const __nv_bfloat162 pl = __floats2bfloat162_rn(p[e] - __low2float(ph), p[e + 1] - __high2float(ph));
                    const __nv_bfloat162 ml = __floats2bfloat162_rn(m[e] - __low2float(mh), m[e + 1] - __high2float(mh));
                    w[e >> 1] = *reinterpret_cast<const unsigned*>(&ph);
                    w[4 + (e >> 1)] = *reinterpret_cast<const unsigned*>(&pl);
                    w[8 + (e >> 1)] = *reinterpret_cast<const unsigned*>(&mh);
                    w[12 + (e >> 1)] = *reinterpret_cast<const unsigned*>(&ml);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) *reinterpret_cast<uint4*>(a_tile + (u * SEL_ROWS + t) * rb + e0 * 2) = o4[u];
            }
            // ---- scores
            const unsigned a_at = tc::smem_u32(a_tile) + (lane & 15) * rb + (lane >> 4) * 16;
            __nv_bfloat162 most[4];                              // of the elements that this lane fetches (NaN stays)
#pragma unroll
            for (int u = 0; u < 4; ++u) most[u] = __float2bfloat162_rn(0.f);
            float acc[4][4];                                     // second and first terms of P, of M
            for (int i = 0; i < nhalf; ++i) {
                asm volatile("cp.async.wait_group %0;" ::"n"(SEL_RING - 2) : "memory");
                __syncthreads();                                 // half stage i is there, and nobody reads i - 1 any more
                load_half(i + SEL_RING - 1);
                const unsigned char* half = smem + (i & (SEL_RING - 1)) * sel_half(c.d);
                if (v < nvec) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint4 x = *reinterpret_cast<const uint4*>(half + (warp * 8 + 2 * q + lower) * rb + v * 16);
                        const __nv_bfloat162* y = reinterpret_cast<const __nv_bfloat162*>(&x);
#pragma unroll
                        for (int u = 0; u < 4; ++u) most[u] = __hmax2_nan(most[u], __habs2(y[u]));
                    }
                }
                const int sign = i & 1;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (sign == 0) acc[u][e] = 0.f;
                        acc[2 + u][e] = sign == 0 ? 0.f : acc[2 + u][e];
                    }
                const unsigned b_at = tc::smem_u32(half) + (warp * 8 + (lane & 7)) * rb + ((lane >> 3) & 1) * 16;
                if (sign == 0) {
#pragma unroll 4
                    for (int ks = 0; ks < c.d >> 4; ++ks) {
                        unsigned bf[2], hi[4], lo[4];
                        ldsm2(b_at + ks * 32, bf);
                        tc::ldsm4(a_at + ks * 32, hi);
                        tc::ldsm4(a_at + SEL_ROWS * rb + ks * 32, lo);
                        tc::mma16816(acc[0], lo, bf[0], bf[1]);
                        tc::mma16816(acc[1], hi, bf[0], bf[1]);
                    }
                } else {
#pragma unroll 4
                    for (int ks = 0; ks < c.d >> 4; ++ks) {
                        unsigned bf[2], hi[4], lo[4];
                        ldsm2(b_at + ks * 32, bf);
                        tc::ldsm4(a_at + 2 * SEL_ROWS * rb + ks * 32, hi);
                        tc::ldsm4(a_at + 3 * SEL_ROWS * rb + ks * 32, lo);
                        tc::mma16816(acc[2], lo, bf[0], bf[1]);
                        tc::mma16816(acc[3], hi, bf[0], bf[1]);
                    }
                    const int p = (i >> 1) * SEL_PAGES + warp * 8 + 2 * (lane & 3);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int t = (lane >> 2) + 8 * h;
                        float x[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            x[e] = (acc[1][2 * h + e] + acc[3][2 * h + e]) + (acc[0][2 * h + e] + acc[2][2 * h + e]);
                        if (t < n_tok) *reinterpret_cast<float2*>(score + t * stride + p) = make_float2(x[0], x[1]);
                    }
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            if (v < nvec) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {                    // (a NaN's bits are larger than any number's)
                    atomicMax(&sh.col[v * 8 + 2 * u], __float_as_uint(__low2float(most[u])) & 0x7fffffffu);
                    atomicMax(&sh.col[v * 8 + 2 * u + 1], __float_as_uint(__high2float(most[u])) & 0x7fffffffu);
                }
            }
            __syncthreads();
        }
    }

    // ---- teams of `tw` warps, a row each: the k-th largest fp32 score, and what cannot be told from it
    // (One warp alone needs no meeting.  Four scores a lane and load; the code is kept small, every block runs it once.)
    const int room = ONE ? SEL_WARPS : rows >= SEL_WARPS ? 1 : SEL_WARPS / rows;
    int tw = 1;
    while (tw < room && nb_all > SEL_SPAN * tw) tw <<= 1;
    const int team = warp / room, mate = warp - team * room;
    const int step = 32 * tw, at0 = mate * 32 + lane;
    int turn = 0;
    auto meet = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(step) : "memory"); };
    // sum (greatest) over the team; the slots alternate, so that one meeting per call is enough
    auto sum_of = [&](int x) {
        x = __reduce_add_sync(0xffffffffu, x);
        if (tw == 1) return x;
        turn ^= 1;
        if (lane == 0) sh.cnt[turn][warp] = x;
        meet();
        x = 0;
        for (int q = 0; q < tw; ++q) x += sh.cnt[turn][team * room + q];
        return x;
    };
    auto most_of = [&](unsigned x) {
        x = __reduce_max_sync(0xffffffffu, x);
        if (tw == 1) return x;
        turn ^= 1;
        if (lane == 0) sh.word[turn][warp] = x;
        meet();
        x = 0u;
        for (int q = 0; q < tw; ++q) x = max(x, sh.word[turn][team * room + q]);
        return x;
    };
    for (int t = team; t < n_tok && mate < tw; t += SEL_WARPS / room) {
        const int nb = pages_of(t), row = row0 + t, take = min(nb, j.k);
        int32_t* idx = j.blk_idx + ((int64_t)row * c.h_kv + head) * j.k;
        if (mate == 0 && lane == 0) j.blk_cnt[(int64_t)row * c.h_kv + head] = take;
        if (nb <= j.k) {
            for (int i = at0; i < j.k; i += step) idx[i] = i < nb ? i : -1;
            continue;
        }
        float* s = score + t * stride;
        const int first = j.n_first, last = nb - j.n_last;       // pages [first, last) compete for `need` places
        int n4 = (nb + 3) >> 2;                                  // float4s of the row
        // the others are out of it, and listed without further ado
        for (int p = at0; p < first; p += step) { s[p] = SEL_NONE; idx[p] = p; }
        for (int p = last + at0; p < n4 * 4; p += step) {
            s[p] = SEL_NONE;
            if (p < nb) idx[j.k - nb + p] = p;
        }
        if (tw > 1) meet(); else __syncwarp();
        int need = j.k - j.n_first - j.n_last;
        if (need == 0) continue;
        float A = 0.f;
        if (ONE) {                                               // (a page's sum is bounded by its own warp's)
            A = __uint_as_float(__reduce_max_sync(0xffffffffu, sh.reach[lane & (SEL_WARPS - 1)]));
        } else {
            if (lane * 4 < c.d) {
                const unsigned char* ar = a_tile + t * rb + lane * 8;
                const uint2 ph = *reinterpret_cast<const uint2*>(ar), mh = *reinterpret_cast<const uint2*>(ar + 2 * SEL_ROWS * rb);
                const uint4 a = *reinterpret_cast<const uint4*>(&sh.col[lane * 4]);
                A = (__uint_as_float(ph.x << 16) - __uint_as_float(mh.x << 16)) * __uint_as_float(a.x) +
                    (__uint_as_float(ph.x & 0xffff0000u) - __uint_as_float(mh.x & 0xffff0000u)) * __uint_as_float(a.y) +
                    (__uint_as_float(ph.y << 16) - __uint_as_float(mh.y << 16)) * __uint_as_float(a.z) +
                    (__uint_as_float(ph.y & 0xffff0000u) - __uint_as_float(mh.y & 0xffff0000u)) * __uint_as_float(a.w);
            }
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) A += __shfl_xor_sync(0xffffffffu, A, m);
            A *= 1.004f;                                         // (first terms are up to 2^-8 short)
        }
        // no score is larger than A and its error: beyond this, or for a NaN, fp32 says nothing
        if (!(A <= 1e36f)) {
            if (mate == 0 && lane == 0) sh.hard[atomicAdd(&sh.n_hard, 1)] = t;
            continue;
        }
        const float E = ((ONE ? SEL_ERR_ONE : SEL_ERR_MMA) + (float)G * 6e-8f) * A + 1e-35f;
        // places of the pages of 32 float4s for which `is` holds, ascending: what a warp writes them with
        const float4* s4 = reinterpret_cast<const float4*>(s);
        auto list = [&](auto is, auto put) {
            int n_put = 0;
            for (int i0 = 0; i0 < n4; i0 += 32) {
                const float4 x = i0 + lane < n4 ? s4[i0 + lane] : make_float4(SEL_NONE, SEL_NONE, SEL_NONE, SEL_NONE);
                const bool y[4] = {is(x.x), is(x.y), is(x.z), is(x.w)};
                int before = n_put;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned m = __ballot_sync(0xffffffffu, y[e]);
                    before += __popc(m & ((1u << lane) - 1u));
                    n_put += __popc(m);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (y[e]) put(before++, 4 * (i0 + lane) + e);
            }
            return n_put;
        };
        // A warp alone with few places to give first leaves aside what cannot have one: if `need` groups of pages have a score of
        // at least t0 each, no page below t0 - 2 E matters.  What remains, mostly a few more than `need`, is two a lane.
        bool left = tw == 1 && need <= 32 && n4 * 4 > SEL_LEFT;
        float va = SEL_NONE, vb = SEL_NONE;                      // number `lane` and 32 + lane of what remains
        int pa = 0, pb = 0, n_left = 0;
        // of the lanes' values (va, vb) the need-th largest, or with `slack` one up to so many places behind it; SEL_NONE if there
        // are not that many
        auto kth_of = [&](int slack) {
            const unsigned ka = sort_key(va), kb = sort_key(vb), none = sort_key(SEL_NONE);
            unsigned hi = __reduce_max_sync(0xffffffffu, max(ka, kb));
            unsigned lo = __reduce_min_sync(0xffffffffu, min(ka == none ? ~0u : ka, kb == none ? ~0u : kb));
            if (__popc(__ballot_sync(0xffffffffu, ka >= lo)) + __popc(__ballot_sync(0xffffffffu, kb >= lo)) < need) return SEL_NONE;
            while (lo < hi) {
                const unsigned mid = lo + ((hi - lo + 1u) >> 1);
                const int ge = __popc(__ballot_sync(0xffffffffu, ka >= mid)) + __popc(__ballot_sync(0xffffffffu, kb >= mid));
                if (ge >= need) lo = mid; else hi = mid - 1u;
                if (ge >= need && ge <= need + slack) {          // the smallest of them
                    lo = __reduce_min_sync(0xffffffffu, min(ka >= mid ? ka : ~0u, kb >= mid ? kb : ~0u));
                    break;
                }
            }
            return key_value(lo);
        };
        if (left) {
            const int step2 = need > 16 ? 64 : 32;               // groups: 32, or 64 where many places are to be given
            for (int i = lane; i < n4; i += 64) {
                const float4 x = s4[i], y = i + 32 < n4 ? s4[i + 32] : make_float4(SEL_NONE, SEL_NONE, SEL_NONE, SEL_NONE);
                va = fmaxf(va, fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)));
                vb = fmaxf(vb, fmaxf(fmaxf(y.x, y.y), fmaxf(y.z, y.w)));
            }
            if (step2 == 32) { va = fmaxf(va, vb); vb = SEL_NONE; }
            const float t0 = fmaxf(__fadd_rd(kth_of(2), -__fmul_ru(2.0f, E)), -2e36f);    // (SEL_NONE is below)
            float* room_v = reinterpret_cast<float*>(smem + left_at) + warp * 2 * SEL_LEFT;
            int* room_p = reinterpret_cast<int*>(room_v + SEL_LEFT);
            __syncwarp();                                        // (the row before has been read out of it)
            n_left = list([&](float x) { return x >= t0; }, [&](int at, int p) {
                if (at < SEL_LEFT) { room_v[at] = s[p]; room_p[at] = p; }
            });
            __syncwarp();
            left = n_left <= SEL_LEFT;
            if (left) {
                const bool x = lane < n_left, y = 32 + lane < n_left;
                va = x ? room_v[lane] : SEL_NONE;
                vb = y ? room_v[32 + lane] : SEL_NONE;
                pa = x ? room_p[lane] : 0;
                pb = y ? room_p[32 + lane] : 0;
            }
        }
        float kth;
        if (left) {
            kth = kth_of(0);
        } else {
            float mn = INFINITY, mx = SEL_NONE;
            for (int i = at0; i < n4; i += step) {
                const float4 x = s4[i];
                mx = fmaxf(mx, fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)));
                mn = fminf(mn, fminf(fminf(x.x == SEL_NONE ? mn : x.x, x.y == SEL_NONE ? mn : x.y), fminf(x.z == SEL_NONE ? mn : x.z, x.w == SEL_NONE ? mn : x.w)));
            }
            // at least `need` scores are >= lo, fewer than that > hi (as keys: integers that order as the scores do)
            unsigned hi = most_of(sort_key(mx)), lo = ~most_of(~sort_key(mn));
            while (lo < hi) {
                const unsigned mid = lo + ((hi - lo + 1u) >> 1);
                const float at = key_value(mid);
                int ge = 0;
#pragma unroll 2
                for (int i = at0; i < n4; i += step) {
                    const float4 x = s4[i];
                    ge += (x.x >= at) + (x.y >= at) + (x.z >= at) + (x.w >= at);
                }
                ge = sum_of(ge);
                if (ge >= need) lo = mid; else hi = mid - 1u;
                if (ge == need) {                                // the smallest of them is the one that is sought
                    mn = INFINITY;
                    for (int i = at0; i < n4; i += step) {
                        const float4 x = s4[i];
                        mn = fminf(mn, fminf(fminf(x.x >= at ? x.x : mn, x.y >= at ? x.y : mn), fminf(x.z >= at ? x.z : mn, x.w >= at ? x.w : mn)));
                    }
                    lo = ~most_of(~sort_key(mn));
                    break;
                }
            }
            kth = key_value(lo);
        }
        // undecided if below <= s <= above
        const float above = __fadd_ru(kth, __fmul_ru(2.0f, E)), below = __fadd_rd(kth, -__fmul_ru(2.0f, E));
        const unsigned before = (1u << lane) - 1u;
        unsigned ua = 0u, ub = 0u;                               // undecided ones among what remains
        int band;
        if (left) {
            ua = __ballot_sync(0xffffffffu, va >= below && va <= above);
            ub = __ballot_sync(0xffffffffu, vb >= below && vb <= above);
            band = __popc(ua) + __popc(ub);
            need -= __popc(__ballot_sync(0xffffffffu, va > above)) + __popc(__ballot_sync(0xffffffffu, vb > above));
        } else {
            int in = 0;                                          // certain ones, and 65536 for every undecided one
            for (int i = at0; i < n4; i += step) {
                const float4 x = s4[i];
                in += (x.x > above ? 1 : x.x >= below ? 65536 : 0) + (x.y > above ? 1 : x.y >= below ? 65536 : 0) +
                      (x.z > above ? 1 : x.z >= below ? 65536 : 0) + (x.w > above ? 1 : x.w >= below ? 65536 : 0);
            }
            in = sum_of(in);
            band = in >> 16;
            need -= in & 0xffff;
        }
        const int at_a = __popc(ua & before), at_b = __popc(ua) + __popc(ub & before);   // places among the undecided ones
        unsigned chosen = 0xffffffffu;                           // of the undecided ones
        if (band != need) {
            if (band > 32) {
                if (mate == 0 && lane == 0) sh.hard[atomicAdd(&sh.n_hard, 1)] = t;
                continue;
            }
            // every warp of the team lists them; each scores its share of them in 64 bits
            if (left) {
                if (ua >> lane & 1u) sh.list[warp][at_a] = pa;
                if (ub >> lane & 1u) sh.list[warp][at_b] = pb;
            } else {
                list([&](float x) { return x >= below && x <= above; }, [&](int at, int p) { sh.list[warp][at] = p; });
            }
            __syncwarp();
            const int mine = lane < band ? sh.list[warp][lane] : INT_MAX;
            const int page_l = lane < band ? page_of(c, b, mine, status) : -1;
            double P[4], M[4];                                   // of elements 4 lane .. 4 lane + 3
            const bool on = lane * 4 < c.d;
#pragma unroll
            for (int e = 0; e < 4; ++e) P[e] = M[e] = 0.0;
            const __nv_bfloat16* qrow = j.Q + (int64_t)row * j.ldq + (int64_t)head * G * c.d + (on ? lane * 4 : 0);
#pragma unroll 4
            for (int g = 0; g < G; ++g) {
                const uint2 w = *reinterpret_cast<const uint2*>(qrow + (int64_t)g * c.d);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned u = e < 2 ? w.x : w.y;
                    const double x = (double)__uint_as_float((e & 1) ? u & 0xffff0000u : u << 16);
                    P[e] += x > 0.0 ? x : 0.0;
                    M[e] += x > 0.0 ? 0.0 : x;
                }
            }
#pragma unroll 2
            for (int q = mate; q < band; q += tw) {
                const int page = __shfl_sync(0xffffffffu, page_l, q);
                double x = 0.0;
                if (page >= 0 && on) {
                    const int64_t base = ((int64_t)page * c.h_kv + head) * c.d + lane * 4;
                    const uint2 u = *reinterpret_cast<const uint2*>(c.kmax + base), z = *reinterpret_cast<const uint2*>(c.kmin + base);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned a = e < 2 ? u.x : u.y, i = e < 2 ? z.x : z.y;
                        x = fma(P[e], (double)__uint_as_float((e & 1) ? a & 0xffff0000u : a << 16),
                                fma(M[e], (double)__uint_as_float((e & 1) ? i & 0xffff0000u : i << 16), x));
                    }
                }
#pragma unroll
                for (int m = 16; m > 0; m >>= 1) x += __shfl_xor_sync(0xffffffffu, x, m);
                if (lane == 0) sh.key[team * room][q] = page < 0 ? 0ull : sort_key(x);
            }
            if (tw > 1) meet(); else __syncwarp();
            const unsigned long long own = lane < band ? sh.key[team * room][lane] : 0ull;
            int rank = 0;
            for (int q = 0; q < band; ++q) {
                const unsigned long long k = __shfl_sync(0xffffffffu, own, q);
                rank += k > own || (k == own && q < lane);       // (the list ascends)
            }
            chosen = __ballot_sync(0xffffffffu, lane < band && rank < need);
            if (!left && mate == 0 && lane < band) s[mine] = rank < need ? -SEL_NONE : SEL_NONE;
            __syncwarp();
        }
        if (mate != 0) continue;                                 // (the first warp has what was decided in 64 bits)
        if (left) {
            const bool ia = va > above || ((ua >> lane & 1u) && (chosen >> (at_a & 31) & 1u));
            const bool ib = vb > above || ((ub >> lane & 1u) && (chosen >> (at_b & 31) & 1u));
            const unsigned ma = __ballot_sync(0xffffffffu, ia), mb = __ballot_sync(0xffffffffu, ib);
            if (ia) idx[first + __popc(ma & before)] = pa;
            if (ib) idx[first + __popc(ma) + __popc(mb & before)] = pb;
        } else {
            float cut = below;                                   // in if s >= cut
            if (band != need) {                                  // the next number above `above`
                cut = above == 0.f ? 1.4e-45f : __uint_as_float(__float_as_uint(above) + (above > 0.f ? 1u : -1u));
            }
            list([&](float x) { return x >= cut; }, [&](int at, int p) { idx[first + at] = p; });
        }
    }
    if (nb_all <= j.k) return;
    __syncthreads();

    // ---- rows that the approximate scores say too little about: 64 bits, by the whole block
    unsigned long long* key = reinterpret_cast<unsigned long long*>(smem);
    for (int h = 0; h < sh.n_hard; ++h) {
        const int t = sh.hard[h], nb = pages_of(t), row = row0 + t, take = j.k;
        int32_t* idx = j.blk_idx + ((int64_t)row * c.h_kv + head) * j.k;
        __syncthreads();
        for (int e = tid; e < c.d; e += SEL_THREADS) {
            double p = 0.0, m = 0.0;
            for (int g = 0; g < G; ++g) {
                const double x = (double)__bfloat162float(j.Q[(int64_t)row * j.ldq + ((int64_t)head * G + g) * c.d + e]);
                p += x > 0.0 ? x : 0.0;
                m += x > 0.0 ? 0.0 : x;
            }
            sh.qp[e] = p; sh.qm[e] = m;
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
                            s = fma(sh.qp[e + q], (double)__bfloat162float(pa[q]), fma(sh.qm[e + q], (double)__bfloat162float(pz[q]), s));
                    }
                }
                k = page >= 0 ? sort_key(s) : 0ull;
            }
            key[p] = k;
        }
        __syncthreads();
        auto count = [&](unsigned long long x) {
            int ge = 0;
            for (int p = tid; p < nb; p += SEL_THREADS) ge += key[p] >= x;
            ge = __reduce_add_sync(0xffffffffu, ge);
            __syncthreads();
            if (lane == 0) sh.cnt[0][warp] = ge;
            __syncthreads();
            int sum = 0;
#pragma unroll
            for (int w = 0; w < SEL_WARPS; ++w) sum += sh.cnt[0][w];
            return sum;
        };
        unsigned long long thr = 0ull;                           // the take-th largest key, bit by bit
        for (int bit = 63; bit >= 0; --bit) {
            const unsigned long long x = thr | 1ull << bit;
            if (count(x) >= take) thr = x;
        }
        int ties = take - (thr == ~0ull ? 0 : count(thr + 1ull));    // of the pages with that key, the lowest
        int out = 0;
        for (int p0 = 0; p0 < nb; p0 += SEL_THREADS) {
            const int p = p0 + tid;
            const unsigned long long k = p < nb ? key[p] : 0ull;
            const bool eq = p < nb && k == thr, gt = p < nb && k > thr;
            const unsigned me = __ballot_sync(0xffffffffu, eq);
            __syncthreads();
            if (lane == 0) sh.tie[warp] = __popc(me);
            __syncthreads();
            int before = __popc(me & ((1u << lane) - 1u)), all = 0;
#pragma unroll
            for (int w = 0; w < SEL_WARPS; ++w) { if (w < warp) before += sh.tie[w]; all += sh.tie[w]; }
            const bool in = gt || (eq && before < ties);
            ties -= min(ties, all);
            const unsigned mi = __ballot_sync(0xffffffffu, in);
            if (lane == 0) sh.cnt[0][warp] = __popc(mi);
            __syncthreads();
            int at = out + __popc(mi & ((1u << lane) - 1u));
#pragma unroll
            for (int w = 0; w < SEL_WARPS; ++w) { if (w < warp) at += sh.cnt[0][w]; out += sh.cnt[0][w]; }
            if (in) idx[at] = p;
        }
    }
}

}  // namespace

cudaError_t launch_cache_select(ada_ctx* ctx, const CacheView& c, const Ragged& r, const SelectJob& j, cudaStream_t s) {
    // scores of a tile: up to 64 KB, whole stages of pages
    const int stride = (c.max_pages + SEL_PAGES - 1) / SEL_PAGES * SEL_PAGES + 4, keys = c.max_pages * 8;
    int rows = SEL_ROWS;
    while (rows > 1 && (rows * stride * 4 > 65536 || rows / 2 * (int64_t)r.B >= r.N)) rows >>= 1;
    const int most = 226 * 1024 - (int)sizeof(SelShared);
    cudaError_t e;
    if (rows == 1) {
        const int scores = stride * 4 + SEL_WARPS * SEL_LEFT * 8;
        if ((e = allow_smem(ctx, 14, k_cache_select<true>, most)) != cudaSuccess) return e;
        prof_begin(ctx, K_CACHE_SELECT, s);
        e = launch_k(ctx, k_cache_select<true>, dim3(r.N, c.h_kv), dim3(SEL_THREADS), ((keys > scores ? keys : scores) + 15) / 16 * 16,
                     s, c, r, j, 1, stride, 0, ctx->status);
    } else {
        const int ring = SEL_RING * sel_half(c.d), room = ((keys > ring ? keys : ring) + 15) / 16 * 16;
        const int smem = room + 4 * SEL_ROWS * sel_row(c.d) + rows * stride * 4;
        if ((e = allow_smem(ctx, 15, k_cache_select<false>, most)) != cudaSuccess) return e;
        prof_begin(ctx, K_CACHE_SELECT, s);
        e = launch_k(ctx, k_cache_select<false>, dim3(r.N / rows + (r.B < r.N ? r.B : r.N), c.h_kv), dim3(SEL_THREADS), smem, s, c, r,
                     j, rows, stride, room, ctx->status);
    }
    prof_end(ctx, s);
    return e;
}

}  // namespace ada
