// Choice of pages (ada_select_blocks): for every new token and key head the k pages whose keys can matter most.
//
//   s(p) = sum_g sum_e max(q_ge kmax_pe, q_ge kmin_pe)  >=  sum_g q_g . key   for every key of page p
// g runs over the heads that share the key head.  max(q a, q b) with a >= b is q a for q > 0 and q b for q < 0, so with
// the sums of the positive and of the negative parts, P_e = sum_g max(q_ge, 0) and M_e = sum_g min(q_ge, 0),
//   s(p) = sum_e P_e kmax_pe + M_e kmin_pe:
// one dot product of 2 d_h elements, whatever the number of heads.
//
// The choice is that of scores in 64 bits, but few of them are ever formed.  A block scores 16 tokens of a sequence
// against all pages on mma.sync: P and M as two bf16 terms each, products exact, fp32 sums.  What that leaves out is
// bounded (E below), so a page whose approximate score is more than 2 E above (below) the k-th largest is
// certainly in (out); the few in between are scored again in 64 bits by the warp that has the row.  Rows with more such
// pages than lanes (equal scores, infinities) are done in 64 bits throughout, by the whole block.
//
// Bound: the bounds of all pages are read once per 16 tokens (from HBM for single tokens, else from L2).
#include "cache_tma.cuh"

namespace ada {

namespace {

constexpr int SEL_THREADS = 256;
constexpr int SEL_WARPS = SEL_THREADS / 32;
constexpr int SEL_PAGES = 64;            // pages per stage: eight for every warp
constexpr int SEL_ROWS = 16;             // tokens of a tile
constexpr int SEL_KEYS = 16;             // scores of a row that a lane keeps in registers
// |approximate - s(p)| <= (SEL_ERR + (G - 1) 2^-24) sum_e (P_e + |M_e|) a_e, a_e the largest |bound| of element e in any
// page: two bf16 terms leave 2^-16 of P, its fp32 sum over G heads (G - 1) 2^-24; d_h / 16 <= 8 matrix instructions for
// either sign add 16 products and the running sum, each of the 17 addends cut at 2^-24 of the largest.  In all 2.4e-5; the
// sums of either sign and of the second terms, a few roundings more, are in the reserve.
constexpr float SEL_ERR = 2.7e-5f;

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
    unsigned col[128];                             // largest |bound| of every element (bits)
    int n_hard, hard[SEL_ROWS];
    int cnt[2][SEL_WARPS], tie[SEL_WARPS];
    unsigned word[2][SEL_WARPS];
    int list[SEL_WARPS][32];
    unsigned long long key[SEL_WARPS][32];
};

// bytes of a row of d elements in shared memory: an odd number of 16-byte pieces, so that ldmatrix has no bank conflict
__host__ __device__ __forceinline__ int sel_row(int d) { return d * 2 + 16; }
__host__ __device__ __forceinline__ int sel_stage(int d) { return 2 * SEL_PAGES * sel_row(d); }

// grid (tiles of `rows` tokens of one sequence, key heads).  Shared memory: two stages of bounds | the tile's P and M as
// bf16 terms | scores [rows][stride]; a row done in 64 bits throughout has its keys in the stages' place.
__global__ void __launch_bounds__(SEL_THREADS)
k_cache_select(const CacheView c, const Ragged r, const SelectJob j, int rows, int stride, int stage_room,
               unsigned* __restrict__ status) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ SelShared sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int head = blockIdx.y, G = j.h / c.h_kv;
    const int rb = sel_row(c.d);
    unsigned char* a_tile = smem + stage_room;                  // [P hi, P lo, M hi, M lo][16][rb]
    float* score = reinterpret_cast<float*>(a_tile + 4 * SEL_ROWS * rb);
    grid_dep_wait();
    grid_dep_launch_next();
    if (blockIdx.x == 0 && head == 0) check_ragged(r, c, status, tid, SEL_THREADS);

    // ---- the tile: the sequence and its first token, by every warp for itself
    int b = -1, t0 = 0;
    {
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
    if (nb_all > j.k) {
        // ---- loads of the bounds: a warp's lanes hold one page at a time, 16 bytes each
        const int nvec = c.d >> 3, nst = (nb_all + SEL_PAGES - 1) / SEL_PAGES;
        int id = -1;                                            // lane q: the table's entry for page w + 8 q of the next stage
        auto fetch_ids = [&](int st) {
            const int p = st * SEL_PAGES + warp + 8 * lane;
            id = lane < 8 && p < nb_all ? page_of(c, b, p, status) : -1;
        };
        const int v = lane & 15, lower = lane >> 4;             // lanes 0..15 the maxima, 16..31 the minima
        const __nv_bfloat16* bounds = (lower ? c.kmin : c.kmax) + (int64_t)head * c.d + v * 8;
        auto load_stage = [&](int st) {
            const unsigned at = tc::smem_u32(smem + (st & 1) * sel_stage(c.d)) + (lower * SEL_PAGES) * rb + v * 16;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int page = __shfl_sync(0xffffffffu, id, q);
                if (v < nvec) cp16(at + (warp + 8 * q) * rb, bounds + (int64_t)max(page, 0) * c.h_kv * c.d, page >= 0);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        if (tid == 0) sh.n_hard = 0;
        if (tid < 128) sh.col[tid] = 0u;
        __syncthreads();
        fetch_ids(0);
        load_stage(0);
        if (nst > 1) fetch_ids(1);
        // ---- P and M of the tile's tokens, two elements a thread
        for (int i = tid; i < SEL_ROWS * (c.d >> 1); i += SEL_THREADS) {
            const int t = i / (c.d >> 1), e = (i - t * (c.d >> 1)) * 2;
            float p[2] = {0.f, 0.f}, m[2] = {0.f, 0.f};
            if (t < n_tok) {
                const __nv_bfloat16* q = j.Q + (int64_t)(row0 + t) * j.ldq + (int64_t)head * G * c.d + e;
                for (int g = 0; g < G; ++g) {
                    const unsigned w = *reinterpret_cast<const unsigned*>(q + (int64_t)g * c.d);
                    const float x[2] = {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
#pragma unroll
                    for (int u = 0; u < 2; ++u) { p[u] += fmaxf(x[u], 0.f); m[u] += fminf(x[u], 0.f); if (x[u] != x[u]) p[u] = x[u]; }
                }
            }
            const __nv_bfloat162 ph = __floats2bfloat162_rn(p[0], p[1]), mh = __floats2bfloat162_rn(m[0], m[1]);
            const __nv_bfloat162 pl = __floats2bfloat162_rn(p[0] - __low2float(ph), p[1] - __high2float(ph));
            const __nv_bfloat162 ml = __floats2bfloat162_rn(m[0] - __low2float(mh), m[1] - __high2float(mh));
            unsigned char* d = a_tile + t * rb + e * 2;
            *reinterpret_cast<__nv_bfloat162*>(d) = ph;
            *reinterpret_cast<__nv_bfloat162*>(d + SEL_ROWS * rb) = pl;
            *reinterpret_cast<__nv_bfloat162*>(d + 2 * SEL_ROWS * rb) = mh;
            *reinterpret_cast<__nv_bfloat162*>(d + 3 * SEL_ROWS * rb) = ml;
        }
        // ---- scores
        const unsigned a_at = tc::smem_u32(a_tile) + (lane & 15) * rb + (lane >> 4) * 16;
        __nv_bfloat162 most[4];                                  // of the elements that this lane fetches (NaN stays)
#pragma unroll
        for (int u = 0; u < 4; ++u) most[u] = __float2bfloat162_rn(0.f);
        for (int st = 0; st < nst; ++st) {
            if (st + 1 < nst) {
                load_stage(st + 1);
                if (st + 2 < nst) fetch_ids(st + 2);
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            } else {
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            }
            __syncthreads();
            const unsigned char* stage = smem + (st & 1) * sel_stage(c.d);
            if (v < nvec) {
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const uint4 x = *reinterpret_cast<const uint4*>(stage + (lower * SEL_PAGES + warp + 8 * q) * rb + v * 16);
                    const __nv_bfloat162* y = reinterpret_cast<const __nv_bfloat162*>(&x);
#pragma unroll
                    for (int u = 0; u < 4; ++u) most[u] = __hmax2_nan(most[u], __habs2(y[u]));
                }
            }
            float acc[4][4];                                     // second and first terms of P, of M
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[u][i] = 0.f;
            const unsigned b_at = tc::smem_u32(stage) + (warp * 8 + (lane & 7)) * rb + ((lane >> 3) & 1) * 16;
            for (int ks = 0; ks < c.d >> 4; ++ks)
#pragma unroll
                for (int sign = 0; sign < 2; ++sign) {
                    unsigned bf[2], hi[4], lo[4];
                    ldsm2(b_at + sign * SEL_PAGES * rb + ks * 32, bf);
                    tc::ldsm4(a_at + 2 * sign * SEL_ROWS * rb + ks * 32, hi);
                    tc::ldsm4(a_at + (2 * sign + 1) * SEL_ROWS * rb + ks * 32, lo);
                    tc::mma16816(acc[2 * sign], lo, bf[0], bf[1]);
                    tc::mma16816(acc[2 * sign + 1], hi, bf[0], bf[1]);
                }
            const int p = st * SEL_PAGES + warp * 8 + 2 * (lane & 3);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = (lane >> 2) + 8 * i;
                float x[2];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    x[e] = (acc[1][2 * i + e] + acc[3][2 * i + e]) + (acc[0][2 * i + e] + acc[2][2 * i + e]);
                if (t < n_tok) *reinterpret_cast<float2*>(score + t * stride + p) = make_float2(x[0], x[1]);
            }
            __syncthreads();
        }
        if (v < nvec) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {                        // (a NaN's bits are larger than any number's)
                atomicMax(&sh.col[v * 8 + 2 * u], __float_as_uint(__low2float(most[u])) & 0x7fffffffu);
                atomicMax(&sh.col[v * 8 + 2 * u + 1], __float_as_uint(__high2float(most[u])) & 0x7fffffffu);
            }
        }
        __syncthreads();
    }

    // ---- teams of `tw` warps, a row each: the k-th largest approximate score, and what cannot be told from it
    const int tw = rows >= SEL_WARPS ? 1 : SEL_WARPS / rows, team = warp / tw, mate = warp - team * tw;
    const int step = 32 * tw, at0 = mate * 32 + lane;
    int turn = 0;
    auto meet = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(step) : "memory"); };
    // sum (least, greatest) over the team; the slots alternate, so that one meeting per call is enough
    auto sum_of = [&](int x) {
        x = __reduce_add_sync(0xffffffffu, x);
        if (tw == 1) return x;
        turn ^= 1;
        if (lane == 0) sh.cnt[turn][warp] = x;
        meet();
        x = 0;
        for (int q = 0; q < tw; ++q) x += sh.cnt[turn][team * tw + q];
        return x;
    };
    auto most_of = [&](unsigned x) {
        x = __reduce_max_sync(0xffffffffu, x);
        if (tw == 1) return x;
        turn ^= 1;
        if (lane == 0) sh.word[turn][warp] = x;
        meet();
        x = 0u;
        for (int q = 0; q < tw; ++q) x = max(x, sh.word[turn][team * tw + q]);
        return x;
    };
    for (int t = team; t < n_tok; t += SEL_WARPS / tw) {
        const int nb = pages_of(t), row = row0 + t, take = min(nb, j.k);
        int32_t* idx = j.blk_idx + ((int64_t)row * c.h_kv + head) * j.k;
        if (mate == 0 && lane == 0) j.blk_cnt[(int64_t)row * c.h_kv + head] = take;
        if (nb <= j.k) {
            for (int i = at0; i < j.k; i += step) idx[i] = i < nb ? i : -1;
            continue;
        }
        float* s = score + t * stride;
        const int first = j.n_first, last = nb - j.n_last;       // pages [first, last) compete for `need` places
        int need = j.k - j.n_first - j.n_last;
        float above = INFINITY, below = INFINITY;                // undecided if below <= s <= above
        bool all_of_them = false;                                // the undecided ones are in
        if (need > 0) {
            float A = 0.f;
            const unsigned char* ar = a_tile + t * rb;
            for (int e = lane; e < c.d; e += 32)
                A += (__bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(ar + e * 2)) -
                      __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(ar + 2 * SEL_ROWS * rb + e * 2))) * __uint_as_float(sh.col[e]);
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) A += __shfl_xor_sync(0xffffffffu, A, m);
            const float E = (SEL_ERR + (float)G * 6e-8f) * A * 1.004f + 1e-35f;   // (first terms are up to 2^-8 short)
            // keys, larger than 0, of the lane's first pages; 0: none
            const bool held = last - first <= SEL_KEYS * step;
            unsigned key[SEL_KEYS];
            bool odd = !(E <= 1e37f);
            unsigned lo = ~0u, hi = 0u;
#pragma unroll
            for (int q = 0; q < SEL_KEYS; ++q) {
                const int p = first + at0 + q * step;
                key[q] = 0u;
                if (p < last) {
                    const float x = s[p];
                    odd = odd || !(fabsf(x) <= 1e37f);
                    key[q] = sort_key(x);
                    lo = min(lo, key[q]); hi = max(hi, key[q]);
                }
            }
            for (int p = first + at0 + SEL_KEYS * step; p < last; p += step) {
                const float x = s[p];
                odd = odd || !(fabsf(x) <= 1e37f);
                lo = min(lo, sort_key(x)); hi = max(hi, sort_key(x));
            }
            hi = most_of(odd ? ~0u : hi);
            if (hi == ~0u) {                                     // (no finite score has that key)
                if (mate == 0 && lane == 0) sh.hard[atomicAdd(&sh.n_hard, 1)] = t;
                continue;
            }
            lo = ~most_of(~lo);
            // at least `need` keys are >= lo, fewer than that > hi
            while (lo < hi) {
                const unsigned mid = lo + ((hi - lo + 1u) >> 1);
                int ge = 0;
#pragma unroll
                for (int q = 0; q < SEL_KEYS; ++q) ge += key[q] >= mid;
                if (!held) for (int p = first + at0 + SEL_KEYS * step; p < last; p += step) ge += sort_key(s[p]) >= mid;
                ge = sum_of(ge);
                if (ge >= need) lo = mid; else hi = mid - 1u;
                if (ge == need) {                                // the smallest of them is the one that is sought
                    unsigned least = ~0u;
#pragma unroll
                    for (int q = 0; q < SEL_KEYS; ++q) if (key[q] >= mid) least = min(least, key[q]);
                    if (!held) for (int p = first + at0 + SEL_KEYS * step; p < last; p += step) { const unsigned k = sort_key(s[p]); if (k >= mid) least = min(least, k); }
                    lo = ~most_of(~least);
                    break;
                }
            }
            const float kth = key_value(lo);
            above = __fadd_ru(kth, __fmul_ru(2.0f, E));
            below = __fadd_rd(kth, -__fmul_ru(2.0f, E));
            int in = 0;                                          // certain ones, and 65536 for every undecided one
            for (int p = first + at0; p < last; p += step) { const float x = s[p]; in += x > above ? 1 : x >= below ? 65536 : 0; }
            in = sum_of(in);
            const int band = in >> 16;
            need -= in & 0xffff;
            if (band == need) {
                all_of_them = true;
            } else if (band <= 32) {
                // every warp of the team lists them; each scores its share of them in 64 bits
                int at = 0;
                for (int p0 = first; p0 < last; p0 += 32) {
                    const int p = p0 + lane;
                    const bool is = p < last && s[p] >= below && s[p] <= above;
                    const unsigned m = __ballot_sync(0xffffffffu, is);
                    if (is) sh.list[warp][at + __popc(m & ((1u << lane) - 1u))] = p;
                    at += __popc(m);
                }
                __syncwarp();
                const int mine = lane < band ? sh.list[warp][lane] : INT_MAX;
                const int page_l = lane < band ? page_of(c, b, mine, status) : -1;
                double P[4], M[4];                               // of elements 4 lane .. 4 lane + 3
                const bool on = lane * 4 < c.d;
#pragma unroll
                for (int e = 0; e < 4; ++e) P[e] = M[e] = 0.0;
                const __nv_bfloat16* qrow = j.Q + (int64_t)row * j.ldq + (int64_t)head * G * c.d + lane * 4;
                for (int g = 0; g < G && on; ++g) {
                    const uint2 w = *reinterpret_cast<const uint2*>(qrow + (int64_t)g * c.d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned u = e < 2 ? w.x : w.y;
                        const double x = (double)__uint_as_float((e & 1) ? u & 0xffff0000u : u << 16);
                        P[e] += x > 0.0 ? x : 0.0;
                        M[e] += x > 0.0 ? 0.0 : x;
                    }
                }
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
                    if (lane == 0) sh.key[team * tw][q] = page < 0 ? 0ull : sort_key(x);
                }
                __syncwarp();
                if (tw > 1) meet();
                if (mate == 0) {
                    const unsigned long long own = lane < band ? sh.key[team * tw][lane] : 0ull;
                    int rank = 0;
                    for (int q = 0; q < band; ++q) {
                        const unsigned long long k = __shfl_sync(0xffffffffu, own, q);
                        rank += k > own || (k == own && q < lane);   // (the list ascends)
                    }
                    if (lane < band) s[mine] = rank < need ? INFINITY : -INFINITY;
                }
                __syncwarp();
            } else {
                if (mate == 0 && lane == 0) sh.hard[atomicAdd(&sh.n_hard, 1)] = t;
                continue;
            }
        }
        if (mate == 0) {                                         // (the first warp has what was decided in 64 bits)
            int at = 0;
            for (int p0 = 0; p0 < nb; p0 += 32) {
                const int p = p0 + lane;
                const bool in = p < nb && (p < first || p >= last || (all_of_them ? s[p] >= below : s[p] > above));
                const unsigned m = __ballot_sync(0xffffffffu, in);
                if (in) idx[at + __popc(m & ((1u << lane) - 1u))] = p;
                at += __popc(m);
            }
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
    const int stride = (c.max_pages + SEL_PAGES - 1) / SEL_PAGES * SEL_PAGES + 4;
    int rows = SEL_ROWS;
    while (rows > 1 && (rows * stride * 4 > 65536 || rows / 2 * (int64_t)r.B >= r.N)) rows >>= 1;
    const int keys = c.max_pages * 8, stages = 2 * sel_stage(c.d);
    const int room = ((keys > stages ? keys : stages) + 15) / 16 * 16;
    const int smem = room + 4 * SEL_ROWS * sel_row(c.d) + rows * stride * 4;
    cudaError_t e = allow_smem(ctx, 14, k_cache_select, 226 * 1024 - (int)sizeof(SelShared));
    if (e != cudaSuccess) return e;
    return launch_k(ctx, k_cache_select, dim3(r.N / rows + (rows > 1 ? (r.B < r.N ? r.B : r.N) : 0), c.h_kv), dim3(SEL_THREADS), smem, s, c, r, j, rows,
                    stride, room, ctx->status);
}

}  // namespace ada
