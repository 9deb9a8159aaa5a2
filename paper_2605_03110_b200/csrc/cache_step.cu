// Attention of single tokens over the paged cache (ada_attention_cached with few rows per key head), and of any tokens
// over the pages that their lists name (ada_attention_blocks).
//
//   out = sum_s 2^(sc q.k_s - m) v_s / sum_s 2^(sc q.k_s - m),   sc = scale log2(e), m the running maximum
// in one pass over the keys.  The heads that share a key head (and, dense, the few new tokens of a sequence) are the
// up to 16 rows of one tile, so that K and V are read once for all of them.  What bounds it is the stream of keys and
// values: from HBM in a decoding step, from L2 where a chunk's tokens list the same pages.  A 128-row tcgen05 tile would be
// empty but for these rows; mma.sync takes 16 rows and leaves its operands in registers, so that nothing but the
// keys and values passes through shared memory.
//
// A warp works alone: 32 keys at a time arrive by TMA in a ring of its own, scores, softmax and products stay in
// its registers, and it shares nothing until the end of a row.  Four warps of a CTA deal a row's granules of 32 keys
// among them (TEAM = 4) or take rows of their own (TEAM = 1, many rows with lists: no barrier at all).
//
// Dense work is cut into units of 128 keys of one (sequence, key head); every CTA takes an equal run of units
// whatever the lengths are, and a row tile that several CTAs share is joined by the one that finishes last (in
// the order of the keys, so that results do not depend on who that is).  Nobody waits for another CTA.
#include "cache_tma.cuh"

namespace ada {

using namespace tc;

namespace {

constexpr int ST_WARPS = 4;
constexpr int ST_THREADS = 32 * ST_WARPS;
constexpr int GK = 32;                     // keys per granule
constexpr int GPU_ = 4;                    // granules per unit of dense work
constexpr int NOWHERE = 0x7fff0000;        // position of keys that are not there: behind every limit
constexpr int SLOT_FLOATS = 16 * 128 + 32; // one partial result: 16 rows x 128, maxima, sums

template <int NDB> __host__ __device__ constexpr int st_stages() { return 6 / NDB; }
template <int NDB> __host__ __device__ constexpr int st_stage_bytes() { return 2 * NDB * GK * 128; }
template <int NDB> __host__ __device__ constexpr int st_ring_bytes() { return ST_WARPS * st_stages<NDB>() * st_stage_bytes<NDB>(); }

struct StepShared {
    unsigned long long full[ST_WARPS][6];
    int2 base[ST_WARPS][6];                // positions of the two halves of a stage
    float m[ST_WARPS][16], l[ST_WARPS][16];
    int abort_flag[2];
    int last;
};
template <int NDB> __host__ __device__ constexpr int st_smem() {
    return st_ring_bytes<NDB>() + ST_WARPS * 16 * NDB * 64 * 4 + (int)sizeof(StepShared);
}
static_assert(st_smem<2>() <= 227 * 1024 && st_smem<1>() <= 227 * 1024, "shared memory budget");

struct StepMaps {
    CUtensorMap k, v;
};

// One row tile's run of keys, as a CTA (TEAM = 4) or a warp (TEAM = 1) works on it.
struct Seg {
    int b, head, row, g0;                  // sequence, key head, first token's row, first of the group's heads
    int rows, n, len;                      // rows of the tile; the sequence's new tokens and its length
    int cnt;                               // list entries (LIST)
    int g_begin, g_end;                    // granules
    int pieces, piece, slot0;              // of how many, which, where the first one's partial result is
    int ctr;
};

template <bool LIST>
struct Work {                              // where a team is in its run of work; the same in all of its lanes
    // dense: units; lists: items
    int64_t at, end;
    // dense
    int b, head, ku, nu, n, off, len;
    int64_t per;

    __device__ __forceinline__ void load_seq(const Ragged& r, const CacheView& c) {
        n = seq_rows(r, b, off);
        len = seq_len(r, c, b);
        nu = n > 0 ? max(1, (len + GK * GPU_ - 1) / (GK * GPU_)) : 0;
    }
    // the next segment, or false
    __device__ __forceinline__ bool next(Seg& s, const Ragged& r, const CacheView& c, const AttendJob& j, int G, int tiles,
                                         int pieces, unsigned* status) {
        if (LIST) {
            while (at < end) {
                const int64_t item = at++;
                const int piece = (int)(item % pieces);
                const int64_t rest = item / pieces;
                const int rt = (int)(rest % tiles);
                const int64_t rh = rest / tiles;
                const int row = (int)(rh / c.h_kv), head = (int)(rh % c.h_kv);
                if (row != off || b < 0) { b = seq_of_row(r, row); off = row; }
                if (b < 0) { b = -1; off = -1; continue; }
                int o;
                s.b = b; s.head = head; s.row = row; s.g0 = rt * 16;
                s.rows = min(16, G - rt * 16);
                s.n = seq_rows(r, b, o);
                s.len = seq_len(r, c, b);
                // the row's own limit, as if it were the only new token
                s.len = j.causal ? max(s.len - s.n + (row - o) + 1, 0) : s.len;
                s.n = 1;
                int cnt = j.blk_cnt[rh];
                if (cnt < 0 || cnt > j.k) { atomicOr(status, ST_BAD_COUNT); cnt = min(max(cnt, 0), j.k); }
                s.cnt = cnt;
                const int g = (int)((((int64_t)cnt << c.shift) + GK - 1) / GK);
                s.g_begin = (int)((int64_t)g * piece / pieces);
                s.g_end = (int)((int64_t)g * (piece + 1) / pieces);
                s.pieces = pieces; s.piece = piece;
                s.slot0 = (int)(rest * pieces);
                s.ctr = (int)rest;
                return true;
            }
            return false;
        }
        if (at >= end) return false;
        while (ku >= nu) {                                  // this (sequence, head) is done: the next one with work
            ku = 0;
            if (++head >= c.h_kv || nu == 0) {
                head = 0;
                if (++b >= r.B) { at = end; return false; }
                load_seq(r, c);
            }
        }
        const int take = (int)min((int64_t)(nu - ku), end - at);
        s.b = b; s.head = head; s.row = off; s.g0 = 0;
        s.n = n; s.len = len; s.cnt = 0;
        s.rows = min(n, j.max_new) * G;
        const int g = (len + GK - 1) / GK;
        s.g_begin = ku * GPU_;
        s.g_end = min((ku + take) * GPU_, g);
        const int64_t first = at - ku;                      // the row tile's units are [first, first + nu)
        const int c0 = (int)(first / per), c1 = (int)((first + nu - 1) / per);
        s.pieces = c1 - c0 + 1;
        s.piece = (int)(at / per) - c0;
        s.slot0 = c0;
        s.ctr = c1;
        at += take; ku += take;
        return true;
    }
};

// where partial result `piece` of a segment lies: dense, CTA c0 + piece has one place for a row tile that began in an
// earlier CTA (2 c) and one for a tile that it begins itself (2 c + 1)
template <bool LIST>
__device__ __forceinline__ float* partial(float* ws, const Seg& s, int piece) {
    const int64_t slot = LIST ? (int64_t)s.slot0 + piece : 2 * ((int64_t)s.slot0 + piece) + (piece == 0 ? 1 : 0);
    return ws + slot * SLOT_FLOATS;
}

template <int NDB, bool LIST, int TEAM>
__global__ void __launch_bounds__(ST_THREADS, 1)
k_cache_step(const __grid_constant__ StepMaps maps, const CacheView c, const Ragged r, const AttendJob j, int tiles,
             int pieces, float* __restrict__ ws, unsigned* __restrict__ counters, unsigned* __restrict__ status) {
    constexpr int NST = st_stages<NDB>();
    constexpr int KS = NDB * 4;                       // 16-element steps of a head row
    constexpr int HALF_TILE = GK * 128;               // one 64-element block of 32 keys: 4 KiB
    extern __shared__ __align__(1024) unsigned char smem[];
    float* mrg = reinterpret_cast<float*>(smem + st_ring_bytes<NDB>());            // [4][16][NDB * 64]
    StepShared& sh = *reinterpret_cast<StepShared*>(smem + st_ring_bytes<NDB>() + ST_WARPS * 16 * NDB * 64 * 4);
    volatile int* abort_flag = sh.abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = j.h / c.h_kv;
    unsigned char* ring = smem + warp * NST * st_stage_bytes<NDB>();
    if ((smem_u32(smem) & 1023u) != 0u) {             // the tiles would not be where the swizzle assumes
        grid_dep_wait();
        if (tid == 0) { atomicOr(status, ST_TIMEOUT); status[2] = 399u; }
        return;
    }
    if (tid == 0) {
        sh.abort_flag[0] = 0;
        sh.abort_flag[1] = wait_limit_units(false);
    }
    if (lane == 0) {
        for (int i = 0; i < NST; ++i) mbar_init(&sh.full[warp][i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (tid == 64) { prefetch_map(&maps.k); prefetch_map(&maps.v); }
    __syncthreads();
    grid_dep_wait();
    grid_dep_launch_next();
    if (blockIdx.x == 0) check_ragged(r, c, status, tid, ST_THREADS);

    // ---------------------------------------------------------------- this team's run of work
    const int w = TEAM == 1 ? 0 : warp;
    Work<LIST> work;
    if (LIST) {
        const int64_t items = (int64_t)r.N * c.h_kv * tiles * pieces;
        const int64_t teams = (int64_t)gridDim.x * (ST_WARPS / TEAM);
        const int64_t team = (int64_t)blockIdx.x * (ST_WARPS / TEAM) + (TEAM == 1 ? warp : 0);
        const int64_t per = (items + teams - 1) / teams;
        work.at = min(team * per, items);
        work.end = min(work.at + per, items);
        work.b = -1; work.off = -1;
        work.head = work.ku = work.nu = work.n = work.len = 0; work.per = 1;
    } else {
        // prefix sums of the sequences' units, 32 at a time, by every warp for itself
        auto units_of = [&](int b) {
            if (b >= r.B) return 0;
            int o;
            const int n = seq_rows(r, b, o);
            if (blockIdx.x == 0 && n > j.max_new) atomicOr(status, ST_BAD_COUNT);
            return n > 0 ? max(1, (seq_len(r, c, b) + GK * GPU_ - 1) / (GK * GPU_)) : 0;
        };
        int64_t U = 0;
        for (int b0 = 0; b0 < r.B; b0 += 32) U += __reduce_add_sync(0xffffffffu, units_of(b0 + lane));
        U *= c.h_kv;
        work.per = max((U + gridDim.x - 1) / gridDim.x, (int64_t)1);
        work.at = min(work.per * blockIdx.x, U);
        work.end = min(work.at + work.per, U);
        work.b = 0; work.head = 0; work.ku = 0; work.nu = 0; work.n = 0; work.off = 0; work.len = 0;
        int64_t before = 0;
        if (work.at < work.end)
            for (int b0 = 0; b0 < r.B; b0 += 32) {
                int sum = units_of(b0 + lane);
                const int own = sum;
#pragma unroll
                for (int m = 1; m < 32; m <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, sum, m);
                    if (lane >= m) sum += y;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, work.at < (before + sum) * c.h_kv);
                if (hit != 0u) {
                    const int l = __ffs(hit) - 1;
                    before += __shfl_sync(0xffffffffu, sum - own, l);
                    work.b = b0 + l;
                    work.load_seq(r, c);
                    const int64_t rest = work.at - before * c.h_kv;
                    work.head = (int)(rest / work.nu);
                    work.ku = (int)(rest % work.nu);
                    break;
                }
                before += __shfl_sync(0xffffffffu, sum, 31);
            }
    }

    // ---------------------------------------------------------------- producer side
    Work<LIST> pwork = work;
    Seg ps;
    ps.g_begin = ps.g_end = 0;
    bool more = pwork.next(ps, r, c, j, G, tiles, pieces, status);
    int pg = ps.g_begin + w;                          // the next granule to fetch
    int batch = -1;                                   // granule of lane 0's page, -1: none fetched for this segment
    int2 pid = make_int2(-1, -1), pbase = make_int2(NOWHERE, NOWHERE);
    unsigned made = 0;
    // fetches the next granule of this warp into the ring, if there is one
    auto produce = [&]() {
        while (more && pg >= ps.g_end) {
            more = pwork.next(ps, r, c, j, G, tiles, pieces, status);
            pg = ps.g_begin + w;
            batch = -1;
        }
        if (!more) return;
        if (batch < 0 || pg >= batch + 32 * TEAM) {
            // lane l: pages of this warp's l-th granule from here on
            batch = pg;
            const int g = pg + lane * TEAM;
            int id[2] = {-1, -1}, base[2] = {NOWHERE, NOWHERE};
            if (g < ps.g_end) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int vk = g * GK + q * 16, e = vk >> c.shift, slot = vk & ((1 << c.shift) - 1);
                    if (q == 1 && c.shift > 4) {
                        id[1] = id[0];
                        base[1] = id[0] >= 0 ? base[0] + 16 : NOWHERE;
                        break;
                    }
                    int p = e;                        // dense: the sequence's e-th page
                    bool ok = true;
                    if (LIST) {
                        ok = e < ps.cnt;
                        if (ok) {
                            const int32_t* list = j.blk_idx + ((int64_t)ps.row * c.h_kv + ps.head) * j.k;
                            p = list[e];
                            // an entry that does not ascend, or names a page that the table has no place for
                            if (p < 0 || p >= c.max_pages || (e > 0 && list[e - 1] >= p)) {
                                atomicOr(status, ST_BAD_INDEX);
                                ok = false;
                            }
                        }
                    }
                    if (ok && (p << c.shift) < ps.len) {     // (pages behind the limit are not looked at)
                        id[q] = page_of(c, ps.b, p, status);
                        if (id[q] >= 0) base[q] = (p << c.shift) + slot;
                    }
                }
            }
            pid = make_int2(id[0], id[1]);
            pbase = make_int2(base[0], base[1]);
        }
        const int l = (pg - batch) / TEAM;
        const int id0 = __shfl_sync(0xffffffffu, pid.x, l), id1 = __shfl_sync(0xffffffffu, pid.y, l);
        const int b0 = __shfl_sync(0xffffffffu, pbase.x, l), b1 = __shfl_sync(0xffffffffu, pbase.y, l);
        if (lane == 0) {
            const int st = made % NST;
            unsigned char* dst = ring + st * st_stage_bytes<NDB>();
            unsigned long long* bar = &sh.full[warp][st];
            sh.base[warp][st] = make_int2(b0, b1);
            if (c.shift > 4) {
                const int slot = (pg * GK) & ((1 << c.shift) - 1);
                mbar_expect_tx(bar, id0 >= 0 ? (unsigned)st_stage_bytes<NDB>() : 0u);
                if (id0 >= 0)
#pragma unroll
                    for (int db = 0; db < NDB; ++db) {
                        tma_load_4d(&maps.k, bar, dst + db * HALF_TILE, db * BK, slot, ps.head, id0);
                        tma_load_4d(&maps.v, bar, dst + (NDB + db) * HALF_TILE, db * BK, slot, ps.head, id0);
                    }
            } else {
                mbar_expect_tx(bar, (unsigned)st_stage_bytes<NDB>() / 2 * ((id0 >= 0) + (id1 >= 0)));
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int id = q == 0 ? id0 : id1;
                    if (id >= 0)
#pragma unroll
                        for (int db = 0; db < NDB; ++db) {
                            tma_load_4d(&maps.k, bar, dst + db * HALF_TILE + q * 2048, db * BK, 0, ps.head, id);
                            tma_load_4d(&maps.v, bar, dst + (NDB + db) * HALF_TILE + q * 2048, db * BK, 0, ps.head, id);
                        }
                }
            }
        }
        ++made;
        pg += TEAM;
    };
#pragma unroll 1
    for (int i = 0; i < NST; ++i) produce();

    // ---------------------------------------------------------------- consumer side
    const int r0 = lane >> 2, c0 = 2 * (lane & 3);
    const unsigned ring_u = smem_u32(ring);
    unsigned used = 0;
    bool ok = true;
    Seg s;
    while (work.next(s, r, c, j, G, tiles, pieces, status)) {
        // A operand: rows r0 and r0 + 8 of the tile (row = token * G + head of the group)
        unsigned qf[KS][4];
        int lim[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = r0 + 8 * i;
            const bool live = row < s.rows;
            const int t = LIST || !live ? 0 : row / G, g = s.g0 + (LIST ? row : row - t * G);
            lim[i] = !live ? 0 : LIST ? s.len : j.causal ? s.len - s.n + t + 1 : s.len;
            const __nv_bfloat16* q = j.Q + (int64_t)(s.row + t) * j.ldq + ((int64_t)s.head * G + g) * c.d;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                qf[k][i] = live && k * 16 < c.d ? *reinterpret_cast<const unsigned*>(q + k * 16 + c0) : 0u;
                qf[k][2 + i] = live && k * 16 < c.d ? *reinterpret_cast<const unsigned*>(q + k * 16 + 8 + c0) : 0u;
            }
        }
        // keys from here on are masked for some row: the first token's limit
        const int lim_all = LIST || !j.causal ? s.len : s.len - s.n + 1;
        float o[NDB * 8][4];
#pragma unroll
        for (int n = 0; n < NDB * 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

        for (int g = s.g_begin + w; g < s.g_end; g += TEAM) {
            const int st = used % NST;
            if (ok) ok = mbar_wait(&sh.full[warp][st], (used / NST) & 1u, abort_flag, 50);
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
                const unsigned kt = ring_u + st * st_stage_bytes<NDB>(), vt = kt + NDB * HALF_TILE;
                const int2 base = sh.base[warp][st];
                // ---- scores: 16 rows x 32 keys
                float sc[4][4];
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int np = 0; np < 2; ++np) {
                        const int key = np * 16 + ((lane >> 4) << 3) + (lane & 7), ch = (k & 3) * 2 + ((lane >> 3) & 1);
                        unsigned bf[4];
                        ldsm4(kt + (k >> 2) * HALF_TILE + key * 128 + ((ch ^ (key & 7)) << 4), bf);
                        mma16816(sc[2 * np], qf[k], bf[0], bf[1]);
                        mma16816(sc[2 * np + 1], qf[k], bf[2], bf[3]);
                    }
                // ---- mask; values of slots that hold nothing of this sequence must not meet a zero probability as NaN
                if (base.x + 15 >= lim_all || base.y + 15 >= lim_all) {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int pos = (n < 2 ? base.x : base.y) + (n & 1) * 8 + c0 + (e & 1);
                            if (pos >= lim[e >> 1]) sc[n][e] = -INFINITY;
                        }
                    if (base.x + 15 >= s.len || base.y + 15 >= s.len) {
                        unsigned char* v = ring + st * st_stage_bytes<NDB>() + NDB * HALF_TILE;
                        for (int q = lane; q < GK * NDB * 8; q += 32) {
                            const int key = (q >> 3) & 31, db = q >> 8;
                            if ((key < 16 ? base.x + key : base.y + key - 16) >= s.len)
                                *reinterpret_cast<uint4*>(v + db * HALF_TILE + key * 128 + (q & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the slot's next load comes through the async proxy)
                        __syncwarp();
                    }
                }
                // ---- running maximum and sum
                float mr[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float x = -INFINITY;
#pragma unroll
                    for (int n = 0; n < 4; ++n) x = fmaxf(x, fmaxf(sc[n][2 * i], sc[n][2 * i + 1]));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                    mr[i] = fmaxf(m[i], x * j.scale);
                }
                if (__any_sync(0xffffffffu, mr[0] > m[0] || mr[1] > m[1])) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float f = m[i] > -INFINITY ? ex2_approx(m[i] - mr[i]) : 0.f;
                        m[i] = mr[i];
                        l[i] *= f;
#pragma unroll
                        for (int n = 0; n < NDB * 8; ++n) { o[n][2 * i] *= f; o[n][2 * i + 1] *= f; }
                    }
                }
                const float ref[2] = {m[0] > -INFINITY ? m[0] : 0.f, m[1] > -INFINITY ? m[1] : 0.f};
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sc[n][e] = ex2_approx(fmaf(sc[n][e], j.scale, -ref[e >> 1]));
                        l[e >> 1] += sc[n][e];
                    }
                // ---- products with the values; the probabilities are rounded to bf16 here, their sum is not
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    unsigned a[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const __nv_bfloat162 p = __floats2bfloat162_rn(sc[2 * ks + (q >> 1)][2 * (q & 1)], sc[2 * ks + (q >> 1)][2 * (q & 1) + 1]);
                        a[q] = *reinterpret_cast<const unsigned*>(&p);
                    }
#pragma unroll
                    for (int np = 0; np < NDB * 4; ++np) {
                        const int key = ks * 16 + (((lane >> 3) & 1) << 3) + (lane & 7), ch = (np & 3) * 2 + (lane >> 4);
                        unsigned bf[4];
                        ldsm4t(vt + (np >> 2) * HALF_TILE + key * 128 + ((ch ^ (key & 7)) << 4), bf);
                        mma16816(o[2 * np], a, bf[0], bf[1]);
                        mma16816(o[2 * np + 1], a, bf[2], bf[3]);
                    }
                }
            }
            __syncwarp();                              // all lanes have read the slot
            if (ok) { ++used; produce(); }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        }
        auto out_row = [&](int row) {
            const int t = LIST ? 0 : row / G, g = s.g0 + (LIST ? row : row - t * G);
            return j.out + (int64_t)(s.row + t) * j.ldo + ((int64_t)s.head * G + g) * c.d;
        };
        if (TEAM == 1) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = r0 + 8 * i;
                if (row < s.rows) {
                    const float f = l[i] > 0.f ? 1.0f / l[i] : 0.f;
                    __nv_bfloat16* dst = out_row(row);
#pragma unroll
                    for (int n = 0; n < NDB * 8; ++n)
                        if (n * 8 < c.d)
                            *reinterpret_cast<__nv_bfloat162*>(dst + n * 8 + c0) = __floats2bfloat162_rn(o[n][2 * i] * f, o[n][2 * i + 1] * f);
                }
            }
            continue;
        }
        // ---- the four warps' shares of the row tile
        constexpr int W = NDB * 64;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = r0 + 8 * i;
            if (row < s.rows) {
                if ((lane & 3) == 0) { sh.m[warp][row] = m[i]; sh.l[warp][row] = l[i]; }
#pragma unroll
                for (int n = 0; n < NDB * 8; ++n)
                    *reinterpret_cast<float2*>(mrg + (warp * 16 + row) * W + n * 8 + c0) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
            }
        }
        __syncthreads();
        const int col = tid % W;
        float* mine = partial<LIST>(ws, s, s.piece);
        for (int row = tid / W; row < s.rows; row += ST_THREADS / W) {
            float M = -INFINITY, L = 0.f, x = 0.f;
#pragma unroll
            for (int q = 0; q < ST_WARPS; ++q) M = fmaxf(M, sh.m[q][row]);
#pragma unroll
            for (int q = 0; q < ST_WARPS; ++q) {
                const float mq = sh.m[q][row], f = mq > -INFINITY ? ex2_approx(mq - M) : 0.f;
                L = fmaf(sh.l[q][row], f, L);
                x = fmaf(mrg[(q * 16 + row) * W + col], f, x);
            }
            if (s.pieces == 1) {
                if (col < c.d) out_row(row)[col] = __float2bfloat16_rn(L > 0.f ? x / L : 0.f);
            } else {
                mine[row * 128 + col] = x;
                if (col == 0) { mine[2048 + row] = M; mine[2064 + row] = L; }
            }
        }
        if (s.pieces > 1) {
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const unsigned before = atomicAdd(&counters[s.ctr], 1u);
                sh.last = before + 1u == (unsigned)s.pieces;
                if (sh.last) counters[s.ctr] = 0u;     // as the next call finds it
            }
            __syncthreads();
            if (sh.last) {                             // the others' results are there: join them in the order of the keys
                __threadfence();
                for (int row = tid / W; row < s.rows; row += ST_THREADS / W) {
                    float M = -INFINITY, L = 0.f, x = 0.f;
                    for (int p = 0; p < s.pieces; ++p) {
                        const float* part = partial<LIST>(ws, s, p);
                        const float mp = __ldcg(part + 2048 + row), lp = __ldcg(part + 2064 + row), xp = __ldcg(part + row * 128 + col);
                        const float Mn = fmaxf(M, mp);
                        const float fa = M > -INFINITY ? ex2_approx(M - Mn) : 0.f, fb = mp > -INFINITY ? ex2_approx(mp - Mn) : 0.f;
                        L = L * fa + lp * fb;
                        x = x * fa + xp * fb;
                        M = Mn;
                    }
                    if (col < c.d) out_row(row)[col] = __float2bfloat16_rn(L > 0.f ? x / L : 0.f);
                }
            }
        }
        __syncthreads();                               // the merge buffer is reused
    }
    // a warp that gave up has copies in flight: they have to land before its shared memory goes
    if (!ok) {
        for (unsigned i = used; i < made; ++i) {
            const unsigned long long t0 = global_ns();
            while (!mbar_try(&sh.full[warp][i % NST], (i / NST) & 1u))
                if (past_limit(2 * (global_ns() - t0), abort_flag)) break;
        }
        if (lane == 0) { atomicOr(status, ST_TIMEOUT); status[2] = 300u + (unsigned)abort_flag[0]; }
    }
}

template <int NDB, bool LIST, int TEAM>
cudaError_t run_step(ada_ctx* ctx, const StepMaps& maps, const CacheView& c, const Ragged& r, const AttendJob& j, int grid,
                     int tiles, int pieces, cudaStream_t s) {
    auto kernel = k_cache_step<NDB, LIST, TEAM>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, st_smem<NDB>());
    if (e != cudaSuccess) return e;
    return launch_k(ctx, kernel, dim3(grid), dim3(ST_THREADS), st_smem<NDB>(), s, maps, c, r, j, tiles, pieces,
                    ctx->cache_part, ctx->cache_ctr, ctx->status);
}

}  // namespace

cudaError_t launch_cache_step(ada_ctx* ctx, const CacheView& c, const Ragged& r, const AttendJob& j, cudaStream_t s) {
    StepMaps maps;
    const int box = c.shift == 4 ? 16 : GK;
    if (!encode_pages(&maps.k, c, c.k, box) || !encode_pages(&maps.v, c, c.v, box)) return cudaErrorInvalidValue;
    const int G = j.h / c.h_kv;
    const bool wide = c.d > 64;
    if (j.blk_idx == nullptr)
        return wide ? run_step<2, false, 4>(ctx, maps, c, r, j, ctx->sm_count, 1, 1, s)
                    : run_step<1, false, 4>(ctx, maps, c, r, j, ctx->sm_count, 1, 1, s);
    const int tiles = (G + 15) / 16;
    const int64_t rows = (int64_t)r.N * c.h_kv * tiles;
    // rows enough for every warp of the GPU: a warp each, nothing to join
    if (rows >= 4 * (int64_t)ctx->sm_count)
        return wide ? run_step<2, true, 1>(ctx, maps, c, r, j, ctx->sm_count, tiles, 1, s)
                    : run_step<1, true, 1>(ctx, maps, c, r, j, ctx->sm_count, tiles, 1, s);
    // few rows: their lists are cut into pieces of at least 4 granules for each warp, as many as fill the SMs
    const int64_t room = ((int64_t)j.k << c.shift) / (4 * ST_WARPS * GK);
    int64_t pieces = (2 * ctx->sm_count) / rows;
    pieces = pieces < room ? pieces : room;
    pieces = pieces < 1 ? 1 : pieces;
    const int64_t items = rows * pieces;
    const int grid = (int)(items < ctx->sm_count ? items : ctx->sm_count);
    return wide ? run_step<2, true, 4>(ctx, maps, c, r, j, grid, tiles, (int)pieces, s)
                : run_step<1, true, 4>(ctx, maps, c, r, j, grid, tiles, (int)pieces, s);
}

}  // namespace ada
