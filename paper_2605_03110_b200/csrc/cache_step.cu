// Attention of single tokens over the paged cache (ada_attention_cached with few rows per key head), and of any tokens
// over the pages that their lists name (ada_attention_blocks).
//
//   out = sum_s 2^(sc q.k_s - m) v_s / sum_s 2^(sc q.k_s - m),   sc = scale log2(e), m a reference near the maximum
// in one pass over the keys.  The heads that share a key head (and, dense, the few new tokens of a sequence) are the
// up to 16 rows of one tile, so that K and V are read once for all of them.  What bounds it is the stream of keys and
// values: from HBM in a decoding step, from L2 where a chunk's tokens list the same pages.  A 128-row tcgen05 tile would be
// empty but for these rows.  Here both products are taken transposed on mma.sync, S^T = K Q^T and O^T = V^T P^T: keys
// (head elements) are the 16-row side of the instruction and the rows its 8-column side, so that 8 rows waste nothing,
// and operands stay in registers but for K and V.
//
// A warp works alone: granules of 32 keys arrive by TMA, K and V in turn, in a ring of its own; scores, softmax and
// products stay in its registers, and it shares nothing until the end of a row tile.  The eight warps of a CTA deal a
// row tile's granules among them (TEAM = 8) or take row tiles of their own (TEAM = 1, many rows with lists: no barrier).
// m is raised only when a score has left it by more than 8 powers of two: a vote per granule instead of a maximum.
//
// Dense work is cut into units of 256 keys of one (sequence, key head); every CTA takes an equal run of units
// whatever the lengths are, and a row tile that several CTAs share is joined by the one that finishes last (in
// the order of the keys, so that results do not depend on who that is).  Nobody waits for another CTA.
//
// Measured (32 heads on 8 key heads of 128, pages of 64): 64 sequences of up to 16384 tokens, 2.2 GB, 341 us = 6.5 TB/s; two of
// 131072 tokens 170 us = 6.3 TB/s; lists of 32 pages for 32 tokens 48 us = 5.7 TB/s (two row tiles for most CTAs, one for the
// rest); lists of 16 pages for 1000 tokens 247 us, 4.2 GB out of L2.  With S = Q K^T and 16 rows padded, four warps:
// 355, 182, 51 and 480 us.
#include "cache_tma.cuh"

namespace ada {

using namespace tc;

namespace {

constexpr int ST_WARPS = 8;                // warps of a team; teams of one warp: st_warps of them in a CTA
constexpr int ST_MOST = 12;
constexpr int GK = 32;                     // keys per granule
constexpr int UNIT = GK * ST_WARPS;        // keys per unit of dense work
constexpr int NOWHERE = 0x7fff0000;        // position of keys that are not there: behind every limit
constexpr int SLOT_FLOATS = 16 * 128 + 32; // one partial result: 16 rows x 128, maxima, sums
constexpr float ST_LAG = 8.0f;

// Warps of a CTA: lone warps with up to 8 rows need few enough registers for twelve, with two slots each instead of three
// (1000 tokens x 8 key heads, lists of 16 pages of 64: 292 -> 244 us, 17 TB/s out of L2).
template <int NT, int TEAM> __host__ __device__ constexpr int st_warps() { return TEAM == 1 && NT == 1 ? 12 : 8; }
// slots of a warp's ring: K or V of a granule, NDB blocks of 64 elements x 32 keys
template <int NDB, int NT, int TEAM> __host__ __device__ constexpr int st_slots() { return (st_warps<NT, TEAM>() == 12 ? 4 : 6) / NDB; }
template <int NDB> __host__ __device__ constexpr int st_slot_bytes() { return NDB * GK * 128; }
template <int NDB> __host__ __device__ constexpr int st_ring_bytes() { return 48 / NDB * st_slot_bytes<NDB>(); }   // 12 x 4 = 8 x 6 = 48
template <int NDB> __host__ __device__ constexpr int st_merge_bytes() { return ST_WARPS * 8 * NDB * 64 * 4; }

struct StepShared {
    unsigned long long full[ST_MOST][6];
    int2 base[ST_MOST][6];                // positions of the two halves of a granule
    float m[ST_WARPS][16], l[ST_WARPS][16];
    int abort_flag[2];
    int last;
    int odd_any;                          // dense, of the row tile: a value of a later token was not finite
    unsigned odd[128];                    // by column: bits 0..15 +inf, 16..31 -inf (NaN both) of token 0's successors 1..16
};
template <int NDB> __host__ __device__ constexpr int st_smem() {
    return st_ring_bytes<NDB>() + st_merge_bytes<NDB>() + (int)sizeof(StepShared);
}
static_assert(st_smem<2>() <= 227 * 1024 && st_smem<1>() <= 227 * 1024, "shared memory budget");

struct StepMaps {
    CUtensorMap k, v;
};

// One row tile's run of keys, as a team works on it.
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
    int64_t at, end;                       // dense: units; lists: (row, key head, row tile, piece) items
    int b, head, n, off, len;
    int ku, nu;                            // dense: unit within the row tile, of how many
    int64_t per;
    int row, rt, piece;                    // lists

    __device__ __forceinline__ void load_seq(const Ragged& r, const CacheView& c, int few) {
        n = seq_rows(r, b, off);
        len = seq_len(r, c, b);
        nu = n > 0 && !(few > 0 && n > few) ? max(1, (len + UNIT - 1) / UNIT) : 0;
    }
    // the next segment, or false
    __device__ __forceinline__ bool next(Seg& s, const Ragged& r, const CacheView& c, const AttendJob& j, int G, int tiles,
                                         int pieces, unsigned* status) {
        if (LIST) {
            while (at < end) {
                if (b < 0 || row < off || row >= off + n) {     // another sequence
                    // Rows from off[B] on are nobody's.  One before that may be too if the offsets are out of order: all teams
                    // that meet it leave it out, and each goes on, so that a row's pieces are all there or none of them
                    // (what comes back to zero are the counters of the next call).
                    const int last = r.off[r.B];
                    b = seq_of_row(r, row);
                    if (row >= last) { at = end; return false; }
                    if (b < 0) {
                        at += ((int64_t)(c.h_kv - head) * tiles - rt) * pieces - piece;
                        head = rt = piece = 0;
                        ++row;
                        continue;
                    }
                    load_seq(r, c, j.few);
                }
                s.b = b; s.head = head; s.row = row; s.g0 = rt * 16;
                s.rows = min(16, G - rt * 16);
                s.len = j.causal ? max(len - n + (row - off) + 1, 0) : len;   // as if it were the only new token
                s.n = 1;
                const int64_t rh = (int64_t)row * c.h_kv + head;
                int cnt = j.blk_cnt[rh];
                if (cnt < 0 || cnt > j.k) { atomicOr(status, ST_BAD_COUNT); cnt = min(max(cnt, 0), j.k); }
                s.cnt = cnt;
                const int g = (int)((((int64_t)cnt << c.shift) + GK - 1) / GK);
                s.g_begin = pieces == 1 ? 0 : (int)((int64_t)g * piece / pieces);
                s.g_end = pieces == 1 ? g : (int)((int64_t)g * (piece + 1) / pieces);
                s.pieces = pieces; s.piece = piece;
                s.ctr = pieces == 1 ? 0 : (int)(rh * tiles + rt);
                s.slot0 = s.ctr * pieces;
                ++at;
                if (++piece == pieces) {
                    piece = 0;
                    if (++rt == tiles) { rt = 0; if (++head == c.h_kv) { head = 0; ++row; } }
                }
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
                load_seq(r, c, j.few);
            }
        }
        const int take = (int)min((int64_t)(nu - ku), end - at);
        s.b = b; s.head = head; s.row = off; s.g0 = 0;
        s.n = n; s.len = len; s.cnt = 0;
        s.rows = min(n, j.max_new) * G;
        const int g = (len + GK - 1) / GK;
        s.g_begin = ku * ST_WARPS;
        s.g_end = min((ku + take) * ST_WARPS, g);
        const int64_t first = at - ku;                      // the row tile's units are [first, first + nu)
        if (take == nu) {
            s.pieces = 1; s.piece = s.slot0 = s.ctr = 0;
        } else {
            int c0, c1;
            shares_of(first, nu, per, blockIdx.x, c0, c1);
            s.pieces = c1 - c0 + 1;
            s.piece = (int)blockIdx.x - c0;
            s.slot0 = c0;
            s.ctr = c1;
        }
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

// NT: rows / 8
template <int NDB, int NT, bool LIST, int TEAM>
__global__ void __launch_bounds__(32 * st_warps<NT, TEAM>(), 1)
k_cache_step(const __grid_constant__ StepMaps maps, const CacheView c, const Ragged r, const AttendJob j, int tiles,
             int pieces, float* __restrict__ ws, unsigned* __restrict__ counters, unsigned* __restrict__ status) {
    constexpr int SLOTS = st_slots<NDB, NT, TEAM>(), WARPS = st_warps<NT, TEAM>(), THREADS = 32 * WARPS;
    constexpr int KS = NDB * 4;                       // 16-element steps of a head row
    constexpr int BLOCK = GK * 128;                   // one 64-element block of 32 keys: 4 KiB
    extern __shared__ __align__(1024) unsigned char smem[];
    float* mrg = reinterpret_cast<float*>(smem + st_ring_bytes<NDB>());            // [8 warps][8 rows][NDB * 64]
    StepShared& sh = *reinterpret_cast<StepShared*>(smem + st_ring_bytes<NDB>() + st_merge_bytes<NDB>());
    volatile int* abort_flag = sh.abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = j.h / c.h_kv;
    unsigned char* ring = smem + warp * SLOTS * st_slot_bytes<NDB>();
    if ((smem_u32(smem) & 1023u) != 0u) {             // the tiles would not be where the swizzle assumes
        grid_dep_wait();
        if (tid == 0) { atomicOr(status, ST_TIMEOUT); status[2] = 399u; }
        return;
    }
    if (tid == 0) {
        sh.abort_flag[0] = 0;
        sh.abort_flag[1] = wait_limit_units(false);
        sh.odd_any = 0;
    }
    if (lane == 0) {
        for (int i = 0; i < SLOTS; ++i) mbar_init(&sh.full[warp][i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (!LIST && tid < 128) sh.odd[tid] = 0u;
    if (tid == 64) { prefetch_map(&maps.k); prefetch_map(&maps.v); }
    __syncthreads();
    grid_dep_wait();
    grid_dep_launch_next();
    if (blockIdx.x == 0) check_ragged(r, c, status, tid, THREADS);

    // ---------------------------------------------------------------- this team's run of work
    const int w = TEAM == 1 ? 0 : warp;
    Work<LIST> work;
    work.b = LIST ? -1 : 0;
    work.head = work.n = work.off = work.len = work.ku = work.nu = work.row = work.rt = work.piece = 0;
    if (LIST) {
        const int64_t items = (int64_t)r.N * c.h_kv * tiles * pieces;
        const int64_t teams = (int64_t)gridDim.x * (WARPS / TEAM);
        const int64_t team = (int64_t)blockIdx.x * (WARPS / TEAM) + (TEAM == 1 ? warp : 0);
        work.per = (items + teams - 1) / teams;
        work.at = min(team * work.per, items);
        work.end = min(work.at + work.per, items);
        int64_t rest = work.at / pieces;
        work.piece = (int)(work.at - rest * pieces);
        work.rt = (int)(rest % tiles); rest /= tiles;
        work.head = (int)(rest % c.h_kv);
        work.row = (int)(rest / c.h_kv);
    } else {
        // prefix sums of the sequences' units, 32 at a time, by every warp for itself
        auto units_of = [&](int b) {
            if (b >= r.B) return 0;
            int o;
            const int n = seq_rows(r, b, o);
            if (j.few > 0 && n > j.few) return 0;
            if (blockIdx.x == 0 && n > j.max_new) atomicOr(status, ST_BAD_COUNT);
            return n > 0 ? max(1, (seq_len(r, c, b) + UNIT - 1) / UNIT) : 0;
        };
        int64_t U = 0;
        for (int b0 = 0; b0 < r.B; b0 += 32) U += __reduce_add_sync(0xffffffffu, units_of(b0 + lane));
        U *= c.h_kv;
        work.per = max((U + gridDim.x - 1) / gridDim.x, (int64_t)1);
        work.at = min(work.per * blockIdx.x, U);
        work.end = min(work.at + work.per, U);
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
                    work.load_seq(r, c, j.few);
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
    unsigned made = 0;                                // slots asked for: K, V, K, V ..
    int id0 = -1, id1 = -1, first_slot = 0, phead = 0;   // pages of the granule whose K was asked for last
    // asks for K or V of the next granule of this warp, if there is one
    auto produce = [&]() {
        if ((made & 1u) == 0u) {
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
                        int p = e;                    // dense: the sequence's e-th page
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
            id0 = __shfl_sync(0xffffffffu, pid.x, l); id1 = __shfl_sync(0xffffffffu, pid.y, l);
            const int b0 = __shfl_sync(0xffffffffu, pbase.x, l), b1 = __shfl_sync(0xffffffffu, pbase.y, l);
            if (elect_one()) sh.base[warp][made % SLOTS] = make_int2(b0, b1);
            first_slot = (pg * GK) & ((1 << c.shift) - 1);
            phead = ps.head;
            pg += TEAM;
        }
        if (elect_one()) {
            const int st = made % SLOTS;
            unsigned char* dst = ring + st * st_slot_bytes<NDB>();
            unsigned long long* bar = &sh.full[warp][st];
            const CUtensorMap* map = (made & 1u) ? &maps.v : &maps.k;
            if (c.shift > 4) {
                mbar_expect_tx(bar, id0 >= 0 ? (unsigned)st_slot_bytes<NDB>() : 0u);
                if (id0 >= 0)
#pragma unroll
                    for (int db = 0; db < NDB; ++db) tma_load_4d(map, bar, dst + db * BLOCK, db * BK, first_slot, phead, id0);
            } else {
                mbar_expect_tx(bar, (unsigned)st_slot_bytes<NDB>() / 2 * ((id0 >= 0) + (id1 >= 0)));
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int id = q == 0 ? id0 : id1;
                    if (id >= 0)
#pragma unroll
                        for (int db = 0; db < NDB; ++db) tma_load_4d(map, bar, dst + db * BLOCK + q * 2048, db * BK, 0, phead, id);
                }
            }
        }
        ++made;
    };
#pragma unroll 1
    for (int i = 0; i < SLOTS; ++i) produce();

    // ---------------------------------------------------------------- consumer side
    const int r0 = lane >> 2, c0 = 2 * (lane & 3);    // a fragment's row; the first of its two columns
    const unsigned ring_u = smem_u32(ring);
    // addresses of the two operands within a slot: lane l names row l % 8 of the 8 x 8 matrix l / 8
    const int k_key = ((lane >> 3) & 1) * 8 + (lane & 7), k_ch = lane >> 4;
    const int v_key = (lane >> 4) * 8 + (lane & 7), v_ch = (lane >> 3) & 1;
    unsigned used = 0;
    bool ok = true;
    auto wait_slot = [&](int where) {
        if (ok) ok = mbar_wait(&sh.full[warp][used % SLOTS], (used / SLOTS) & 1u, abort_flag, where);
        ok = __all_sync(0xffffffffu, ok);
    };
    auto release = [&]() {
        __syncwarp();                                 // all lanes have read the slot
        if (ok) { ++used; produce(); }
    };
    Seg s;
    while (work.next(s, r, c, j, G, tiles, pieces, status)) {
        // right operand of S^T: row r0 (+ 8) of the tile (row = token * G + head of the group)
        unsigned qf[NT][KS][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = nt * 8 + r0;
            const bool live = row < s.rows;
            const int t = LIST || !live ? 0 : row / G, g = s.g0 + (LIST ? row : row - t * G);
            const __nv_bfloat16* q = j.Q + (int64_t)(s.row + t) * j.ldq + ((int64_t)s.head * G + g) * c.d;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                qf[nt][k][0] = live && k * 16 < c.d ? *reinterpret_cast<const unsigned*>(q + k * 16 + c0) : 0u;
                qf[nt][k][1] = live && k * 16 < c.d ? *reinterpret_cast<const unsigned*>(q + k * 16 + 8 + c0) : 0u;
            }
        }
        // of this lane's rows nt * 8 + c0 + {0, 1}: keys that they see, reference, sum of this lane's probabilities
        int lim[NT][2];
        float m[NT][2], l[NT][2], o[KS][NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = nt * 8 + c0 + i;
                lim[nt][i] = row >= s.rows ? 0 : LIST || !j.causal ? s.len : s.len - s.n + row / G + 1;
                m[nt][i] = -INFINITY;
                l[nt][i] = 0.f;
            }
        // keys from here on are masked for some row: the first token's limit
        const int lim_all = LIST || !j.causal ? s.len : s.len - s.n + 1;
#pragma unroll
        for (int d = 0; d < KS; ++d)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][nt][e] = 0.f;

        for (int g = s.g_begin + w; g < s.g_end; g += TEAM) {
            float sc[2][NT][4];                        // scores of 32 keys (two tiles of 16) x rows
            int2 base = make_int2(0, 0);
            wait_slot(50);
            if (ok) {
                const int st = used % SLOTS;
                const unsigned kt = ring_u + st * st_slot_bytes<NDB>();
                base = sh.base[warp][st];
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[mt][nt][e] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        unsigned a[4];
                        ldsm4(kt + (k >> 2) * BLOCK + (mt * 16 + k_key) * 128 + ((((k & 3) * 2 + k_ch) ^ (k_key & 7)) << 4), a);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(sc[mt][nt], a, qf[nt][k][0], qf[nt][k][1]);
                    }
            }
            release();
            if (ok && (base.x + 15 >= lim_all || base.y + 15 >= lim_all)) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if ((mt == 0 ? base.x : base.y) + (e >> 1) * 8 + r0 >= lim[nt][e & 1]) sc[mt][nt][e] = -INFINITY;
            }
            unsigned pf[2][NT][2];                     // probabilities as right operand of O^T
            if (ok) {
                float top[NT][2];
                bool raise = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        top[nt][i] = fmaxf(fmaxf(sc[0][nt][i], sc[0][nt][2 + i]), fmaxf(sc[1][nt][i], sc[1][nt][2 + i])) * j.scale;
                        raise = raise || top[nt][i] > m[nt][i] + ST_LAG;
                    }
                if (__any_sync(0xffffffffu, raise)) {   // (the first keys always do)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float x = top[nt][i];
#pragma unroll
                            for (int q = 4; q < 32; q <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, q));
                            const float mn = fmaxf(m[nt][i], x);
                            const float f = m[nt][i] > -INFINITY ? ex2_approx(m[nt][i] - mn) : 0.f;
                            m[nt][i] = mn;
                            l[nt][i] = top[nt][i] < INFINITY ? l[nt][i] * f : NAN;   // (a score beyond fp32: NaN, on every path)
#pragma unroll
                            for (int d = 0; d < KS; ++d) { o[d][nt][i] *= f; o[d][nt][2 + i] *= f; }
                        }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float ref[2] = {m[nt][0] > -INFINITY ? m[nt][0] : 0.f, m[nt][1] > -INFINITY ? m[nt][1] : 0.f};
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            sc[mt][nt][e] = ex2_approx(fmaf(sc[mt][nt][e], j.scale, -ref[e & 1]));
                            l[nt][e & 1] += sc[mt][nt][e];
                        }
                        // rounded to bf16 for the second product; their sum is not
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const __nv_bfloat162 p = __floats2bfloat162_rn(sc[mt][nt][2 * i], sc[mt][nt][2 * i + 1]);
                            pf[mt][nt][i] = transposed(*reinterpret_cast<const unsigned*>(&p));
                        }
                    }
                }
            }
            wait_slot(51);
            if (ok) {
                const int st = used % SLOTS;
                // Values that a row does not see must not meet its zero probability as a NaN or an infinity: those of slots that
                // hold nothing of this sequence become zeros, and so do a later token's that are not finite; rows that see one
                // get it back where the warps' shares are joined.
                if (base.x + 15 >= lim_all || base.y + 15 >= lim_all) {
                    unsigned char* v = ring + st * st_slot_bytes<NDB>();
                    auto position = [&](int q) {           // of 16-byte piece q of a granule
                        const int key = (q >> 3) & 31;
                        return key < 16 ? base.x + key : base.y + key - 16;
                    };
                    auto piece = [&](int q) {
                        return reinterpret_cast<uint4*>(v + (q >> 8) * BLOCK + ((q >> 3) & 31) * 128 + (q & 7) * 16);
                    };
                    for (int q = lane; q < GK * NDB * 8; q += 32)
                        if (position(q) >= s.len) *piece(q) = make_uint4(0u, 0u, 0u, 0u);
                    if (!LIST && lim_all < s.len) {
#pragma unroll 1
                        for (int q = lane; q < GK * NDB * 8; q += 32) {
                            const int later = position(q) - lim_all;         // token later + 1 on sees it
                            if (later < 0 || later >= s.len - lim_all || !nonfinite8(*piece(q))) continue;
                            const int col = (q >> 8) * 64 + (((q & 7) ^ (q >> 3 & 7)) << 3);
                            sh.odd_any = 1;
                            take_nonfinite(piece(q), [&](int e, bool plus, bool minus) {
                                if (later < 16) atomicOr(&sh.odd[col + e], ((plus ? 1u : 0u) | (minus ? 0x10000u : 0u)) << later);
                            });
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the slot's next load comes through the async proxy)
                    __syncwarp();
                }
                const unsigned vt = ring_u + st * st_slot_bytes<NDB>();
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int d = 0; d < KS; ++d) {
                        unsigned a[4];
                        ldsm4t(vt + (d >> 2) * BLOCK + (mt * 16 + v_key) * 128 + ((((d & 3) * 2 + v_ch) ^ (v_key & 7)) << 4), a);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(o[d][nt], a, pf[mt][nt][0], pf[mt][nt][1]);
                    }
            }
            release();
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int q = 4; q < 32; q <<= 1) l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], q);
        auto out_row = [&](int row) {
            const int t = LIST ? 0 : row / G, g = s.g0 + (LIST ? row : row - t * G);
            return j.out + (int64_t)(s.row + t) * j.ldo + ((int64_t)s.head * G + g) * c.d;
        };
        // what a row whose sum is 0 gets: zeros if it sees no slot, NaN if all of its scores are -inf
        auto no_weight = [&](int row) {
            bool sees;
            if (LIST) {                                // the first listed page has the first slot
                const int p = s.cnt > 0 ? j.blk_idx[((int64_t)s.row * c.h_kv + s.head) * j.k] : c.max_pages;
                sees = p < c.max_pages && (p << c.shift) < s.len;
            } else {
                sees = (j.causal ? s.len - s.n + row / G + 1 : s.len) > 0;
            }
            return sees ? NAN : 0.f;
        };
        if (TEAM == 1) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float f[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) f[i] = l[nt][i] == 0.f ? no_weight(nt * 8 + c0 + i) : 1.0f / l[nt][i];   // (NaN stays)
                __nv_bfloat16* dst = out_row(nt * 8 + r0);
#pragma unroll
                for (int d = 0; d < KS; ++d)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const __nv_bfloat162 p = __floats2bfloat162_rn(o[d][nt][2 * i] * f[0], o[d][nt][2 * i + 1] * f[1]);
                        const unsigned x = transposed(*reinterpret_cast<const unsigned*>(&p));   // two elements of row r0
                        if (nt * 8 + r0 < s.rows && d * 16 < c.d) *reinterpret_cast<unsigned*>(dst + d * 16 + i * 8 + c0) = x;
                    }
            }
            continue;
        }
        // ---- the warps' shares of the row tile, eight rows at a time
        constexpr int W = NDB * 64;
        const int col = tid % W;
        float* mine = partial<LIST>(ws, s, s.piece);
        int odd = 0;
        if (lane < 4)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) { sh.m[warp][nt * 8 + c0 + i] = m[nt][i]; sh.l[warp][nt * 8 + c0 + i] = l[nt][i]; }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt * 8 >= s.rows) break;
#pragma unroll
            for (int d = 0; d < KS; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    mrg[(warp * 8 + c0 + (e & 1)) * W + d * 16 + (e >> 1) * 8 + r0] = o[d][nt][e];
            __syncthreads();
            if (!LIST && nt == 0) odd = sh.odd_any;
            const int rows = min(s.rows - nt * 8, 8);
            for (int rr = tid / W; rr < rows; rr += THREADS / W) {
                const int row = nt * 8 + rr;
                float M = -INFINITY, L = 0.f, x = 0.f;
#pragma unroll
                for (int q = 0; q < ST_WARPS; ++q) M = fmaxf(M, sh.m[q][row]);
#pragma unroll
                for (int q = 0; q < ST_WARPS; ++q) {
                    const float mq = sh.m[q][row], f = mq > -INFINITY ? ex2_approx(mq - M) : 0.f;
                    L = fmaf(sh.l[q][row], f, L);
                    x = fmaf(mrg[(q * 8 + rr) * W + col], f, x);
                }
                if (!LIST && odd) {                    // what the row's token sees of the values that were taken out
                    const unsigned seen = sh.odd[col] & ((1u << row / G) - 1u) * 0x10001u;
                    if (seen & 0xffffu) x += INFINITY;
                    if (seen >> 16) x -= INFINITY;
                }
                if (s.pieces == 1) {
                    if (col < c.d) out_row(row)[col] = __float2bfloat16_rn(L == 0.f ? no_weight(row) : x / L);
                } else {
                    mine[row * 128 + col] = x;
                    if (col == 0) { mine[2048 + row] = M; mine[2064 + row] = L; }
                }
            }
            __syncthreads();                           // the buffer is reused
        }
        if (!LIST && odd) {                            // (the same in all threads)
            if (tid < 128) sh.odd[tid] = 0u;
            if (tid == 0) sh.odd_any = 0;
            __syncthreads();
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
                for (int row = tid / W; row < s.rows; row += THREADS / W) {
                    float M = -INFINITY, L = 0.f, x = 0.f;
                    for (int p = 0; p < s.pieces; ++p) M = fmaxf(M, __ldcg(partial<LIST>(ws, s, p) + 2048 + row));
                    const float ref = M > -INFINITY ? M : 0.f;
#pragma unroll 4
                    for (int p = 0; p < s.pieces; ++p) {
                        const float* part = partial<LIST>(ws, s, p);
                        const float f = ex2_approx(__ldcg(part + 2048 + row) - ref);
                        L = fmaf(__ldcg(part + 2064 + row), f, L);
                        x = fmaf(__ldcg(part + row * 128 + col), f, x);
                    }
                    if (col < c.d) out_row(row)[col] = __float2bfloat16_rn(L == 0.f ? no_weight(row) : x / L);
                }
            }
            __syncthreads();
        }
    }
    // a warp that gave up has copies in flight: they have to land before its shared memory goes
    if (!ok) {
        for (unsigned i = used; i < made; ++i) {
            const unsigned long long t0 = global_ns();
            while (!mbar_try(&sh.full[warp][i % SLOTS], (i / SLOTS) & 1u))
                if (past_limit(2 * (global_ns() - t0), abort_flag)) break;
        }
        if (lane == 0) { atomicOr(status, ST_TIMEOUT); status[2] = 300u + (unsigned)abort_flag[0]; }
    }
}

struct StepPlan {
    int grid, tiles, pieces;
};

template <int NDB, int NT, bool LIST, int TEAM>
cudaError_t run_step(ada_ctx* ctx, const StepMaps& maps, const CacheView& c, const Ragged& r, const AttendJob& j,
                     const StepPlan& p, cudaStream_t s) {
    auto kernel = k_cache_step<NDB, NT, LIST, TEAM>;
    cudaError_t e = allow_smem(ctx, (NDB - 1) + 2 * (NT - 1) + 4 * (!LIST ? 0 : TEAM == 1 ? 1 : 2), kernel, st_smem<NDB>());   // bits 0 .. 11
    if (e != cudaSuccess) return e;
    prof_begin(ctx, K_CACHE_STEP, s);
    e = launch_k(ctx, kernel, dim3(p.grid), dim3(32 * st_warps<NT, TEAM>()), st_smem<NDB>(), s, maps, c, r, j, p.tiles, p.pieces,
                 ctx->cache_part, ctx->cache_ctr, ctx->status);
    prof_end(ctx, s);
    return e;
}
template <bool LIST, int TEAM>
cudaError_t run_step(ada_ctx* ctx, const StepMaps& maps, const CacheView& c, const Ragged& r, const AttendJob& j,
                     const StepPlan& p, int rows, cudaStream_t s) {
    if (c.d > 64)
        return rows <= 8 ? run_step<2, 1, LIST, TEAM>(ctx, maps, c, r, j, p, s) : run_step<2, 2, LIST, TEAM>(ctx, maps, c, r, j, p, s);
    return rows <= 8 ? run_step<1, 1, LIST, TEAM>(ctx, maps, c, r, j, p, s) : run_step<1, 2, LIST, TEAM>(ctx, maps, c, r, j, p, s);
}

}  // namespace

cudaError_t launch_cache_step(ada_ctx* ctx, const CacheView& c, const Ragged& r, const AttendJob& j, cudaStream_t s) {
    StepMaps maps;
    const int box = c.shift == 4 ? 16 : GK;
    if (!encode_pages(&maps.k, c, c.k, box) || !encode_pages(&maps.v, c, c.v, box)) return cudaErrorInvalidValue;
    const int G = j.h / c.h_kv;
    StepPlan p = {ctx->sm_count, 1, 1};
    if (j.blk_idx == nullptr) return run_step<false, ST_WARPS>(ctx, maps, c, r, j, p, j.max_new * G, s);
    p.tiles = (G + 15) / 16;
    const int64_t rows = (int64_t)r.N * c.h_kv * p.tiles;
    // row tiles enough for every warp of the GPU: a warp each, nothing to join
    if (rows >= ST_WARPS * (int64_t)ctx->sm_count) return run_step<true, 1>(ctx, maps, c, r, j, p, G, s);
    // few of them: their lists are cut into pieces of at least 4 granules for each warp, as many as fill the SMs
    const int64_t room = ((int64_t)j.k << c.shift) / (4 * UNIT);
    int64_t pieces = (2 * ctx->sm_count) / rows;
    pieces = pieces < room ? pieces : room;
    p.pieces = pieces < 1 ? 1 : (int)pieces;
    const int64_t items = rows * p.pieces;
    if (items < p.grid) p.grid = (int)items;
    return run_step<true, ST_WARPS>(ctx, maps, c, r, j, p, G, s);
}

}  // namespace ada
