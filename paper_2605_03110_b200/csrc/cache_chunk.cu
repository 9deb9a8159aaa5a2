// Attention of chunks of new tokens over the paged cache (ada_attention_cached) on the 5th-generation tensor cores.
//
// The same softmax(scale q K^T) V in one pass over the keys as in cache_step.cu, for as many rows as a tile holds:
// the G heads that share a key head times 128 / G consecutive tokens are the 128 rows of a tile, two tiles (512 columns
// of TMEM: two score tiles, two accumulators) are a CTA's work item, and both read the same tiles of 128 keys.
//   warp 0      TMA: queries, and pages of K and V into a ring of slots (one slot = K or V of 128 keys)
//   warp 1      tcgen05.mma: S_t = Q_t K^T, O_t += P_t V; while tile 0's softmax runs, tile 1's products do
//   warps 2, 3  look at the values that not every row sees (a chunk's own): a NaN there must not reach the rows before it
//   warps 4..7  softmax of tile 0, one row per thread: S out of TMEM into registers, 2^(s - m), P back into TMEM as bf16
//               over its own scores, where the second product takes it from as its left operand
//   warps 8..11 the same for tile 1 (they have most of the registers, for a row's 128 scores)
// V needs no transposed copy: its tiles are MN-major right operands as the pages hold them.
// A row's reference maximum m is raised only when the running maximum has left it by more than 8 powers of two
// (then the accumulator is rescaled in TMEM); O / l does not depend on it.
//
// Work: items (sequence, 2 x 128 / G tokens, key head) cost as many units as they see key tiles; every CTA takes an
// equal run of units.  An item that several CTAs share is joined, 32 rows at a time, by the warp that finishes last,
// in the order of the keys; nobody waits for another CTA.
//
// Measured (32 heads on 8 key heads of 128): 2048 tokens after 6145 others, called again and again, 264 us = 911 TFLOP/s, 65 %
// of what cuBLAS sustains; a few calls on a GPU that was idle before (higher clocks) 228 us = 1055 TFLOP/s, 63 % of its
// best.  Two tiles and 128 keys take 3500 cycles, of them 2048 the tensor core's: each tile's chain is 600 for scores into registers
// and maxima, 1600 for exponentials (special-function unit and multipliers shared by the two sets), 1250 until the next
// scores are there (half of the second product, the first one, the signals).  An item's output takes 2.8 us, a share's
// 3.5, joining two shares 6 (11 before the last one's own came straight out of TMEM: 230 us against 224 at the time).
// On the way, idle GPU: MMAs issued behind `if (lane == 0)` 335 us, behind elect_one() 242; exponentials in two unrolled copies
// that miss the instruction cache 253, in one 232.
// Registers: 352 bytes of spill stores and 400 of loads (d_h above 64; 344 and 380 up to it).  Compiled with the other roles
// empty, the softmax role has 180 and 164 of them, nearly all with its key loop alone: 128 scores and 32 probabilities do
// not leave room in 216 registers for all of an item's state.  The rest is the producer's and the issuer's, in 72.
#include "cache_tma.cuh"

namespace ada {

using namespace tc;

namespace {

constexpr int CH_THREADS = 384;
constexpr int CH_KEYS = 128;                      // keys per tile
constexpr int BLK_BYTES = 128 * BK * 2;           // 128 rows x 64 elements: 16 KiB
constexpr float CH_LAG = 8.0f;
constexpr int PART_FLOATS = 256 * 128 + 2 * 256;  // one item's partial result: 4 columns x rows x 32, maxima, sums

template <int NDB> __host__ __device__ constexpr int ch_slots() { return 10 / NDB; }

struct ChunkShared {
    unsigned long long q_full, q_empty, full[10], empty[10], s_full[2], p_full[2][2], o_full[2], o_empty[2];
    unsigned tmem_base;
    int abort_flag[2];
    int start[5];                                 // b, p, head, place within the item: where the CTA's run begins; turn
    long long range[3];                           // first place, one past the last, places per CTA
    struct { int slot, from, to, found[2]; } look; // values to look at: number of the slot's load (-1: no more), its rows; answers
    int odd_item;                                 // the CTA's latest item (from 1) with entries in here:
    int odd[2][128];                              // first key whose value in a column is inf, -inf; NaN: both (see clean_values)
};
template <int NDB> __host__ __device__ constexpr int ch_smem() { return 14 * BLK_BYTES + (int)sizeof(ChunkShared); }
static_assert(ch_smem<2>() <= 227 * 1024, "shared memory budget");

struct ChunkMaps {
    CUtensorMap q, k, v;
};

struct Item {
    int b, head, row0, n_tok;             // first token's row; tokens of both tiles
    int first_lim;                        // keys that the first token sees
    int kv;                               // the sequence's length: keys behind it are nobody's
    int units[2];                         // key tiles of either tile of rows (0: no rows)
    int ku, take;                         // the CTA's units of it
    int pieces, piece, c0, c1;
};

// tq tokens per row tile.  Work is dealt out in places: `turn` of them for an item and one for each of its units behind them; a
// CTA has the units whose places are in its run.  Where a CTA's run holds several items, an item's queries and output take about
// as long as CH_TURN units; where items are longer than that, each of their shares has that to do, and turn is 0.
// (8 sequences of 1 to 517 new tokens, 32 heads: 146 us without, 142 with 2 places, 139 with 3; one of 17 after 3000, in shares:
// 23.0 without, 24.4 with 3.)
constexpr int CH_TURN = 3;
struct ChunkWork {
    long long at, end, per;
    int b, p, head, place, turn;          // place: of the item that many are behind
    int n, off, len, nu, P;

    static __device__ __forceinline__ int limit(int n, int len, int tok, int causal) {   // keys that the tokens below `tok` see
        return max(causal ? len - n + min(tok, n) : len, 0);
    }
    static __device__ __forceinline__ int units(int n, int len, int p, int tq, int causal) {
        return max((limit(n, len, (p + 1) * 2 * tq, causal) + CH_KEYS - 1) / CH_KEYS, 1);
    }
    // items of a sequence of n new tokens: none if it is the other kernel's
    static __device__ __forceinline__ int items(int n, int tq, int max_new, int few) {
        return n <= few ? 0 : (min(n, max_new) + 2 * tq - 1) / (2 * tq);
    }
    __device__ __forceinline__ void load_seq(const Ragged& r, const CacheView& c, int tq, int max_new, int few) {
        n = seq_rows(r, b, off);
        len = seq_len(r, c, b);
        P = items(n, tq, max_new, few);
    }
    __device__ __forceinline__ bool next(Item& it, const Ragged& r, const CacheView& c, int tq, int causal, int max_new, int few) {
        if (at >= end) return false;
        while (P == 0 || place >= nu + turn) {
            place = 0;
            if (P == 0 || ++head >= c.h_kv) {
                head = 0;
                if (P == 0 || ++p >= P) {
                    p = 0;
                    if (++b >= r.B) { at = end; return false; }
                    load_seq(r, c, tq, max_new, few);
                    if (P == 0) continue;
                }
                nu = units(n, len, p, tq, causal);
            }
        }
        if (place < turn) {
            at += turn - place;
            place = turn;
            if (at >= end) return false;
        }
        const int t0 = p * 2 * tq, ku = place - turn;
        it.b = b; it.head = head; it.row0 = off + t0;
        it.n_tok = min(min(n, max_new) - t0, 2 * tq);
        it.first_lim = causal ? len - n + t0 + 1 : len;
        it.kv = len;
        it.units[0] = min((limit(n, len, t0 + tq, causal) + CH_KEYS - 1) / CH_KEYS, nu);
        it.units[1] = it.n_tok > tq ? nu : 0;
        it.ku = ku;
        it.take = (int)min((long long)(nu - ku), end - at);
        const long long first = at - ku;
        shares_of(first, nu, per, blockIdx.x, it.c0, it.c1);
        it.pieces = it.c1 - it.c0 + 1;
        it.piece = (int)blockIdx.x - it.c0;
        at += it.take; place += it.take;
        return true;
    }
    // key tiles of row tile t in this CTA's share of the item
    static __device__ __forceinline__ int tiles_of(const Item& it, int t) { return max(min(it.units[t] - it.ku, it.take), 0); }
};

__device__ __forceinline__ float max3(float a, unsigned b, unsigned c) {      // NaN if one of them is
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
    return d;
}
__device__ __forceinline__ unsigned long long pack2(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(unsigned long long v, float& a, float& b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// p = 2^(x scale + nref) of 64 scores, as bf16 pairs; their sum.  The special-function unit takes 8 cycles for a warp's
// 32 exponentials, as long as everything else in this loop: CH_POLY of every 8 pairs go through the multipliers
// instead: y = n + f with n the nearest integer (left in the low bits by adding 1.5 x 2^23), 2^f on [-1/2, 1/2] a cubic
// that is off by at most 1.02e-4 of itself (fitted for least relative error with a value of exactly 1 at 0; a bf16 is
// rounded by up to 3.9e-3), n added to the exponent.  Arguments are cut at -127, where exactly 0 comes out: for masked
// scores too.
constexpr int CH_POLY = 2;
__device__ __forceinline__ void exp_pairs(const unsigned (&a)[32], const unsigned (&b)[32], float scale, float nref,
                                          unsigned (&w)[32], float& sum) {
    const unsigned long long sc2 = pack2(scale, scale), nr2 = pack2(nref, nref);
    const unsigned long long big = pack2(12582912.f, 12582912.f), nbig = pack2(-12582912.f, -12582912.f);
    const unsigned long long neg = pack2(-1.f, -1.f), c0 = pack2(1.f, 1.f);
    const unsigned long long c1 = pack2(0.6932829f, 0.6932829f), c2 = pack2(0.24221095f, 0.24221095f), c3 = pack2(0.055008933f, 0.055008933f);
    unsigned long long s2[2] = {0ull, 0ull};
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const unsigned (&x)[32] = i < 16 ? a : b;
        const int e = 2 * (i & 15);
        const unsigned long long y2 = fma2(pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), sc2, nr2);
        float p0, p1;
        unpack2(y2, p0, p1);
        if ((i & 7) < CH_POLY) {
            const unsigned long long y = pack2(fmaxf(p0, -127.f), fmaxf(p1, -127.f));
            const unsigned long long t = add2(y, big), f = fma2(add2(t, nbig), neg, y);
            const unsigned long long q = fma2(fma2(fma2(c3, f, c2), f, c1), f, c0);
            float t0, t1;
            unpack2(t, t0, t1);
            unpack2(q, p0, p1);
            p0 = __uint_as_float(__float_as_uint(p0) + (__float_as_uint(t0) << 23));
            p1 = __uint_as_float(__float_as_uint(p1) + (__float_as_uint(t1) << 23));
        } else {
            p0 = ex2_approx(p0);
            p1 = ex2_approx(p1);
        }
        s2[i & 1] = add2(s2[i & 1], pack2(p0, p1));
        const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
        w[i] = *reinterpret_cast<const unsigned*>(&h);
    }
    float u0, u1, v0, v1;
    unpack2(s2[0], u0, u1);
    unpack2(s2[1], v0, v1);
    sum += (u0 + u1) + (v0 + v1);
}

// Values of keys that some rows of an item see and others do not (a chunk's own tokens, causal), as they lie in a slot, from
// row `from` to row `to`: one that is not finite would meet the zero probabilities of the rows before it.  So it becomes
// zero for all of them, and odd[][column] says from which key on a row has seen one: such rows get it back at the item's
// end (restore_values).  Rows in shared memory are 128 bytes of 64 elements, 16-byte pieces swizzled.
// Who looks at them: the issuing warp itself made a mixed batch of 8 sequences 142 -> 155 us and 2048 tokens after 6145
// 263 -> 267; two warps that are otherwise idle, a key tile ahead of it, 146 and 264.
template <int NDB>
__device__ __forceinline__ void clean_values(unsigned char* v, int from, int to, int key0, int lane, ChunkShared& sh) {
    for (int q = from * 8 + lane; q < to * 8; q += 32)
        for (int db = 0; db < NDB; ++db) {
            uint4* at = reinterpret_cast<uint4*>(v + db * BLK_BYTES + q * 16);
            if (!nonfinite8(*at)) continue;
            const int key = q >> 3, col = db * 64 + (((q & 7) ^ (key & 7)) << 3);
            take_nonfinite(at, [&](int e, bool pos, bool neg) {
                if (pos) atomicMin(&sh.odd[0][col + e], key0 + key);
                if (neg) atomicMin(&sh.odd[1][col + e], key0 + key);
            });
        }
}
// the accumulator in TMEM of a row that sees `lim` keys
template <int NDB>
__device__ __forceinline__ void restore_values(unsigned t_o, int lim, const ChunkShared& sh) {
#pragma unroll 1
    for (int q = 0; q < NDB * 2; ++q) {
        unsigned y[32];
        tmem_ld32_issue(t_o + q * 32, y);
        tmem_ld_wait(y);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const int col = q * 32 + e;
            float x = __uint_as_float(y[e]);
            if (lim > sh.odd[0][col]) x += INFINITY;
            if (lim > sh.odd[1][col]) x -= INFINITY;
            y[e] = __float_as_uint(x);
        }
        tmem_st32(t_o + q * 32, y);
    }
}

template <int NDB>
__global__ void __launch_bounds__(CH_THREADS, 1)
k_cache_chunk(const __grid_constant__ ChunkMaps maps, const CacheView c, const Ragged r, const AttendJob j, int tq,
              float* __restrict__ ws, unsigned* __restrict__ counters, unsigned* __restrict__ status) {
    constexpr int SLOTS = ch_slots<NDB>();
    constexpr int SLOT_BYTES = NDB * BLK_BYTES;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char* qs = smem;                              // two tiles of queries
    unsigned char* ring = smem + 2 * NDB * BLK_BYTES;
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(smem + 14 * BLK_BYTES);
    volatile int* abort_flag = sh.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = j.h / c.h_kv;
    if ((smem_u32(smem) & 1023u) != 0u) {
        grid_dep_wait();
        if (threadIdx.x == 0) { atomicOr(status, ST_TIMEOUT); status[2] = 499u; }
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(&sh.q_full, 1); mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < SLOTS; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&sh.s_full[t], 1); mbar_init(&sh.p_full[t][0], 4); mbar_init(&sh.p_full[t][1], 4);
            mbar_init(&sh.o_full[t], 1); mbar_init(&sh.o_empty[t], 4);
        }
        sh.abort_flag[0] = 0;
        sh.abort_flag[1] = wait_limit_units(false);
        sh.odd_item = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&sh.tmem_base)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 64) { prefetch_map(&maps.q); prefetch_map(&maps.k); prefetch_map(&maps.v); }
    grid_dep_wait();
    grid_dep_launch_next();
    if (warp == 0) {
        // every CTA's first unit: units of all sequences, 32 at a time (a lane adds up the items of its own)
        auto units_of = [&](int b, int& items) {
            items = 0;
            long long u = 0;
            if (b >= r.B) return u;
            int o;
            const int n = seq_rows(r, b, o), len = seq_len(r, c, b);
            if (blockIdx.x == 0 && n > j.max_new) atomicOr(status, ST_BAD_COUNT);
            const int P = items = ChunkWork::items(n, tq, j.max_new, j.few);
            for (int p = 0; p < P; ++p) u += ChunkWork::units(n, len, p, tq, j.causal);
            return u;
        };
        long long U = 0, I = 0;                    // units, items (both of one key head)
        long long first = 0;
        int first_items = 0;
        for (int b0 = 0; b0 < r.B; b0 += 32) {
            int items;
            const long long u = units_of(b0 + lane, items);
            if (b0 == 0) { first = u; first_items = items; }
            unsigned long long x = (unsigned long long)u, y = (unsigned long long)items;
#pragma unroll
            for (int m = 16; m > 0; m >>= 1) {
                x += __shfl_xor_sync(0xffffffffu, x, m);
                y += __shfl_xor_sync(0xffffffffu, y, m);
            }
            U += (long long)x; I += (long long)y;
        }
        // An equal run for every CTA, but not so short that joining an item's shares (about as long as a unit each, one
        // after the other) takes longer than the units saved: n units in runs of m cost m + n / m, least at sqrt(n).
        const float share = I > 0 ? sqrtf((float)U / (float)I) : 1.f;
        const int turn = I * c.h_kv >= (long long)gridDim.x ? CH_TURN : 0;
        U = (U + turn * I) * c.h_kv;
        const long long per = max((U + gridDim.x - 1) / gridDim.x, (long long)max(share, 1.f));
        const long long at = min(per * blockIdx.x, U), end = min(at + per, U);
        int b = 0, p = 0, head = 0, place = 0;
        long long before = 0;
        if (at < end)
            for (int b0 = 0; b0 < r.B; b0 += 32) {
                int items = first_items;
                long long own = b0 == 0 ? first : units_of(b0 + lane, items);
                own += turn * items;
                long long sum = own;
#pragma unroll
                for (int m = 1; m < 32; m <<= 1) {
                    const long long y = __shfl_up_sync(0xffffffffu, sum, m);
                    if (lane >= m) sum += y;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, at < (before + sum) * c.h_kv);
                if (hit != 0u) {
                    const int l = __ffs(hit) - 1;
                    before += __shfl_sync(0xffffffffu, sum - own, l);
                    b = b0 + l;
                    int o;
                    const int n = seq_rows(r, b, o), len = seq_len(r, c, b);
                    long long rest = at - before * c.h_kv;
                    int u = ChunkWork::units(n, len, 0, tq, j.causal) + turn;
                    while (rest >= (long long)u * c.h_kv) {
                        rest -= (long long)u * c.h_kv;
                        ++p;
                        u = ChunkWork::units(n, len, p, tq, j.causal) + turn;
                    }
                    head = (int)(rest / u);
                    place = (int)(rest % u);
                    break;
                }
                before += __shfl_sync(0xffffffffu, sum, 31);
            }
        if (lane == 0) {
            sh.start[0] = b; sh.start[1] = p; sh.start[2] = head; sh.start[3] = place; sh.start[4] = turn;
            sh.range[0] = at; sh.range[1] = end; sh.range[2] = per;
        }
    } else if (blockIdx.x == 0 && warp == 2) {
        check_ragged(r, c, status, lane, 32);
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const unsigned tmem_base = sh.tmem_base;
    ChunkWork work;
    work.at = sh.range[0]; work.end = sh.range[1]; work.per = sh.range[2];
    work.b = sh.start[0]; work.p = sh.start[1]; work.head = sh.start[2]; work.place = sh.start[3]; work.turn = sh.start[4];
    work.n = work.off = work.len = work.nu = work.P = 0;
    if (work.at < work.end) {
        work.load_seq(r, c, tq, j.max_new, j.few);
        work.nu = ChunkWork::units(work.n, work.len, work.p, tq, j.causal);
    }
    Item it;
    // Registers: 384 x 168 at launch = 128 x 72 + 256 x 216.  (Inside the roles' branches: where they meet the compiler
    // has to assume the smaller number.)
    if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) {
        // ------------------------------------------------ TMA producer
        bool ok = true;
        unsigned put = 0;                          // slots filled: K, V, K, V ...
        const int np = CH_KEYS >> min(c.shift, 7); // pages per key tile
        const int ps = 1 << c.shift;
        int k = 0;                                 // items
        for (; ok && work.next(it, r, c, tq, j.causal, j.max_new, j.few); ++k) {
            if (k > 0) ok = mbar_wait(&sh.q_empty, (unsigned)(k - 1) & 1u, abort_flag, 30);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;                        // (k items' queries have been asked for)
            const int two = it.units[1] > 0 ? 2 : 1;
            if (elect_one()) {
                mbar_expect_tx(&sh.q_full, (unsigned)(two * NDB * tq * G * 128));
                for (int t = 0; t < two; ++t)
                    for (int db = 0; db < NDB; ++db)
                        tma_load_4d(&maps.q, &sh.q_full, qs + (t * NDB + db) * BLK_BYTES, db * BK, 0, it.head, it.row0 + t * tq);
            }
            int page = -1, batch = -1;             // lane l: the sequence's page batch + l
            const int pages = (it.kv + ps - 1) >> c.shift;
            for (int u = 0; u < it.take && ok; ++u) {
                const int p0 = (it.ku + u) * np;
                if (batch < 0 || p0 + np > batch + 32) {
                    batch = p0;
                    page = p0 + lane < pages ? page_of(c, it.b, p0 + lane, status) : -1;
                }
                const int mine = __shfl_sync(0xffffffffu, page, (p0 - batch + lane) & 31);
                const bool have = lane < np && mine >= 0;
                const unsigned bytes = (unsigned)__popc(__ballot_sync(0xffffffffu, have)) * (unsigned)(ps * 128 * NDB);
                for (int kv = 0; kv < 2 && ok; ++kv, ++put) {
                    const int st = put % SLOTS;
                    ok = mbar_wait(&sh.empty[st], ((put / SLOTS) & 1u) ^ 1u, abort_flag, 31);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(&sh.full[st], bytes);
                    __syncwarp();
                    if (have)
                        for (int db = 0; db < NDB; ++db)
                            tma_load_4d(kv == 0 ? &maps.k : &maps.v, &sh.full[st],
                                        ring + st * SLOT_BYTES + db * BLK_BYTES + lane * ps * 128, db * BK, 0, it.head, mine);
                }
            }
        }
        // every copy has to land before the CTA may exit
        if (lane == 0) {
            const unsigned long long t0 = global_ns();
            while (k > 0 && !mbar_try(&sh.q_full, (unsigned)(k - 1) & 1u))
                if (past_limit(2 * (global_ns() - t0), abort_flag)) { *abort_flag = 33; break; }
            for (unsigned i = put > (unsigned)SLOTS ? put - SLOTS : 0u; i < put; ++i)
                while (!mbar_try(&sh.full[i % SLOTS], (i / SLOTS) & 1u))
                    if (past_limit(2 * (global_ns() - t0), abort_flag)) { *abort_flag = 33; break; }
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issuer (the elected lane; the warp stays together)
        bool ok = true;
        unsigned got = 0;                          // slots consumed
        unsigned n_p[2] = {0u, 0u}, n_o[2] = {0u, 0u};
        const unsigned lead = elect_one();
        const unsigned idesc_s = instr_desc(CH_KEYS);
        const unsigned idesc_o = instr_desc(NDB * 64) | (1u << 16);          // right operand MN-major
        // asks warps 2 and 3 for the values of unit u, load number `slot`, a unit ahead, if not every row sees them all; one
        // request at a time: it has been answered before the next one is made
        bool asked = false;
        auto look = [&](int u, unsigned slot) {
            const int key0 = (it.ku + u) * CH_KEYS;
            if (it.first_lim - key0 >= CH_KEYS) return;
            if (lane == 0) {
                sh.look.slot = (int)slot;
                sh.look.from = max(it.first_lim - key0, 0);
                sh.look.to = min(max(it.kv - key0, 0), CH_KEYS);
            }
            __syncwarp();
            asm volatile("bar.arrive 1, 96;" ::: "memory");
            asked = true;
        };
        auto looked = [&]() {
            asm volatile("bar.sync 2, 96;" ::: "memory");
            asked = false;
            return (sh.look.found[0] | sh.look.found[1]) != 0;
        };
        for (int k = 0; ok && work.next(it, r, c, tq, j.causal, j.max_new, j.few); ++k) {
            const int nt[2] = {ChunkWork::tiles_of(it, 0), ChunkWork::tiles_of(it, 1)};
            const int two = it.units[1] > 0 ? 2 : 1;
            look(0, got + 1);
            ok = mbar_wait(&sh.q_full, (unsigned)k & 1u, abort_flag, 35);
            auto wait_slot = [&](unsigned i, int where) {
                ok = ok && mbar_wait(&sh.full[i % SLOTS], (i / SLOTS) & 1u, abort_flag, where);
                ok = __all_sync(0xffffffffu, ok);
            };
            auto issue_s = [&](int t, unsigned slot) {
                const unsigned a = desc_lo(smem_u32(qs + t * NDB * BLK_BYTES));
                const unsigned b = desc_lo(smem_u32(ring + (slot % SLOTS) * SLOT_BYTES));
#pragma unroll
                for (int q = 0; q < NDB * 4; ++q)
                    umma_ss(tmem_base + t * 128, a + (q >> 2) * (BLK_BYTES >> 4) + 2 * (q & 3), b + (q >> 2) * (BLK_BYTES >> 4) + 2 * (q & 3), idesc_s, q != 0, lead);
                umma_commit_lead(&sh.s_full[t], lead);
            };
            wait_slot(got, 36);
            if (!ok) break;
            tcgen05_fence_after();
            {
                for (int t = 0; t < two; ++t)
                    if (nt[t] > 0) issue_s(t, got);
                umma_commit_lead(&sh.empty[got % SLOTS], lead);
                if (it.take == 1) umma_commit_lead(&sh.q_empty, lead);
            }
            for (int u = 0; u < it.take && ok; ++u, got += 2) {
                const unsigned sv = got + 1, sk = got + 2;
                wait_slot(sv, 38);
                if (!ok) break;
                const bool ahead = u + 1 < it.take;
                if (ahead) wait_slot(sk, 37);
                if (!ok) break;
                // values that a row does not see meet probabilities of zero: warps 2 and 3 have looked at them
                if (asked) {
                    if (looked()) {
                        if (sh.odd_item != k + 1) {                          // the entries of items before: nobody needs them any more
                            for (int t = 0; t < 2; ++t)
                                if (n_o[t] > 0) ok = ok && mbar_wait(&sh.o_empty[t], (n_o[t] - 1u) & 1u, abort_flag, 44);
                            ok = __all_sync(0xffffffffu, ok);
                            if (!ok) break;
                            for (int q = lane; q < 2 * 128; q += 32) sh.odd[0][q] = INT_MAX;
                            __syncwarp();
                        }
                        clean_values<NDB>(ring + (sv % SLOTS) * SLOT_BYTES, sh.look.from, sh.look.to, (it.ku + u) * CH_KEYS, lane, sh);
                        if (lane == 0) sh.odd_item = k + 1;
                        __threadfence_block();
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                }
                if (ahead) look(u + 1, sv + 2);
                for (int t = 0; t < two; ++t) {
                    if (u >= nt[t]) continue;
                    // the accumulator is overwritten: the previous item's rows have been read out
                    if (u == 0 && n_o[t] > 0) ok = mbar_wait(&sh.o_empty[t], (n_o[t] - 1u) & 1u, abort_flag, 40);
                    const unsigned b = desc_lo_mn(smem_u32(ring + (sv % SLOTS) * SLOT_BYTES), BLK_BYTES);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                            // as soon as half of the probabilities are there
                        ok = ok && mbar_wait(&sh.p_full[t][h], n_p[t] & 1u, abort_flag, 39);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        tcgen05_fence_after();
#pragma unroll
                            for (int q = 4 * h; q < 4 * h + 4; ++q)
                                umma_ts(tmem_base + 256 + t * 128, tmem_base + t * 128 + q * 8, b + q * (2048 >> 4), idesc_o, (u | q) != 0, lead);
                    }
                    if (!ok) break;
                    ++n_p[t];
                    {
                        if (u + 1 < nt[t]) issue_s(t, sk);
                        else umma_commit_lead(&sh.o_full[t], lead);
                    }
                    if (u + 1 >= nt[t]) ++n_o[t];
                }
                if (!ok) break;
                {
                    umma_commit_lead(&sh.empty[sv % SLOTS], lead);
                    if (ahead) umma_commit_lead(&sh.empty[sk % SLOTS], lead);
                    if (u + 2 == it.take) umma_commit_lead(&sh.q_empty, lead);   // the item's last scores are under way
                }
            }
        }
        if (asked) looked();
        if (lane == 0) sh.look.slot = -1;
        __syncwarp();
        asm volatile("bar.arrive 1, 96;" ::: "memory");
    } else if (warp < 4) {
        // ------------------------------------------------ values that meet zero probabilities (see clean_values)
        bool ok = true;
        for (;;) {
            asm volatile("bar.sync 1, 96;" ::: "memory");
            const int slot = sh.look.slot, from = sh.look.from, to = sh.look.to;
            if (slot < 0) break;
            // (the slot's load before this one is long done: warp 1 has waited for it)
            if (ok) ok = mbar_wait(&sh.full[(unsigned)slot % SLOTS], ((unsigned)slot / SLOTS) & 1u, abort_flag, 45);
            ok = __all_sync(0xffffffffu, ok);
            bool odd = false;
            if (ok) {
                unsigned char* v = ring + ((unsigned)slot % SLOTS) * SLOT_BYTES;
                const int i = (warp - 2) * 32 + lane;
#pragma unroll 4
                for (int q = from * 8 + i; q < to * 8; q += 64)
#pragma unroll
                    for (int db = 0; db < NDB; ++db) odd |= nonfinite8(*reinterpret_cast<const uint4*>(v + db * BLK_BYTES + q * 16));
                for (int q = to * 8 + i; q < CH_KEYS * 8; q += 64)           // nobody's: whatever it is becomes zero
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
                        *reinterpret_cast<uint4*>(v + db * BLK_BYTES + q * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            odd = __any_sync(0xffffffffu, odd);
            if (lane == 0) sh.look.found[warp - 2] = odd;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            asm volatile("bar.arrive 2, 96;" ::: "memory");
        }
    } else {
        // ------------------------------------------------ softmax and output
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int quad = warp & 3, t = (warp - 4) >> 2;
        const int i = quad * 32 + lane;                                     // row of the tile
        const unsigned t_s = tmem_base + ((unsigned)(quad * 32) << 16) + t * 128;
        const unsigned t_o = t_s + 256;
        const int tok = i / G, g = i - tok * G;                             // within the tile
        bool ok = true;
        unsigned n_s = 0, n_o = 0;
        for (int k = 1; work.next(it, r, c, tq, j.causal, j.max_new, j.few); ++k) {
            if (it.units[t] == 0 && t == 1) continue;                       // no rows in this tile
            const int nt = ChunkWork::tiles_of(it, t);
            const int tok_i = t * tq + tok;                                 // within the item
            const bool live = tok < tq && tok_i < it.n_tok;
            const int lim = !live ? 0 : j.causal ? min(it.first_lim + tok_i, it.kv) : it.kv;
            const int lim_tile = j.causal ? it.first_lim + t * tq : it.kv;   // smallest of the tile's live rows
            float m = -INFINITY, l = 0.f;
            for (int u = 0; u < nt; ++u) {
                if (ok) ok = mbar_wait(&sh.s_full[t], n_s & 1u, abort_flag, 41);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ++n_s;
                tcgen05_fence_after();
                unsigned x[2][32], z[2][32];
                const int k0 = (it.ku + u) * CH_KEYS;
                tmem_ld32_issue(t_s, x[0]);
                tmem_ld32_issue(t_s + 32, x[1]);
                tmem_ld32_issue(t_s + 64, z[0]);
                tmem_ld32_issue(t_s + 96, z[1]);
                tmem_ld_wait(x[0]); tmem_ld_wait(x[1]); tmem_ld_wait(z[0]); tmem_ld_wait(z[1]);
                if (k0 + CH_KEYS > lim_tile) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (k0 + q * 32 + e >= lim) x[q][e] = 0xff800000u;
                            if (k0 + 64 + q * 32 + e >= lim) z[q][e] = 0xff800000u;
                        }
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    mx[0] = max3(mx[0], x[0][e], x[0][e + 1]);
                    mx[1] = max3(mx[1], x[1][e], x[1][e + 1]);
                    mx[2] = max3(mx[2], z[0][e], z[0][e + 1]);
                    mx[3] = max3(mx[3], z[1][e], z[1][e + 1]);
                }
                const float top = max3(mx[0], __float_as_uint(mx[1]), __float_as_uint(max3(mx[2], __float_as_uint(mx[3]), __float_as_uint(mx[3])))) * j.scale;
                const float m_new = fmaxf(m, top);
                if (!(top < INFINITY)) l = NAN;                             // a NaN, or an overflow, that the row sees
                if (u == 0) {
                    m = m_new;
                } else {
                    const bool raise = m_new > m + CH_LAG;
                    if (__any_sync(0xffffffffu, raise)) {
                        // (the scores' barrier also says that the previous tile's product is done)
                        const float f = raise ? (m > -INFINITY ? ex2_approx(m - m_new) : 0.f) : 1.0f;
#pragma unroll
                        for (int q = 0; q < NDB * 2; ++q) {
                            unsigned y[32];
                            tmem_ld32_issue(t_o + q * 32, y);
                            tmem_ld_wait(y);
#pragma unroll
                            for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * f);
                            tmem_st32(t_o + q * 32, y);
                        }
                        l *= f;
                        if (raise) m = m_new;
                    }
                }
                const float ref = m > -INFINITY ? m : 0.f;
                // (one copy of this code for both halves: with all of it unrolled a key tile's instructions no longer fit the
                // instruction cache nearest to the scheduler)
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    unsigned w[32];
                    exp_pairs(x[0], x[1], j.scale, -ref, w, l);
                    tmem_st32(t_s + h * 32, w);
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.p_full[t][h]);
#pragma unroll
                    for (int e = 0; e < 32; ++e) { x[0][e] = z[0][e]; x[1][e] = z[1][e]; }
                }
            }
            if (!ok) break;
            // ---- the item's rows
            if (nt > 0) {
                ok = mbar_wait(&sh.o_full[t], n_o & 1u, abort_flag, 43);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                ++n_o;
                tcgen05_fence_after();
                // (no later item's number can be there before this one's o_empty)
                if (sh.odd_item == k) restore_values<NDB>(t_o, lim, sh);
            }
            __nv_bfloat16* dst = j.out + (int64_t)(it.row0 + tok_i) * j.ldo + ((int64_t)it.head * G + g) * c.d;
            // of a row whose sum is 0: it sees no slot, and gets zeros, or all of its scores are -inf
            const float none = lim > 0 ? NAN : 0.f;
            if (it.pieces == 1) {
                const float f = l == 0.f ? none : 1.0f / l;                  // (NaN stays)
#pragma unroll
                for (int q = 0; q < NDB * 2; ++q) {
                    unsigned y[32];
                    if (nt > 0) { tmem_ld32_issue(t_o + q * 32, y); tmem_ld_wait(y); }
                    else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = 0u;
                    }
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            if (q * 32 + e < c.d) {
                                unsigned w[4];
#pragma unroll
                                for (int v = 0; v < 4; ++v) {
                                    const __nv_bfloat162 p = __floats2bfloat162_rn(__uint_as_float(y[e + 2 * v]) * f, __uint_as_float(y[e + 2 * v + 1]) * f);
                                    w[v] = *reinterpret_cast<const unsigned*>(&p);
                                }
                                *reinterpret_cast<uint4*>(dst + q * 32 + e) = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                    }
                }
            } else if (__any_sync(0xffffffffu, live)) {
                // a share of an item: unnormalised, four columns of a row together (a warp's lanes write next to each other)
                auto part = [&](int piece) { return ws + (2 * (int64_t)(it.c0 + piece) + (piece == 0 ? 1 : 0)) * PART_FLOATS; };
                const int at = t * 128 + i;
                unsigned* ctr = counters + ((size_t)it.c1 * 2 + t) * 4 + quad;
                // the one that comes last joins the shares, its own out of TMEM: where the others are all there already, it
                // need not be written
                unsigned last = 0u;
                if (lane == 0) last = ld_acquire(ctr) + 1u == (unsigned)it.pieces;
                last = __shfl_sync(0xffffffffu, last, 0);
                if (!last) {
                    float4* mine = reinterpret_cast<float4*>(part(it.piece)) + at;
#pragma unroll
                    for (int q = 0; q < NDB * 2; ++q) {
                        unsigned y[32];
                        if (nt > 0) { tmem_ld32_issue(t_o + q * 32, y); tmem_ld_wait(y); }
                        else {
#pragma unroll
                            for (int e = 0; e < 32; ++e) y[e] = 0u;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            __stcg(mine + (q * 8 + e) * 256, make_float4(__uint_as_float(y[4 * e]), __uint_as_float(y[4 * e + 1]),
                                                                         __uint_as_float(y[4 * e + 2]), __uint_as_float(y[4 * e + 3])));
                    }
                    __stcg(part(it.piece) + 128 * 256 + at, m);
                    __stcg(part(it.piece) + 128 * 256 + 256 + at, l);
                    __threadfence();
                    __syncwarp();
                    if (lane == 0) last = atomicAdd(ctr, 1u) + 1u == (unsigned)it.pieces;
                    last = __shfl_sync(0xffffffffu, last, 0);
                }
                if (last) {
                    if (lane == 0) *ctr = 0u;                                // as the next call finds it
                    __threadfence();
                    float M = m, L = 0.f;
#pragma unroll 2
                    for (int p = 0; p < it.pieces; ++p)
                        if (p != it.piece) M = fmaxf(M, __ldcg(part(p) + 128 * 256 + at));
                    const float Mr = M > -INFINITY ? M : 0.f;
#pragma unroll 2
                    for (int p = 0; p < it.pieces; ++p) {
                        const bool own = p == it.piece;
                        L = fmaf(own ? l : __ldcg(part(p) + 128 * 256 + 256 + at),
                                 ex2_approx((own ? m : __ldcg(part(p) + 128 * 256 + at)) - Mr), L);
                    }
                    const float f = L == 0.f ? none : 1.0f / L;
                    // 64 columns at a time, in the order of the keys whoever joins them
#pragma unroll 1
                    for (int q = 0; q < NDB; ++q) {
                        float y[64];
#pragma unroll
                        for (int e = 0; e < 64; ++e) y[e] = 0.f;
#pragma unroll 1
                        for (int p = 0; p < it.pieces; ++p) {
                            if (p != it.piece) {
                                const float4* o = reinterpret_cast<const float4*>(part(p)) + q * 16 * 256 + at;
                                float4 z[16];
#pragma unroll
                                for (int e = 0; e < 16; ++e) z[e] = __ldcg(o + e * 256);
                                const float fp = ex2_approx(__ldcg(part(p) + 128 * 256 + at) - Mr);
#pragma unroll
                                for (int e = 0; e < 16; ++e) {
                                    y[4 * e] = fmaf(z[e].x, fp, y[4 * e]);
                                    y[4 * e + 1] = fmaf(z[e].y, fp, y[4 * e + 1]);
                                    y[4 * e + 2] = fmaf(z[e].z, fp, y[4 * e + 2]);
                                    y[4 * e + 3] = fmaf(z[e].w, fp, y[4 * e + 3]);
                                }
                            } else if (nt > 0) {
                                const float fp = ex2_approx(m - Mr);
#pragma unroll
                                for (int v = 0; v < 2; ++v) {
                                    unsigned o[32];
                                    tmem_ld32_issue(t_o + q * 64 + v * 32, o);
                                    tmem_ld_wait(o);
#pragma unroll
                                    for (int e = 0; e < 32; ++e) y[v * 32 + e] = fmaf(__uint_as_float(o[e]), fp, y[v * 32 + e]);
                                }
                            }
                        }
                        if (live) {
#pragma unroll
                            for (int e = 0; e < 64; e += 8)
                                if (q * 64 + e < c.d) {
                                    unsigned w[4];
#pragma unroll
                                    for (int v = 0; v < 4; ++v) {
                                        const __nv_bfloat162 h = __floats2bfloat162_rn(y[e + 2 * v] * f, y[e + 2 * v + 1] * f);
                                        w[v] = *reinterpret_cast<const unsigned*>(&h);
                                    }
                                    *reinterpret_cast<uint4*>(dst + q * 64 + e) = make_uint4(w[0], w[1], w[2], w[3]);
                                }
                        }
                    }
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (nt > 0 && lane == 0) mbar_arrive(&sh.o_empty[t]);
        }
        tcgen05_fence_before();
    }
    __syncthreads();
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
    if (threadIdx.x == 0 && sh.abort_flag[0] != 0) {
        atomicOr(status, ST_TIMEOUT);
        status[2] = 400u + (unsigned)sh.abort_flag[0];
    }
}

// queries as (element, head of the group, key head, token): a box is 64 elements of G heads x tq tokens
bool encode_queries(CUtensorMap* map, const CacheView& c, const Ragged& r, const AttendJob& j, int G, int tq) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)G, (cuuint64_t)c.h_kv, (cuuint64_t)r.N};
    const cuuint64_t strides[3] = {(cuuint64_t)c.d * 2, (cuuint64_t)G * c.d * 2, (cuuint64_t)j.ldq * 2};
    const cuuint32_t box[4] = {(cuuint32_t)BK, (cuuint32_t)G, 1, (cuuint32_t)tq};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16*>(j.Q), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NDB>
cudaError_t run_chunk(ada_ctx* ctx, const ChunkMaps& maps, const CacheView& c, const Ragged& r, const AttendJob& j, int tq,
                      cudaStream_t s) {
    cudaError_t e = allow_smem(ctx, 11 + NDB, k_cache_chunk<NDB>, ch_smem<NDB>());                // bits 12, 13
    if (e != cudaSuccess) return e;
    prof_begin(ctx, K_CACHE_CHUNK, s);
    e = launch_k(ctx, k_cache_chunk<NDB>, dim3(ctx->sm_count), dim3(CH_THREADS), ch_smem<NDB>(), s, maps, c, r, j, tq,
                 ctx->cache_part, ctx->cache_ctr, ctx->status);
    prof_end(ctx, s);
    return e;
}

}  // namespace

cudaError_t launch_cache_chunk(ada_ctx* ctx, const CacheView& c, const Ragged& r, const AttendJob& j, cudaStream_t s) {
    const int G = j.h / c.h_kv, tq = 128 / G;
    const int ps = 1 << c.shift;
    ChunkMaps maps;
    if (!encode_pages(&maps.k, c, c.k, ps < 128 ? ps : 128) || !encode_pages(&maps.v, c, c.v, ps < 128 ? ps : 128) ||
        !encode_queries(&maps.q, c, r, j, G, tq))
        return cudaErrorInvalidValue;
    return c.d > 64 ? run_chunk<2>(ctx, maps, c, r, j, tq, s) : run_chunk<1>(ctx, maps, c, r, j, tq, s);
}

size_t cache_part_floats() { return (size_t)PART_FLOATS; }

}  // namespace ada
