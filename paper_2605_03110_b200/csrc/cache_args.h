// Argument checks of the calls on a paged cache (no CUDA in here; pointers are looked at, not followed).
#pragma once

#include <stdint.h>

#include "../../include/ada.h"

namespace ada {

constexpr int SELECT_MAX_PAGES = 16384;  // of a sequence: the scores of a row are in shared memory
constexpr int MAX_GROUP = 128;           // heads that share a key head: rows of one tile

inline bool lies16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool between(int64_t x, int64_t lo, int64_t hi) { return x >= lo && x <= hi; }

// log2 of the page size, -1 if there is no kernel for it
inline int page_shift(int64_t page_size) {
    for (int s = 4; s <= 7; ++s)
        if (page_size == (int64_t)1 << s) return s;
    return -1;
}

inline ada_status check_cache(const ada_kv_cache* kv, int64_t B, const int32_t* off, const int32_t* len, int64_t N,
                              ada_dtype dt) {
    if (kv == nullptr || off == nullptr || len == nullptr) return ADA_ERR_INVALID_ARG;
    if (kv->k == nullptr || kv->v == nullptr || kv->table == nullptr || (kv->kmin == nullptr) != (kv->kmax == nullptr))
        return ADA_ERR_INVALID_ARG;
    if (dt != ADA_F32 && dt != ADA_BF16) return ADA_ERR_INVALID_ARG;
    if (B < 1 || N < 1 || kv->n_pages < 1 || kv->max_pages < 1 || kv->table_ld < kv->max_pages || kv->h_kv < 1 ||
        kv->d_h < 1 || kv->page_size < 1)
        return ADA_ERR_INVALID_ARG;
    if (dt != ADA_BF16 || kv->d_h % 16 != 0 || kv->d_h > 128) return ADA_ERR_UNSUPPORTED;
    const int shift = page_shift(kv->page_size);
    if (shift < 0) return ADA_ERR_UNSUPPORTED;
    // indexes of rows, pages, slots of a sequence and TMA coordinates are 32-bit; addresses are not
    if (!between(B, 1, 1 << 20) || !between(N, 1, 1 << 28) || !between(kv->n_pages, 1, 0x7fffffff) ||
        !between(kv->h_kv, 1, 4096) || !between(kv->max_pages, 1, (int64_t)0x3fffffff >> shift) ||
        kv->table_ld >= (int64_t)1 << 40)
        return ADA_ERR_UNSUPPORTED;
    if (kv->page_stride < kv->h_kv * kv->page_size * kv->d_h) return ADA_ERR_INVALID_ARG;
    if (kv->page_stride % 8 != 0 || kv->page_stride >= (int64_t)1 << 38 || !lies16(kv->k) || !lies16(kv->v) ||
        !lies16(kv->kmin) || !lies16(kv->kmax))
        return ADA_ERR_UNSUPPORTED;
    return ADA_OK;
}

// rows of `heads` heads side by side
inline ada_status check_rows(const void* p, int64_t heads, int64_t d, int64_t ld) {
    if (p == nullptr || heads < 1) return ADA_ERR_INVALID_ARG;
    if (heads > 4096 * MAX_GROUP) return ADA_ERR_UNSUPPORTED;
    if (ld < heads * d) return ADA_ERR_INVALID_ARG;
    return !lies16(p) || ld % 8 != 0 || ld >= (int64_t)1 << 38 ? ADA_ERR_UNSUPPORTED : ADA_OK;
}

inline ada_status check_heads(const ada_kv_cache* kv, int64_t h) {
    if (h < 1 || h % kv->h_kv != 0) return ADA_ERR_INVALID_ARG;
    return h / kv->h_kv <= MAX_GROUP ? ADA_OK : ADA_ERR_UNSUPPORTED;
}

// scale of the scores (0: 1 / sqrt(d_h)) is one
inline bool scale_ok(double scale) { return scale >= 0.0 && scale <= 1e30; }   // also rejects NaN

// where the results of an attention call go: apart from the queries, or over them row by row (a row is read before it is written)
inline ada_status check_out(const void* Q, int64_t ldq, const void* out, int64_t ldo) {
    return out == Q && ldo != ldq ? ADA_ERR_INVALID_ARG : ADA_OK;
}

// int32 arrays of na and nb entries have none in common (b may be NULL)
inline bool apart(const int32_t* a, int64_t na, const int32_t* b, int64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return b == nullptr || x + (uintptr_t)na * 4 <= y || y + (uintptr_t)nb * 4 <= x;
}

inline ada_status check_append(const ada_kv_cache* kv, int64_t B, const int32_t* off, const int32_t* len, int64_t N,
                               const int32_t* len_out, const int32_t* pos0, const void* K, int64_t ldk,
                               const void* V, int64_t ldv, const void* Q, int64_t h, int64_t ldq, const void* q_out,
                               int64_t ldqo, const void* q_norm, const void* k_norm, double eps, const double* inv_freq,
                               int64_t rot, const int32_t* rep_idx, const int32_t* rep_cnt, uint32_t flags) {
    ada_status st;
    if ((st = check_rows(K, kv->h_kv, kv->d_h, ldk)) != ADA_OK || (st = check_rows(V, kv->h_kv, kv->d_h, ldv)) != ADA_OK)
        return st;
    if ((flags & ~ADA_ROPE_PAIRS) != 0 || (rep_idx == nullptr) != (rep_cnt == nullptr)) return ADA_ERR_INVALID_ARG;
    // the new lengths are written while other blocks still read these
    if (len_out != nullptr && !(apart(len_out, B, len, B) && apart(len_out, B, off, B + 1) && apart(len_out, B, pos0, B) &&
                                apart(len_out, B, rep_cnt, B) && apart(len_out, B, rep_idx, N)))
        return ADA_ERR_INVALID_ARG;
    if (Q != nullptr) {
        if ((st = check_rows(Q, h, kv->d_h, ldq)) != ADA_OK || (st = check_rows(q_out, h, kv->d_h, ldqo)) != ADA_OK) return st;
        if ((st = check_out(Q, ldq, q_out, ldqo)) != ADA_OK) return st;
    } else if (q_out != nullptr || q_norm != nullptr) {
        return ADA_ERR_INVALID_ARG;
    }
    if (inv_freq != nullptr) {
        if (rot < 2 || rot > kv->d_h) return ADA_ERR_INVALID_ARG;
        if (rot % 16 != 0) return ADA_ERR_UNSUPPORTED;
    }
    if ((q_norm != nullptr || k_norm != nullptr) && !(eps >= 0.0 && eps <= 1e30)) return ADA_ERR_INVALID_ARG;
    return lies16(q_norm) && lies16(k_norm) ? ADA_OK : ADA_ERR_UNSUPPORTED;
}

inline ada_status check_select(const ada_kv_cache* kv, int64_t k, int64_t n_first, int64_t n_last, const int32_t* blk_idx,
                               const int32_t* blk_cnt, uint32_t flags) {
    if (kv->kmin == nullptr || blk_idx == nullptr || blk_cnt == nullptr || (flags & ~ADA_ATTN_CAUSAL) != 0 || k < 1 ||
        n_first < 0 || n_last < 0 || n_first > k || n_last > k - n_first)
        return ADA_ERR_INVALID_ARG;
    return kv->max_pages <= SELECT_MAX_PAGES && k <= SELECT_MAX_PAGES ? ADA_OK : ADA_ERR_UNSUPPORTED;
}

}  // namespace ada
