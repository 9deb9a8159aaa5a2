"""The operators on a paged cache in 64 bits, token by token, for the tests (torch on the CPU, plain loops)."""
import math

import torch

F64 = torch.float64


class Pages:
    """A cache on the CPU: K, V (pages, hk, ps, d), table (B, P), all tensors of one test."""

    def __init__(self, K, V, table, kmin=None, kmax=None):
        self.K, self.V, self.table, self.kmin, self.kmax = K, V, table, kmin, kmax
        self.ps = K.shape[2]

    def slots(self, b, head, n):
        """Keys and values of the first n slots of sequence b, in 64 bits."""
        at = [(int(self.table[b, t // self.ps]), t % self.ps) for t in range(n)]
        return (torch.stack([X[p, head, s].to(F64) for p, s in at]) if n else torch.zeros((0, X.shape[3]), dtype=F64)
                for X in (self.K, self.V))


def sees(n, length, i, causal):
    return max(length - n + i + 1, 0) if causal else length


def attend(cache, Q, off, length, h_kv, causal=True, scale=0.0, lists=None):
    """(out, sum of p |v|): rows of no sequence are None.  lists[i][j]: pages of token i, key head j."""
    N, h, d = Q.shape
    G = h // h_kv
    scale = scale or 1.0 / math.sqrt(d)
    out, weight = torch.zeros((N, h, d), dtype=F64), torch.zeros((N, h, d), dtype=F64)
    for b in range(len(off) - 1):
        n = off[b + 1] - off[b]
        if n == 0:
            continue
        for j in range(h_kv):
            k, v = cache.slots(b, j, length[b])
            for i in range(n):
                row, lim = off[b] + i, sees(n, length[b], i, causal)
                pos = torch.arange(lim)
                if lists is not None:
                    pos = pos[torch.isin(pos // cache.ps, torch.tensor(lists[row][j], dtype=torch.long))]
                if len(pos) == 0:
                    continue
                s = Q[row, j * G:(j + 1) * G].to(F64) @ k[pos].T * scale
                p = torch.softmax(s, dim=1)
                out[row, j * G:(j + 1) * G] = p @ v[pos]
                weight[row, j * G:(j + 1) * G] = p @ v[pos].abs()
    return out, weight


def tolerance(out, weight, V):
    """The probabilities are rounded to bf16 (half a step: 2^-8 of each), the output once more; what fp32 adds (scores
    of up to a few dozen, sums over the keys) is below 2^-12 of the largest value."""
    return 2.0 ** -8 * weight + 2.0 ** -8 * out.abs() + 2.0 ** -12 * float(V.abs().max())


def select(cache, Q, off, length, h_kv, k, n_first, n_last, causal=True):
    """Lists as Python lists, by token and key head (None for rows of no sequence)."""
    N, h, d = Q.shape
    G = h // h_kv
    got = [None] * N
    for b in range(len(off) - 1):
        n = off[b + 1] - off[b]
        for i in range(n):
            row = off[b] + i
            seen = -(-sees(n, length[b], i, causal) // cache.ps)
            got[row] = []
            for j in range(h_kv):
                if seen <= k:
                    got[row].append(list(range(seen)))
                    continue
                q = Q[row, j * G:(j + 1) * G].to(F64)
                score = []
                for p in range(seen):
                    page = int(cache.table[b, p])
                    lo, hi = cache.kmin[page, j].to(F64), cache.kmax[page, j].to(F64)
                    forced = p < n_first or p >= seen - n_last
                    score.append(math.inf if forced else float(torch.maximum(q * lo, q * hi).sum()))
                order = sorted(range(seen), key=lambda p: (-score[p], p))
                got[row].append(sorted(order[:k]))
    return got


def turned(x, pos, inv_freq, pairs):
    """Rotation of the first 2 len(inv_freq) elements of a head."""
    x = x.clone()
    half = len(inv_freq)
    a = pos * inv_freq
    i = torch.arange(half)
    u, v = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    x[..., u], x[..., v] = x[..., u] * a.cos() - x[..., v] * a.sin(), x[..., v] * a.cos() + x[..., u] * a.sin()
    return x


def normed(x, w, eps):
    return x if w is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.to(F64)


def append(cache, K, V, off, length, Q=None, q_norm=None, k_norm=None, eps=1e-6, inv_freq=None, pairs=False, pos0=None,
           lists=None):
    """Writes to copies: (K64, V, kmin64, kmax64, q64, lengths).  lists[b]: the tokens that are kept."""
    f = inv_freq if inv_freq is not None else torch.zeros(0, dtype=F64)
    K64, V2 = cache.K.to(F64), cache.V.clone()
    lo, hi = (x.to(F64) if x is not None else None for x in (cache.kmin, cache.kmax))
    q64 = None if Q is None else Q.to(F64).clone()
    lengths = list(length)
    for b in range(len(off) - 1):
        n = off[b + 1] - off[b]
        first = length[b] if pos0 is None else pos0[b]
        for i in range(n if Q is not None else 0):
            q64[off[b] + i] = turned(normed(Q[off[b] + i].to(F64), q_norm, eps), first + i, f, pairs)
        kept = range(n) if lists is None else lists[b]
        for t, i in enumerate(kept):
            slot = length[b] + t
            page = int(cache.table[b, slot // cache.ps])
            K64[page, :, slot % cache.ps] = turned(normed(K[off[b] + i].to(F64), k_norm, eps), first + i, f, pairs)
            V2[page, :, slot % cache.ps] = V[off[b] + i]
        lengths[b] = length[b] + len(kept)
        for p in range(length[b] // cache.ps, -(-lengths[b] // cache.ps)):
            if len(kept) and lo is not None:
                page = int(cache.table[b, p])
                live = K64[page, :, :min(cache.ps, lengths[b] - p * cache.ps)]
                lo[page], hi[page] = live.amin(1), live.amax(1)
    return K64, V2, lo, hi, q64, lengths
