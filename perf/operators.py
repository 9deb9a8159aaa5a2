"""Performance cases of the operators on a paged key / value cache.

After a prompt a model goes on from the keys and values that it keeps.  Each case is one call that a
serving program makes for one layer: new tokens are appended to the cache (`append`), attend to it
(`attend`), pick the pages that matter to them (`select`) and attend to those alone (`blocks`).

The cache is a pool of pages of `ps` tokens: K and V are (pages, hk, ps, d) bf16, `table` names the pages
of every sequence in order, `kmin` and `kmax` (pages, hk, d) hold the elementwise bounds of a page's keys.
New tokens of all sequences stand one after the other, those of sequence b at off[b] .. off[b + 1].

  append  per-head RMS norm of queries and keys (`norm`), rotation of their first `rot` elements
          (`inter`: neighbouring elements are a pair, else element i and i + rot / 2), queries written
          out, keys and values written behind the `len` tokens that the sequence has, the bounds of every
          page that was written.  `keep` < 1: only a list of each sequence's tokens goes to the cache (the
          representatives of a prompt), rotated at the positions that they have in the prompt.
  attend  softmax(q K^T / sqrt(d)) V for every new token and head over the sequence's cache, the new
          tokens' own keys included; head i reads key / value head i // (h // hk).  `causal`: a token
          sees itself and what came before it, else all.
  select  for every new token and key / value head the `k` pages with the largest
          sum over its heads and the elements of max(q * kmax, q * kmin), an upper bound of the sum over the
          heads of q . key for every key of the page; the first and the last page always; ascending, -1 behind
          the count; a token that sees k pages or fewer takes them all.  Ties go to the lower page.
  blocks  attend, over the listed pages alone.

  B sequences get up to `new` tokens each behind up to `past` older ones.  `spread`: the lengths vary from
  sequence to sequence; `mixed`: every other sequence gets a single token (a step of continuous batching).
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
THETA = 10000.0
_CTX = {}


def _case(name, op, h, hk, d, ps, B, new, past, spread=False, mixed=False, causal=True, norm=False, rot=0,
          inter=False, keep=1.0, k=0):
    c = {"op": op, "h": h, "hk": hk, "d": d, "ps": ps, "B": B, "new": new, "past": past, "spread": spread,
         "mixed": mixed, "causal": causal, "norm": norm, "rot": rot, "inter": inter, "keep": keep, "k": k}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one decoding step of 64 sequences, grouped heads, normed queries and keys: launch latency counts
        _case("append-step-64", "append", 32, 8, 128, 64, 64, 1, 2047, spread=True, norm=True, rot=128),
        # prompts of four sequences through a GPT-J-sized layer: neighbouring pairs, half of the head rotated
        _case("append-prompts", "append", 32, 32, 128, 64, 4, 2005, 200, spread=True, rot=64, inter=True),
        # the representatives of a long OPT-6.7B-sized prompt go to the cache, a sixth of its tokens
        _case("append-reps-8192", "append", 32, 32, 128, 64, 1, 8192, 0, rot=128, keep=1377 / 8192),
        # the smallest call: one token of a GPT-2-sized model, small pages
        _case("attend-step-1", "attend", 12, 12, 64, 16, 1, 1, 776),
        # one decoding step of a batch with grouped heads, lengths of all sizes
        _case("attend-step-64", "attend", 32, 8, 128, 64, 64, 1, 16383, spread=True),
        # a decoding step of two long texts: few rows, the keys have to be split
        _case("attend-step-long", "attend", 32, 8, 128, 64, 2, 1, 131071),
        # a chunk of a long prompt
        _case("attend-chunk-2048", "attend", 32, 8, 128, 64, 1, 2048, 6145),
        # a step of continuous batching: chunks of prompts beside single tokens, one key head per head
        _case("attend-mixed", "attend", 32, 32, 128, 32, 8, 517, 4096, spread=True, mixed=True),
        # page selection of a decoding step over long texts
        _case("select-step-32", "select", 32, 8, 128, 64, 32, 1, 32767, k=32),
        # page selection of a chunk, every token its own pages
        _case("select-chunk-1000", "select", 32, 8, 128, 64, 1, 1000, 15384, k=16),
        # the attention of that decoding step
        _case("blocks-step-32", "blocks", 32, 8, 128, 64, 32, 1, 32767, k=32),
        # the attention of that chunk
        _case("blocks-chunk-1000", "blocks", 32, 8, 128, 64, 1, 1000, 15384, k=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "select", "blocks"])
    h, hk = rng.choice([(12, 12), (32, 32), (32, 8), (16, 8), (32, 4), (14, 2), (8, 1)])
    d = rng.choice([64, 128, 128, 80])
    ps = rng.choice([16, 32, 64, 64, 128])
    step = rng.random() < 0.5
    spread, mixed = rng.random() < 0.6, rng.random() < 0.3
    if op == "append":
        B = _log(rng, 1, 200) if step else _log(rng, 1, 6)
        new = 1 if step else _log(rng, 2, 8000 // B)
        rot = rng.choice([0, d, d, 32])
        return _case(None, op, h, hk, d, ps, B, new, _log(rng, 1, 2000), spread, mixed, norm=rng.random() < 0.5,
                     rot=rot, inter=rng.random() < 0.5, keep=1.0 if step or rng.random() < 0.6 else rng.uniform(0.05, 0.9))
    if op == "attend":
        B = _log(rng, 1, 60) if step else _log(rng, 1, 6)
        new = rng.choice([1, 1, 2, 5]) if step else _log(rng, 8, 1500 // B)
        past = _log(rng, 1, 120000 // B) if step else _log(rng, 1, 8000)
        return _case(None, op, h, hk, d, ps, B, new, past, spread, mixed, causal=rng.random() < 0.8)
    B = _log(rng, 1, 40) if step else _log(rng, 1, 3)
    new = 1 if step else _log(rng, 8, 700 // B)
    k = _log(rng, 4, 40) if op == "select" or step else _log(rng, 4, max(4, 1000 // ps))
    return _case(None, op, h, hk, d, ps, B, new, _log(rng, 100, min(16000, ps * 600)), spread, mixed, k=k)


def _lengths(case):
    """New tokens and older tokens of every sequence: a matter of the case alone."""
    r = np.random.default_rng([case["B"], case["new"], case["past"]])
    n = np.full(case["B"], case["new"])
    past = np.full(case["B"], case["past"])
    if case["spread"]:
        n[1:] = r.integers(1, case["new"] + 1, case["B"] - 1)
        past[1:] = r.integers(0, case["past"] + 1, case["B"] - 1)
    if case["mixed"]:
        n[1::2] = 1
    return n, past


def _kept(case, n):
    """How many of a sequence's new tokens go to the cache."""
    return n if case["keep"] >= 1 else np.maximum(1, (n * case["keep"]).astype(np.int64))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").bfloat16()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = np.random.default_rng(seed)
    n, past = _lengths(case)
    kept = _kept(case, n)
    B, h, hk, d, ps = (case[x] for x in ("B", "h", "hk", "d", "ps"))
    N, total = int(n.sum()), past + kept
    pages = -(-total // ps)
    n_pages = int(pages.sum()) + 3
    table = np.full((B, int(pages.max()) + 1), -1, dtype=np.int32)
    at = r.permutation(n_pages)[:int(pages.sum())].astype(np.int32)
    for b, p in enumerate(np.split(at, np.cumsum(pages)[:-1])):
        table[b, :len(p)] = p
    cuda = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, dtype=t)).cuda()  # noqa: E731
    s = {"case": case, "N": N, "max_new": int(n.max()), "max_len": int(total.max()),
         "off": cuda(np.concatenate([[0], np.cumsum(n)]), np.int32), "table": cuda(table, np.int32)}
    if case["op"] == "append":
        # the projection writes queries, keys and values of a token side by side
        qkv = _randn(g, N, (h + 2 * hk) * d)
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([h * d, hk * d, hk * d], 1))
        s["q_norm"], s["k_norm"] = ((1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16() for _ in range(2)) \
            if case["norm"] else (None, None)
        rot = case["rot"]
        s["inv_freq"] = THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot) if rot else None
        s["len"] = cuda(past, np.int32)
        if case["keep"] < 1:
            idx = np.zeros(N, dtype=np.int32)
            for b, o in enumerate(np.concatenate([[0], np.cumsum(n)[:-1]])):
                idx[o:o + kept[b]] = np.sort(r.permutation(n[b])[:kept[b]])
            s["rep_idx"], s["rep_cnt"] = cuda(idx, np.int32), cuda(kept, np.int32)
        else:
            s["rep_idx"] = s["rep_cnt"] = None
    else:
        s["len"] = cuda(total, np.int32)
        s["q"] = 2 * _randn(g, N, h, d)
    s["K"], s["V"] = _randn(g, n_pages, hk, ps, d), _randn(g, n_pages, hk, ps, d)
    if case["op"] != "append":
        # channels of a key head have their own mean and scale, pages a drift of their own
        s["K"] *= 0.5 + torch.rand((hk, 1, d), generator=g, device="cuda").bfloat16()
        s["K"] += _randn(g, hk, 1, d)
        s["K"] += 0.5 * _randn(g, n_pages, hk, 1, d)
    s["kmin"], s["kmax"] = s["K"].amin(2), s["K"].amax(2)
    s["out"] = torch.empty_like(s["q"]) if case["op"] in ("attend", "blocks") else None
    if case["op"] == "blocks":
        s["idx"], s["cnt"] = _lists(s, g)
    return s


def _seq(s):
    """The sequence of every new token and its place among the sequence's new tokens."""
    i = torch.arange(s["N"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["off"][1:].contiguous(), i, right=True)
    return b, i - s["off"][b]


def _limits(s):
    """How many tokens of the cache every new token sees."""
    b, i = _seq(s)
    n = s["off"][1:] - s["off"][:-1]
    return b, (s["len"][b] - n[b] + i + 1 if s["case"]["causal"] else s["len"][b]).clamp(min=0)


def _pages_seen(s):
    b, lim = _limits(s)
    return b, lim, (lim + s["case"]["ps"] - 1) // s["case"]["ps"]


def _lists(s, g):
    """Lists as a selection leaves them: first and last page, others in between, ascending."""
    hk, k = s["case"]["hk"], s["case"]["k"]
    _, _, seen = _pages_seen(s)
    P = s["table"].shape[1]
    w = torch.rand((s["N"], hk, max(P, k)), generator=g, device="cuda")
    p = torch.arange(w.shape[2], device="cuda")
    last = (seen - 1).view(-1, 1, 1)
    w = torch.where((p == 0) | (p == last), 2.0, w).where(p <= last, -1.0)
    top = w.topk(k, dim=2)
    idx = top.indices.where(top.values >= 0, 1 << 30).sort(2).values
    cnt = seen.clamp(max=k).view(-1, 1).expand(-1, hk)
    return idx.where(idx < (1 << 30), -1).int().contiguous(), cnt.int().contiguous()


# ---------------------------------------------------------------- plain forms
def _normed(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _rotated(x, pos, case, inv_freq):
    rot = case["rot"]
    if not rot:
        return x
    a = pos.double().unsqueeze(1) * inv_freq
    c, s = a.cos().float().unsqueeze(1), a.sin().float().unsqueeze(1)
    if case["inter"]:
        u, v = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([u * c - v * s, v * c + u * s], -1).flatten(-2)
    else:
        u, v = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([u * c - v * s, v * c + u * s], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(s):
    case, ps = s["case"], s["case"]["ps"]
    b, i = _seq(s)
    q = _rotated(_normed(s["q"].float(), s["q_norm"]), s["len"][b] + i, case, s["inv_freq"]).bfloat16()
    n = s["off"][1:] - s["off"][:-1] if s["rep_cnt"] is None else s["rep_cnt"]
    src = torch.arange(s["N"], device="cuda") if s["rep_idx"] is None else s["off"][b] + s["rep_idx"]
    row = (i < n[b]).nonzero().squeeze(1)
    src, b, i = src[row], b[row], i[row]
    pos = s["len"][b] + (src - s["off"][b])
    k = _rotated(_normed(s["k"][src].float(), s["k_norm"]), pos, case, s["inv_freq"]).bfloat16()
    slot = s["len"][b] + i
    page = s["table"][b, slot // ps]
    s["K"][page, :, slot % ps] = k
    s["V"][page, :, slot % ps] = s["v"][src]
    new_len = s["len"] + n
    t = torch.arange(-(-s["max_new"] // ps) + 1, device="cuda") + (s["len"] // ps).unsqueeze(1)
    at = (t < ((new_len + ps - 1) // ps).unsqueeze(1)).nonzero()
    bb, tt = at[:, 0], t[at[:, 0], at[:, 1]]
    page = s["table"][bb, tt]
    live = ((tt * ps).unsqueeze(1) + torch.arange(ps, device="cuda") < new_len[bb].unsqueeze(1)).view(-1, 1, ps, 1)
    keys = s["K"][page]
    s["kmin"][page] = keys.where(live, math.inf).amin(2)
    s["kmax"][page] = keys.where(live, -math.inf).amax(2)
    return q, new_len.int()


def _plain_attend(s):
    case = s["case"]
    B, h, hk, d, ps = (case[x] for x in ("B", "h", "hk", "d", "ps"))
    b, i = _seq(s)
    _, lim = _limits(s)
    P = -(-s["max_len"] // ps)
    table = s["table"][:, :P].clamp(min=0)
    k = s["K"][table].transpose(1, 2).reshape(B, hk, P * ps, d).float()
    v = s["V"][table].transpose(1, 2).reshape(B, hk, P * ps, d)
    slot = torch.arange(P * ps, device="cuda")
    v = v.where((slot < s["len"].unsqueeze(1)).view(B, 1, -1, 1), 0).float()
    q = torch.zeros((B, s["max_new"], h, d), device="cuda")
    q[b, i] = s["q"].float()
    q = q.view(B, s["max_new"], hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(B, hk, -1, d)
    full = torch.zeros((B, s["max_new"]), dtype=torch.int32, device="cuda")
    full[b, i] = lim.int()
    x = torch.matmul(q, k.transpose(2, 3)).view(B, hk, h // hk, s["max_new"], -1) * (1.0 / math.sqrt(d))
    x = x.masked_fill(slot >= full.view(B, 1, 1, -1, 1), -math.inf)
    x = (x - x.amax(-1, keepdim=True).clamp(min=-3e38)).exp()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hk, -1, P * ps), v).view(B, hk, h // hk, s["max_new"], d) / l.clamp(min=1e-38)
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, s["max_new"], h, d)[b, i])
    return s["out"]


def _plain_select(s):
    case = s["case"]
    B, h, hk, d, k = (case[x] for x in ("B", "h", "hk", "d", "k"))
    b, _, seen = _pages_seen(s)
    i = _seq(s)[1]
    table = s["table"].clamp(min=0)
    P = table.shape[1]
    q = s["q"].double().view(-1, hk, h // hk, d)
    both = torch.cat([q.clamp(min=0).sum(2), q.clamp(max=0).sum(2)], -1)
    x = torch.zeros((B, s["max_new"], hk, 2 * d), dtype=torch.float64, device="cuda")
    x[b, i] = both
    bounds = torch.cat([s["kmax"][table], s["kmin"][table]], -1).double()
    score = torch.einsum("bnhe,bphe->bnhp", x, bounds)[b, i]
    p = torch.arange(P, device="cuda")
    last = (seen - 1).view(-1, 1, 1)
    score = torch.where((p == 0) | (p == last), math.inf, score).where(p <= last, -math.inf)
    if P < k:
        score = torch.nn.functional.pad(score, (0, k - P), value=-math.inf)
    take = min(k, P)
    order = score.argsort(dim=2, descending=True, stable=True)[..., :k]
    count = seen.clamp(max=take).view(-1, 1, 1)
    idx = order.where(torch.arange(k, device="cuda") < count, 1 << 30).sort(2).values
    return idx.where(idx < (1 << 30), -1).int(), count.squeeze(2).expand(-1, hk).int().contiguous()


def _plain_blocks(s):
    case = s["case"]
    h, hk, d, ps, k = (case[x] for x in ("h", "hk", "d", "ps", "k"))
    b, lim = _limits(s)
    page = s["table"][b.view(-1, 1, 1), s["idx"].clamp(min=0)].clamp(min=0)
    head = torch.arange(hk, device="cuda").view(1, -1, 1)
    slot = (s["idx"] * ps).unsqueeze(3) + torch.arange(ps, device="cuda")
    live = (torch.arange(k, device="cuda") < s["cnt"].unsqueeze(2)).unsqueeze(3) & (slot < lim.view(-1, 1, 1, 1))
    live = live.view(-1, hk, 1, k * ps)
    keys = s["K"][page, head].view(-1, hk, k * ps, d).float()
    vals = s["V"][page, head].view(-1, hk, k * ps, d).where(live.transpose(2, 3), 0).float()
    q = s["q"].float().view(-1, hk, h // hk, d)
    x = torch.matmul(q, keys.transpose(2, 3)) * (1.0 / math.sqrt(d))
    x = x.masked_fill(~live, -math.inf)
    x = (x - x.amax(-1, keepdim=True).clamp(min=-3e38)).exp()
    o = torch.matmul(x, vals) / x.sum(-1, keepdim=True).clamp(min=1e-38)
    s["out"].copy_(o.view(-1, h, d))
    return s["out"]


# ---------------------------------------------------------------- one pass
def _library():
    """The binding and a context: a program makes one context and keeps it."""
    from paper_2605_03110_b200 import binding as ada
    if "ctx" not in _CTX:
        _CTX["ctx"] = ada.ada_create(1, 128, 128, ada.ADA_BF16)
    return ada, _CTX["ctx"]


def _own(s):
    ada, ctx = _library()
    case = s["case"]
    if "cache" not in s:
        s["cache"] = ada.KVCache(s["K"], s["V"], s["table"], s["kmin"], s["kmax"])
    causal = ada.ADA_ATTN_CAUSAL if case["causal"] else 0
    if case["op"] == "append":
        return ada.ada_cache_append(ctx, s["cache"], s["k"], s["v"], s["off"], s["len"], Q=s["q"], q_norm=s["q_norm"],
                                    k_norm=s["k_norm"], eps=EPS, inv_freq=s["inv_freq"], rep_idx=s["rep_idx"],
                                    rep_cnt=s["rep_cnt"], flags=ada.ADA_ROPE_PAIRS if case["inter"] else 0)
    if case["op"] == "attend":
        return ada.ada_attention_cached(ctx, s["cache"], s["q"], s["off"], s["len"], s["max_new"], out=s["out"],
                                        flags=causal)
    if case["op"] == "select":
        return ada.ada_select_blocks(ctx, s["cache"], s["q"], s["off"], s["len"], case["k"], n_first=1, n_last=1,
                                     flags=causal)
    return ada.ada_attention_blocks(ctx, s["cache"], s["q"], s["off"], s["len"], s["idx"], s["cnt"], out=s["out"],
                                    flags=causal)


def run(state):
    if own:
        got = _own(state)
    else:
        got = {"append": _plain_append, "attend": _plain_attend, "select": _plain_select,
               "blocks": _plain_blocks}[state["case"]["op"]](state)
    if state["case"]["op"] == "append":
        return {"q": got[0], "len": got[1], "K": state["K"], "V": state["V"], "kmin": state["kmin"], "kmax": state["kmax"]}
    if state["case"]["op"] == "select":
        return {"idx": got[0], "cnt": got[1]}
    return got


def work(case):
    n, past = _lengths(case)
    kept = _kept(case, n)
    B, h, hk, d, ps, k = (case[x] for x in ("B", "h", "hk", "d", "ps", "k"))
    N, total = int(n.sum()), past + kept
    row = 2 * d
    if case["op"] == "append":
        # queries in and out, kept keys and values in and out, the keys that began a page, the bounds
        touched = -(-total // ps) - past // ps
        byte = 2 * N * h * row + 4 * int(kept.sum()) * hk * row + int((past % ps).sum() + 2 * touched.sum()) * hk * row
        return {"bytes": byte, "flops": (N * h + int(kept.sum()) * hk) * d * (7 if case["norm"] else 3)}
    lim = np.concatenate([np.arange(t - m + 1, t + 1) if case["causal"] else np.full(m, t) for m, t in zip(n, total)])
    if case["op"] == "attend":
        return {"bytes": 2 * N * h * row + 2 * int(total.sum()) * hk * row, "flops": 4 * h * d * int(lim.sum())}
    seen = -(-lim // ps)
    pages = int((-(-total // ps)).sum())
    if case["op"] == "select":
        return {"bytes": N * h * row + 2 * pages * hk * row + 4 * N * hk * (k + 1), "flops": 4 * d * hk * int(seen.sum())}
    # every listed page once for each sequence at least
    keys = int(np.minimum(seen, k).sum()) * ps
    once = sum(min(int(t), int(m) * k * ps) for m, t in zip(n, total))
    return {"bytes": 2 * N * h * row + 2 * once * hk * row + 4 * N * hk * (k + 1), "flops": 4 * h * d * keys}


# ---------------------------------------------------------------- the definition, in 64 bits
def _turn64(x, pos, case, inv_freq):
    """Rotation of pairs as a product of complex numbers; x (n, heads, d)."""
    rot = case["rot"]
    if not rot:
        return x
    w = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None] * inv_freq)[:, None]
    y = x.clone()
    if case["inter"]:
        y[..., :rot] = torch.view_as_real(torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * w).flatten(-2)
    else:
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * w
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def _unit64(x, w):
    return x if w is None else x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()


def _exact_append(s, n, past):
    case, ps = s["case"], s["case"]["ps"]
    q = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    K, V, lo, hi = (s[x].double() for x in ("K", "V", "kmin", "kmax"))
    o = 0
    for b in range(case["B"]):
        m, old = int(n[b]), int(past[b])
        here = torch.arange(m, device="cuda")
        q[o:o + m] = _turn64(_unit64(s["q"][o:o + m].double(), s["q_norm"]), old + here, case, s["inv_freq"])
        if s["rep_idx"] is not None:
            here = s["rep_idx"][o:o + int(_kept(case, n)[b])].long()
        k = _turn64(_unit64(s["k"][o + here].double(), s["k_norm"]), old + here, case, s["inv_freq"])
        v = s["v"][o + here].double()
        end = old + len(here)
        for p in range(old // ps, -(-end // ps)):
            a, z = max(old, p * ps), min(end, (p + 1) * ps)
            page = int(s["table"][b, p])
            K[page, :, a - p * ps:z - p * ps] = k[a - old:z - old].transpose(0, 1)
            V[page, :, a - p * ps:z - p * ps] = v[a - old:z - old].transpose(0, 1)
            live = K[page, :, :z - p * ps]
            lo[page], hi[page] = live.amin(1), live.amax(1)
        o += m
    return {"q": q, "len": None, "K": K, "V": V, "kmin": lo, "kmax": hi}


def _keys64(s, b, length):
    """Keys and values of a sequence as (hk, length, d)."""
    ps = s["case"]["ps"]
    p = s["table"][b, :-(-length // ps)].long()
    return (s[x][p].double().transpose(0, 1).flatten(1, 2)[:, :length] for x in ("K", "V"))


def _exact_attend(s, n, past, listed_pages):
    case = s["case"]
    h, hk, d, ps = (case[x] for x in ("h", "hk", "d", "ps"))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    o = 0
    for b in range(case["B"]):
        m, total = int(n[b]), int(past[b] + n[b])
        k, v = _keys64(s, b, total)
        at = torch.arange(total, device="cuda")
        for a in range(0, m, 128):
            z = min(m, a + 128)
            q = s["q"][o + a:o + z].double().view(z - a, hk, h // hk, d)
            x = torch.einsum("thgd,hsd->thgs", q, k) / math.sqrt(d)
            seen = total - m + torch.arange(a, z, device="cuda") + 1 if case["causal"] else torch.full((z - a,), total, device="cuda")
            ok = (at < seen[:, None])[:, None].expand(-1, hk, -1)
            if listed_pages:
                chosen = torch.zeros((z - a, hk, -(-total // ps) + 1), dtype=torch.bool, device="cuda")
                pages = s["idx"][o + a:o + z].long()
                chosen.scatter_(2, pages.where(pages >= 0, chosen.shape[2] - 1), True)
                chosen[..., -1] = False
                ok = ok & chosen[:, :, at // ps]
            p = torch.softmax(x.masked_fill(~ok[:, :, None], -math.inf), -1)
            out[o + a:o + z] = torch.einsum("thgs,hsd->thgd", p, v).reshape(z - a, h, d)
        o += m
    return out


def exact(case, seed):
    n, past = _lengths(case)
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s, n, past)
    if case["op"] == "select":
        return None                               # whole numbers only
    return _exact_attend(s, n, past, case["op"] == "blocks")
