"""The paged cache on the GPU against plain loops in 64 bits: appending with norm and rotation, attention of single
tokens and chunks, choice of pages, attention on the chosen pages, and a run of all of them."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ada():
    from paper_2605_03110_b200 import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def ctx(ada):
    c = ada.ada_create(1, 128, 128, ada.ADA_BF16)
    yield c
    ada.ada_destroy(c)


def fine(ada, ctx):
    st, _ = ada.ada_device_status(ctx)
    assert st == 0, ada.status_string(st)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """Sequences with news[b] new tokens out of lens[b] in all, their pages scattered over a pool.  Slots behind a
    sequence's length hold NaN, table entries that nobody needs hold nonsense."""

    def __init__(self, ada, seed, h, hk, d, ps, news, lens, pad=0, planes=False, drift=0.0):
        g = torch.Generator().manual_seed(seed)
        self.h, self.hk, self.d, self.ps = h, hk, d, ps
        self.news, self.lens = news, lens
        B = len(news)
        need = [-(-n // ps) for n in lens]
        pool = sum(need) + 4
        perm = torch.randperm(pool, generator=g).tolist()
        width = max(need) + 2
        table = torch.tensor([-7, 1 << 30] * (width * B), dtype=torch.int32)[:width * B].view(B, width).clone()
        KV = torch.randn((pool, 2, hk, ps, d), generator=g)
        KV += drift * torch.randn((pool, 2, hk, 1, d), generator=g)
        KV = KV.bfloat16()
        free = set(range(pool))
        for b in range(B):
            for p in range(need[b]):
                page = perm.pop()
                free.discard(page)
                table[b, p] = page
                KV[page, :, :, max(0, min(ps, lens[b] - p * ps)):] = math.nan
        for page in free:
            KV[page] = math.nan
        self.N = sum(news) + pad
        self.off = [sum(news[:b]) for b in range(B + 1)]
        self.Q = (1.5 * torch.randn((self.N, h, d), generator=g)).bfloat16()
        kmin = torch.full((pool, hk, d), math.nan).bfloat16()
        kmax = kmin.clone()
        for b in range(B):
            for p in range(need[b]):
                page = int(table[b, p])
                live = KV[page, 0, :, :min(ps, lens[b] - p * ps)]
                kmin[page], kmax[page] = live.amin(1), live.amax(1)
        self.cpu = ref.Pages(KV[:, 0], KV[:, 1], table, kmin, kmax)
        if planes:                               # K and V as planes of one tensor
            KVd = KV.cuda()
            Kd, Vd = KVd[:, 0], KVd[:, 1]
        else:
            Kd, Vd = KV[:, 0].contiguous().cuda(), KV[:, 1].contiguous().cuda()
        self.cache = ada.KVCache(Kd, Vd, table.cuda(), kmin.cuda(), kmax.cuda())
        self.d_off, self.d_len, self.d_Q = i32(self.off), i32(lens), self.Q.cuda()
        self.max_new = max(news + [1])

    def check(self, got, causal, scale=0.0, lists=None):
        out, weight = ref.attend(self.cpu, self.Q, self.off, self.lens, self.hk, causal, scale, lists)
        n = self.off[-1]
        V = torch.nan_to_num(self.cpu.V.float())
        far = (got.cpu().double() - out).abs() - ref.tolerance(out, weight, V)
        assert bool((far[:n] <= 0).all()), (float(far[:n].max()), got.isnan().sum())


HEADS = [(4, 4, 64), (8, 2, 128), (7, 1, 80), (6, 3, 16), (16, 1, 128), (2, 2, 48)]
STEPS = [
    ([1], [1]),
    ([1, 1, 1], [17, 1, 300]),
    ([1, 0, 1, 1], [128, 64, 129, 127]),
    ([1] * 40, [(37 * b) % 211 + 1 for b in range(40)]),
    ([1, 1], [2500, 33]),
    ([1, 1], [0, 5]),
]


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
@pytest.mark.parametrize("h,hk,d", HEADS)
def test_single_tokens(ada, ctx, h, hk, d, ps):
    for seed, (news, lens) in enumerate(STEPS):
        c = Case(ada, seed, h, hk, d, ps, news, lens)
        for causal in (True, False):
            out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new,
                                           flags=ada.ADA_ATTN_CAUSAL if causal else 0)
            fine(ada, ctx)
            c.check(out, causal)


@pytest.mark.parametrize("news,lens", [([2, 3, 1], [40, 3, 700]), ([4, 4], [3, 1000]), ([2, 0, 4], [1, 50, 129])])
@pytest.mark.parametrize("h,hk,d,ps", [(8, 2, 128, 64), (3, 1, 64, 16), (4, 4, 80, 32)])
def test_a_few_tokens_each(ada, ctx, h, hk, d, ps, news, lens):
    """Rows of one 16-row tile that see different numbers of keys; sequences shorter than their new tokens."""
    c = Case(ada, 3, h, hk, d, ps, news, lens)
    for causal in (True, False):
        out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 4, flags=int(causal))
        fine(ada, ctx)
        c.check(out, causal)


CHUNKS = [
    ([17], [17]),
    ([130], [400]),
    ([40, 0, 1, 300], [45, 10, 129, 300]),
    ([33, 64], [20, 1000]),                    # the first has fewer slots than new tokens: rows that see nothing
    ([260], [384]),
    ([1, 1, 70], [1, 513, 70]),
]


@pytest.mark.parametrize("ps", [16, 64, 128])
@pytest.mark.parametrize("h,hk,d", HEADS)
def test_chunks(ada, ctx, h, hk, d, ps):
    for seed, (news, lens) in enumerate(CHUNKS):
        c = Case(ada, 50 + seed, h, hk, d, ps, news, lens, planes=seed % 2 == 1)
        for causal in (True, False):
            out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, max(c.max_new, 17),
                                           flags=int(causal))
            fine(ada, ctx)
            c.check(out, causal)


@pytest.mark.parametrize("h,hk,few", [(4, 4, 16), (8, 2, 4), (14, 2, 2), (16, 1, 1), (34, 2, 0)])
def test_few_tokens_and_chunks_in_one_call(ada, ctx, h, hk, few):
    """Sequences on either side of the line between the two kernels, in one call; and one sequence alone."""
    for news, lens in (([few + 1, few, 1, 0, 60], [90, 300, 5, 3, 700]), ([few, few + 1], [2000, few]), ([few + 1], [1500])):
        c = Case(ada, few, h, hk, 64, 32, news, lens, pad=1)
        for causal in (True, False):
            out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new, flags=int(causal))
            fine(ada, ctx)
            c.check(out, causal)


@pytest.mark.parametrize("max_new", [1, 50])
def test_pages_behind_the_32_bit_range(ada, ctx, max_new):
    """A pool of more than 2^31 elements, the sequence's pages at its far end."""
    h, hk, d, ps, pool = 8, 2, 128, 64, 135000
    K, V = (torch.empty((pool, hk, ps, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert K.numel() > 2 ** 31
    kmin, kmax = (torch.empty((pool, hk, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pages = [pool - 1, pool - 7, 0, 131072, 131071, pool - 2]
    table = i32([pages + [-1]])
    cache = ada.KVCache(K, V, table, kmin, kmax)
    g = torch.Generator(device="cuda").manual_seed(9)
    total = 350
    x = torch.randn((total, (h + 2 * hk) * d), generator=g, device="cuda").bfloat16()
    q, k, v = (y.unflatten(1, (-1, d)) for y in x.split([h * d, hk * d, hk * d], 1))
    ada.ada_cache_append(ctx, cache, k, v, i32([0, total]), i32([0]))
    small = ref.Pages(K[pages].cpu(), V[pages].cpu(), torch.arange(6, dtype=torch.int32).view(1, 6), kmin[pages].cpu(), kmax[pages].cpu())
    q = q[-max_new:].contiguous()
    out = ada.ada_attention_cached(ctx, cache, q, i32([0, max_new]), i32([total]), max_new)
    idx, cnt = ada.ada_select_blocks(ctx, cache, q, i32([0, max_new]), i32([total]), 4)
    some = ada.ada_attention_blocks(ctx, cache, q, i32([0, max_new]), i32([total]), idx, cnt)
    fine(ada, ctx)
    assert lists_of(idx, cnt) == ref.select(small, q.cpu(), [0, max_new], [total], hk, 4, 1, 1)
    for got, lists in ((out, None), (some, lists_of(idx, cnt))):
        want, weight = ref.attend(small, q.cpu(), [0, max_new], [total], hk, True, 0.0, lists)
        tol = ref.tolerance(want, weight, v.float().cpu())
        assert bool(((got.cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("h,hk", [(128, 1), (40, 1), (66, 2), (12, 2)])
def test_wide_groups(ada, ctx, h, hk):
    """Groups that do not divide a tile's 128 rows, and the largest; single tokens of more than 16 heads a key head."""
    for news, lens in (([1, 1], [200, 77]), ([9, 3], [30, 300])):
        c = Case(ada, h, h, hk, 64, 32, news, lens)
        out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new)
        fine(ada, ctx)
        c.check(out, True)


@pytest.mark.parametrize("max_new", [1, 40])
def test_rows_behind_the_last_sequence_and_strides(ada, ctx, max_new):
    """Queries and outputs as columns of wider rows; padding rows and columns keep what they hold."""
    h, hk, d = 8, 2, 64
    news = [1, 1, 1] if max_new == 1 else [40, 3, 17]
    c = Case(ada, 8, h, hk, d, 16, news, [50, 200, 20], pad=5, planes=True)
    wide = torch.full((c.N, (h + 2 * hk) * d), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, hk * d:(hk + h) * d] = c.d_Q.flatten(1)
    Q = wide[:, hk * d:(hk + h) * d].unflatten(1, (h, d))
    room = torch.full((c.N, (h + 1) * d), 5.0, dtype=torch.bfloat16, device="cuda")
    out = room[:, d:].unflatten(1, (h, d))
    ada.ada_attention_cached(ctx, c.cache, Q, c.d_off, c.d_len, max_new, out=out)
    fine(ada, ctx)
    c.check(out, True)
    assert bool((room[:, :d] == 5.0).all()) and bool((room[c.off[-1]:] == 5.0).all())


@pytest.mark.parametrize("news", [[1], [90]])
def test_scale_and_large_scores(ada, ctx, news):
    """Scores far apart: the maximum moves from tile to tile, most probabilities vanish."""
    c = Case(ada, 9, 4, 2, 128, 32, news, [900])
    grow = (1.5 ** (torch.arange(900) // 100)).view(1, -1, 1)
    for t in range(900):
        page, s = int(c.cpu.table[0, t // 32]), t % 32
        c.cpu.K[page, :, s] = (c.cpu.K[page, :, s].float() * grow[0, t]).bfloat16()
    c.cache.K.copy_(c.cpu.K)
    for scale in (0.0, 1.0, 0.01):
        out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new, scale=scale)
        fine(ada, ctx)
        # scores of up to a few thousand: their fp32 error (2^-22 of the largest) turns into one of the probabilities
        S = float(c.Q.abs().max()) * float(torch.nan_to_num(c.cpu.K.float()).abs().max()) * 128 * (scale or 128 ** -0.5)
        ref_out, weight = ref.attend(c.cpu, c.Q, c.off, c.lens, 2, True, scale)
        V = torch.nan_to_num(c.cpu.V.float())
        tol = ref.tolerance(ref_out, weight, V) + 2 * S * 2.0 ** -22 * float(V.abs().max())
        assert bool(((out.cpu().double() - ref_out).abs() <= tol).all())


@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("n", [1, 3, 90, 700])
def test_nan_and_infinity_that_a_token_sees(ada, ctx, n, lists):
    """A NaN in a key gives NaN in the rows that see it, and only there, wherever it lies in a tile; so does a score of
    +inf; one of -inf has no weight."""
    length, j = 900, 1
    c = Case(ada, 21, 4, 2, 128, 32, [n], [length])
    pages = -(-length // 32)
    idx = torch.arange(pages, dtype=torch.int32, device="cuda").expand(n, 2, pages).contiguous()
    cnt = torch.full((n, 2), pages, dtype=torch.int32, device="cuda")
    seen_from = torch.arange(length - n, length)             # a token's own slot
    for value in (math.nan, math.inf):
        for slot in (0, 2, 5, 18, 127, 450, length - 60, length - 1):
            page, at = int(c.cpu.table[0, slot // 32]), slot % 32
            c.cache.K.copy_(c.cpu.K)
            c.cache.K[page, j, at, 7] = value
            if lists:
                out = ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt)
            else:
                out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, n)
            fine(ada, ctx)
            bad = (seen_from >= slot).view(-1, 1).expand(n, 4) & (torch.arange(4) // 2 == j)
            if value == math.inf:
                bad = bad & (c.Q[:, :, 7] > 0)
            assert torch.equal(out.cpu().isnan().all(-1), bad), slot
            assert torch.equal(out.cpu().isnan().any(-1), bad), slot
            assert bool(out.cpu().isfinite().all(-1)[~bad].all())


def attend_by(ada, ctx, c, how):
    """A call of either kind over all that the new tokens see: dense, causal or not, or over lists of every page."""
    if how != "lists":
        return ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new, flags=int(how == "causal"))
    pages = c.cache.table.shape[1] - 2
    idx = torch.arange(pages, dtype=torch.int32, device="cuda").expand(c.N, c.hk, pages).contiguous()
    cnt = torch.zeros((c.N, c.hk), dtype=torch.int32)
    for b, n in enumerate(c.lens):
        cnt[c.off[b]:c.off[b + 1]] = -(-n // c.ps)
    return ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt.cuda())


@pytest.mark.parametrize("how", ["causal", "all", "lists"])
@pytest.mark.parametrize("h,hk,d,ps,n,length", [(4, 2, 128, 32, 1, 900), (4, 2, 128, 32, 3, 900), (2, 2, 128, 64, 16, 500),
                                                (3, 1, 48, 16, 4, 129), (4, 2, 128, 32, 90, 900), (4, 2, 128, 32, 700, 900),
                                                (16, 1, 64, 128, 130, 130), (6, 1, 80, 16, 60, 40), (4, 2, 64, 16, 7, 5)])
def test_nan_and_infinity_in_values(ada, ctx, h, hk, d, ps, n, length, how):
    """A value that is NaN or infinite makes its element so in the rows that see its slot, and changes nothing else: not a
    bit of the rows before it, whose probability of that slot is zero."""
    c = Case(ada, 25, h, hk, d, ps, [n], [length])
    clean = attend_by(ada, ctx, c, how).cpu()
    fine(ada, ctx)
    j, heads = hk - 1, slice((hk - 1) * (h // hk), h)
    limit = torch.tensor([ref.sees(n, length, i, how != "all") for i in range(n)])
    first = max(length - n, 0)
    for slot in sorted({0, 5, 127, first, first + 1, first + n // 2, length - 60, length - 2, length - 1}):
        if not 0 < slot + 1 <= length:
            continue
        sees = limit > slot
        for values, elements in (((math.nan,), [7]), ((math.inf,), [0]), ((-math.inf,), [d - 1]), ((math.nan,), list(range(d))),
                                 ((math.inf, -math.inf), [d // 2 + 3]), ((-math.inf, math.nan), [1, d - 2])):
            want = clean.float()
            c.cache.V.copy_(c.cpu.V)
            for k, value in enumerate(values):               # the second one in the slot before
                at = max(slot - k, 0)
                c.cache.V[int(c.cpu.table[0, at // ps]), j, at % ps, elements] = value
                for e in elements:
                    before = want[:, heads, e]
                    new = torch.where((limit > at).view(-1, 1), torch.full_like(before, value), before)
                    if k > 0 and at < slot:                  # both: +inf - inf and NaN are NaN
                        new = torch.where(sees.view(-1, 1), torch.full_like(before, math.nan), new)
                    want[:, heads, e] = new
            got = attend_by(ada, ctx, c, how).cpu().float()
            fine(ada, ctx)
            assert torch.equal(got.isnan(), want.isnan()), (slot, values, elements)
            assert torch.equal(got.nan_to_num(9e9, 8e9, -8e9), want.nan_to_num(9e9, 8e9, -8e9)), (slot, values, elements)


@pytest.mark.parametrize("news,lens,h,hk", [([40] * 20, [40 + 31 * b for b in range(20)], 16, 16),
                                            ([60, 3, 1, 200, 17], [700, 90, 4, 200, 17], 8, 2),
                                            ([300, 300], [2500, 280], 4, 1)])
def test_nan_in_values_of_one_sequence(ada, ctx, news, lens, h, hk):
    """Many items of many sequences and heads on an SM: a NaN in the last value of some of them is seen by that token alone."""
    c = Case(ada, 26, h, hk, 64, 32, news, lens)
    clean = attend_by(ada, ctx, c, "causal").cpu()
    fine(ada, ctx)
    for b, j in {(0, 0), (len(news) // 2, hk - 1), (len(news) - 1, hk // 2), (1, 0)}:
        c.cache.V.copy_(c.cpu.V)
        at = lens[b] - 1
        c.cache.V[int(c.cpu.table[b, at // 32]), j, at % 32, 20] = math.nan
        got = attend_by(ada, ctx, c, "causal").cpu()
        fine(ada, ctx)
        want = clean.clone()
        want[c.off[b + 1] - 1, j * (h // hk):(j + 1) * (h // hk), 20] = math.nan
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num()), (b, j)


SPANS = [([1], [900]), ([3], [900]), ([90], [900]), ([700], [900]), ([6], [4]), ([90], [80])]


@pytest.mark.parametrize("how", ["causal", "lists"])
@pytest.mark.parametrize("news,lens", SPANS)
def test_scores_beyond_fp32(ada, ctx, news, lens, how):
    """Scores that leave the range of fp32, in the product or only with the scale: NaN in every row that sees a slot, on
    every path, where one is +inf or all are -inf; zeros where there is none."""
    c = Case(ada, 27, 4, 2, 128, 32, news, lens)
    n, length = news[0], lens[0]
    some = torch.tensor([ref.sees(n, length, i, True) > 0 for i in range(n)])
    scaled = lambda s: (attend_by(ada, ctx, c, how) if s is None else call(s)).cpu()          # noqa: E731

    def call(scale):
        if how != "lists":
            return ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new, scale=scale)
        pages = -(-length // 32)
        idx = torch.arange(pages, dtype=torch.int32, device="cuda").expand(n, 2, pages).contiguous()
        cnt = torch.full((n, 2), pages, dtype=torch.int32, device="cuda")
        return ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt, scale=scale)

    def nan_rows(out):
        fine(ada, ctx)
        assert bool((out[~some] == 0).all()) and bool(out[some].isnan().all())

    c.cache.K.mul_(2.0 ** 40)                            # a product of 2^40, times 1e30
    nan_rows(scaled(1e30))
    Q = c.d_Q
    c.cache.K.copy_(torch.where(c.cpu.K.isnan(), c.cpu.K, torch.full_like(c.cpu.K, 1e30)))
    for sign in (1.0, -1.0):                             # the product itself; every score -inf
        c.d_Q = torch.full_like(Q, sign * 1e30)
        nan_rows(scaled(None))
    # every score -inf but one slot's: that slot has all the weight
    slot = max(length - n, 0)
    page = int(c.cpu.table[0, slot // 32])
    c.cache.K[page, :, slot % 32] = 0.0
    out = scaled(None)
    fine(ada, ctx)
    v = c.cpu.V[page, :, slot % 32].repeat_interleave(2, 0)
    assert bool((out[~some] == 0).all()) and torch.equal(out[some], v.expand(int(some.sum()), 4, 128))


@pytest.mark.parametrize("scale", [1e-300, 1e-50, 1e-44, 1e-39, 1e-30])
@pytest.mark.parametrize("news,lens", SPANS)
def test_tiny_scale(ada, ctx, news, lens, scale):
    """A scale that fp32 holds as a subnormal number, or not at all: equal weights, as far as a row sees."""
    c = Case(ada, 28, 4, 2, 128, 32, news, lens)
    pages = -(-lens[0] // 32)
    idx = torch.arange(pages, dtype=torch.int32, device="cuda").expand(c.N, 2, pages).contiguous()
    cnt = torch.full((c.N, 2), pages, dtype=torch.int32, device="cuda")
    for out in (ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new, scale=scale),
                ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt, scale=scale)):
        fine(ada, ctx)
        c.check(out, True, scale=scale)


@pytest.mark.parametrize("news,lens", [([1] * 5, [3, 900, 64, 2000, 1]), ([200], [5000]), ([1, 90, 2, 300], [700, 90, 2, 1000])])
def test_output_over_the_queries(ada, ctx, news, lens):
    c = Case(ada, 22, 8, 2, 128, 64, news, lens)
    out = c.d_Q.clone()
    assert ada.ada_attention_cached(ctx, c.cache, out, c.d_off, c.d_len, c.max_new, out=out) is out
    fine(ada, ctx)
    c.check(out, True)
    k = 4
    idx, cnt = ada.ada_select_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, k)
    apart = ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt)
    over = c.d_Q.clone()
    ada.ada_attention_blocks(ctx, c.cache, over, c.d_off, c.d_len, idx, cnt, out=over)
    fine(ada, ctx)
    assert torch.equal(over, apart)


def test_long_sequence_split_over_all_sms(ada, ctx):
    """One row tile of 20000 keys: every SM has a share, joined in the order of the keys; repeated calls agree."""
    c = Case(ada, 10, 4, 1, 64, 128, [1], [20000])
    out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 1)
    c.check(out, True)
    for _ in range(10):
        assert torch.equal(ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 1), out)
    c = Case(ada, 11, 16, 1, 64, 128, [20], [6000])
    out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 20)
    c.check(out, True)
    for _ in range(10):
        assert torch.equal(ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 20), out)
    fine(ada, ctx)


def test_many_sequences(ada, ctx):
    """More sequences than lanes and threads, many of them without new tokens."""
    B = 300
    news = [1 if b % 3 else 0 for b in range(B)]
    lens = [(b * 7) % 90 + 1 for b in range(B)]
    c = Case(ada, 12, 4, 2, 64, 16, news, lens)
    out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 1)
    fine(ada, ctx)
    c.check(out, True)
    out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 100)
    fine(ada, ctx)
    c.check(out, True)


# ---------------------------------------------------------------- choice of pages
def lists_of(idx, cnt):
    idx, cnt = idx.cpu(), cnt.cpu()
    assert all(bool((idx[i, j, int(cnt[i, j]):] == -1).all()) for i in range(idx.shape[0]) for j in range(idx.shape[1]))
    return [[idx[i, j, :int(cnt[i, j])].tolist() for j in range(idx.shape[1])] for i in range(idx.shape[0])]


@pytest.mark.parametrize("h,hk,d", HEADS)
@pytest.mark.parametrize("news,lens", [([1, 1, 1], [1000, 40, 16]), ([30, 0, 2], [700, 5, 300]), ([3], [2])])
def test_select(ada, ctx, h, hk, d, news, lens):
    for ps, k, first, last in ((16, 8, 1, 1), (32, 3, 0, 0), (16, 5, 2, 3), (64, 1, 0, 1), (16, 64, 1, 1)):
        c = Case(ada, 20, h, hk, d, ps, news, lens, drift=0.5)
        for causal in (True, False):
            idx, cnt = ada.ada_select_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, k, first, last, flags=int(causal))
            fine(ada, ctx)
            want = ref.select(c.cpu, c.Q, c.off, c.lens, hk, k, first, last, causal)
            assert lists_of(idx, cnt) == want


@pytest.mark.parametrize("distinct", [0, 3, 40])
@pytest.mark.parametrize("news,pages", [([1], 65), ([1], 130), ([1], 512), ([1], 700), ([5], 68), ([5], 257), ([5], 512)])
def test_select_few_places_of_many_pages(ada, ctx, news, pages, distinct):
    """Few places, many places, on either side of what a warp keeps for itself; pages all different, or with the bounds of
    a few, so that scores are equal in groups."""
    c = Case(ada, 24, 4, 2, 64, 16, news, [16 * pages], drift=0.5)
    if distinct:
        for p in range(pages):
            at, like = int(c.cpu.table[0, p]), int(c.cpu.table[0, (p * 7) % distinct])
            c.cpu.kmin[at], c.cpu.kmax[at] = c.cpu.kmin[like], c.cpu.kmax[like]
        c.cache.kmin.copy_(c.cpu.kmin)
        c.cache.kmax.copy_(c.cpu.kmax)
    for k, first, last in ((1, 0, 0), (2, 1, 0), (17, 1, 1), (18, 0, 1), (20, 1, 1), (34, 1, 1), (35, 1, 1), (64, 30, 2), (64, 0, 0)):
        idx, cnt = ada.ada_select_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, k, first, last)
        fine(ada, ctx)
        assert lists_of(idx, cnt) == ref.select(c.cpu, c.Q, c.off, c.lens, 2, k, first, last), (k, first, last)


def test_select_ties_go_to_the_lower_page(ada, ctx):
    """Pages with the same bounds, and queries of zeros: every score equal."""
    c = Case(ada, 21, 4, 2, 64, 16, [2], [1600])
    c.cache.kmin.copy_(c.cache.kmin[:1].nan_to_num().expand_as(c.cache.kmin).clone())
    c.cache.kmax.copy_(c.cache.kmax[:1].nan_to_num().expand_as(c.cache.kmax).clone())
    for Q in (c.d_Q, torch.zeros_like(c.d_Q)):
        idx, cnt = ada.ada_select_blocks(ctx, c.cache, Q, c.d_off, c.d_len, 10, 0, 2)
        fine(ada, ctx)
        assert lists_of(idx, cnt) == [[list(range(8)) + [98, 99]] * 2] * 2


def test_select_near_ties(ada, ctx):
    """Scores that differ by less than fp32 tells apart: the 64-bit order decides."""
    c = Case(ada, 22, 2, 2, 128, 16, [1], [16 * 700])
    base = torch.randn(128).bfloat16()
    for p in range(700):
        page = int(c.cpu.table[0, p])
        k = base.clone()
        k[p % 128] = (k[p % 128].float() * (1 + 2.0 ** -7)).bfloat16()
        c.cpu.kmin[page] = k
        c.cpu.kmax[page] = k
    c.cache.kmin.copy_(c.cpu.kmin)
    c.cache.kmax.copy_(c.cpu.kmax)
    Q = c.Q.float()
    Q[..., 0] = 1e4
    Q[..., 1:] *= 2.0 ** -10
    c.Q = Q.bfloat16()
    idx, cnt = ada.ada_select_blocks(ctx, c.cache, c.Q.cuda(), c.d_off, c.d_len, 40, 1, 1)
    fine(ada, ctx)
    assert lists_of(idx, cnt) == ref.select(c.cpu, c.Q, c.off, c.lens, 2, 40, 1, 1)


@pytest.mark.parametrize("width", [300, 1024, 2100, 4096, 8192, 16384])
@pytest.mark.parametrize("news,lens", [([40, 1, 0, 3], [1500, 700, 20, 90]), ([1, 1, 1], [4000, 16, 333])])
def test_wide_tables(ada, ctx, news, lens, width):
    """A table for far longer texts than there are: the same pages, whether a call may look at all of it or at its front."""
    c = Case(ada, 29, 4, 2, 64, 16, news, lens, pad=1, drift=0.5)
    B, used = c.cache.table.shape
    wide = torch.full((B, width), -3, dtype=torch.int32, device="cuda")
    wide[:, :used] = c.cache.table
    want = ref.select(c.cpu, c.Q, c.off, c.lens, 2, 9, 1, 1)[:c.off[-1]]
    out = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new)
    for table in (wide, wide[:, :used], wide[:, :used + 100]):
        cache = ada.KVCache(c.cache.K, c.cache.V, table, c.cache.kmin, c.cache.kmax)
        idx, cnt = ada.ada_select_blocks(ctx, cache, c.d_Q, c.d_off, c.d_len, 9)
        got = ada.ada_attention_cached(ctx, cache, c.d_Q, c.d_off, c.d_len, c.max_new)
        fine(ada, ctx)
        assert lists_of(idx[:c.off[-1]], cnt[:c.off[-1]]) == want
        assert torch.equal(got, out)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("close", [2, 9, 30])
@pytest.mark.parametrize("news,pages", [([1], 100), ([1], 700), ([1], 1500), ([3], 100), ([3], 700), ([5], 100), ([5], 700), ([16], 300)])
def test_select_scores_that_fp32_cannot_tell_apart(ada, ctx, news, pages, close, sign):
    """`close` pages around the last place differ by less than an fp32 score can show, all others by far more: few enough
    to be scored again one by one, whose order in 64 bits runs against that of the pages."""
    hk, d, ps = 2, 64, 16
    n = news[0]
    g = torch.Generator().manual_seed(pages + close)
    table = torch.randperm(pages, generator=g).int().view(1, -1)
    for above in (3, 40):                                    # places that are given for certain: few and many
        bound = torch.zeros((pages, hk, d))
        order = torch.randperm(pages, generator=g)
        ahead, near_, rest = order[:above], order[above:above + close].sort().values, order[above + close:]
        bound[ahead, :, 0] = 112.0
        bound[rest, :, 0] = (8.0 + 0.25 * (torch.arange(len(rest)) % 128)).view(-1, 1)
        bound[near_, :, 0] = 96.0
        # 2^-14 (1 + i / 128), more for the higher page: 2^-21 a step, where a score of 96 has a last place of 2^-17
        bound[near_, :, 1] = (1.0 + torch.arange(close) / 128.0).view(-1, 1)
        bound[..., 0] *= sign
        Q = torch.zeros((n, 4, d))
        Q[..., 0] = sign
        Q[..., 1] = 2.0 ** -14
        Q *= 2.0 ** (torch.arange(n) % 3).view(-1, 1, 1)
        Q = Q.bfloat16()
        k_ = bound.bfloat16()
        assert torch.equal(k_.float(), bound)
        kmin = torch.empty_like(k_)
        kmin[table[0].long()] = k_
        KV = torch.zeros((pages, hk, ps, d), dtype=torch.bfloat16, device="cuda")
        cache = ada.KVCache(KV, KV, table.cuda(), kmin.cuda(), kmin.cuda())
        cpu = ref.Pages(KV, KV, table, kmin, kmin)
        length = pages * ps
        for need in {1, close // 2, close - 1} - {0}:
            k = above + need
            # causal tokens of one sequence: all of them see the last page
            idx, cnt = ada.ada_select_blocks(ctx, cache, Q.cuda(), i32([0, n]), i32([length]), k, 0, 0)
            fine(ada, ctx)
            want = ref.select(cpu, Q, [0, n], [length], hk, k, 0, 0)
            assert all(x == sorted(ahead.tolist() + near_[close - need:].tolist()) for row in want for x in row)
            assert lists_of(idx, cnt) == want, (above, need)


def test_select_infinite_bounds(ada, ctx):
    """A page whose score is NaN comes last, an infinite one first."""
    c = Case(ada, 23, 2, 2, 64, 16, [1], [1600])
    page = [int(x) for x in c.cpu.table[0, :100]]
    c.cache.kmax[page[40]] = math.inf
    c.cache.kmin[page[50]] = -math.inf
    c.cache.kmax[page[50]] = -math.inf
    idx, cnt = ada.ada_select_blocks(ctx, c.cache, c.d_Q.abs(), c.d_off, c.d_len, 99, 0, 0)
    assert all(50 not in x and 40 in x for x in lists_of(idx, cnt)[0])
    c.cache.kmin[page[60]] = math.nan
    Q = c.d_Q.clone()
    idx, cnt = ada.ada_select_blocks(ctx, c.cache, Q, c.d_off, c.d_len, 98, 0, 0)
    assert all(60 not in x for x in lists_of(idx, cnt)[0])


# ---------------------------------------------------------------- attention on chosen pages
@pytest.mark.parametrize("ps,k", [(16, 5), (32, 4), (64, 3), (128, 2)])
@pytest.mark.parametrize("h,hk,d", HEADS + [(40, 2, 64)])
def test_blocks(ada, ctx, h, hk, d, ps, k):
    for seed, (news, lens) in enumerate([([1, 1], [900, 33]), ([37, 0, 3], [500, 9, 2]), ([320 // hk], [400])]):
        c = Case(ada, 30 + seed, h, hk, d, ps, news, lens)
        idx, cnt = ada.ada_select_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, k, 1, 1)
        for causal in (True, False):
            out = ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt, flags=int(causal))
            fine(ada, ctx)
            c.check(out, causal, lists=lists_of(idx, cnt))


@pytest.mark.parametrize("h,hk,d,ps,n", [(8, 2, 128, 64, 610), (32, 2, 64, 16, 600), (6, 6, 80, 32, 200), (40, 2, 128, 16, 205)])
def test_blocks_of_many_rows(ada, ctx, h, hk, d, ps, n):
    """Row tiles enough for a warp each; lists of all lengths, none among them, padding rows behind."""
    c = Case(ada, 34, h, hk, d, ps, [n - 3, 0, 3], [n + 150, 4, 90], pad=2)
    g = torch.Generator().manual_seed(n)
    k = 7
    idx, cnt = torch.full((c.N, hk, k), -9, dtype=torch.int32), torch.zeros((c.N, hk), dtype=torch.int32)
    lists = [[[] for _ in range(hk)] for _ in range(c.N)]
    for i in range(n):
        pages = -(-c.lens[0 if i < n - 3 else 2] // ps)
        for j in range(hk):
            m = min(int(torch.randint(0, k + 1, (1,), generator=g)), pages)
            lists[i][j] = sorted(torch.randperm(pages, generator=g)[:m].tolist())
            idx[i, j, :m] = torch.tensor(lists[i][j], dtype=torch.int32)
            cnt[i, j] = m
    out = torch.full((c.N, h, d), 9.0, dtype=torch.bfloat16, device="cuda")
    ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx.cuda(), cnt.cuda(), out=out)
    fine(ada, ctx)
    c.check(out, True, lists=lists)
    assert bool((out[n:] == 9.0).all())


def test_blocks_with_lists_of_any_kind(ada, ctx):
    """Empty lists, lists of one page, pages that the token does not see (no slot of theirs counts), long lists."""
    c = Case(ada, 33, 4, 2, 128, 16, [4, 1], [700, 800], pad=2)
    k = 50
    lists = [[[], [0]], [[43], list(range(44))], [list(range(0, 44, 2)), [3, 43]], [[42], [1, 2, 3]],
             [list(range(50)), [49]]]
    idx = torch.full((c.N, 2, k), -5, dtype=torch.int32)
    cnt = torch.full((c.N, 2), 1 << 20, dtype=torch.int32)
    for i, row in enumerate(lists):
        for j, x in enumerate(row):
            idx[i, j, :len(x)] = torch.tensor(x, dtype=torch.int32)
            cnt[i, j] = len(x)
    out = torch.full((c.N, 4, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, idx.cuda(), cnt.cuda(), out=out)
    fine(ada, ctx)
    c.check(out, True, lists=lists)
    assert bool((out[5:] == 9.0).all())


# ---------------------------------------------------------------- appending
def near(got, want, row_max):
    """bf16 rounding of the value, and fp32 arithmetic on what enters it."""
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -19 * row_max
    return bool(((got.cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("ps", [16, 64])
@pytest.mark.parametrize("h,hk,d,rot,pairs,norm", [(4, 2, 128, 128, False, True), (3, 3, 64, 32, True, False),
                                                   (8, 1, 80, 80, False, True), (2, 2, 16, 16, True, True),
                                                   (5, 5, 96, 0, False, False), (2, 1, 128, 64, False, False)])
def test_append(ada, ctx, h, hk, d, rot, pairs, norm, ps):
    g = torch.Generator().manual_seed(d + rot)
    # (no more rows than sequences: the form for single tokens, also where they are not spread one to each)
    for news, olds, pad in (([1, 1, 1], [0, 15, 200], 3), ([70, 0, 33], [5, 9, 64], 3), ([700], [0], 3),
                            ([1, 1, 1, 1], [0, 15, 16, 200], 0), ([5, 0, 0, 1, 0, 0, 0, 0], [14, 3, 0, 31, 1, 2, 3, 4], 2),
                            ([0] * 30 + [20] + [0] * 10, [5] * 41, 21)):
        lens = [a + b for a, b in zip(news, olds)]
        c = Case(ada, 40, h, hk, d, ps, news, lens, pad=pad, planes=True)
        qkv = torch.randn((c.N, (h + 2 * hk) * d), generator=g).bfloat16()
        qkv[c.off[-1]:] = math.nan                       # padding is not read
        Q, K, V = (x.unflatten(1, (-1, d)) for x in qkv.split([h * d, hk * d, hk * d], 1))
        dQ, dK, dV = (x.unflatten(1, (-1, d)) for x in qkv.cuda().split([h * d, hk * d, hk * d], 1))
        w = [(1 + 0.1 * torch.randn(d, generator=g)).bfloat16() for _ in range(2)] if norm else [None, None]
        f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1)) if rot else None
        pos0 = [7 + 1000000 * b for b in range(len(news))] if pairs else None
        want = ref.append(c.cpu, K, V, c.off, olds, Q, *w, 1e-6, f, pairs, pos0)
        q_out = torch.full((c.N, h, d), 3.0, dtype=torch.bfloat16, device="cuda")
        q, n = ada.ada_cache_append(ctx, c.cache, dK, dV, c.d_off, i32(olds), Q=dQ, q_out=q_out,
                                    q_norm=None if w[0] is None else w[0].cuda(),
                                    k_norm=None if w[1] is None else w[1].cuda(),
                                    inv_freq=None if f is None else f.cuda(), pos0=None if pos0 is None else i32(pos0),
                                    flags=ada.ADA_ROPE_PAIRS if pairs else 0)
        fine(ada, ctx)
        assert n.tolist() == want[5] == lens
        big = 6.0 * (1.5 if norm else 1.0)
        m = c.off[-1]
        assert near(q[:m], want[4][:m], big) and bool((q[m:] == 3.0).all())
        live = ~want[0].isnan()
        assert bool((live == ~c.cache.K.isnan().cpu()).all())
        assert near(c.cache.K.cpu().nan_to_num(), want[0].nan_to_num(), big)
        assert torch.equal(c.cache.V.cpu().nan_to_num(), want[1].nan_to_num())
        touched = ~torch.isnan(want[2])
        assert near(c.cache.kmin.cpu()[touched], want[2][touched], big)
        assert near(c.cache.kmax.cpu()[touched], want[3][touched], big)
        assert bool(c.cache.kmin.isnan().cpu()[~touched].all())


@pytest.mark.parametrize("news", [[1, 1, 1], [40, 2, 9]])
def test_append_of_keys_and_values_alone(ada, ctx, news):
    """No queries, no bounds, a norm without rotation, and neither."""
    c = Case(ada, 45, 2, 2, 48, 16, news, [n + 5 for n in news])
    cache = ada.KVCache(c.cache.K, c.cache.V, c.cache.table)
    g = torch.Generator().manual_seed(4)
    K, V = (torch.randn((c.N, 2, 48), generator=g).bfloat16() for _ in range(2))
    w = (1 + 0.1 * torch.randn(48, generator=g)).bfloat16()
    for weight in (w, None):
        want = ref.append(ref.Pages(c.cpu.K, c.cpu.V, c.cpu.table), K, V, c.off, [5] * 3, None, None, weight, 1e-5)
        q, n = ada.ada_cache_append(ctx, cache, K.cuda(), V.cuda(), c.d_off, i32([5] * 3), eps=1e-5,
                                    k_norm=None if weight is None else weight.cuda())
        fine(ada, ctx)
        assert q is None and n.tolist() == [x + 5 for x in news]
        assert near(cache.K.cpu().nan_to_num(), want[0].nan_to_num(), 8.0)
        assert torch.equal(cache.V.cpu().nan_to_num(), want[1].nan_to_num())


def test_append_in_place_and_far_positions(ada, ctx):
    """q_out may be Q; positions of tens of millions turn by the right angle."""
    c = Case(ada, 41, 2, 2, 64, 32, [3, 2], [3, 2])
    f = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    pos0 = [50_000_001, 2_000_000_000]
    K, V = torch.randn(5, 2, 64).bfloat16(), torch.randn(5, 2, 64).bfloat16()
    want = ref.append(c.cpu, K, V, c.off, [0, 0], c.Q, None, None, 1e-6, f, False, pos0)
    Q = c.d_Q.clone()
    q, n = ada.ada_cache_append(ctx, c.cache, K.cuda(), V.cuda(), c.d_off, i32([0, 0]), Q=Q, q_out=Q, inv_freq=f.cuda(),
                                pos0=i32(pos0))
    fine(ada, ctx)
    assert q.data_ptr() == Q.data_ptr()
    # an angle of 2e9 in 64 bits is good to 2^-22, next to nothing here
    assert near(q, want[4], 8.0)
    assert near(c.cache.K.cpu().nan_to_num(), want[0].nan_to_num(), 8.0)


@pytest.mark.parametrize("news", [[5], [5, 0, 0, 0, 0, 1]])
def test_positions_behind_the_largest_int32(ada, ctx, news):
    """Positions go on behind 2^31 - 1, in both forms of the append (several tokens; no more rows than sequences)."""
    B = len(news)
    c = Case(ada, 46, 2, 2, 64, 32, news, [max(n, 1) for n in news])
    f = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    pos0 = [2 ** 31 - 3] * B
    K, V = torch.randn(c.N, 2, 64).bfloat16(), torch.randn(c.N, 2, 64).bfloat16()
    want = ref.append(c.cpu, K, V, c.off, [0] * B, c.Q, None, None, 1e-6, f, False, pos0)
    q, _ = ada.ada_cache_append(ctx, c.cache, K.cuda(), V.cuda(), c.d_off, i32([0] * B), Q=c.d_Q, inv_freq=f.cuda(), pos0=i32(pos0))
    fine(ada, ctx)
    # (the angle, up to 2^31 radians, is rounded to 64 bits: 2^-22, times an element of up to 8, half of near()'s 2^-19 x 8)
    assert near(q, want[4], 8.0)
    for got, w in ((c.cache.K, want[0]), (c.cache.kmin, want[2]), (c.cache.kmax, want[3])):
        assert near(got.cpu().nan_to_num(), w.nan_to_num(), 8.0)


def test_append_of_representatives(ada, ctx):
    """Only the listed tokens are kept, rotated where they stood; the queries are not affected."""
    news, olds = [50, 20, 10], [3, 0, 8]
    lists = [[0, 1, 7, 8, 30, 49], [], list(range(10))]
    lens = [o + len(x) for o, x in zip(olds, lists)]
    c = Case(ada, 42, 4, 2, 64, 16, news, [max(x, 1) for x in lens])
    g = torch.Generator().manual_seed(1)
    K, V = (torch.randn((c.N, 2, 64), generator=g).bfloat16() for _ in range(2))
    f = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    idx = torch.full((c.N,), -1, dtype=torch.int32)
    for b, x in enumerate(lists):
        idx[c.off[b]:c.off[b] + len(x)] = torch.tensor(x, dtype=torch.int32)
    want = ref.append(c.cpu, K, V, c.off, olds, c.Q, None, None, 1e-6, f, False, [5, 6, 7], lists)
    q, n = ada.ada_cache_append(ctx, c.cache, K.cuda(), V.cuda(), c.d_off, i32(olds), Q=c.d_Q, inv_freq=f.cuda(),
                                pos0=i32([5, 6, 7]), rep_idx=idx.cuda(), rep_cnt=i32([len(x) for x in lists]))
    fine(ada, ctx)
    assert n.tolist() == lens
    assert near(q, want[4], 8.0)
    assert near(c.cache.K.cpu().nan_to_num(), want[0].nan_to_num(), 8.0)
    assert torch.equal(c.cache.V.cpu().nan_to_num(), want[1].nan_to_num())
    assert near(c.cache.kmax.cpu().nan_to_num(), want[3].nan_to_num(), 8.0)


def test_append_of_representatives_to_few_rows(ada, ctx):
    """The form for single tokens with lists: kept tokens that share a page."""
    news, olds = [6, 0, 0, 1, 0, 0, 0], [14, 2, 0, 3, 1, 1, 1]
    lists = [[0, 2, 3, 5], [], [], [0], [], [], []]
    lens = [o + len(x) for o, x in zip(olds, lists)]
    c = Case(ada, 44, 4, 2, 64, 16, news, [max(x, 1) for x in lens])
    g = torch.Generator().manual_seed(2)
    K, V = (torch.randn((c.N, 2, 64), generator=g).bfloat16() for _ in range(2))
    f = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    idx = torch.full((c.N,), -1, dtype=torch.int32)
    for b, x in enumerate(lists):
        idx[c.off[b]:c.off[b] + len(x)] = torch.tensor(x, dtype=torch.int32)
    pos0 = [100 * b for b in range(7)]
    want = ref.append(c.cpu, K, V, c.off, olds, c.Q, None, None, 1e-6, f, False, pos0, lists)
    q, n = ada.ada_cache_append(ctx, c.cache, K.cuda(), V.cuda(), c.d_off, i32(olds), Q=c.d_Q, inv_freq=f.cuda(),
                                pos0=i32(pos0), rep_idx=idx.cuda(), rep_cnt=i32([len(x) for x in lists]))
    fine(ada, ctx)
    assert n.tolist() == lens and near(q, want[4], 8.0)
    for got, w in ((c.cache.K, want[0]), (c.cache.kmin, want[2]), (c.cache.kmax, want[3])):
        assert near(got.cpu().nan_to_num(), w.nan_to_num(), 8.0)
    assert torch.equal(c.cache.V.cpu().nan_to_num(), want[1].nan_to_num())


def test_bounds_of_a_page_that_was_taken_back(ada, ctx):
    """Tokens that were taken back (a shorter length) have no part in the bounds formed next."""
    c = Case(ada, 43, 1, 1, 16, 16, [1], [12])
    page = int(c.cpu.table[0, 0])
    c.cache.K[page, 0, 8:] = 100.0
    K = torch.zeros((1, 1, 16), dtype=torch.bfloat16, device="cuda")
    ada.ada_cache_append(ctx, c.cache, K, K, c.d_off, i32([6]))
    fine(ada, ctx)
    live = torch.cat([c.cpu.K[page, 0, :6].float(), torch.zeros(1, 16)])
    assert torch.equal(c.cache.kmax[page, 0].cpu().float(), live.amax(0))
    assert torch.equal(c.cache.kmin[page, 0].cpu().float(), live.amin(0))


# ---------------------------------------------------------------- faults
def status(ada, ctx):
    return ada.ada_device_status(ctx)[0]


@pytest.mark.parametrize("max_new", [1, 30])
def test_bad_pages_and_offsets_are_reported(ada, ctx, max_new):
    news = [max_new, 1]
    c = Case(ada, 60, 4, 2, 64, 16, news, [200, 50])
    good = ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, max_new)
    fine(ada, ctx)
    table = c.cache.table.clone()
    for bad in (-1, c.cache.K.shape[0], 1 << 30):
        c.cache.table[0, 3] = bad
        ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, max_new)
        assert status(ada, ctx) == 5
        ada.ada_select_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 4)
        assert status(ada, ctx) == 5
        ada.ada_cache_append(ctx, c.cache, c.d_Q[:, :2], c.d_Q[:, :2], c.d_off, i32([60, 0]))
        assert status(ada, ctx) == (5 if max_new == 1 or 60 + max_new > 48 else 0)
        c.cache.table.copy_(table)
    for off in ([0, max_new + 1, max_new], [0, -1, 1], [1, 2, 3], [0, 1, 1000]):
        for call in (lambda o: ada.ada_attention_cached(ctx, c.cache, c.d_Q, o, c.d_len, max_new),
                     lambda o: ada.ada_select_blocks(ctx, c.cache, c.d_Q, o, c.d_len, 4),
                     lambda o: ada.ada_cache_append(ctx, c.cache, c.d_Q[:, :2], c.d_Q[:, :2], o, i32([0, 0]))):
            call(i32(off))
            assert status(ada, ctx) == 5
    for lens in ([-1, 50], [1 << 29, 50]):
        ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, i32(lens), max_new)
        assert status(ada, ctx) == 5
    if max_new > 1:                                # more new tokens than max_new
        ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, max_new - 1)
        assert status(ada, ctx) == 5
        ada.ada_attention_cached(ctx, c.cache, c.d_Q, c.d_off, c.d_len, 1)
        assert status(ada, ctx) == 5
    c2 = Case(ada, 60, 4, 2, 64, 16, news, [200, 50])
    out = ada.ada_attention_cached(ctx, c2.cache, c2.d_Q, c2.d_off, c2.d_len, max_new)
    fine(ada, ctx)
    assert torch.equal(out, good)


@pytest.mark.parametrize("off", [[0, 3, 2, 3, 4], [0, 1, -5, 3, 4], [1, 2, 3, 4, 4], [3, 4, 0, 1, 2], [0, 1, 2, 1000, 4], [0, 0, 4, 4, 1]])
def test_calls_after_faulty_offsets(ada, ctx, off):
    """Whatever the offsets say, a call leaves the workspace as the next one needs it: nobody has asked for the status
    (which would clear it) in between."""
    c = Case(ada, 63, 8, 2, 64, 128, [1] * 4, [9000, 5000, 8192, 7000])
    many = Case(ada, 64, 8, 2, 64, 64, [30, 40, 20, 50], [3000, 900, 700, 4000])
    k = 64
    idx = torch.arange(k, dtype=torch.int32, device="cuda").expand(4, 2, k).contiguous()
    cnt = torch.full((4, 2), k, dtype=torch.int32, device="cuda")
    cnt[1:] = torch.tensor([[40, 3], [64, 64], [55, 50]])

    def run(o, o_many):
        return (ada.ada_attention_blocks(ctx, c.cache, c.d_Q, o, c.d_len, idx, cnt),            # lists in pieces
                ada.ada_attention_cached(ctx, c.cache, c.d_Q, o, c.d_len, 1),
                ada.ada_attention_cached(ctx, many.cache, many.d_Q, o_many, many.d_len, 50))

    good = run(c.d_off, many.d_off)
    fine(ada, ctx)
    bad = [run(i32(off), i32([30 * x for x in off])) for _ in range(3)]
    after = [run(c.d_off, many.d_off) for _ in range(3)]
    assert status(ada, ctx) == 5
    assert all(torch.equal(x, y) for got in after for x, y in zip(got, good))
    assert all(torch.equal(x, y) for got in bad for x, y in zip(got, bad[0]))
    again = run(c.d_off, many.d_off)
    fine(ada, ctx)
    assert all(torch.equal(x, y) for x, y in zip(again, good))


def test_bad_lists_are_reported(ada, ctx):
    c = Case(ada, 61, 4, 2, 64, 16, [1], [200])
    for idx, cnt in (([3, 3, 4], 3), ([4, 3, 5], 3), ([-1, 3, 4], 3), ([1, 2, 1000], 3), ([1, 2, 3], 4), ([1, 2, 3], -1)):
        i = i32([idx, [0, 1, 2]]).view(1, 2, 3)
        ada.ada_attention_blocks(ctx, c.cache, c.d_Q, c.d_off, c.d_len, i, i32([[cnt, 3]]))
        assert status(ada, ctx) == 5
    K = c.d_Q[:, :2]
    for idx, cnt in (([0], 2), ([0], -1), ([1], 1), ([-1], 1)):
        ada.ada_cache_append(ctx, c.cache, K, K, c.d_off, i32([0]), rep_idx=i32(idx), rep_cnt=i32([cnt]))
        assert status(ada, ctx) == 5


def test_nonfinite_and_full_tables_are_reported(ada, ctx):
    c = Case(ada, 62, 4, 2, 64, 16, [2], [200])
    cap = c.cache.table.shape[1] * 16
    c.cache.table.clamp_(0, 3)
    K = c.d_Q[:, :2].clone()
    before = c.cache.K.clone()
    _, n = ada.ada_cache_append(ctx, c.cache, K, K, c.d_off, i32([cap]))
    assert status(ada, ctx) == 5 and n.tolist() == [cap]
    assert torch.equal(before.nan_to_num(), c.cache.K.nan_to_num())
    K[1, 1, 3] = math.inf
    ada.ada_cache_append(ctx, c.cache, K, c.d_Q[:, :2], c.d_off, i32([0]))
    assert status(ada, ctx) == 6
    K[1, 1, 3] = math.nan
    ada.ada_cache_append(ctx, c.cache, c.d_Q[:, :2], K, c.d_off, i32([0]))
    assert status(ada, ctx) == 6


# ---------------------------------------------------------------- streams, graphs, a run of all
def test_another_stream_and_two_contexts_at_once(ada):
    a, b = (ada.ada_create(1, 128, 128, ada.ADA_F32) for _ in range(2))    # (a context's storage type does not matter)
    cases = [Case(ada, 70 + i, 8, 2, 128, 64, n, l) for i, (n, l) in enumerate([([1, 1], [5000, 9000]), ([300], [3000])])]
    want = [ada.ada_attention_cached(a, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [ada.ada_attention_cached(x, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new, stream=s,
                                        out=torch.zeros_like(c.d_Q)) for x, c, s in zip((a, b), cases, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    for x in (a, b):
        fine(ada, x)
        ada.ada_destroy(x)


def test_fresh_outputs_on_another_stream(ada):
    """A call on another stream than the current one, which has a long queue: its outputs are its own, cleared in time."""
    own = ada.ada_create(1, 128, 128, ada.ADA_BF16)
    cases = [Case(ada, 72 + i, 8, 2, 128, 64, n, l) for i, (n, l) in enumerate([([1, 1], [5000, 900]), ([300], [3000])])]

    def run(c, **kw):
        out = ada.ada_attention_cached(own, c.cache, c.d_Q, c.d_off, c.d_len, c.max_new, **kw)
        idx, cnt = ada.ada_select_blocks(own, c.cache, c.d_Q, c.d_off, c.d_len, 5, **kw)
        return out, idx, cnt, ada.ada_attention_blocks(own, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt, **kw)

    want = [run(c) for c in cases]
    X = torch.randn((8192, 8192), device="cuda").bfloat16()
    Y = torch.empty_like(X)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        for _ in range(20):
            torch.matmul(X, X, out=Y)
        got = [run(c, stream=side) for c in cases]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b))
    fine(ada, own)
    ada.ada_destroy(own)


def test_kernel_times_and_launches_without_overlap(ada, ctx):
    """Every kernel of the calls is in the per-kernel timing; without dependent launches the results are the same."""
    c = Case(ada, 31, 8, 2, 64, 16, [70, 1], [900, 300])
    K, V = (torch.randn(71, 2, 64, device="cuda").bfloat16() for _ in range(2))

    def run():
        pages = ada.KVCache(*(x.clone() for x in (c.cache.K, c.cache.V, c.cache.table, c.cache.kmin, c.cache.kmax)))
        ada.ada_cache_append(ctx, pages, K, V, c.d_off, i32([830, 299]))
        out = ada.ada_attention_cached(ctx, pages, c.d_Q, c.d_off, c.d_len, 70)
        idx, cnt = ada.ada_select_blocks(ctx, pages, c.d_Q, c.d_off, c.d_len, 6)
        return out, idx, cnt, ada.ada_attention_blocks(ctx, pages, c.d_Q, c.d_off, c.d_len, idx, cnt)

    want = run()
    ada.ada_profile_enable(ctx, True)
    ada.ada_set_dependent_launch(ctx, False)
    try:
        got = run()
        times = {k: v for k, v in ada.ada_profile_read(ctx).items() if v[0]}
    finally:
        ada.ada_profile_enable(ctx, False)
        ada.ada_set_dependent_launch(ctx, True)
    fine(ada, ctx)
    assert {k: n for k, (n, _) in times.items()} == {"cache_append": 1, "cache_bounds": 1, "cache_step": 2, "cache_chunk": 1,
                                                     "cache_select": 1}
    assert all(t > 0 for _, t in times.values())
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_captured_step(ada, ctx):
    """A decoding step as a graph: append, choose, attend; replayed over growing lengths that live on the device."""
    h, hk, d, ps, k = 8, 2, 64, 16, 4
    c = Case(ada, 80, h, hk, d, ps, [1, 1], [300, 70])
    lens = i32([200, 60])
    nxt = torch.empty_like(lens)
    g = torch.Generator(device="cuda").manual_seed(5)
    K, V = (torch.randn((2, hk, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    f = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).cuda()
    q = torch.empty_like(c.d_Q)
    idx, cnt = torch.empty((2, hk, k), dtype=torch.int32, device="cuda"), torch.empty((2, hk), dtype=torch.int32, device="cuda")
    dense, sparse = torch.zeros_like(q), torch.zeros_like(q)

    def step():
        ada.ada_cache_append(ctx, c.cache, K, V, c.d_off, lens, len_out=nxt, Q=c.d_Q, q_out=q, inv_freq=f)
        ada.ada_attention_cached(ctx, c.cache, q, c.d_off, nxt, 1, out=dense)
        ada.ada_select_blocks(ctx, c.cache, q, c.d_off, nxt, k, blk_idx=idx, blk_cnt=cnt)
        ada.ada_attention_blocks(ctx, c.cache, q, c.d_off, nxt, idx, cnt, out=sparse)
        lens.copy_(nxt)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(9):
        K.normal_(generator=g)
        V.normal_(generator=g)
        graph.replay()
    fine(ada, ctx)
    assert lens.tolist() == [210, 70]
    cpu = ref.Pages(c.cache.K.cpu(), c.cache.V.cpu(), c.cpu.table, c.cache.kmin.cpu(), c.cache.kmax.cpu())
    Q = q.cpu()
    for out, lists in ((dense, None), (sparse, lists_of(idx, cnt))):
        want, weight = ref.attend(cpu, Q, c.off, [210, 70], hk, True, 0.0, lists)
        tol = ref.tolerance(want, weight, cpu.V.float().nan_to_num())
        assert bool(((out.cpu().double() - want).abs() <= tol).all())
    assert lists_of(idx, cnt) == ref.select(cpu, Q, c.off, [210, 70], hk, k, 1, 1)


@pytest.mark.parametrize("mode", ["global", "relaxed"])
def test_first_call_while_a_graph_is_captured(ada, mode):
    """It would have to allocate: refused, the capture goes on, and the context serves as if nothing had been."""
    own = ada.ada_create(1, 128, 128, ada.ADA_BF16)
    c = Case(ada, 81, 8, 2, 64, 16, [1, 1], [3000, 70])
    other = Case(ada, 82, 8, 2, 64, 16, [200], [300])
    x = torch.zeros(4, device="cuda")
    idx, cnt = torch.zeros((2, 2, 4), dtype=torch.int32, device="cuda"), torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode=mode):
        for call in (lambda: ada.ada_attention_cached(own, c.cache, c.d_Q, c.d_off, c.d_len, 1),
                     lambda: ada.ada_attention_cached(own, other.cache, other.d_Q, other.d_off, other.d_len, 200),
                     lambda: ada.ada_attention_blocks(own, c.cache, c.d_Q, c.d_off, c.d_len, idx, cnt)):
            with pytest.raises(ada.AdaError) as e:
                call()
            assert e.value.status == 4
        x += 1
    for _ in range(3):
        for y in (c, other):
            y.check(ada.ada_attention_cached(own, y.cache, y.d_Q, y.d_off, y.d_len, y.max_new), True)
    graph.replay()
    torch.cuda.synchronize()
    assert x.tolist() == [1.0] * 4
    fine(ada, own)
    ada.ada_destroy(own)


def test_prompt_to_generation(ada, ctx):
    """What the library is for, from end to end: the prompt's representatives are selected, the prompt's attention
    runs on them, their keys and values go to the cache, and the next chunk and token attend to it."""
    T, h, hk, d, ps = 300, 4, 2, 32, 16
    g = torch.Generator().manual_seed(3)
    protos = torch.randn((40, h * d), generator=g)
    X = (protos[torch.randint(0, 40, (T,), generator=g)] + 0.05 * torch.randn((T, h * d), generator=g)).bfloat16()
    own = ada.ada_create(1, T, h * d, ada.ADA_BF16)
    rep, cnt, _ = ada.ada_select_full(own, X.cuda().unsqueeze(0), 0.3)
    Xh = X.cuda().view(T, h, d)
    near_idx, _ = ada.ada_nearest_rep(own, X.cuda().unsqueeze(0), rep, cnt)
    ada.ada_attention_reps(own, Xh, Xh, Xh, rep[0], cnt, nearest_idx=near_idx[0])
    R = rep[0, :int(cnt[0])].tolist()
    assert 30 <= len(R) < 120
    pool = 20
    K, V = (torch.full((pool, hk, ps, d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kmin, kmax = torch.zeros((2, pool, hk, d), dtype=torch.bfloat16, device="cuda")
    cache = ada.KVCache(K, V, torch.randperm(pool, generator=g).int().cuda().view(1, pool), kmin, kmax)
    f = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    _, n = ada.ada_cache_append(own, cache, Xh[:, :hk], Xh[:, hk:], i32([0, T]), i32([0]), inv_freq=f.cuda(), rep_idx=rep[0],
                                rep_cnt=cnt)
    k64 = [ref.turned(X.view(T, h, d)[t, :hk].double(), t, f, False) for t in R]
    v64 = [X.view(T, h, d)[t, hk:].double() for t in R]
    at = T
    for m in (33, 1, 1):                           # a chunk, then single tokens; positions go on from the prompt's
        Y = torch.randn((m, (h + 2 * hk) * d), generator=g).bfloat16()
        q, k, v = (x.unflatten(1, (-1, d)) for x in Y.cuda().split([h * d, hk * d, hk * d], 1))
        q, n = ada.ada_cache_append(own, cache, k, v, i32([0, m]), n, Q=q, inv_freq=f.cuda(), pos0=i32([at]))
        out = ada.ada_attention_cached(own, cache, q, i32([0, m]), n, m)
        idx, c = ada.ada_select_blocks(own, cache, q, i32([0, m]), n, pool)
        every = ada.ada_attention_blocks(own, cache, q, i32([0, m]), n, idx, c)
        fine(ada, own)
        Y = Y.double()
        for i in range(m):
            k64.append(ref.turned(Y[i, h * d:(h + hk) * d].view(hk, d), at + i, f, False))
            v64.append(Y[i, (h + hk) * d:].view(hk, d))
        at += m
        assert int(n[0]) == len(k64)
        for i in range(m):
            Kt, Vt = torch.stack(k64)[:len(k64) - m + i + 1], torch.stack(v64)[:len(k64) - m + i + 1]
            qi = ref.turned(Y[i, :h * d].view(h, d), at - m + i, f, False)
            for x in range(h):
                s = Kt[:, x // 2] @ qi[x] / math.sqrt(d)
                p = torch.softmax(s, 0)
                # queries and keys are rounded to bf16 here: a score is off by up to 2 x 2^-8 of |q||k| / sqrt(d)
                slack = 2 * 2.0 ** -8 * float((Kt[:, x // 2].abs() @ qi[x].abs()).max()) / math.sqrt(d)
                want, weight = p @ Vt[:, x // 2], p @ Vt[:, x // 2].abs()
                tol = 2.0 ** -8 * (weight + want.abs()) + (math.exp(2 * slack) - 1) * weight + 1e-3
                for got in (out, every):
                    assert bool(((got[i, x].cpu().double() - want).abs() <= tol).all())
    ada.ada_destroy(own)
