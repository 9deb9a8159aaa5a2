"""What the calls on a paged cache refuse, without a GPU: the library's argument checks (compiled as host code), the
binding's checks of tensors; and the tests' own reference against an independent statement."""
import math
import subprocess

import pytest
import torch

import cache_ref as ref
from paper_2605_03110_b200 import build as ada_build


@pytest.fixture(scope="module")
def ada():
    ada_build.build()
    from paper_2605_03110_b200 import binding
    binding.lib()
    return binding


def run_host_code(tmp_path, body):
    src = tmp_path / "args.cc"
    src.write_text('#include "cache_args.h"\n#include <cmath>\n#include <initializer_list>\n#undef NDEBUG\n#include <assert.h>\nusing namespace ada;\n'
                   'int main() {' + body + "return 0; }")
    exe = str(tmp_path / "args")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", ada_build.CSRC, "-o", exe, str(src)], check=True)
    subprocess.run([exe], check=True)


PREFIX = """
    char* at = (char*)4096; int32_t* ints = (int32_t*)at;
    const ada_kv_cache good = {at, at, at, at, ints, 8, 8, 100, 2 * 64 * 128, 64, 2, 128};
    const ada_status OK = ADA_OK, BAD = ADA_ERR_INVALID_ARG, NO = ADA_ERR_UNSUPPORTED;
"""


def test_cache_arguments(tmp_path):
    run_host_code(tmp_path, PREFIX + """
    auto is = [&](ada_kv_cache kv) { return check_cache(&kv, 3, ints, ints, 7, ADA_BF16); };
    assert(is(good) == OK);
    assert(check_cache(nullptr, 3, ints, ints, 7, ADA_BF16) == BAD);
    assert(check_cache(&good, 3, nullptr, ints, 7, ADA_BF16) == BAD && check_cache(&good, 3, ints, nullptr, 7, ADA_BF16) == BAD);
    assert(check_cache(&good, 0, ints, ints, 7, ADA_BF16) == BAD && check_cache(&good, 3, ints, ints, 0, ADA_BF16) == BAD);
    assert(check_cache(&good, 3, ints, ints, 7, ADA_F32) == NO && check_cache(&good, 3, ints, ints, 7, (ada_dtype)5) == BAD);
    assert(check_cache(&good, (1 << 20) + 1, ints, ints, 7, ADA_BF16) == NO);
    assert(check_cache(&good, 3, ints, ints, (1 << 28) + 1, ADA_BF16) == NO);
    ada_kv_cache kv;
    #define WITH(field, value, want) kv = good; kv.field = value; assert(is(kv) == want)
    WITH(k, nullptr, BAD); WITH(v, nullptr, BAD); WITH(table, nullptr, BAD); WITH(kmin, nullptr, BAD); WITH(kmax, nullptr, BAD);
    kv = good; kv.kmin = kv.kmax = nullptr; assert(is(kv) == OK);
    WITH(k, at + 8, NO); WITH(v, at + 2, NO); WITH(kmin, at + 8, NO); WITH(kmax, at + 4, NO);
    WITH(table_ld, 7, BAD); WITH(max_pages, 0, BAD); WITH(n_pages, 0, BAD); WITH(n_pages, (int64_t)1 << 31, NO);
    WITH(page_stride, 2 * 64 * 128 - 8, BAD); WITH(page_stride, 2 * 64 * 128 + 4, NO); WITH(page_stride, 4 * 64 * 128, OK);
    WITH(page_stride, (int64_t)1 << 38, NO);
    for (int64_t ps : {1, 8, 24, 48, 256}) { WITH(page_size, ps, NO); }
    kv = good; kv.page_size = 256; kv.page_stride *= 4; assert(is(kv) == NO);
    for (int64_t ps : {16, 32, 64}) { WITH(page_size, ps, OK); }
    WITH(page_size, 0, BAD); WITH(page_size, 128, BAD); WITH(d_h, 0, BAD); WITH(d_h, 72, NO); WITH(d_h, 144, NO); WITH(d_h, 16, OK);
    WITH(h_kv, 0, BAD); WITH(h_kv, 3, BAD);
    kv = good; kv.max_pages = kv.table_ld = (int64_t)1 << 24; assert(is(kv) == NO);        // 2^30 slots
    kv = good; kv.max_pages = kv.table_ld = ((int64_t)1 << 24) - 1; assert(is(kv) == OK);
    """)


def test_call_arguments(tmp_path):
    run_host_code(tmp_path, PREFIX + """
    assert(check_rows(at, 4, 128, 512) == OK && check_rows(at, 4, 128, 520) == OK);
    assert(check_rows(nullptr, 4, 128, 512) == BAD && check_rows(at, 0, 128, 512) == BAD && check_rows(at, 4, 128, 504) == BAD);
    assert(check_rows(at + 8, 4, 128, 512) == NO && check_rows(at, 4, 128, 516) == NO);
    assert(check_rows(at, 4, 128, (int64_t)1 << 38) == NO && check_rows(at, (int64_t)1 << 40, 128, 512) == NO);
    assert(check_heads(&good, 2) == OK && check_heads(&good, 256) == OK && check_heads(&good, 258) == NO);
    assert(check_heads(&good, 0) == BAD && check_heads(&good, 3) == BAD);
    assert(scale_ok(0.0) && scale_ok(1.0) && !scale_ok(-1.0) && !scale_ok(NAN) && !scale_ok(INFINITY));
    int32_t *out = ints + 16, *pos = nullptr;
    const double* f = (double*)at;
    auto app = [&](const void* K, int64_t ldk, const void* Q, int64_t h, const void* qo, int64_t ldqo, const void* qn,
                   const void* kn, double eps, const double* fr, int64_t rot, const int32_t* ri, const int32_t* rc,
                   const int32_t* lo, uint32_t fl) {
        return check_append(&good, 3, ints, ints, 7, lo, pos, K, ldk, at, 256, Q, h, 512, qo, ldqo, qn, kn, eps, fr, rot, ri, rc, fl);
    };
    assert(app(at, 256, at, 4, at, 512, at, at, 1e-6, f, 128, ints, ints, out, 1) == OK);
    assert(app(at, 256, nullptr, 0, nullptr, 0, nullptr, at, 0.0, nullptr, 0, nullptr, nullptr, nullptr, 0) == OK);
    assert(app(nullptr, 256, at, 4, at, 512, at, at, 1e-6, f, 128, ints, ints, out, 0) == BAD);
    assert(app(at, 128, at, 4, at, 512, at, at, 1e-6, f, 128, ints, ints, out, 0) == BAD);
    assert(app(at, 256, at, 4, nullptr, 512, at, at, 1e-6, f, 128, ints, ints, out, 0) == BAD);
    assert(app(at, 256, nullptr, 4, at, 512, nullptr, at, 1e-6, f, 128, ints, ints, out, 0) == BAD);
    assert(app(at, 256, nullptr, 4, nullptr, 512, at, at, 1e-6, f, 128, ints, ints, out, 0) == BAD);
    assert(app(at, 256, at, 4, at, 520, at, at, 1e-6, f, 128, ints, ints, out, 0) == BAD);      // in place, other rows
    assert(app(at, 256, at, 4, at + 64, 520, at, at, 1e-6, f, 128, ints, ints, out, 0) == OK);
    assert(app(at, 256, at, 4, at, 512, at + 2, at, 1e-6, f, 128, ints, ints, out, 0) == NO);
    assert(app(at, 256, at, 4, at, 512, at, at, -1.0, f, 128, ints, ints, out, 0) == BAD);
    assert(app(at, 256, at, 4, at, 512, at, at, NAN, f, 128, ints, ints, out, 0) == BAD);
    assert(app(at, 256, at, 4, at, 512, nullptr, nullptr, NAN, f, 128, ints, ints, out, 0) == OK);
    for (int64_t rot : {0, -16, 130, 144}) assert(app(at, 256, at, 4, at, 512, at, at, 0.0, f, rot, ints, ints, out, 0) == BAD);
    for (int64_t rot : {2, 8, 40, 120}) assert(app(at, 256, at, 4, at, 512, at, at, 0.0, f, rot, ints, ints, out, 0) == NO);
    assert(app(at, 256, at, 4, at, 512, at, at, 0.0, f, 128, ints, nullptr, out, 0) == BAD);
    assert(app(at, 256, at, 4, at, 512, at, at, 0.0, f, 128, ints, ints, ints, 0) == BAD);      // new lengths over the old
    // off has 4 entries, lengths, positions and counts 3, the list 7
    for (int i = -8; i <= 8; ++i) {
        const int32_t* lo = ints + i;
        assert((app(at, 256, at, 4, at, 512, at, at, 0.0, f, 128, nullptr, nullptr, lo, 0) == OK) == (i <= -3 || i >= 4));
        assert((app(at, 256, at, 4, at, 512, at, at, 0.0, f, 128, ints, ints, lo, 0) == OK) == (i <= -3 || i >= 7));
        pos = ints + 4;
        assert((app(at, 256, at, 4, at, 512, at, at, 0.0, f, 128, nullptr, nullptr, lo, 0) == OK) == (i <= -3 || i >= 7));
        pos = nullptr;
    }
    assert(check_out(at, 512, at, 512) == OK && check_out(at, 512, at, 520) == BAD && check_out(at, 512, at + 16, 520) == OK);
    assert(app(at, 256, at, 4, at, 512, at, at, 0.0, f, 128, ints, ints, out, 2) == BAD);
    assert(check_select(&good, 4, 1, 1, ints, ints, 1) == OK && check_select(&good, 4, 2, 2, ints, ints, 0) == OK);
    assert(check_select(&good, 4, 3, 2, ints, ints, 0) == BAD && check_select(&good, 0, 0, 0, ints, ints, 0) == BAD);
    assert(check_select(&good, 4, -1, 0, ints, ints, 0) == BAD && check_select(&good, 4, 0, -1, ints, ints, 0) == BAD);
    assert(check_select(&good, 4, 0, INT64_MAX, ints, ints, 0) == BAD);
    assert(check_select(&good, 4, 0, 0, nullptr, ints, 0) == BAD && check_select(&good, 4, 0, 0, ints, nullptr, 0) == BAD);
    assert(check_select(&good, 4, 0, 0, ints, ints, 2) == BAD && check_select(&good, 16385, 0, 0, ints, ints, 0) == NO);
    ada_kv_cache kv = good; kv.max_pages = 16385; assert(check_select(&kv, 4, 0, 0, ints, ints, 0) == NO);
    kv = good; kv.kmin = kv.kmax = nullptr; assert(check_select(&kv, 4, 0, 0, ints, ints, 0) == BAD);
    """)


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_native_calls_without_a_context(ada):
    t = bf(64)
    calls = {
        "cache_append": [None, None, 1, t, t, None, 1, t, 64, t, 64, 1, None, 0, 0, None, 0, None, None, 1e-6, None, 0, None,
                         None, None, 0, 0],
        "attention_cached": [None, None, 1, t, t, 1, 1, t, 1, 64, 1, 0.0, t, 64, 0, 0],
        "select_blocks": [None, None, 1, t, t, 1, t, 1, 64, 1, 4, 1, 1, t, t, 0, 0],
        "attention_blocks": [None, None, 1, t, t, 1, t, 1, 64, 1, t, t, 4, 0.0, t, 64, 0, 0],
    }
    for name, args in calls.items():
        call = getattr(ada._fast, name)
        assert call(*args) == 1
        for i, a in enumerate(args):
            if a is t:
                for wrong in (4096, None, "x"):
                    with pytest.raises(AttributeError):
                        call(*args[:i], wrong, *args[i + 1:])
        with pytest.raises(TypeError):
            call(*args[:-1])


def test_cache_tensors(ada):
    K, V, table = bf(5, 2, 16, 64), bf(5, 2, 16, 64), torch.zeros((3, 4), dtype=torch.int32)
    both = bf(5, 2, 2, 16, 64)
    c = ada.KVCache(both[:, 0], both[:, 1], table, bf(5, 2, 64), bf(5, 2, 64))
    assert c._c.page_stride == 2 * 2 * 16 * 64 and c._c.max_pages == 4 and c._c.page_size == 16
    for args, error in (((K, V[:4], table), ValueError), ((K[0], V[0], table), ValueError),
                        ((K, both[:, 1], table), ValueError), ((K.transpose(1, 2), V.transpose(1, 2), table), ValueError),
                        ((K, V, table.long()), TypeError), ((K, V, table.T), ValueError), ((K, V, table[0]), ValueError),
                        ((K, V.half(), table), TypeError), ((K.half(), V.half(), table), TypeError),
                        ((K, V, table, bf(5, 2, 64)), ValueError), ((K, V, table, bf(5, 2, 16), bf(5, 2, 16)), ValueError),
                        ((K, V, table, bf(5, 64, 2).transpose(1, 2), bf(5, 2, 64)), ValueError),
                        ((K, V, table, bf(5, 2, 64).float(), bf(5, 2, 64)), TypeError)):
        with pytest.raises(error):
            ada.KVCache(*args)


def test_tables_whose_rows_overlap(ada):
    """Rows one behind the other in memory are read at the table's stride: one row expanded to several, or rows closer than
    they are long, would be read where the table is not."""
    K, V = bf(5, 2, 16, 64), bf(5, 2, 16, 64)
    flat = torch.zeros(64, dtype=torch.int32)
    for table in (flat[:4].view(1, 4).expand(3, 4), flat.as_strided((3, 4), (3, 1)), flat.as_strided((2, 4), (1, 1))):
        with pytest.raises(ValueError, match="overlap"):
            ada.KVCache(K, V, table)
    for table, ld in ((flat.as_strided((3, 4), (4, 1)), 4), (flat.as_strided((3, 4), (9, 1)), 9), (flat[:4].view(1, 4), 4),
                      (flat[:4].view(1, 4).expand(1, 4), 4), (flat.as_strided((1, 4), (2, 1)), 4), (flat.as_strided((1, 4), (50, 1)), 4)):
        c = ada.KVCache(K, V, table)
        assert c._c.table_ld == ld and c._c.max_pages == 4
        last = (table.shape[0] - 1) * ld + 3               # what a kernel reads of it lies in it
        assert last <= sum((n - 1) * s for n, s in zip(table.shape, table.stride()) if n > 1)


def test_call_tensors(ada):
    from types import SimpleNamespace
    ctx = SimpleNamespace(addr=None, device=0)
    stream = SimpleNamespace(cuda_stream=0)
    c = ada.KVCache(bf(5, 2, 16, 64), bf(5, 2, 16, 64), torch.zeros((3, 4), dtype=torch.int32), bf(5, 2, 64), bf(5, 2, 64))
    Q, K, off, n = bf(7, 4, 64), bf(7, 2, 64), i32(0, 3, 7), i32(5, 9)
    idx, cnt = torch.zeros((7, 2, 4), dtype=torch.int32), torch.zeros((7, 2), dtype=torch.int32)
    attend = lambda *a, **k: ada.ada_attention_cached(ctx, c, *a, stream=stream, **k)       # noqa: E731
    select = lambda *a, **k: ada.ada_select_blocks(ctx, c, *a, stream=stream, **k)          # noqa: E731
    blocks = lambda *a, **k: ada.ada_attention_blocks(ctx, c, *a, stream=stream, **k)       # noqa: E731
    append = lambda *a, **k: ada.ada_cache_append(ctx, c, *a, stream=stream, **k)           # noqa: E731
    for call in (lambda: attend(Q, off, n, 4), lambda: select(Q, off, n, 4), lambda: blocks(Q, off, n, idx, cnt),
                 lambda: append(K, K, off, n, Q=Q)):
        with pytest.raises(ada.AdaError) as e:             # all is well but the context
            call()
        assert e.value.status == 1
    many = i32(0, 1, 2, 3, 4)
    for call, error in (
            (lambda: attend(Q, many, n, 4), ValueError), (lambda: attend(Q, off[:1], n, 4), ValueError),
            (lambda: attend(Q, off.long(), n, 4), TypeError), (lambda: attend(Q, off, n.long(), 4), TypeError),
            (lambda: attend(Q, off, n[:1], 4), ValueError), (lambda: attend(Q.half(), off, n, 4), TypeError),
            (lambda: attend(Q[..., :32], off, n, 4), ValueError), (lambda: attend(Q[:, :, ::2], off, n, 4), ValueError),
            (lambda: attend(Q[:, ::2], off, n, 4), ValueError), (lambda: attend(Q[0], off, n, 4), ValueError),
            (lambda: attend(Q, off, n, 4, out=Q.float()), TypeError), (lambda: attend(Q, off, n, 4, out=K), ValueError),
            (lambda: select(Q, off, n, 4, blk_idx=idx[:, :, :3], blk_cnt=cnt), ValueError),
            (lambda: select(Q, off, n, 4, blk_idx=idx.long(), blk_cnt=cnt), TypeError),
            (lambda: select(Q, off, n, 4, blk_idx=idx, blk_cnt=cnt[:3]), ValueError),
            (lambda: select(Q, off, n, 4, blk_cnt=cnt), ValueError),
            (lambda: blocks(Q, off, n, idx[:6], cnt), ValueError), (lambda: blocks(Q, off, n, idx[:, :1], cnt), ValueError),
            (lambda: blocks(Q, off, n, idx, cnt.float()), TypeError),
            (lambda: append(Q, K, off, n), ValueError), (lambda: append(K, K[:3], off, n), ValueError),
            (lambda: append(K, K, off, n, Q=Q[:3]), ValueError), (lambda: append(K, K, off, n, Q=Q, q_out=K), ValueError),
            (lambda: append(K, K, off, n, inv_freq=torch.zeros(32)), TypeError),
            (lambda: append(K, K, off, n, k_norm=bf(32)), ValueError),
            (lambda: append(K, K, off, n, k_norm=torch.zeros(64)), TypeError),
            (lambda: append(K, K, off, n, pos0=off.long()), TypeError),
            (lambda: append(K, K, off, n, rep_idx=i32(0, 1), rep_cnt=n), ValueError),
            (lambda: append(K, K, off, n, len_out=i32(0)), ValueError)):
        with pytest.raises(error):
            call()
    c.index = 0                                            # a cache on a GPU: tensors from elsewhere are refused
    for call in (lambda: attend(Q, off, n, 4), lambda: append(K, K, off, n), lambda: select(Q, off, n, 4),
                 lambda: blocks(Q, off, n, idx, cnt)):
        with pytest.raises(ValueError, match="device"):
            call()


@pytest.mark.parametrize("index,device", [(-1, 0), (1, 0), (0, 1), (-1, -1)])
def test_a_cache_on_another_device_than_the_context(ada, monkeypatch, index, device):
    """A cache in host memory, or on a GPU that is not the context's: nothing of it reaches the library."""
    from types import SimpleNamespace

    class There(torch.Tensor):
        """A CPU tensor that says where it is."""
        def get_device(self):
            return index

    reached = []
    native = SimpleNamespace(**{name: lambda *a: reached.append(a) or 0 for name in
                                ("cache_append", "attention_cached", "select_blocks", "attention_blocks")})
    monkeypatch.setattr(ada, "_fast", native)
    g = lambda t: t.as_subclass(There)                                                       # noqa: E731
    stream = SimpleNamespace(cuda_stream=0)
    c = ada.KVCache(g(bf(5, 2, 16, 64)), g(bf(5, 2, 16, 64)), g(torch.zeros((3, 4), dtype=torch.int32)), g(bf(5, 2, 64)),
                    g(bf(5, 2, 64)))
    Q, K, off, n = g(bf(7, 4, 64)), g(bf(7, 2, 64)), g(i32(0, 3, 7)), g(i32(5, 9))
    idx, cnt = g(torch.zeros((7, 2, 4), dtype=torch.int32)), g(torch.zeros((7, 2), dtype=torch.int32))
    calls = (lambda x: ada.ada_attention_cached(x, c, Q, off, n, 4, out=Q, stream=stream),
             lambda x: ada.ada_select_blocks(x, c, Q, off, n, 4, blk_idx=idx, blk_cnt=cnt, stream=stream),
             lambda x: ada.ada_attention_blocks(x, c, Q, off, n, idx, cnt, out=Q, stream=stream),
             lambda x: ada.ada_cache_append(x, c, K, K, off, n, len_out=off[:2].clone(), stream=stream))
    for call in calls:
        with pytest.raises(ada.AdaError, match="device") as e:
            call(SimpleNamespace(addr=4096, device=device))
        assert e.value.status == 1 and not reached
        if index >= 0:
            call(SimpleNamespace(addr=4096, device=index))
            assert len(reached) == 1
            reached.clear()


def test_outputs_are_made_on_the_stream_of_the_call(ada, monkeypatch):
    """What a call allocates or clears for itself is ordered with its kernels: made under the stream that was passed."""
    import contextlib
    from types import SimpleNamespace
    at, made = [None], []

    @contextlib.contextmanager
    def on(stream):
        at.append(stream)
        yield
        at.pop()

    class OnGPU(torch.Tensor):
        """A CPU tensor that says it is on a GPU."""
        def get_device(self):
            return 0

        def new_empty(self, *a, **k):
            made.append(at[-1])
            return super().new_empty(*a, **k)

        def new_zeros(self, *a, **k):
            made.append(at[-1])
            return super().new_zeros(*a, **k)

    def count(make):
        def counted(*a, **k):
            made.append(at[-1])
            return make(*a, **k).as_subclass(OnGPU)
        return counted

    g = lambda t: t.as_subclass(OnGPU)                                                       # noqa: E731
    stream, ctx = SimpleNamespace(cuda_stream=0), SimpleNamespace(addr=None, h=None, device=0)
    c = ada.KVCache(g(bf(5, 2, 16, 64)), g(bf(5, 2, 16, 64)), g(torch.zeros((3, 4), dtype=torch.int32)), g(bf(5, 2, 64)),
                    g(bf(5, 2, 64)))
    Q, K, off, n = g(bf(7, 4, 64)), g(bf(7, 2, 64)), g(i32(0, 3, 7)), g(i32(5, 9))
    idx, cnt = g(torch.zeros((7, 2, 4), dtype=torch.int32)), g(torch.zeros((7, 2), dtype=torch.int32))
    X, lists, one = g(bf(1, 7, 256)), g(torch.zeros((1, 7), dtype=torch.int32)), g(i32(1))
    heads = g(torch.zeros((4, 7), dtype=torch.int32))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", count(torch.empty))
    monkeypatch.setattr(torch, "zeros", count(torch.zeros))
    for outputs, call in (
            (1, lambda: ada.ada_attention_cached(ctx, c, Q, off, n, 4, stream=stream)),
            (0, lambda: ada.ada_attention_cached(ctx, c, Q, off, n, 4, out=Q, stream=stream)),
            (1, lambda: ada.ada_attention_blocks(ctx, c, Q, off, n, idx, cnt, stream=stream)),
            (2, lambda: ada.ada_select_blocks(ctx, c, Q, off, n, 4, stream=stream)),
            (0, lambda: ada.ada_select_blocks(ctx, c, Q, off, n, 4, blk_idx=idx, blk_cnt=cnt, stream=stream)),
            (2, lambda: ada.ada_cache_append(ctx, c, K, K, off, n, Q=Q, stream=stream)),
            (1, lambda: ada.ada_cache_append(ctx, c, K, K, off, n, stream=stream)),
            (1, lambda: ada.ada_attention_reps(ctx, Q, Q, Q, lists[0], one, stream=stream)),
            (3, lambda: ada.ada_normalize(ctx, X, want_xhat=True, rep_idx=lists, rep_cnt=one, stream=stream)),
            (3, lambda: ada.ada_select_full(ctx, X, 0.3, stream=stream)),
            (8, lambda: ada.ada_cascade_step(ctx, X, 0.3, lists, one, stream=stream)),
            (2, lambda: ada.ada_nearest_rep(ctx, X, lists, one, stream=stream)),
            (3, lambda: ada.ada_select_full_heads(ctx, Q, 0.3, stream=stream)),
            (8, lambda: ada.ada_cascade_step_heads(ctx, Q, 0.3, heads, heads[:, 0], stream=stream))):
        made.clear()
        with pytest.raises(ada.AdaError) as e:             # (there is no context)
            call()
        assert e.value.status == 1 and made == [stream] * outputs


def test_reference_against_dense_attention():
    """The loops of the reference against torch's attention in 64 bits, and its rotation against complex numbers."""
    g = torch.Generator().manual_seed(0)
    K, V = (torch.randn((6, 2, 16, 32), generator=g).bfloat16() for _ in range(2))
    table = torch.tensor([[4, 1, 0], [2, 5, 3]], dtype=torch.int32)
    Q = torch.randn((7, 4, 32), generator=g).bfloat16()
    out, weight = ref.attend(ref.Pages(K, V, table), Q, [0, 5, 7], [40, 20], 2)
    for b, (o, n, total) in enumerate(((0, 5, 40), (5, 2, 20))):
        k, v = (x[table[b].long()].transpose(0, 1).reshape(2, 48, 32)[:, :total].double() for x in (K, V))
        q = Q[o:o + n].double().transpose(0, 1)
        mask = torch.ones(n, total, dtype=torch.bool).tril(total - n)
        want = torch.nn.functional.scaled_dot_product_attention(q, k.repeat_interleave(2, 0), v.repeat_interleave(2, 0), mask)
        assert float((out[o:o + n].transpose(0, 1) - want).abs().max()) < 1e-12
    x = torch.randn((3, 32), generator=g, dtype=torch.float64)
    f = 100.0 ** (-torch.arange(0, 16, 2, dtype=torch.float64) / 16)
    z = torch.view_as_complex(x[:, :16].reshape(3, 8, 2).contiguous()) * torch.exp(1j * 5 * f)
    assert float((ref.turned(x, 5, f, True)[:, :16] - torch.view_as_real(z).flatten(1)).abs().max()) < 1e-12
    z = torch.complex(x[:, :8], x[:, 8:16]) * torch.exp(1j * 5 * f)
    assert float((ref.turned(x, 5, f, False)[:, :16] - torch.cat([z.real, z.imag], 1)).abs().max()) < 1e-12
    assert math.isclose(float(ref.normed(x, torch.ones(32), 0.0).square().mean()), 1.0)


