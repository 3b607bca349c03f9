"""CPU-side checks of a step of drafted tokens: host-checkable argument errors, the rotary frequencies, the binding's refusals.
No compute call is made here."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import paper_2506_07311_amd as pa
from paper_2506_07311_amd import binding

INVALID, UNSUPPORTED, SMALL = 1, 2, 3
i32, i64, f32, f64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_size_t
P, NULL = ctypes.c_void_p(0x4000), ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2506_07311_amd import build
        build.build()
    return binding.load_library()


def desc(**kw):
    d = dict(k_cache=0x1000, v_cache=0x2000, page_stride=16 * 8 * 128, token_stride=8 * 128, head_stride=128, num_pages=4,
             page_size=16, num_kv_heads=8, head_dim=128, dtype=1)
    d.update(kw)
    return binding._Desc(**d)


def call(fn, args, **change):
    """fn with its named arguments, some of them changed."""
    assert set(change) <= set(args), change
    args = dict(args, **change)
    return fn(*(ctypes.byref(a) if isinstance(a, binding._Desc) else a for a in args.values()))


def test_plan_refusals(lib):
    L = ctypes.c_void_p(0x6000)                                   # (lengths that are written are not those that are read)
    a = dict(ctx=P, new=P, batch=i32(2), parents=NULL, page=i32(16), table=P, max_blocks=i32(4), num=P, free=P, count=P, rows=i32(8),
             seq_lens=L, cu=P, ids=P, pos=P, rope=NULL, mask=P, words=i32(1), shortage=P, stream=NULL)
    for bad in (dict(batch=i32(-1)), dict(page=i32(0)), dict(page=i32(12)), dict(max_blocks=i32(0)), dict(max_blocks=i32(-1)),
                dict(rows=i32(-1)), dict(words=i32(0)), dict(words=i32(-1)), dict(mask=ctypes.c_void_p(0x4004)), dict(ctx=NULL),
                dict(new=NULL), dict(table=NULL), dict(num=NULL), dict(free=NULL), dict(count=NULL), dict(seq_lens=NULL),
                dict(cu=NULL), dict(ids=NULL), dict(pos=NULL), dict(shortage=NULL), dict(seq_lens=P), dict(ctx=L), dict(new=L)):
        assert call(lib.paged_plan_step, a, **bad) == INVALID, bad
    assert call(lib.paged_plan_step, a, batch=i32(0)) == 0
    r = dict(keep=P, batch=i32(2), page=i32(16), table=P, max_blocks=i32(4), num=P, free=P, count=P, max_free=i32(9), stream=NULL)
    for bad in (dict(batch=i32(-1)), dict(page=i32(3)), dict(max_blocks=i32(0)), dict(max_free=i32(-1)), dict(keep=NULL),
                dict(table=NULL), dict(num=NULL), dict(free=NULL), dict(count=NULL)):
        assert call(lib.paged_release_blocks, r, **bad) == INVALID, bad
    assert call(lib.paged_release_blocks, r, batch=i32(0)) == 0


def test_rope_append_refusals(lib):
    a = dict(cache=desc(), q=P, qs=i64(0), qo=P, qos=i64(0), hq=i32(32), k=P, ks=i64(0), v=P, vs=i64(0), rope=P, ids=P, pos=P, T=i32(3),
             table=P, batch=i32(2), max_blocks=i32(4), inv=P, rot=i32(128), inter=i32(0), mscale=f32(1.0), stream=NULL)
    fn = lib.paged_rope_append
    for bad in (dict(T=i32(-1)), dict(rot=i32(7)), dict(rot=i32(130)), dict(rot=i32(-2)), dict(q=NULL), dict(qo=NULL), dict(k=NULL),
                dict(v=NULL), dict(hq=i32(0)), dict(rope=NULL), dict(inv=NULL), dict(inv=ctypes.c_void_p(0x4004)), dict(ids=NULL),
                dict(pos=NULL), dict(table=NULL), dict(batch=i32(0)), dict(max_blocks=i32(0)), dict(mscale=f32(float("nan"))),
                dict(qs=i64(4088)), dict(qos=i64(4088)), dict(ks=i64(1016)), dict(vs=i64(-1024)), dict(qs=i64(8192)),
                dict(cache=desc(page_size=12))):
        assert call(fn, a, **bad) == INVALID, bad                 # (qs: q and its output are one, with other strides)
    for bad in (dict(ks=i64(1028)), dict(vs=i64(1025)), dict(qs=i64(4097), qos=i64(4097)), dict(k=ctypes.c_void_p(0x4008)),
                dict(cache=desc(dtype=7)), dict(cache=desc(head_dim=100))):
        assert call(fn, a, **bad) == UNSUPPORTED, bad
    assert call(fn, a, T=i32(0)) == 0
    assert call(fn, a, q=NULL, qo=NULL, k=NULL, v=NULL) == 0


def test_tree_attention_refusals(lib):
    a = dict(cache=desc(), q=P, out=P, lse=NULL, cu=P, total=i32(6), max_q=i32(3), mask=P, words=i32(1), table=P, lens=P, batch=i32(2),
             hq=i32(32), max_blocks=i32(4), max_len=i32(64), scale=f32(0.1), ws=ctypes.c_void_p(0x10000), bytes=size(1 << 40),
             stream=NULL)
    fn = lib.paged_attention_tree
    for bad in (dict(total=i32(-1)), dict(max_q=i32(-1)), dict(max_q=i32(65)), dict(words=i32(0)), dict(mask=NULL), dict(q=NULL),
                dict(out=NULL), dict(cu=NULL), dict(table=NULL), dict(lens=NULL), dict(batch=i32(-1)), dict(hq=i32(12)),
                dict(hq=i32(0)), dict(max_blocks=i32(3)), dict(max_len=i32(-1)), dict(scale=f32(float("nan"))),
                dict(mask=ctypes.c_void_p(0x4004)), dict(ws=ctypes.c_void_p(0x10010)), dict(cache=desc(num_pages=0))):
        assert call(fn, a, **bad) == INVALID, bad
    for bad in (dict(q=ctypes.c_void_p(0x4008)), dict(out=ctypes.c_void_p(0x4004)), dict(cache=desc(head_dim=264)),
                dict(cache=desc(token_stride=1025))):
        assert call(fn, a, **bad) == UNSUPPORTED, bad
    assert call(fn, a, ws=NULL) == SMALL and call(fn, a, bytes=size(16)) == SMALL
    assert call(fn, a, batch=i32(0)) == 0 and call(fn, a, total=i32(0)) == 0
    assert call(fn, a, max_q=i32(0), words=i32(0)) == 0           # no sequence brings a query: nothing to do


def test_tree_workspace_bound(lib):
    for args in ((1, 8, 8, 64, 5, 5, 128), (64, 32, 8, 128, 300, 8, 32768), (0, 8, 8, 64, 0, 0, 0), (16, 64, 8, 128, 256, 16, 131072)):
        n = binding.paged_attention_tree_workspace_bytes(*args)
        assert n > 0 and n % 256 == 0


def test_accept_refusals(lib):
    a = dict(cache=desc(), cu=P, lens=P, batch=i32(2), max_q=i32(8), parents=P, tokens=P, targets=P, path=P, max_path=i32(8),
             path_lens=P, nxt=P, kept=ctypes.c_void_p(0x6000), table=P, max_blocks=i32(4), stream=NULL)
    fn = lib.paged_tree_accept
    for bad in (dict(batch=i32(-1)), dict(max_q=i32(-1)), dict(max_path=i32(0)), dict(parents=NULL), dict(tokens=NULL),
                dict(targets=NULL), dict(parents=NULL, tokens=NULL, targets=NULL), dict(path=NULL), dict(path_lens=NULL),
                dict(cu=NULL), dict(lens=NULL), dict(table=NULL), dict(max_blocks=i32(0)), dict(cache=desc(k_cache=0)), dict(kept=P)):
        assert call(fn, a, **bad) == INVALID, bad
    assert call(fn, a, max_q=i32(9000), max_path=i32(9000)) == UNSUPPORTED
    assert call(fn, a, batch=i32(0)) == 0


def test_rope_frequencies():
    """Against the formulas, evaluated another way, within the last bits of the power function."""
    for r in (2, 20, 64, 128):
        i = np.arange(r // 2)
        f = np.exp(-2.0 * i / r * math.log(10000.0))
        got, m = pa.pa_rope_frequencies(r)
        assert got.dtype == torch.float64 and np.allclose(got.numpy(), f, rtol=1e-13) and m == 1.0
        got, _ = pa.pa_rope_frequencies(r, scaling="linear", factor=4.0)
        assert np.allclose(got.numpy(), f / 4.0, rtol=1e-13)
        got, _ = pa.pa_rope_frequencies(r, 500000.0, "base", factor=8.0)
        if r > 2:                                                 # ends: unscaled, and slowed by the factor
            slow = math.exp(-(r - 2.0) / r * math.log(500000.0))
            assert got[0] == 1.0 and math.isclose(float(got[-1]), slow / 8.0, rel_tol=1e-12)
        got, _ = pa.pa_rope_frequencies(r, scaling="parts", factor=8.0, context=4096.0, slow=1.0, fast=4.0)
        turns = 4096.0 * f / (2.0 * math.pi)
        for x, y, n in zip(got.tolist(), f, turns):
            want = y if n >= 4 else y / 8 if n <= 1 else y / 8 + (y - y / 8) * (n - 1) / 3
            assert math.isclose(x, want, rel_tol=1e-11)
        got, m = pa.pa_rope_frequencies(r, scaling="ramp", factor=8.0, context=4096.0)
        assert math.isclose(m, 0.1 * math.log(8.0) + 1.0, rel_tol=1e-6)
        assert all(y / 8 * (1 - 1e-12) <= x <= y * (1 + 1e-12) for x, y in zip(got.tolist(), f))
        if r == 128:
            assert math.isclose(float(got[0]), 1.0) and math.isclose(float(got[-1]), f[-1] / 8, rel_tol=1e-12)
            lo, hi = (r * math.log(4096.0 / (2 * math.pi * t)) / (2 * math.log(10000.0)) for t in (32.0, 1.0))
            lo, hi = math.floor(lo), math.ceil(hi)
            at = (lo + hi) // 2
            keep = 1.0 - (at - lo) / (hi - lo)
            assert math.isclose(float(got[at]), f[at] * keep + f[at] / 8 * (1 - keep), rel_tol=1e-11)
    for bad in (dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=64, base=1.0), dict(rotary_dim=64, factor=0.5),
                dict(rotary_dim=64, base=float("nan")), dict(rotary_dim=64, scaling="other"),
                dict(rotary_dim=64, scaling="parts", slow=4.0, fast=1.0), dict(rotary_dim=64, scaling="ramp", context=0.0)):
        with pytest.raises(pa.PagedAttnError):
            pa.pa_rope_frequencies(**bad)


def test_binding_refuses_host_tensors():
    k = torch.zeros(4, 16, 2, 64)
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(pa.PagedAttnError):
        pa.paged_plan_step(n, n, torch.zeros(2, 4, dtype=torch.int32), n, n, n[:1], 16, 4)
    with pytest.raises(pa.PagedAttnError):
        pa.paged_release_blocks(n, torch.zeros(2, 4, dtype=torch.int32), n, n, n[:1], 16)
    with pytest.raises(pa.PagedAttnError):
        pa.paged_rope_append(k, k, k[0], None, None, n, None, None, None, torch.zeros(32, dtype=torch.float64))
    with pytest.raises(pa.PagedAttnError):
        pa.paged_attention_tree(k, k, k[0], n, 4, torch.zeros(4, 1, dtype=torch.int64), n, n, 64, 1.0)
    with pytest.raises(pa.PagedAttnError):
        pa.paged_tree_accept(k, k, n, n, 4, n, n, n)
