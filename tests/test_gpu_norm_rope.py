"""Norms of heads and rotary positions of several numbers against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2506_07311_amd as pa
from paper_2506_07311_amd import PagedAttnError
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def ints(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).to(DEV)


class Case:
    """Tokens of three sequences on their way into a cache of four times as many slots."""

    def __init__(self, dtype=torch.bfloat16, T=37, hq=8, hkv=2, d=128, page=16, rot=None, axes=1, per_head=False, weights=True, f32_weights=False,
                 pad=0, apart=False, seed=0, far=100000):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.T, self.hq, self.hkv, self.d, self.page = T, hq, hkv, d, page
        rows = T + pad
        rot = d if rot is None else rot
        if apart:                                                 # parts of one projection
            x = torch.randn(rows, (hq + 2 * hkv) * d, generator=g).to(dtype).to(DEV)
            self.q, self.k, self.v = (y.view(rows, -1, d) for y in x.split([hq * d, hkv * d, hkv * d], 1))
        else:
            self.q, self.k, self.v = (torch.randn(rows, h, d, generator=g).to(dtype).to(DEV) for h in (hq, hkv, hkv))
        ids = np.sort(rng.integers(0, 3, T))
        start = rng.integers(0, 3 * page, 3)
        places = np.concatenate([start[s] + np.arange((ids == s).sum()) for s in range(3)])
        blocks = int(places.max()) // page + 2
        pages = 3 * blocks + 5
        table = rng.permutation(pages)[:3 * blocks].reshape(3, blocks)
        self.table_np, self.ids_np, self.places_np = table, ids, places
        self.table = ints(table)
        self.ids, self.places = ints(np.concatenate([ids, np.full(pad, -1)])), ints(np.concatenate([places, np.full(pad, -1)]))
        self.rope = ints(rng.integers(0, far, (axes, rows)) if axes > 1 else rng.integers(0, far, rows))
        self.pair_axes = ints(rng.integers(0, axes, rot // 2)) if axes > 1 else None
        self.freq = (10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / max(rot, 1))).to(DEV)
        kind = torch.float32 if f32_weights else dtype
        self.qw, self.kw = ((1 + 0.3 * torch.randn((h, d) if per_head else (d,), generator=g)).to(kind).to(DEV) if weights else None
                            for h in (hq, hkv))
        self.k_cache, self.v_cache = (torch.randn(pages, page, hkv, d, generator=g).to(dtype).to(DEV) for _ in range(2))

    def tokens(self):
        return self.q, self.k, self.v, self.rope, self.ids, self.places, self.table, self.freq

    def expect(self, what="qk", **kw):
        kw.setdefault("axes_of", self.pair_axes)
        return [ref.norm_rope(x, self.rope, self.freq, w, **kw) for x, w in ((self.q, self.qw), (self.k, self.kw))]

    def slots(self):
        return self.table_np[self.ids_np, self.places_np // self.page], self.places_np % self.page


def near(got, want, size, dtype, what=""):
    """Half a step of the type, and of the 32-bit arithmetic before it: the angle's rounding to 32 bits is at most pi 2^-24 and sine and cosine
    add 2^-22, the norm's sum of at most 256 squares in trees of 2^-24 steps, its root and quotient stay below 2^-20 together, the weight's sum
    and product 2^-23; each relative to the pair's size: 2^-19."""
    got = got.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        tol = torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -19 * size * (1 + torch.finfo(dtype).eps) + torch.finfo(dtype).tiny
        bad = ~(np.abs(got - want) <= tol)
    bad &= ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), (what, int(bad.sum()), np.abs(got - want)[bad][:3], tol[bad][:3])


def check(c, dtype, call, **kw):
    k_before, v_before = c.k_cache.clone(), c.v_cache.clone()
    q_in = c.q.clone()
    (qr, qs), (kr, ks) = c.expect(**kw)
    out = call()
    near(out, qr, qs, dtype, "q")
    page, place = c.slots()
    near(c.k_cache[page, place], kr[:c.T], ks[:c.T], dtype, "K")
    assert torch.equal(c.v_cache[page, place], c.v[:c.T])
    k_before[page, place], v_before[page, place] = c.k_cache[page, place], c.v_cache[page, place]
    assert torch.equal(k_before, c.k_cache) and torch.equal(v_before, c.v_cache)   # no other slot
    return q_in


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 32), (256, 256), (80, 32), (80, 20), (96, 24), (112, 14), (8, 8), (40, 6), (128, 0), (200, 2)])
@pytest.mark.parametrize("inter", [False, True])
def test_sizes(dtype, d, rot, inter):
    c = Case(TYPES[dtype], d=d, rot=rot, axes=3 if rot else 1, seed=d + rot)
    check(c, TYPES[dtype], lambda: pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw,
                                                             pair_axes=c.pair_axes, interleaved=inter), interleaved=inter)


@pytest.mark.parametrize("T,hq,hkv", [(1, 1, 1), (1, 64, 8), (3, 7, 7), (200, 12, 4), (1030, 5, 1), (2100, 8, 2)])
@pytest.mark.parametrize("apart,pad", [(False, 0), (True, 5)])
def test_tokens_and_heads(T, hq, hkv, apart, pad):
    c = Case(T=T, hq=hq, hkv=hkv, apart=apart, pad=pad, axes=2, per_head=True, seed=T)
    check(c, torch.bfloat16, lambda: pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw,
                                                               pair_axes=c.pair_axes, weight_offset=1.0, eps=1e-3, mscale=1.25),
          offset=1.0, eps=1e-3, mscale=1.25)


@pytest.mark.parametrize("f32_weights,per_head,weights", [(True, False, True), (True, True, True), (False, False, False)])
@pytest.mark.parametrize("axes", [1, 4])
def test_weights(f32_weights, per_head, weights, axes):
    c = Case(f32_weights=f32_weights, per_head=per_head, weights=weights, axes=axes, page=64, seed=3)
    check(c, torch.bfloat16, lambda: pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw,
                                                               pair_axes=c.pair_axes))


def test_one_of_the_norms():
    c = Case(seed=4)
    out = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw, norm_k=False)
    near(out, *c.expect()[0], torch.bfloat16)
    page, place = c.slots()
    near(c.k_cache[page, place], *ref.norm_rope(c.k, c.rope, c.freq, norm=False), torch.bfloat16)
    out = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), norm_q=False, norm_k=False)
    near(out, *ref.norm_rope(c.q, c.rope, c.freq, norm=False), torch.bfloat16)


@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (80, 20, False), (128, 64, True)])
def test_in_place(d, rot, inter):
    c = Case(d=d, rot=rot, T=300, hq=20, seed=5)
    (qr, qs), _ = c.expect(interleaved=inter)
    out = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw, q_out=c.q, interleaved=inter)
    assert out.data_ptr() == c.q.data_ptr()
    near(out, qr, qs, torch.bfloat16)


def test_parts_absent_and_head_major():
    c = Case(seed=6)
    q, k, v, rope, ids, places, table, freq = c.tokens()
    before = c.k_cache.clone()
    out = pa.paged_norm_rope_append(c.k_cache, c.v_cache, q, None, None, rope, None, None, None, freq, q_weight=c.qw)
    near(out, *c.expect()[0], torch.bfloat16)
    assert torch.equal(before, c.k_cache)
    kc, vc = (x.transpose(1, 2).contiguous() for x in (c.k_cache, c.v_cache))
    assert pa.paged_norm_rope_append(kc, vc, None, k, v, rope, ids, places, table, freq, k_weight=c.kw, head_major=True) is None
    page, place = c.slots()
    near(kc.transpose(1, 2)[page, place], *c.expect()[1], torch.bfloat16)


def test_rows_without_a_page():
    c = Case(seed=7)
    table = c.table_np.copy()
    table[1] = -1                                                 # not mapped
    c.table.copy_(ints(table))
    lost = (c.ids_np == 1) | (np.arange(c.T) % 5 == 0)
    c.places[torch.arange(0, c.T, 5)] = -3
    before = c.k_cache.clone()
    pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw)
    page, place = c.slots()
    kr, ks = c.expect()[1]
    near(c.k_cache[page[~lost], place[~lost]], kr[~lost], ks[~lost], torch.bfloat16)
    before[page[~lost], place[~lost]] = c.k_cache[page[~lost], place[~lost]]
    assert torch.equal(before, c.k_cache)


@pytest.mark.parametrize("dtype,size", [("fp32", 1e25), ("bf16", 1e30), ("fp32", 1e-30), ("fp32", 2e-38), ("bf16", 1e-28), ("fp16", 1e-6)])
def test_far_magnitudes(dtype, size):
    """Squares beyond the range of fp32."""
    c = Case(TYPES[dtype], seed=8)
    c.q.copy_((c.q.double() * size).to(TYPES[dtype]))
    out = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw, eps=0.0)
    near(out, *c.expect(eps=0.0)[0], TYPES[dtype])


def test_values_that_are_not_finite_stay_in_their_head():
    c = Case(torch.float32, seed=9)
    c.q[3, 2, 5], c.q[4, 1, 0], c.k[2, 1, 7] = float("nan"), float("inf"), -float("inf")
    c.q[6, 0] = 0.0
    out = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw)
    (qr, qs), (kr, ks) = c.expect()
    bad = np.zeros(qr.shape[:2], bool)
    bad[3, 2] = bad[4, 1] = True
    near(out[torch.from_numpy(~bad).to(DEV)], qr[~bad], qs[~bad], torch.float32)
    assert torch.isnan(out[3, 2]).all() and torch.isnan(out[4, 1, 0]) and (out[6, 0] == 0).all()
    page, place = c.slots()
    ok = np.ones(kr.shape[:2], bool)
    ok[2, 1] = False
    near(c.k_cache[page, place][torch.from_numpy(ok).to(DEV)], kr[ok], ks[ok], torch.float32)


def test_far_positions():
    c = Case(torch.float32, axes=3, far=2 ** 31 - 1, seed=10)
    check(c, torch.float32, lambda: pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw,
                                                              pair_axes=c.pair_axes))


def test_axes_out_of_range_read_nothing():
    """Numbers of a position that do not exist count as the nearest that does."""
    c = Case(axes=2, seed=11)
    wild = torch.where(torch.arange(64, device=DEV) % 2 == 0, -7, 900).to(torch.int32)
    tame = wild.clamp(0, 1)
    a = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), pair_axes=wild)
    b = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), pair_axes=tame)
    assert torch.equal(a, b)


def test_captured_and_on_another_stream():
    c = Case(T=1200, pad=3, axes=3, seed=12)
    kw = dict(q_weight=c.qw, k_weight=c.kw, pair_axes=c.pair_axes)
    want = pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), **kw)
    want_k = c.k_cache.clone()
    out = torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_out=out, **kw)
    for i in range(3):
        out.zero_(), c.k_cache.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        page, place = c.slots()
        assert torch.equal(c.k_cache[page, place], want_k[page, place])
        c.q.add_(0)
    out.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_out=out, stream=side, **kw)
    side.synchronize()
    assert torch.equal(out, want)


def test_refusals():
    c = Case(axes=2, seed=13)
    q, k, v, rope, ids, places, table, freq = c.tokens()
    run = lambda *t, **kw: pa.paged_norm_rope_append(c.k_cache, c.v_cache, *t, **dict(dict(pair_axes=c.pair_axes), **kw))  # noqa: E731
    full = (q, k, v, rope, ids, places, table, freq)
    for kw in (dict(q_weight=c.qw[:64]), dict(q_weight=c.qw.half()), dict(k_weight=c.kw[None].repeat(3, 1)), dict(pair_axes=None),
               dict(pair_axes=c.pair_axes[:9]), dict(pair_axes=c.pair_axes.long()), dict(eps=-1.0), dict(eps=float("nan")),
               dict(weight_offset=float("nan")), dict(q_out=q[:-1]), dict(q_weight=c.qw, k_weight=c.kw.float()),
               dict(q_weight=c.qw.cpu()), dict(mscale=float("nan"))):
        with pytest.raises(PagedAttnError):
            run(*full, **kw)
    for change in (dict(q=q.float()), dict(k=k[:, :1]), dict(v=None), dict(ids=ids[:-1]), dict(rope=rope[None]), dict(freq=freq.float()),
                   dict(q=q.cpu()), dict(table=table[0]), dict(k=k.transpose(0, 1))):
        args = dict(q=q, k=k, v=v, rope=rope, ids=ids, places=places, table=table, freq=freq)
        args.update(change)
        with pytest.raises(PagedAttnError):
            run(*args.values())
