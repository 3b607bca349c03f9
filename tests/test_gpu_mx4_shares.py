"""Attention over the 4-bit cache where workgroups share a call's keys: several pieces of several sequences a workgroup, long walks, pieces
that are done again.  Samples of sequences and KV heads against the definition in 64 bits; all of it against other places of the pages."""
import numpy as np
import pytest
import torch

import paper_2506_07311_amd as pa
from tests import mx4_reference as ref
from tests.test_gpu_mx4 import TYPES, ints

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Records:
    """Sequences whose records are any bytes, with scales of 1/4, 1/2 and 1; other pages and slots behind a sequence are blocks of NaN."""

    def __init__(self, lens, hkv, d, page=16, seed=0):
        self.lens, self.hkv, self.d, self.page = list(lens), hkv, d, page
        g = torch.Generator(device=DEV).manual_seed(seed)
        blocks = [-(-n // page) for n in lens]
        self.pages = sum(blocks) + 5
        size = pa.pa_mx4_record_bytes(page, d)
        self.cache = torch.randint(0, 256, (self.pages, hkv, size), generator=g, device=DEV, dtype=torch.uint8)
        scales = self.cache[:, :, page * d:]
        scales.remainder_(3).add_(125)
        order = np.random.default_rng(seed).permutation(self.pages)
        self.table_np = np.full((len(lens), max(max(blocks), 1) + 2), -1)
        at = 0
        for s, b in enumerate(blocks):
            self.table_np[s, :b] = order[at:at + b]
            at += b
            if lens[s] % page:
                scales[self.table_np[s, b - 1]].view(hkv, -1, page)[..., lens[s] % page:] = 255
        scales[torch.from_numpy(order[at:]).to(DEV)] = 255
        self.table = ints(self.table_np)

    def moved(self, seed):
        """The same sequences in other pages."""
        to = torch.from_numpy(np.random.default_rng(seed).permutation(self.pages)).to(DEV)
        cache = torch.empty_like(self.cache)
        cache[to] = self.cache
        return cache, torch.where(self.table >= 0, to[self.table.clamp(min=0).long()], -1).to(torch.int32)

    def head(self, s, h):
        """K and V [len, d] in 64 bits."""
        pages = torch.from_numpy(self.table_np[s, :-(-self.lens[s] // self.page)]).to(DEV)
        return [torch.from_numpy(ref.values(*x).reshape(-1, self.d)[:self.lens[s]]).to(DEV)
                for x in ref.unpacked(self.cache[pages, h:h + 1], self.page, self.d)]

    def set_scale(self, s, h, token, block, what, value):
        P, d = self.page, self.d
        self.cache[self.table_np[s, token // P], h, P * d + (what * (d // 32) + block) * P + token % P] = value


def run(c, q, new, scale, loose=0, cache=None, table=None):
    out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 5.0, device=DEV)
    top = min(max(c.lens) + loose, c.table.shape[1] * c.page)
    pa.paged_attention_mx4(c.cache if cache is None else cache, q, ints(np.cumsum([0, *new])), max(new), c.table if table is None else table,
                           ints(c.lens), top, scale, out=out, lse=lse)
    return out, lse


def check(c, G, new, dtype, seed=0, heads=3):
    t, hkv = TYPES[dtype], c.hkv
    total, scale = sum(new), 0.5 * c.d ** -0.5
    q = torch.randn(total + 3, G * hkv, c.d, generator=torch.Generator().manual_seed(seed)).to(t).to(DEV)
    out, lse = run(c, q, new, scale)
    assert (out[total:] == 3).all() and (lse[total:] == 5).all()
    for again in (run(c, q, new, scale), run(c, q, new, scale, 0, *c.moved(seed + 1))):
        assert torch.equal(out.view(torch.int16), again[0].view(torch.int16)) and torch.equal(lse.view(torch.int32), again[1].view(torch.int32))
    cu = np.cumsum([0, *new])
    for s, n in enumerate(new):
        rows = slice(cu[s], cu[s + 1])
        if n == 0:
            continue
        if c.lens[s] == 0:
            assert (out[rows] == 0).all() and torch.isneginf(lse[rows]).all()
            continue
        for h in sorted({(5 * s + i * hkv // heads) % hkv for i in range(heads)}):
            k, v = c.head(s, h)
            mine = slice(h * G, h * G + G)
            near(out[rows, mine], lse[rows, mine], q[rows, mine], k, v, c.lens[s] - n, scale, t)
    return out, lse


def attention(q, k, v, n_ctx, scale):
    """q [n, G, d], k and v [len, d], 64-bit: (out, lse, sum p |v|, largest sum |q k| scale); row i sees keys j <= n_ctx + i."""
    n, G, d = q.shape
    q = q.reshape(n * G, d)
    sees = torch.arange(len(k), device=DEV) <= n_ctx + torch.arange(n, device=DEV).repeat_interleave(G)[:, None]
    lost_k, lost_v = torch.isnan(k), torch.isnan(v)
    k, v = k.nan_to_num(0.0), v.nan_to_num(0.0)
    x = (q @ k.t().contiguous() * scale).masked_fill(~sees, -np.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse.clamp(min=-1e300)[:, None])
    out, mass = p @ v, p @ v.abs()
    size = ((q.abs() @ k.abs().t().contiguous()) * sees).amax(1) * scale
    sees = sees.double()
    out[(sees @ lost_v.double()) > 0] = np.nan
    rows = (sees @ lost_k.any(1).double()) > 0
    out[rows], lse[rows] = np.nan, np.nan
    return [y.cpu().numpy().reshape(n, G, *y.shape[1:]) for y in (out, lse, mass, size)]


def near(out, lse, q, k, v, n_ctx, scale, dtype):
    """Bounds: a score is a 32-bit sum of up to 3 x 256 exact products, off by less than 2^-18 of the sum of their magnitudes, and rounded once
    more; a weight has two 16-bit terms (2^-17; three: 2^-24), exp2 is good to 2^-22.  Sums over the keys are rounded up to three times every 32
    keys, each time by up to 2^-24 of what is summed, with either sign: six deviations of that.  The output is rounded once."""
    want, want_lse, mass, size = attention(q.double(), k, v, n_ctx, scale)
    score = 2.0 ** -17 * size
    sums = 6 * 2.0 ** -24 * np.sqrt(len(k) / 32 + 1) + 2.0 ** -20
    weight = (2.0 ** -17 if dtype != torch.float32 else 2.0 ** -20) + sums + 2 * score
    tol = torch.finfo(dtype).eps / 2 * np.abs(want) + weight[..., None] * mass + torch.finfo(dtype).tiny
    got, none = out.double().cpu().numpy(), np.isnan(want)
    assert (np.isnan(got) == none).all()
    err, tol = np.abs(got - want)[~none], tol[~none] * (1 + torch.finfo(dtype).eps)
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))
    got, none, empty = lse.double().cpu().numpy(), np.isnan(want_lse), np.isinf(want_lse)
    assert (np.isnan(got) == none).all() and (np.isneginf(got) == empty).all()
    some = ~(none | empty)
    assert (np.abs(got - want_lse)[some] <= (sums + score + 2.0 ** -22 * np.abs(want_lse))[some]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_many_ragged_sequences(dtype, d):
    """64 sequences on 32 workgroups a KV head: several pieces a workgroup, empty sequences among them."""
    lens = [(37 * i * i) % 300 for i in range(64)]
    lens[5] = lens[41] = 0
    lens[20], lens[63] = 4500, 5000
    check(Records(lens, 8, d, seed=d), 4, [0 if i in (7, 30) else 1 for i in range(64)], dtype, heads=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_pieces(dtype, d):
    """64 KV heads leave 4 workgroups each: 100 and more steps of 32 keys a wave, page ids 32 steps at a time from any place on."""
    c = Records([30001, 0, 9000, 64, 40000, 8191, 33, 12345, 1, 700], 64, d, page=32 if d == 64 else 16, seed=d)
    check(c, 1, [1] * 10, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [5, 12, 40])
def test_long_pieces_of_many_rows(dtype, d, new):
    """The same with 20 to 160 rows a sequence and KV head: two, four or eight workgroups, row blocks that end inside a piece."""
    c = Records([10001, 0, 3000, 64, 13000, 2731, 33, 4100, 1, 700], 64, d, seed=new)
    check(c, 4, [new, 1, new, new, new, max(1, new // 2), 1, new, 0, 1], dtype, heads=1)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_whole_contexts_around_the_steps_that_page_ids_come_in(dtype, d):
    """256 sequences of 8 KV heads, a workgroup each, whose four waves have 32 and 64 steps, one less, one more."""
    lens = [1 + i % 3 for i in range(256)]
    for i, n in enumerate((3968, 3969, 4095, 4096, 4097, 4224, 8064, 8191, 8192, 8193, 8200, 12288, 12289)):
        lens[17 * i + 3] = n
    check(Records(lens, 8, d, page=64, seed=1), 4, [1] * 256, dtype, heads=1)


PIECES = {"few": ([3000, 30], 2), "many": ([10001, 0, 3000, 64, 4800, 33, 4100, 1, 700, 8], 64)}


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 12, 40])
@pytest.mark.parametrize("pieces", PIECES)
def test_nan_blocks_in_cut_contexts(dtype, d, new, pieces):
    """A V block of NaN in a piece in the middle, and one next to the end that some rows do not see; a K block: its KV head alone."""
    lens, hkv = PIECES[pieces]
    c = Records(lens, hkv, d, seed=new)
    n = lens[0]
    c.set_scale(0, 0, n // 3, d // 32 - 1, 1, 255)
    c.set_scale(0, hkv // 3, n - 1 - new // 2, 0, 1, 255)
    c.set_scale(0, 2 * hkv // 3, n - 1 - new // 2, 1, 0, 255)
    G = 4 if new > 1 else 1
    total = [min(new, x) if x else 1 for x in lens]
    out, lse = check(c, G, total, dtype, heads=3)
    nan = torch.isnan(out).cpu().numpy().reshape(-1, hkv, G, d)
    want = np.zeros_like(nan)
    sees = np.arange(total[0]) >= new - 1 - new // 2
    want[:total[0], 0, :, d - 32:] |= True
    want[:total[0], hkv // 3, :, :32] |= sees[:, None, None]
    want[:total[0], 2 * hkv // 3] |= sees[:, None, None]
    assert np.array_equal(nan, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 12, 40])
@pytest.mark.parametrize("pieces", PIECES)
def test_means_of_the_largest_values_in_cut_contexts(dtype, d, new, pieces):
    """V of up to 3/2 2^127, the largest scale that an append leaves."""
    lens, hkv = PIECES[pieces]
    c = Records(lens, hkv, d, seed=new)
    P = c.page
    v = c.cache[:, :, P * d + P * d // 32:]
    v[v != 255] = 252
    c.cache[:, :, P * d // 2:P * d] &= 0x77                       # (all of one sign, so that sums do not cancel)
    out, _ = check(c, 4 if new > 1 else 1, [min(new, x) if x else 1 for x in lens], dtype, heads=2)
    assert torch.isfinite(out).all()
