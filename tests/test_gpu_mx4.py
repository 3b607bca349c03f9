"""The cache of 4-bit elements: what is stored, bit for bit, and attention over it, against definitions in 64 bits."""
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


class Cache:
    """Sequences in a 4-bit cache whose other slots, and pages, hold bytes of 255: blocks of NaN."""

    def __init__(self, lens, hkv=2, d=128, page=16, seed=0, spread=3, room=2, extra=0):
        rng = np.random.default_rng(seed)
        self.lens, self.hkv, self.d, self.page = list(lens), hkv, d, page
        blocks = [-(-n // page) for n in self.lens]
        pages = sum(blocks) + 3
        order = rng.permutation(pages)
        self.table_np = np.full((len(lens), max(max(blocks), 1) + room), -1)
        at = 0
        for s, b in enumerate(blocks):
            self.table_np[s, :b] = order[at:at + b]
            at += b
        self.table = ints(self.table_np)
        size = pa.pa_mx4_record_bytes(page, d)
        self.cache = torch.full((pages, hkv + extra, size), 255, dtype=torch.uint8, device=DEV)[:, :hkv]
        total = sum(self.lens)
        g = torch.Generator().manual_seed(seed)
        scale = torch.exp2(torch.randint(-spread, spread + 1, (2, total, hkv, 1), generator=g).float())
        self.k_new, self.v_new = (torch.randn(2, total, hkv, d, generator=g) * scale).to(DEV)
        self.ids = ints(np.repeat(np.arange(len(lens)), self.lens))
        self.places = ints(np.concatenate([np.arange(n) for n in self.lens] + [np.zeros(0)]))

    def fill(self, dtype=torch.float32):
        self.k_new, self.v_new = self.k_new.to(dtype), self.v_new.to(dtype)
        pa.paged_kv_append_mx4(self.cache, self.k_new, self.v_new, self.ids, self.places, self.table)
        return self

    def held(self):
        """[(K, V) [len, hkv, d]] in 64 bits, from the cache's bytes."""
        kv = [ref.values(*x).swapaxes(1, 2) for x in ref.unpacked(self.cache, self.page, self.d)]   # [pages, P, Hkv, d]
        res = []
        for s, n in enumerate(self.lens):
            pages = self.table_np[s, :-(-n // self.page)]
            res.append([x[pages].reshape(-1, self.hkv, self.d)[:n] for x in kv])
        return res


def stored_as_defined(c):
    """The bytes of every slot: the sequences' by definition, all others 255 still."""
    want = torch.full(tuple(c.cache.shape), 255, dtype=torch.uint8).numpy()
    page, place = c.table_np[c.ids.cpu(), c.places.cpu() // c.page], (c.places.cpu() % c.page).numpy()
    P, d, w = c.page, c.d, c.d // 32
    for what, x in enumerate((c.k_new, c.v_new)):
        codes, scales = ref.quantised(x.double().cpu().numpy())
        b = codes[..., 0::2] + 16 * codes[..., 1::2]              # [T, hkv, d / 2]
        j = np.arange(d // 2)
        for t in range(len(place)):
            at = place[t] * (d // 2) + j if what == 0 else P * d // 2 + (place[t] // 8 * 16 + j // w) * 8 * w + place[t] % 8 * w + j % w
            want[page[t], :, at] = b[t].T
            want[page[t], :, P * d + what * P * w + np.arange(w) * P + place[t]] = scales[t].T
    return np.array_equal(want, c.cache.cpu().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page,hkv", [(16, 1), (32, 3), (128, 8)])
def test_append_bit_for_bit(dtype, d, page, hkv):
    c = Cache([1, 37, 0, page, 3 * page + 7], hkv, d, page, seed=d + page, extra=1).fill(TYPES[dtype])
    assert stored_as_defined(c)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_append_of_all_kinds_of_values(dtype):
    """Every exponent, ties between codes, zeros of both signs, subnormal numbers, the largest, infinities and NaN."""
    t = TYPES[dtype]
    info = torch.finfo(t)
    c = Cache([96, 64], hkv=2, d=128, seed=1)
    x = torch.randn(160, 2, 128, generator=torch.Generator().manual_seed(2))
    step = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 7.9, 6.0, 4.0, 0.5, 0.0, -0.0, -0.25, -5.0]).repeat(8)
    lo, hi = int(np.log2(info.smallest_normal)), int(np.log2(info.max))
    for i in range(64):
        x[i] = step * 2.0 ** (lo + (hi - 3 - lo) * i / 63 // 1)
    x[64:70] = 0.0
    x[70, :, :32], x[71, :, 40], x[72, 0, 5], x[73, 1, 127] = info.max, info.smallest_normal / 4, float("nan"), -float("inf")
    x[74], x[75] = -0.0, info.min
    x[76] = info.smallest_normal * torch.rand(128)
    x = x.to(t).to(DEV)
    c.k_new, c.v_new = x, x.flip(0).contiguous()
    c.fill(t)
    assert stored_as_defined(c)


def test_append_of_every_bf16_number():
    bits = torch.arange(65536, dtype=torch.int32)
    x = bits.to(torch.int16).view(torch.bfloat16).reshape(-1, 1, 64)          # blocks of one exponent
    y = bits.reshape(256, 256).t().reshape(-1).to(torch.int16).view(torch.bfloat16).reshape(-1, 1, 64)   # of all
    c = Cache([1024], hkv=1, d=64, page=64)
    c.k_new, c.v_new = x.to(DEV).contiguous(), y.to(DEV).contiguous()
    c.fill(torch.bfloat16)
    assert stored_as_defined(c)


def test_append_leaves_padded_and_unmapped_rows():
    c = Cache([40, 20], page=16)
    c.table_np[1, 1] = -1
    c.table.copy_(ints(c.table_np))
    c.places[::3] = -1
    c.fill(torch.bfloat16)
    keep = ((c.places >= 0) & ~((c.ids == 1) & (c.places >= 16))).cpu()
    c.ids, c.places, c.k_new, c.v_new = c.ids[keep.to(DEV)], c.places[keep.to(DEV)], c.k_new[keep.to(DEV)], c.v_new[keep.to(DEV)]
    assert stored_as_defined(c)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d,page,hkv", [(64, 16, 3), (128, 64, 8), (256, 32, 1)])
def test_gather(dtype, d, page, hkv):
    c = Cache([1, 0, 77, 200, 9], hkv, d, page, seed=3).fill()
    first = [0, 0, 13, 64, 9]
    for begin in (None, first):
        begin_np = np.zeros(5, int) if begin is None else np.array(begin)
        n = np.array(c.lens) - begin_np
        k, v = (torch.full((n.sum() + 2, hkv, d), 7.0, dtype=TYPES[dtype], device=DEV) for _ in range(2))
        pa.paged_kv_gather_mx4(c.cache, c.table, ints(c.lens), cu_lens=ints(np.cumsum([0, *n])), max_seq_len=200, out_k=k, out_v=v,
                               first_lens=None if begin is None else ints(begin))
        for got, i in ((k, 0), (v, 1)):
            want = np.concatenate([x[i][b:] for x, b in zip(c.held(), begin_np)])
            assert torch.equal(got[:-2].cpu(), torch.from_numpy(want).to(TYPES[dtype])) and (got[-2:] == 7).all()


def test_gather_of_every_code_and_scale():
    c = Cache([256], hkv=1, d=64, page=256)
    kv = c.cache[c.table_np[0, 0], 0]
    P, d = 256, 64
    codes = torch.arange(P * d // 2, device=DEV) % 251
    kv[:P * d // 2], kv[P * d // 2:P * d] = codes.to(torch.uint8), codes.flip(0).to(torch.uint8)
    kv[P * d:] = (torch.arange(P * d // 16, device=DEV) % 256).to(torch.uint8)
    k, v = (torch.empty(256, 1, 64, device=DEV) for _ in range(2))
    pa.paged_kv_gather_mx4(c.cache, c.table, ints([256]), cu_lens=ints([0, 256]), max_seq_len=256, out_k=k, out_v=v)
    for got, want in zip((k, v), c.held()[0]):
        np.testing.assert_array_equal(got.cpu().numpy(), want.astype(np.float32))


def attend(c, new, hq, dtype=torch.bfloat16, seed=0, scale=None, pad=0, q=None, loose=0, expect=True):
    """Runs the call, checks it, and returns (out, lse, q)."""
    t = TYPES[dtype] if isinstance(dtype, str) else dtype
    g = torch.Generator().manual_seed(seed + 100)
    total = sum(new)
    if q is None:
        q = torch.randn(total + pad, hq, c.d, generator=g).to(t).to(DEV)
    scale = c.d ** -0.5 if scale is None else scale
    out, lse = torch.full_like(q, 3.0), torch.full((total + pad, hq), 5.0, device=DEV)
    cu = np.cumsum([0, *new])
    longest = max(max(c.lens), 1)
    top = min(longest + loose, c.table.shape[1] * c.page)
    pa.paged_attention_mx4(c.cache, q, ints(cu), max(new) + loose, c.table, ints(c.lens), top, scale, out=out, lse=lse)
    assert (out[total:] == 3).all() and (lse[total:] == 5).all()
    if expect:
        for s, (k, v) in enumerate(c.held()):
            if new[s]:
                near(out[cu[s]:cu[s + 1]], lse[cu[s]:cu[s + 1]], q[cu[s]:cu[s + 1]], k, v, c.lens[s] - new[s], scale, t)
    return out, lse, q


def near(out, lse, q, k, v, n_ctx, scale, dtype):
    """Bounds.  A score is a 32-bit sum of up to 3 x 256 exact products: off by less than 2^-18 of the sum of their magnitudes; the rounding of
    score times log2 e less the reference is 2^-23 of a number of at most twice that size.  exp2 is good to 2^-22, a weight in two
    16-bit terms to 2^-17 (three: 2^-24), sums of weights and products to 2^-19 for the lengths here.  The output is rounded once."""
    want, want_lse, mass, size = ref.attention(q.double().cpu().numpy(), k, v, n_ctx, scale)
    score = 2.0 ** -17 * size
    weight = (2.0 ** -16 if dtype != torch.float32 else 2.0 ** -18) + 2 * score
    tol = torch.finfo(dtype).eps / 2 * np.abs(want) + weight[..., None] * mass + torch.finfo(dtype).tiny
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= tol * (1 + torch.finfo(dtype).eps)).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
    got = lse.double().cpu().numpy()
    empty = np.isinf(want_lse)
    assert (np.isneginf(got) == empty).all()
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want_lse)
    assert (off[~empty] <= (2.0 ** -18 + score + 2.0 ** -22 * np.abs(want_lse))[~empty]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv,new", [(8, 2, 1), (4, 4, 3), (32, 1, 1), (7, 1, 9), (16, 2, 17), (6, 2, 50)])
def test_attention(dtype, d, hq, hkv, new):
    """Rows of a KV head from 3 to 153: every shape, with row blocks that end inside a tile."""
    lens = [new, new + 1, new + 31, 290, 700 + new]
    c = Cache(lens, hkv, d, page=16, seed=hq + new).fill()
    rng = np.random.default_rng(new)
    attend(c, [new if i == 0 else int(rng.integers(1, new + 1)) for i in range(5)], hq, dtype, pad=2)


@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_lengths_and_pages(page, n):
    c = Cache([n, max(1, n - 1)], 2, 128, page, seed=n, room=0).fill()
    attend(c, [1, 1], 8)
    attend(c, [n if n < 70 else 5, 1], 8, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_contexts_are_cut_and_joined(dtype, d):
    c = Cache([9000, 30, 3001], 1, d, page=64, seed=d).fill()
    attend(c, [1, 1, 1], 4, dtype)
    attend(c, [5, 7, 1], 4, dtype, seed=1)
    attend(c, [20, 3, 9], 4, dtype, seed=2)


def test_whole_prompts():
    c = Cache([333, 1, 128, 517], 2, 128, page=32, seed=5).fill()
    attend(c, [333, 1, 128, 517], 8)
    attend(c, [300, 1, 64, 200], 8, "fp16", seed=1)


@pytest.mark.parametrize("new", [1, 6, 30, 90])
def test_padded_batch(new):
    """Sequences without a token, without a query, and bounds that are not tight."""
    c = Cache([0, 400, 0, 250, 1], 2, 128, seed=6, room=9).fill()
    out, lse, _ = attend(c, [1, new, 0, 0, 1], 4, loose=70)
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()
    out, lse, _ = attend(c, [new, 1, 0, 1, 0], 4, seed=2)         # queries of a sequence that has no token
    assert (out[:new] == 0).all() and torch.isneginf(lse[:new]).all()


def test_more_queries_than_tokens():
    c = Cache([3, 40], 1, 64, seed=7).fill()
    out, lse, _ = attend(c, [8, 2], 2)
    assert (out[:5] == 0).all() and torch.isneginf(lse[:5]).all()


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0, 1e-6])
def test_scales(scale):
    c = Cache([200, 77], 2, 128, seed=8).fill()
    attend(c, [3, 1], 4, scale=scale)


@pytest.mark.parametrize("dtype,size", [("bf16", 1e30), ("bf16", 1e-30), ("fp16", 6e4), ("fp16", 1e-7), ("fp32", 1e25), ("fp32", 1e-25)])
def test_sizes_of_queries(dtype, size):
    c = Cache([200], 2, 128, seed=9).fill()
    g = torch.Generator().manual_seed(1)
    q = (torch.rand(2, 4, 128, generator=g) * size).to(TYPES[dtype]).to(DEV)
    attend(c, [2], 4, dtype, q=q, scale=float(1.0 / size / 128))


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_blocks_reach_those_that_see_them(new, d):
    hq, hkv, n = 4, 2, 350
    c = Cache([n, n], hkv, d, seed=10).fill()
    clean, clean_lse, q = attend(c, [new, new], hq)
    last = n - new // 2 - 1                                       # rows before it do not see it
    page, slot = c.table_np[0, last // 16], last % 16
    P, w = 16, d // 32
    c.cache[page, 1, P * d + P * w + 1 * P + slot] = 255          # V, head 1, its second 32 elements
    page1, slot1 = c.table_np[1, 100 // 16], 100 % 16
    c.cache[page1, 0, P * d + 0 * P + slot1] = 255                # K, head 0, seen by all rows of sequence 1
    out, lse, _ = attend(c, [new, new], hq, q=q, expect=False)
    i = torch.arange(new, device=DEV)
    sees = n - new + i >= last
    assert sees.any() and (new == 1 or not sees.all())
    want = clean.clone()
    want[:new][sees, 2:, 32:64] = float("nan")
    want[new:, :2] = float("nan")
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    ok = ~torch.isnan(want)
    torch.testing.assert_close(out[ok], want[ok], rtol=2 ** -7, atol=1e-4)
    assert torch.isnan(lse[new:, :2]).all()
    k, v = c.held()[0]                                            # (V has no part in them; near() says why so near)
    _, want_lse, _, size = ref.attention(q[:new].double().cpu().numpy(), k, np.zeros_like(v), n - new, d ** -0.5)
    for got in (lse, clean_lse):
        assert (np.abs(got[:new].double().cpu().numpy() - want_lse) <= 2.0 ** -18 + 2.0 ** -17 * size + 2.0 ** -22 * np.abs(want_lse)).all()


def test_means_of_large_values_are_finite():
    """512 values of 2^126: their sums of weights leave the range of fp32, their means do not."""
    c = Cache([512, 300], 1, 128, seed=11)
    c.v_new = torch.sign(c.v_new) * 6.0 * 2.0 ** 124
    c.v_new[:, :, :64] = 6.0 * 2.0 ** 125
    c.fill()
    for new in (1, 9, 40):
        attend(c, [new, 2], 8, "fp32" if new == 9 else "bf16", seed=new)


@pytest.mark.parametrize("lead", [200.0, -200.0])
def test_weights_far_apart(lead):
    """A key that leads by e^200, early and late: what went before counts for nothing, or what follows."""
    c = Cache([600], 1, 64, seed=12)
    q = torch.zeros(1, 2, 64, device=DEV)
    q[..., 0] = 8.0
    c.k_new[:, :, 0] = 0.0
    c.k_new[[3, 500], :, 0] = torch.tensor([lead, -lead], device=DEV)[:, None]
    c.fill()
    attend(c, [1], 2, "fp32", q=q)


def test_queries_of_nan_and_infinity_stay_in_their_rows():
    c = Cache([300], 1, 128, seed=13).fill()
    _, _, q = attend(c, [20], 4)
    q[3, 1, 5], q[7, 2, 9] = float("nan"), float("inf")
    out, lse, _ = attend(c, [20], 4, q=q, expect=False)
    bad = torch.zeros(20, 4, dtype=torch.bool, device=DEV)
    bad[3, 1] = bad[7, 2] = True
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()


def test_cache_views_and_far_pages():
    """A part of a larger cache, and pages beyond 2^32 bytes."""
    size = pa.pa_mx4_record_bytes(16, 128)
    pages = (1 << 32) // (2 * size) + 4000
    big = pa.pa_mx4_cache(pages, 16, 2, 128).view(pages, 2, size)
    c = Cache([500, 90], 2, 128, seed=14).fill()
    far = pages - c.cache.shape[0]
    big[far:] = c.cache
    table = torch.where(c.table >= 0, c.table + far, -1).to(torch.int32)
    q = torch.randn(5, 8, 128, device=DEV).bfloat16()
    args = (ints([0, 4, 5]), 4)
    want = pa.paged_attention_mx4(c.cache, q, *args, c.table, ints(c.lens), 500, 0.1)
    assert torch.equal(want, pa.paged_attention_mx4(big, q, *args, table, ints(c.lens), 500, 0.1))
    k, v = (torch.randn(2, 2, 128, device=DEV).bfloat16() for _ in range(2))
    for cache, t in ((c.cache, c.table), (big, table)):
        pa.paged_kv_append_mx4(cache, k, v, ints([0, 1]), ints([499, 0]), t)
    assert torch.equal(big[far:], c.cache)
    got = [torch.empty(590, 2, 128, device=DEV) for _ in range(4)]
    for cache, t, o in ((c.cache, c.table, got[:2]), (big, table, got[2:])):
        pa.paged_kv_gather_mx4(cache, t, ints(c.lens), cu_lens=ints([0, 500, 590]), max_seq_len=500, out_k=o[0], out_v=o[1])
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])


def test_results_do_not_depend_on_the_run_or_stream():
    c = Cache([3000, 77, 1200], 2, 128, seed=15).fill()
    q = torch.randn(7, 8, 128, device=DEV).bfloat16()
    args = (ints([0, 1, 5, 7]), 4, c.table, ints(c.lens), 3000, 0.1)
    want = pa.paged_attention_mx4(c.cache, q, *args)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        assert torch.equal(want, pa.paged_attention_mx4(c.cache, q, *args))
        with torch.cuda.stream(side):
            other = pa.paged_attention_mx4(c.cache, q, *args, stream=side)
        side.synchronize()
        assert torch.equal(want, other)


def test_two_captured_steps_that_share_a_workspace():
    c = Cache([2000, 150], 2, 128, seed=16).fill()
    q1, q2 = torch.randn(2, 8, 128, device=DEV).bfloat16(), torch.randn(9, 8, 128, device=DEV).bfloat16()
    lens = ints(c.lens)
    ws = torch.empty(max(pa.paged_attention_mx4_workspace_bytes(2, 8, 2, 128, n, m, 2000) for n, m in ((2, 1), (9, 8))), dtype=torch.uint8,
                     device=DEV)
    calls = [(q1, ints([0, 1, 2]), 1, c.table, lens, 2000, 0.1), (q2, ints([0, 8, 9]), 8, c.table, lens, 2000, 0.1)]
    want = [pa.paged_attention_mx4(c.cache, *x) for x in calls]
    outs, graphs = [torch.empty_like(x) for x in want], []
    side = torch.cuda.Stream()
    for x, out in zip(calls, outs):
        side.wait_stream(torch.cuda.current_stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            pa.paged_attention_mx4(c.cache, *x, out=out, workspace=ws)
    for i in range(4):
        for g, out, w in zip(graphs, outs, want):
            out.zero_(), ws.fill_(255 if i % 2 else 0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w), i


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d,inter", [(64, False), (128, True), (256, False)])
def test_norm_rope_append_into_four_bits(dtype, d, inter):
    """Stored is what the 32-bit rows round to.  A row's element is known to 2^-19 of its pair's size: its code is that of a number
    within this distance, its block's scale that of a magnitude within it."""
    t = TYPES[dtype]
    T, hq, hkv = 130, 4, 2
    c = Cache([100, 30], hkv, d, seed=17)
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(T, h, d, generator=g).to(t).to(DEV) for h in (hq, hkv, hkv))
    rope = ints(np.random.default_rng(1).integers(0, 50000, (3, T)))
    axes = ints(np.arange(d // 2) % 3)
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).to(DEV)
    qw, kw = (1 + 0.3 * torch.randn(2, d, generator=g)).to(t).to(DEV)
    out = pa.paged_norm_rope_append_mx4(c.cache, q, k, v, rope, c.ids, c.places, c.table, freq, q_weight=qw, k_weight=kw, pair_axes=axes,
                                        interleaved=inter)
    want, size = ref.norm_rope(q, rope, freq, qw, axes_of=axes.cpu(), interleaved=inter)
    assert (np.abs(out.double().cpu().numpy() - want) <= torch.finfo(t).eps / 2 * np.abs(want) + 2.0 ** -18 * size).all()
    want, size = ref.norm_rope(k, rope, freq, kw, axes_of=axes.cpu(), interleaved=inter)
    err = 2.0 ** -19 * size
    held = c.held()
    got_k, got_v = (np.concatenate([h[i] for h in held]) for i in range(2))
    ends = [ref.values(*ref.quantised(want + s * err)) for s in (-1, 0, 1)]
    lo, hi = np.minimum.reduce(ends), np.maximum.reduce(ends)
    assert ((got_k >= lo) & (got_k <= hi)).all()
    assert (got_k != ends[1]).mean() < 1e-3                       # (2 x 2^-19 of an element's size next to one of 7 borders)
    np.testing.assert_array_equal(got_v, ref.values(*ref.quantised(v.double().cpu().numpy())))


def test_a_run_as_a_server_makes_it():
    """Plan, norms and positions into the 4-bit cache, attention: a prompt, then three steps of one or several tokens, two sequences."""
    hq, hkv, d, page = 8, 2, 128, 16
    g = torch.Generator().manual_seed(5)
    cache = pa.pa_mx4_cache(80, page, hkv, d)
    cache.fill_(255)
    table, num = ints(np.full((2, 40), -1)), ints([0, 0])
    free, count = ints(np.random.default_rng(2).permutation(80)), ints([80])
    ctx = ints([0, 0])
    freq, mscale = pa.pa_rope_frequencies(d, 10000.0, "linear", factor=2.0)
    freq = freq.to(DEV)
    qw, kw = (1 + 0.1 * torch.randn(2, d, generator=g)).bfloat16().to(DEV)
    for width, new in ((150, [150, 61]), (1, [1, 1]), (4, [4, 2]), (1, [1, 1])):
        rows = 2 * width
        new_t = ints(new)
        plan = pa.paged_plan_step(ctx, new_t, table, num, free, count, page, rows, mask_words=0)
        qkv = torch.randn(rows, (hq + 2 * hkv) * d, generator=g).bfloat16().to(DEV)
        q, k, v = (x.view(rows, -1, d) for x in qkv.split([hq * d, hkv * d, hkv * d], 1))
        q = pa.paged_norm_rope_append_mx4(cache, q, k, v, plan.rope_positions, plan.seq_ids, plan.positions, table, freq, q_weight=qw,
                                          k_weight=kw, mscale=mscale)
        lse = torch.zeros(rows, hq, device=DEV)
        out = pa.paged_attention_mx4(cache, q, plan.cu_q_lens, width, table, plan.seq_lens, 40 * page, d ** -0.5, lse=lse)
        ctx = plan.seq_lens.clone()
        assert plan.shortage.tolist() == [0, 0]
        lens, cu = ctx.tolist(), plan.cu_q_lens.tolist()
        k_all, v_all = (torch.empty(sum(lens), hkv, d, device=DEV) for _ in range(2))
        pa.paged_kv_gather_mx4(cache, table, ctx, cu_lens=ints([0, lens[0], sum(lens)]), max_seq_len=max(lens), out_k=k_all, out_v=v_all)
        k_all, v_all = k_all.double().cpu().numpy(), v_all.double().cpu().numpy()
        for s in range(2):
            part = slice(0, lens[0]) if s == 0 else slice(lens[0], None)
            r = slice(cu[s], cu[s + 1])
            near(out[r], lse[r], q[r], k_all[part], v_all[part], lens[s] - new[s], d ** -0.5, torch.bfloat16)
        # what was stored of this step is what its rows round to, V exactly
        kept = np.concatenate([v_all[lens[0] - new[0]:lens[0]], v_all[sum(lens) - new[1]:]])
        live = (plan.positions >= 0).cpu().numpy()
        np.testing.assert_array_equal(kept, ref.values(*ref.quantised(v.double().cpu().numpy()[live])))


def test_shared_pages_are_copied_before_a_write():
    """The page manager over a 4-bit cache: a shared prefix, a private copy of its last page, and an append there."""
    hkv, d, page = 3, 64, 32
    cache = pa.pa_mx4_cache(10, page, hkv + 1, d)[:, :hkv]        # (a part of a larger one)
    cache.fill_(255)
    table = torch.zeros(2, 5, dtype=torch.int32, device=DEV)
    pool = pa.pa_pool_create(10, page, 2, 5, table)
    pa.pa_pool_reserve(pool, 0, 64)
    k, v = torch.randn(2, 64, hkv, d, device=DEV)
    pa.paged_kv_append_mx4(cache, k, v, ints(np.zeros(64)), ints(np.arange(64)), table)
    pa.pa_pool_share_prefix(pool, 1, 0, 64)
    before = cache.clone()
    pa.pa_pool_make_writable_mx4(pool, cache, 1, 40, head_dim=d)
    rows = table.cpu()
    assert rows[0, 0] == rows[1, 0] and rows[0, 1] != rows[1, 1]
    assert torch.equal(cache[rows[0, 1]], cache[rows[1, 1]])
    pa.paged_kv_append_mx4(cache, k[:1], v[:1], ints([1]), ints([40]), table)
    assert not torch.equal(cache[rows[0, 1]], cache[rows[1, 1]])
    other = torch.arange(10) != rows[1, 1]
    assert torch.equal(before[other.to(DEV)], cache[other.to(DEV)])
    pa.pa_pool_make_writable_mx4(pool, cache, 1, 40)              # private already
    assert torch.equal(rows, table.cpu())
    with pytest.raises(PagedAttnError):
        pa.pa_pool_make_writable_mx4(pool, cache, 1, 40, head_dim=128)
    with pytest.raises(PagedAttnError):
        pa.pa_pool_make_writable_mx4(pool, cache, 1, 64, head_dim=d)
    pa.pa_pool_destroy(pool)


def test_prompts_beside_decode_steps():
    """Rows of one sequence, a bound for all: the work is shared by keys."""
    c = Cache([1500, 900, 2000, 64, 700], 2, 128, seed=18).fill()
    attend(c, [1, 300, 1, 64, 1], 8)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 12])
def test_many_sequences(dtype, new):
    """More than a wave looks at in one go, and units for the whole machine."""
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(0, 150, 140)]
    c = Cache(lens, 2, 64, seed=19).fill()
    attend(c, [min(n, int(rng.integers(0, new + 1))) if i % 7 else min(n, new) for i, n in enumerate(lens)], 4, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_long_context_among_short_ones(dtype, d):
    c = Cache([9000, 10, 700, 1, 33, 2000, 0, 64], 8, d, page=32, seed=20).fill()
    attend(c, [1] * 6 + [0, 1], 16, dtype)


def test_calls_beside_each_other():
    """Two streams, each with its workspace."""
    c = Cache([4000, 300], 2, 128, seed=21).fill()
    q = [torch.randn(2 * n, 8, 128, device=DEV).bfloat16() for n in (1, 5)]
    args = [(x, ints([0, n, 2 * n]), n, c.table, ints(c.lens), 4000, 0.1) for x, n in zip(q, (1, 5))]
    want = [pa.paged_attention_mx4(c.cache, *a) for a in args]
    streams = [torch.cuda.Stream() for _ in args]
    torch.cuda.synchronize()
    outs = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    calls = [pa.prepare_attention_mx4(c.cache, *a, out=o, stream=s) for a, o, s in zip(args, outs, streams)]
    for _ in range(20):
        for call in calls:
            call()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_refusals():
    c = Cache([40, 9], 2, 128).fill(torch.bfloat16)
    q = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    good = dict(cache=c.cache, q=q, cu=ints([0, 1, 2]), max_q=1, table=c.table, lens=ints(c.lens), max_len=40, scale=0.1)
    pa.paged_attention_mx4(*good.values())
    for change in (dict(q=q.double()), dict(q=q[:, :3]), dict(q=q.transpose(0, 1)), dict(cu=ints([0, 1])),
                   dict(lens=ints([40])), dict(table=c.table[:1]), dict(table=c.table.long()), dict(cache=c.cache[..., :-16]),
                   dict(cache=c.cache.cpu()), dict(cache=c.cache.to(torch.int32)), dict(max_len=100000), dict(scale=float("nan")),
                   dict(max_q=-1)):
        with pytest.raises(PagedAttnError):
            pa.paged_attention_mx4(*dict(good, **change).values())
    # a shape that says the page's tokens: heads of another size are refused (a record of 16 x 128 is as large as one of 32 x 64)
    four = c.cache.view(c.cache.shape[0], 2, 16, 136)
    assert torch.equal(pa.paged_attention_mx4(*dict(good, cache=four).values()), pa.paged_attention_mx4(*good.values()))
    for change in (dict(q=q[..., :64].contiguous()), dict(cache=four[:, :, :8]), dict(cache=four[..., :68]), dict(cache=four.transpose(2, 3))):
        with pytest.raises(PagedAttnError):
            pa.paged_attention_mx4(*dict(dict(good, cache=four), **change).values())
    with pytest.raises(PagedAttnError):
        pa.paged_attention_mx4(*good.values(), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(PagedAttnError):
        pa.paged_attention_mx4(*good.values(), out=torch.empty(2, 4, 128, device=DEV))
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device=DEV)
    for args in ((k, k[:2], ints([0] * 3), ints([0] * 3), c.table), (k, k.float(), ints([0] * 3), ints([0] * 3), c.table),
                 (k, k, ints([0] * 2), ints([0] * 3), c.table), (k[:, :1], k[:, :1], ints([0] * 3), ints([0] * 3), c.table),
                 (k.int(), k.int(), ints([0] * 3), ints([0] * 3), c.table), (k, k, ints([0] * 3), ints([0] * 3), c.table[0])):
        with pytest.raises(PagedAttnError):
            pa.paged_kv_append_mx4(c.cache, *args)
    for change in (dict(out_v=k[:2]), dict(out_k=k.int()), dict(cu_lens=ints([0, 1])), dict(first_lens=ints([0])), dict(out_k=k[:, :1])):
        kw = dict(dict(cu_lens=ints([0, 1, 3]), max_seq_len=40, out_k=k, out_v=k.clone(), first_lens=None), **change)
        with pytest.raises(PagedAttnError):
            pa.paged_kv_gather_mx4(c.cache, c.table, ints(c.lens), **kw)
    rope = ints([0, 1])
    with pytest.raises(PagedAttnError):
        pa.paged_norm_rope_append_mx4(c.cache, None, None, None, rope, None, None, None, torch.zeros(64, dtype=torch.float64, device=DEV))
    with pytest.raises(PagedAttnError):
        pa.paged_norm_rope_append_mx4(c.cache, q[..., :96].contiguous(), None, None, rope, None, None, None,
                                      torch.zeros(16, dtype=torch.float64, device=DEV))


def test_a_captured_decode_loop():
    """One graph of plan, norms and positions into the cache, attention and the lengths' step, replayed with eager work in between: each
    replay as the calls one by one on a cache of their own."""
    hq, hkv, d, page, B = 8, 2, 128, 16, 3
    g = torch.Generator().manual_seed(6)
    freq = pa.pa_rope_frequencies(d)[0].to(DEV)
    qw, kw = (1 + 0.1 * torch.randn(2, d, generator=g)).bfloat16().to(DEV)
    q_in, out = torch.zeros(B, hq, d, dtype=torch.bfloat16, device=DEV), torch.zeros(B, hq, d, dtype=torch.bfloat16, device=DEV)
    k_in, v_in = (torch.zeros(B, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    new = ints([1] * B)

    class Side:
        def __init__(self):
            self.cache = pa.pa_mx4_cache(60, page, hkv, d)
            self.cache.fill_(255)
            self.table, self.num = ints(np.full((B, 20), -1)), ints([0] * B)
            self.free, self.count, self.ctx = ints(np.arange(60)), ints([60]), ints([0] * B)
            self.cu, self.lens, self.ids, self.at, self.rope = (ints(np.zeros(n)) for n in (B + 1, B, B, B, B))
            self.short, self.q = ints([0, 0]), torch.zeros_like(q_in)
            self.ws = torch.empty(pa.paged_attention_mx4_workspace_bytes(B, hq, hkv, d, B, 1, 20 * page), dtype=torch.uint8, device=DEV)

        def step(self, o):
            pa.paged_plan_step(self.ctx, new, self.table, self.num, self.free, self.count, page, B, mask_words=0, seq_lens=self.lens,
                               cu_q_lens=self.cu, seq_ids=self.ids, positions=self.at, rope_positions=self.rope, shortage=self.short)
            pa.paged_norm_rope_append_mx4(self.cache, q_in, k_in, v_in, self.rope, self.ids, self.at, self.table, freq, q_weight=qw, k_weight=kw,
                                          q_out=self.q)
            pa.paged_attention_mx4(self.cache, self.q, self.cu, 1, self.table, self.lens, 20 * page, d ** -0.5, out=o, workspace=self.ws)
            self.ctx.add_(new)

    one, other = Side(), Side()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        one.step(out)
    want = torch.zeros_like(out)
    for i in range(40):
        for x in (q_in, k_in, v_in):
            x.copy_(torch.randn(x.shape, generator=g).bfloat16())
        graph.replay()
        other.step(want)
        torch.cuda.synchronize()
        assert one.ctx.tolist() == [i + 1] * B and one.short.tolist() == [0, 0]
        assert torch.equal(out, want) and torch.equal(one.cache, other.cache) and bool(torch.isfinite(out.float()).all())


def test_captured_append_and_gather():
    c = Cache([300, 77, 5], 2, 128, seed=22)
    k, v = (torch.zeros(382, 2, 128, device=DEV) for _ in range(2))
    lens, cu = ints(c.lens), ints(np.cumsum([0, *c.lens]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pa.paged_kv_append_mx4(c.cache, c.k_new, c.v_new, c.ids, c.places, c.table)
        pa.paged_kv_gather_mx4(c.cache, c.table, lens, cu_lens=cu, max_seq_len=300, out_k=k, out_v=v)
    for i in range(3):
        c.k_new.mul_(-1.5), c.v_new.add_(0.1)
        k.zero_(), v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, x in ((k, c.k_new), (v, c.v_new)):
            np.testing.assert_array_equal(got.cpu().numpy(), ref.values(*ref.quantised(x.double().cpu().numpy())))
