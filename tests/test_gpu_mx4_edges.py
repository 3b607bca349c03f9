"""The 4-bit cache at the edges of its range: values whose sums leave fp32, outputs with room between sequences, norms beyond fp32's
range, calls whose work is shared by places."""
import numpy as np
import numpy as np
import pytest
import torch

import paper_2506_07311_amd as pa
from tests import mx4_reference as ref
from tests import test_gpu_norm_rope as norms
from tests.test_gpu_mx4 import TYPES, Cache, attend, ints

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 5, 9, 40])
@pytest.mark.parametrize("n", [128, 512, 4000])
def test_means_that_the_join_of_waves_would_lose(dtype, d, new, n):
    """Equal weights and V of 2^118 to 2^123, to 3 / 2 of that: sums within a wave stay in the range of fp32, those of 2, 4 or 8 waves that share
    the keys do not, the means do.  (4 to 160 rows: every shape, whole and cut.)"""
    q = torch.zeros(new, 4, d, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=DEV)
    for e in range(118, 124):
        c = Cache([n], 1, d, seed=e)
        c.v_new = torch.exp2(torch.full_like(c.v_new, e)) * (1 + 0.5 * (torch.arange(d, device=DEV) % 3 == 0))
        c.fill()
        attend(c, [new], 4, dtype, q=q)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("starts,rows", [([0, 1024, 2048, 3072], 4096), ([3, 200, 300, 700], 900), ([0, 90, 91, 400], 402), ([0, 10, 90, 93], 120),
                                         ([5, 20000, 40001, 60000], 70000)])
@pytest.mark.parametrize("part", [False, True])
def test_gather_into_rows_with_room_between_sequences(dtype, starts, rows, part):
    """A sequence's rows begin at its own offset, whatever room is left behind the one before it; where they have less room than tokens,
    the first tokens are taken.  All other rows stay as they were."""
    hkv, d = 2, 128
    c = Cache([80, 0, 3, 77], hkv, d, seed=5).fill()
    first = np.array([13, 0, 0, 64]) if part else np.zeros(4, int)
    ends = np.array([*starts[1:], rows])
    want = [torch.full((rows + 9, hkv, d), 7.0, dtype=TYPES[dtype]) for _ in range(2)]
    for s, kv in enumerate(c.held()):
        for i, x in enumerate(kv):
            x = x[first[s]:][:ends[s] - starts[s]]
            want[i][starts[s]:starts[s] + len(x)] = torch.from_numpy(x).to(TYPES[dtype])
    k, v = (torch.full((rows + 9, hkv, d), 7.0, dtype=TYPES[dtype], device=DEV) for _ in range(2))
    pa.paged_kv_gather_mx4(c.cache, c.table, ints(c.lens), cu_lens=ints([*starts, rows]), max_seq_len=80, out_k=k, out_v=v,
                           first_lens=ints(first) if part else None)
    assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])


def test_gather_of_many_sequences():
    """More sequences than a wave looks at in one go, empty ones among them; few and many rows."""
    rng = np.random.default_rng(3)
    for most in (9, 60):
        lens = [int(x) for x in rng.integers(0, most, 200)]
        lens[0] = lens[63] = lens[64] = lens[199] = 0
        c = Cache(lens, 2, 64, seed=most).fill()
        k, v = (torch.full((sum(lens) + 1, 2, 64), 7.0, device=DEV) for _ in range(2))
        pa.paged_kv_gather_mx4(c.cache, c.table, ints(lens), cu_lens=ints(np.cumsum([0, *lens])), max_seq_len=most, out_k=k, out_v=v)
        for got, i in ((k, 0), (v, 1)):
            want = np.concatenate([x[i] for x in c.held()])
            assert np.array_equal(got[:-1].cpu().numpy(), want.astype(np.float32)) and (got[-1] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 5, 12, 40])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 25])
@pytest.mark.parametrize("n", [300, 3000])
def test_large_scores(dtype, new, size, n):
    """Scores are multiples of size / 2 up to 6 size, exact in fp32, with one largest a row: its V row comes out.  (The two steps of a weight
    and its sum, a product and a quotient: 2^-15 of V.  The score times log2 e is rounded before a logarithm of at most 2^24 is added.)"""
    d, hq = 64, 4
    c = Cache([n], 1, d, seed=9)
    g = torch.Generator().manual_seed(n + new)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0])
    k = torch.zeros(n, 1, d)
    k[:, 0, :hq] = grid[torch.randint(0, 7, (n, hq), generator=g)] * torch.where(torch.rand(n, hq, generator=g) < 0.5, -1.0, 1.0)
    k[:, 0, hq:] = 4.0                                            # (every block's scale is 1)
    best = torch.arange(hq) * 37 + 50
    k[best, 0] = 0.0
    k[best, 0, torch.arange(hq)] = 6.0
    c.k_new = k.to(DEV)
    c.fill()
    q = torch.zeros(new, hq, d, device=DEV)
    q[:, torch.arange(hq), torch.arange(hq)] = size
    out, lse, _ = attend(c, [new], hq, dtype, q=q.to(TYPES[dtype]), scale=1.0, expect=False)
    v = torch.from_numpy(c.held()[0][1][best.numpy(), 0])
    err = (out.double().cpu() - v).abs()
    assert (err <= (2.0 ** -15 + torch.finfo(TYPES[dtype]).eps / 2) * v.abs()).all()
    assert ((lse.double().cpu() - 6 * size).abs() <= 2.0 ** -22 * 6 * size + 2.0 ** -18).all()


@pytest.mark.parametrize("dtype,size", [("fp32", 3e38), ("fp32", 1e-39), ("fp32", 3e-43), ("bf16", 3e38), ("bf16", 1e-39)])
@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (80, 20, False), (256, 128, True)])
def test_norms_of_the_largest_and_of_subnormal_numbers(dtype, size, d, rot, inter):
    """Heads whose root of the mean, or its inverse, fp32 does not hold as a normal number, without an eps."""
    t = TYPES[dtype]
    c = norms.Case(t, d=d, rot=rot, seed=8)
    g = torch.Generator().manual_seed(1)
    for x in (c.q, c.k):
        x.copy_(torch.sign(x) * (size * (0.5 + 0.5 * torch.rand(x.shape, generator=g, dtype=torch.float64).to(DEV))).to(t))
    c.q[5, 1] = 0.0                                               # 0 / 0
    c.q[6, 0, 1:], c.q[6, 0, 0] = 0.0, size
    norms.check(c, t, lambda: pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw, eps=0.0,
                                                        interleaved=inter), eps=0.0, interleaved=inter)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("per_head", [False, True])
def test_norms_of_heads_far_apart(dtype, per_head):
    """Subnormal, ordinary and very large heads in turn and in any order, several of a token in the same lanes."""
    t = TYPES[dtype]
    c = norms.Case(t, T=4100, hq=20, hkv=4, d=128, per_head=per_head, seed=9)
    g = torch.Generator().manual_seed(4)
    for x in (c.q, c.k):
        size = torch.tensor([1e-39, 1.0, 1e30], dtype=torch.float64)[torch.randint(0, 3, (*x.shape[:2], 1), generator=g)]
        x.copy_((x.double().cpu() * size).to(t))
    norms.check(c, t, lambda: pa.paged_norm_rope_append(c.k_cache, c.v_cache, *c.tokens(), q_weight=c.qw, k_weight=c.kw, eps=0.0), eps=0.0)


@pytest.mark.parametrize("dtype,size", [("fp32", 1e-39), ("bf16", 1e-39), ("fp32", 3e38)])
def test_norms_of_subnormal_numbers_into_four_bits(dtype, size):
    t, d = TYPES[dtype], 128
    c = Cache([40], 2, d, seed=3)
    g = torch.Generator().manual_seed(2)
    k = (torch.sign(torch.randn(40, 2, d, generator=g)) * size * (0.25 + 0.75 * torch.rand(40, 2, d, generator=g, dtype=torch.float64))).to(t).to(DEV)
    freq = torch.zeros(0, dtype=torch.float64, device=DEV)
    pa.paged_norm_rope_append_mx4(c.cache, None, k, k, c.places, c.ids, c.places, c.table, freq, eps=0.0)
    want, size = ref.norm_rope(k, c.places, freq, eps=0.0)
    ends = [ref.values(*ref.quantised(want + s * 2.0 ** -19 * size)) for s in (-1, 0, 1)]   # (the bound on an element that the other tests take)
    got = c.held()[0][0]
    assert ((got >= np.minimum.reduce(ends)) & (got <= np.maximum.reduce(ends))).all()


F = np.float32


def steps_of_rotation(a, b, c, s):
    """(a c - b s, a s + b c) in fp32, each product and sum rounded by itself."""
    return a * c - b * s, a * s + b * c


def next_to_borders(rng, c, s):
    """Per element of c and s (fp32) a pair (a, b) of fp32 numbers whose a c - b s lies so near to a border between two codes of scale 1 that
    the separately rounded steps are on one side of it, or on it, and both fused forms on the other.  (0, 0) where none was found."""
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5])
    best = np.zeros((2, *c.shape), F)

    def code(x):
        return ref.quantised(np.concatenate([x[..., None], np.full((*x.shape, 31), 6.0)], -1))[0][..., 0]

    for _ in range(60):
        a = rng.uniform(4, 60, c.shape).astype(F)
        border = rng.choice(borders, c.shape)
        b = ((a.astype(np.float64) * c - border) / s).astype(F)
        for step in range(-6, 7):
            y = (b.view(np.int32) + step).view(F)
            apart = a * c - y * s
            first = (a.astype(np.float64) * c - (y * s)).astype(F)     # a product of two 24-bit numbers is exact in 64 bits
            second = ((a * c) - y.astype(np.float64) * s).astype(F)
            hit = (code(apart) != code(first)) & (code(apart) != code(second)) & (np.abs(apart) < 4)
            best[0], best[1] = np.where(hit, a, best[0]), np.where(hit, y, best[1])
    return best


def test_rotation_on_the_way_to_four_bits_rounds_each_step():
    """Codes are those of products and sums in fp32 that are rounded one by one: elements next to borders, where a fused product would give
    other ones."""
    T, d = 64, 64
    rng = np.random.default_rng(4)
    position = rng.integers(1, 60, T)
    freq = np.geomspace(1.0, 0.02, d // 2)
    angle = position[:, None] * freq
    c, s = np.cos(angle).astype(F), np.sin(angle).astype(F)
    s_safe = np.where(np.abs(s) < 0.05, F(1), s)
    k = np.zeros((T, 1, d), F)
    k[:, 0, :d // 2], k[:, 0, d // 2:] = next_to_borders(rng, c, s_safe)
    k[:, 0][:, np.r_[0, d // 2]] = 0.0
    lost = np.concatenate([np.abs(s) < 0.05] * 2, 1)
    k[:, 0][lost] = 0.0
    k[:, 0, 0], k[:, 0, d // 2] = 5.5 * c[:, 0], -5.5 * s[:, 0]        # (the first pair: about 5.5, which makes the scale 1)
    left, right = steps_of_rotation(k[:, 0, :d // 2], k[:, 0, d // 2:], c, s)
    found = (k[:, 0, 1:d // 2] != 0)
    assert found.mean() > 0.8
    cache = Cache([T], 1, d, seed=1)
    k_dev = torch.from_numpy(k).to(DEV)
    pa.paged_norm_rope_append_mx4(cache.cache, None, k_dev, k_dev, ints(position), cache.ids, cache.places, cache.table,
                                  torch.from_numpy(freq).to(DEV), norm_k=False)
    got = cache.held()[0][0][:, 0]
    want = ref.values(*ref.quantised(np.concatenate([left, right], 1).astype(np.float64)))
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,inter", [(64, True), (128, False), (256, False)])
def test_norms_on_the_way_to_four_bits_round_each_step(dtype, d, inter):
    """Codes of whole heads are those of fp32 steps, rounded one by one: squares summed in fours, then neighbours, the mean and eps, an inverse
    root to a unit in the last place, the products with it, with the weight (its offset added), with cosine and sine, their sum."""
    T, hkv, t = 200, 2, TYPES[dtype]
    g = torch.Generator().manual_seed(d)
    rng = np.random.default_rng(d)
    k = torch.randn(T, hkv, d, generator=g).to(t)
    w = (0.2 * torch.randn(hkv, d, generator=g)).to(t)
    position = rng.integers(0, 60, T)
    freq = np.geomspace(1.0, 0.02, d // 2)
    cache = Cache([T], hkv, d, seed=2)
    k_dev = k.to(DEV)
    pa.paged_norm_rope_append_mx4(cache.cache, None, k_dev, k_dev, ints(position), cache.ids, cache.places, cache.table,
                                  torch.from_numpy(freq).to(DEV), k_weight=w.to(DEV), weight_offset=1.0, eps=1e-5, interleaved=inter)
    got = cache.held()[0][0]
    x = k.float().numpy()
    sq = (x * x).reshape(T, hkv, d // 4, 4)
    total = ((sq[..., 0] + sq[..., 1]) + sq[..., 2]) + sq[..., 3]
    while total.shape[-1] > 1:
        total = total[..., 0::2] + total[..., 1::2]
    mean = total * F(1.0 / d) + F(1e-5)
    angle = position[:, None] * freq
    c, s = (f(angle).astype(F)[:, None] for f in (np.cos, np.sin))
    root = (1.0 / np.sqrt(mean.astype(np.float64))).astype(F)
    ok = np.zeros((T, hkv), bool)
    for step in (-1, 0, 1):
        z = x * (root.view(np.int32) + step).view(F) * (w.float().numpy() + F(1))
        lead = (slice(0, None, 2), slice(1, None, 2)) if inter else (slice(0, d // 2), slice(d // 2, None))
        turned = np.empty_like(z)
        turned[..., lead[0]], turned[..., lead[1]] = steps_of_rotation(z[..., lead[0]], z[..., lead[1]], c, s)
        ok |= (ref.values(*ref.quantised(turned.astype(np.float64))) == got).all(-1)
    assert ok.all(), int((~ok).sum())
