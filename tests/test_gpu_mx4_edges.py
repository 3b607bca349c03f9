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
