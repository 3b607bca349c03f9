"""The 4-bit cache at the edges of its range: values whose sums leave fp32, outputs with room between sequences, norms beyond fp32's
range, calls whose work is shared by places."""
import numpy as np
import numpy as np
import pytest
import torch

import paper_2506_07311_amd as pa
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
