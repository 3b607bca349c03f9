"""The 4-bit cache at the edges of its range: values whose sums leave fp32, outputs with room between sequences, norms beyond fp32's
range, calls whose work is shared by places."""
import numpy as np
import pytest
import torch

from tests.test_gpu_mx4 import Cache, attend

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
