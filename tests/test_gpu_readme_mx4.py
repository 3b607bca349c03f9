"""README's example of normalised heads and a cache of 4-bit elements runs as written, after those before it."""
import os
import re

import numpy as np
import pytest
import torch

from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_readme_mx4_example_runs():
    text = open(os.path.join(ROOT, "README.md")).read()
    blocks = re.findall(r"```python\n(.*?)```", text, re.S)
    at = next(i for i, b in enumerate(blocks) if "pa_mx4_cache" in b)
    scope = {}
    for b in blocks[:at + 1]:
        exec(compile(b, "README.md", "exec"), scope)
    torch.cuda.synchronize()
    n, out, q, P, d = scope["n"], scope["out"], scope["q"], scope["P"], scope["d"]
    assert P == scope["cache"].shape[2] and tuple(out.shape) == (n, scope["Hq"], d)
    cache = scope["cache"].flatten(2)[:-(-n // P)]
    k, v = (ref.values(*x).swapaxes(1, 2).reshape(-1, scope["Hkv"], d)[:n] for x in ref.unpacked(cache, P, d))
    np.testing.assert_array_equal(v, ref.values(*ref.quantised(scope["v_new"].double().cpu().numpy())))
    want, _, mass, _ = ref.attention(q.double().cpu().numpy(), k, v, 0, d ** -0.5)
    # half a step of bf16, and of weights and scores what test_gpu_mx4.py derives, amply
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * mass).all()
