"""README's example of a step of drafted tokens runs as written, after the one before it."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_readme_step_example_runs():
    text = open(os.path.join(ROOT, "README.md")).read()
    blocks = re.findall(r"```python\n(.*?)```", text, re.S)
    at = next(i for i, b in enumerate(blocks) if "paged_plan_step" in b)
    scope = {}
    for b in blocks[:at + 1]:
        exec(compile(b, "README.md", "exec"), scope)
    torch.cuda.synchronize()
    plan, n = scope["plan"], 13
    assert plan.shortage.tolist() == [0, 0] and plan.seq_lens.tolist() == [5, 8] and plan.cu_q_lens.tolist() == [0, 5, 13]
    assert plan.positions.tolist() == [0, 1, 2, 3, 4, 0, 1, 2, 3, 4, 5, 6, 7, -1, -1, -1]
    assert plan.rope_positions.tolist()[:n] == [0, 1, 1, 2, 2, 0, 1, 2, 3, 1, 2, 2, 1]
    assert bool(torch.isfinite(scope["out"][:n].float()).all()) and bool((scope["out"][:n] != 0).any(-1).all())
    kept = scope["path_lens"].tolist()
    assert scope["ctx_lens"].tolist() == kept and all(1 <= k <= 8 for k in kept)
    assert [r[0] for r in scope["path"].tolist()] == [0, 0]
    for s, (k, row) in enumerate(zip(kept, (0, 5))):                              # the path follows parents, tokens and targets
        path = scope["path"][s].tolist()
        for a, b in zip(path[:k], path[1:k]):
            assert int(scope["parents"][row + b]) == a and int(scope["tokens"][row + b]) == int(scope["targets"][row + a])
        assert int(scope["next_tokens"][s]) == int(scope["targets"][row + path[k - 1]]) and path[k:] == [-1] * (8 - k)
