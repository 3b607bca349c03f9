"""Calls given a stream that is not the current one, which allocate what they were not given: results and workspaces are that
stream's memory while the call is still to run, whatever the current stream allocates meanwhile."""
import pytest
import torch

from tests.test_gpu_step import DEV, ancestors, check_tree, ints, make_tree_call, pa, run_tree  # noqa: F401

pytestmark = pytest.mark.gpu


def overwrite(sizes, times=6):
    """New tensors of these sizes on the current stream, filled and dropped again."""
    for _ in range(times):
        keep = [torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) for n in sizes]
        del keep


@pytest.mark.parametrize("external", [False, True])
def test_a_step_on_another_stream_with_memory_of_its_own(pa, external):  # noqa: F811
    c = make_tree_call([3000, 90, 1200], [8, 3, 40], 8, 2, 128, 16, torch.bfloat16, ancestors(4), seed=5)
    rows, B = c["q"].shape[0], 3
    parents = ints([max(i - 2, -1) for n in c["news"] for i in range(n)])
    ctx, new = ints([a - b for a, b in zip(c["host_lens"], c["news"])]), ints(c["news"])
    tokens, targets = ints([i % 3 for i in range(rows)]), ints([(i + 1) % 3 for i in range(rows)])
    inv = torch.ones(64, dtype=torch.float64, device=DEV)
    blocks = [-(-n // 16) for n in c["host_lens"]]
    k_new, v_new = (torch.randn(rows, 2, 128, device=DEV).bfloat16() for _ in range(2))

    def step(stream):
        k, v = c["k"].clone(), c["v"].clone()
        path, lens = torch.empty(B, 40, dtype=torch.int32, device=DEV), ints([0] * B)
        num, free, count = ints(blocks), ints([0]), ints([0])
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)                     # (the calls wait while the current stream goes on)
        given = stream
        if stream is not None and external:
            class Handle:                                         # what another library calls a stream
                cuda_stream = stream.cuda_stream
            given = Handle()
        p = pa.paged_plan_step(ctx, new, c["table"], num, free, count, 16, rows, parents=parents, stream=given)
        q = pa.paged_rope_append(k, v, c["q"], k_new, v_new, p.rope_positions, p.seq_ids, p.positions, c["table"], inv, stream=given)
        out = pa.paged_attention_tree(k, v, q, p.cu_q_lens, 40, p.tree_mask, c["table"], p.seq_lens, 3000, c["scale"], stream=given)
        _, _, nxt, kept = pa.paged_tree_accept(k, v, p.cu_q_lens, p.seq_lens, 40, c["table"], path, lens, parents=parents,
                                               tokens=tokens, targets=targets, stream=given)
        if stream is not None:
            ws = pa.paged_attention_tree_workspace_bytes(B, 8, 2, 128, rows, 40, 3000)
            overwrite([ws, out.numel() * 2, out.numel() * 2, rows * 8, rows * 4, 512, 512, 512])
            torch.cuda.current_stream().wait_stream(stream)
        return [x.clone() for x in (*p, q, out, nxt, kept, k, v, path, lens)]

    want = step(None)
    got = step(torch.cuda.Stream())
    for a, b in zip(want, got):
        assert torch.equal(a, b) or bool((a.isnan() == b.isnan()).all()) and torch.equal(a.nan_to_num(), b.nan_to_num())


def test_attention_on_another_stream_with_memory_of_its_own(pa):  # noqa: F811
    c = make_tree_call([5000, 90], [8, 3], 8, 2, 128, 16, torch.bfloat16, ancestors(4), seed=5)
    args = (c["k"], c["v"], c["q"], c["cu"], 8, c["mask"], c["table"], c["lens"], 5000, c["scale"])
    d_args = (c["k"], c["v"], c["q"][:2].contiguous(), c["table"], c["lens"], 5000, c["scale"])
    p_args = (c["k"], c["v"], c["q"], c["cu"], 8, c["table"], c["lens"], 5000, c["scale"], True)
    for fn, a, nbytes in ((pa.paged_attention_tree, args, pa.paged_attention_tree_workspace_bytes(2, 8, 2, 128, 11, 8, 5000)),
                          (pa.paged_attention_decode, d_args, pa.paged_attention_workspace_bytes(2, 8, 128, 2, 5000)),
                          (pa.paged_attention_prefill, p_args, pa.paged_attention_workspace_bytes(2, 8, 128, 11, 5000))):
        want = fn(*a).clone()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = fn(*a, stream=side)
        overwrite([nbytes, want.numel() * 2])
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
    check_tree(c, *run_tree(pa, c))


def test_a_captured_call_on_a_forked_stream_with_memory_of_its_own(pa):  # noqa: F811
    """A stream that joins a capture: what its call allocates lives in the graph, whose replays with the program's own work
    between repeat the eager result."""
    c = make_tree_call([3000, 90], [8, 3], 8, 2, 128, 16, torch.bfloat16, ancestors(4), seed=5)
    args = (c["k"], c["v"], c["q"], c["cu"], 8, c["mask"], c["table"], c["lens"], 3000, c["scale"])
    side = torch.cuda.Stream()
    pa.paged_attention_tree(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = pa.paged_attention_tree(*args, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for turn in range(4):
        c["q"].copy_(c["q"].roll(1, 0))
        graph.replay()
        overwrite([out.numel() * 2, 1 << 20], 2)
        if turn % 2:
            torch.cuda.synchronize()
        assert torch.equal(out, pa.paged_attention_tree(*args))
