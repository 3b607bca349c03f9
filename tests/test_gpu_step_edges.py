"""A step of drafted tokens where it is used otherwise than usual: scales of any sign, the portable kernel, pools whose offsets
pass 32 bits, many sequences, loose bounds, other streams, captured graphs that share a workspace, values that are not finite."""
import numpy as np
import pytest
import torch

from tests import step_reference as R
from tests.test_gpu_step import DEV, ancestors, any_mask, bits, check_tree, half_step, ints, make_tree_call, pa, run_tree  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
@pytest.mark.parametrize("hq,d,dtype,n", [(4, 64, torch.bfloat16, 5), (16, 128, torch.float16, 20), (16, 128, torch.float32, 20)])
def test_scales_of_any_sign(pa, hq, d, dtype, n, scale):  # noqa: F811
    """Scores change sign with the scale; of 0, every weight is one; of 3, next to all of a row's weight lies on one key:
    scores then are sums of 128 products of up to 180 in 32 bits, 128 independent roundings of deviation 180 * 2^-24 / sqrt(3); six
    deviations of their sum are 4.2e-4, of the score and so of the weight's logarithm."""
    c = make_tree_call([n, 700, 1100], [n, 3, n], hq, 2, d, 16, dtype, any_mask(3), seed=4)
    c["scale"] = scale
    out, lse = run_tree(pa, c)
    if scale == 3.0:
        row, extra = 0, 3e-5 + 4.2e-4
        for s, m in enumerate(c["news"]):
            k, v = (x.double().numpy() for x in c["seqs"][s])
            q = c["q"][row:row + m].double().cpu().numpy()
            ref, ref_lse, wide = R.tree_attention(k, v, q, c["masks"][s], c["host_lens"][s] - m, scale, spread=True)
            near = half_step(dtype) * (np.abs(ref) + 6 / 3 ** 0.5 * wide) + extra * np.abs(v).max()
            assert (np.abs(out[row:row + m].double().cpu().numpy() - ref) <= near).all(), s
            seen = np.isfinite(ref_lse)
            got = lse[row:row + m].double().cpu().numpy()
            assert (np.abs(got[seen] - ref_lse[seen]) <= 4.2e-4 + 2e-6 * np.abs(ref_lse[seen])).all() and (got[~seen] == -np.inf).all()
            row += m
    else:
        check_tree(c, out, lse, f"{scale}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 80])
def test_the_portable_kernel_takes_the_same_calls(pa, d, dtype):  # noqa: F811
    from paper_2506_07311_amd import binding
    c = make_tree_call([5, 64, 300, 0, 65], [5, 1, 33, 0, 65], 8, 2, d, 16, dtype, any_mask(5), seed=9, pad=1)
    binding.pa_set_option("force_generic", 1)
    try:
        out, lse = run_tree(pa, c)
    finally:
        binding.pa_set_option("force_generic", 0)
    check_tree(c, out, lse, f"{d}")


@pytest.mark.parametrize("dtype,d,hq,hkv", [(torch.bfloat16, 128, 8, 2), (torch.float32, 64, 4, 4)])
def test_many_sequences(pa, dtype, d, hq, hkv):  # noqa: F811
    """More sequences than a wave has lanes, in order and out of it, some without tokens; once short, once cut over workgroups."""
    rng = np.random.default_rng(14)
    for most in (90, 1500):
        news = [int(x) for x in rng.integers(0, 9, 150)]
        lens = [n + int(rng.integers(0, most)) if n else int(rng.integers(0, 40)) for n in news]
        c = make_tree_call(lens, news, hq, hkv, d, 16, dtype, ancestors(7), seed=2)
        out, lse = run_tree(pa, c)
        check_tree(c, out, lse, f"{most}")


def test_a_full_machine_of_short_contexts(pa):  # noqa: F811
    """So many row blocks that each is one workgroup's, up to 1024 keys."""
    rng = np.random.default_rng(15)
    news = [int(x) for x in rng.integers(1, 3, 70)]
    lens = [n + int(rng.integers(0, 1000)) for n in news]
    lens[3] = 1024
    c = make_tree_call(lens, news, 8, 8, 64, 16, torch.bfloat16, ancestors(7), seed=2)
    out, lse = run_tree(pa, c)
    check_tree(c, out, lse)


@pytest.mark.parametrize("how", ["chain", "tree", None])
def test_plans_of_long_sequences(pa, how):  # noqa: F811
    """Thousands of new tokens in a sequence, whose chains of parents run through all of them."""
    new, rng = [2500, 70, 1], np.random.default_rng(4)
    if how is None:
        parents = None
    else:
        parents = [i - 1 if how == "chain" else int(rng.integers(max(0, i - 200), i)) if i else -1 for n in new for i in range(n)]
    rows, words, ctx = sum(new), 40, [100, 0, 7]
    table = torch.full((3, 200), -1, dtype=torch.int32, device=DEV)
    p = pa.paged_plan_step(ints(ctx), ints(new), table, ints([0] * 3), ints(range(400)), ints([400]), 16, rows, mask_words=words,
                           parents=None if parents is None else ints(parents))
    ref = R.plan(ctx, new, parents, table.cpu().numpy() * 0 - 1, [0] * 3, list(range(400)), 16, rows, words)
    assert p.shortage.tolist() == [0, 0] and p.rope_positions.tolist() == list(ref["rope_positions"])
    assert torch.equal(p.tree_mask, bits(np.array(ref["tree_mask"], dtype=np.uint64).reshape(rows, words)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_chunk_of_many_tokens(pa, dtype):  # noqa: F811
    """As many rows as a chunk of a prompt brings, each with a mask of its own."""
    c = make_tree_call([650, 90, 300], [400, 3, 300], 4, 2, 64, 16, dtype, any_mask(3), seed=4)
    out, lse = run_tree(pa, c)
    check_tree(c, out, lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_bounds_may_be_loose(pa, dtype):  # noqa: F811
    """max_q_len, the masks' words and the rows of q beyond what the sequences bring, as a captured step has them."""
    c = make_tree_call([2000, 7, 90], [3, 7, 1], 8, 2, 64, 16, dtype, ancestors(4), seed=5, pad=50)
    mask = torch.full((c["q"].shape[0], 3), -1, dtype=torch.int64, device=DEV)
    mask[:, 0] = c["mask"][:, 0]
    c["table"] = torch.cat([c["table"], torch.full((3, 9), -1, dtype=torch.int32, device=DEV)], 1)
    for max_q, longest in ((7, 2000), (150, 2000), (150, 2048)):
        ws = pa.paged_attention_tree_workspace_bytes(3, 8, 2, 64, c["q"].shape[0], max_q, longest)
        ws = torch.full((ws,), 0xFF, dtype=torch.uint8, device=DEV)
        out, lse = torch.full_like(c["q"], 9.0), torch.full(c["q"].shape[:2], 7.0, device=DEV)
        pa.paged_attention_tree(c["k"], c["v"], c["q"], c["cu"], max_q, mask, c["table"], c["lens"], longest, c["scale"], out=out,
                                lse=lse, workspace=ws)
        # (with bounds of 600 rows and of contexts over 255 the weights are of 16 bits: check_tree's allowance goes by the bound)
        if max_q == 7 or dtype == torch.float32:
            check_tree(c, out, lse, f"{max_q}")
        else:
            check_one_term(c, out)


def check_one_term(c, out):
    """check_tree's bound for weights of 16 bits, whatever the call's number of rows."""
    row = 0
    for s, n in enumerate(c["news"]):
        k, v = (x.double().numpy() for x in c["seqs"][s])
        ref, _, wide = R.tree_attention(k, v, c["q"][row:row + n].double().cpu().numpy(), c["masks"][s], c["host_lens"][s] - n, c["scale"],
                                        spread=True)
        near = half_step(c["q"].dtype) * (np.abs(ref) + 6 / 3 ** 0.5 * wide) + 3e-5 * np.abs(v).max()
        assert (np.abs(out[row:row + n].double().cpu().numpy() - ref) <= near).all(), s
        row += n
    assert bool((out[row:] == 9.0).all())


def test_a_bound_that_is_too_small_leaves_rows(pa):  # noqa: F811
    """A sequence with more tokens than max_q_len says: nothing outside its rows is written, and what is covered is right."""
    c = make_tree_call([2000, 2040], [40, 40], 8, 2, 64, 16, torch.bfloat16, ancestors(4), seed=5, pad=3)
    ws = pa.paged_attention_tree_workspace_bytes(2, 8, 2, 64, 83, 9, 2048)
    ws = torch.full((ws + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full_like(c["q"], 9.0)
    c["table"] = torch.cat([c["table"], torch.full_like(c["table"], -1)], 1)
    pa.paged_attention_tree(c["k"], c["v"], c["q"], c["cu"], 9, c["mask"], c["table"], c["lens"], 2048, c["scale"], out=out,
                            workspace=ws[:-4096])
    assert bool((ws[-4096:] == 0xFF).all()) and bool((out[80:] == 9.0).all())
    full, _ = run_tree(pa, c)
    # (two roundings of the output, half a step of up to its largest each, and the wider call's weights of 16 bits)
    assert float((out[:9].float() - full[:9].float()).abs().max()) <= 2.0 ** -6 * float(full.abs().max())


@pytest.mark.parametrize("dtype,n,heads", [(torch.bfloat16, 4, (16, 16)), (torch.bfloat16, 40, (32, 8)), (torch.float32, 4, (8, 8))])
@pytest.mark.parametrize("head_major", [False, True])
def test_pools_whose_offsets_pass_32_bits(pa, dtype, n, heads, head_major):  # noqa: F811
    """Pages at both ends of a pool of over 2^32 elements: appending, attention and acceptance do what they do in a small pool, bit
    for bit.  Head-major: pages so long that a head's offset in one passes 32 bits, too."""
    hq, hkv, d = heads[0], heads[1], 128
    P = 1 << 21 if head_major else 16
    NP = (1 << 32) // (P * hkv * d) + 1 if head_major else (1 << 32) // (P * hkv * d) + 40
    ctx, B = 150, 2
    blocks = R.blocks(ctx + n, P)
    rng = np.random.default_rng(3)
    far = [NP - 1, 0] if head_major else rng.choice(np.concatenate([np.arange(20), np.arange(NP - 30, NP)]), B * blocks, replace=False)
    big_table = np.full((B, blocks + 1), -1)
    big_table[:, :blocks] = np.reshape(far, (B, blocks))
    small_P = 16
    small_blocks = R.blocks(ctx + n, small_P)
    small_table = np.arange(B * small_blocks).reshape(B, small_blocks)
    shape = (NP, hkv, P, d) if head_major else (NP, P, hkv, d)
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = B * (ctx + n)
    k_new, v_new, q = (torch.randn(rows, h, d, generator=g, device=DEV).to(dtype) for h in (hkv, hkv, hq))
    inv = torch.from_numpy(10000.0 ** (-np.arange(d // 2) * 2.0 / d)).to(DEV)
    seq_ids, positions = ints(np.repeat(np.arange(B), ctx + n)), ints(np.tile(np.arange(ctx + n), B))
    qs = torch.stack([q[b * (ctx + n) + ctx:(b + 1) * (ctx + n)] for b in range(B)]).view(B * n, hq, d)
    mask = bits([[(1 << (i + 1)) - 1] for i in range(n)] * B)
    cu, lens = ints([0, n, 2 * n]), ints([ctx + n] * B)
    path = ints([[0, 2, 3] + [-1] * (n - 3)] * B)
    results = []
    for table, make, major, page in ((big_table, lambda: torch.empty(shape, dtype=dtype, device=DEV), head_major, P),
                                     (small_table, lambda: torch.zeros(B * small_blocks, small_P, hkv, d, dtype=dtype, device=DEV), False, small_P)):
        k, v, table = make(), make(), ints(table)
        turned = pa.paged_rope_append(k, v, q, k_new, v_new, positions, seq_ids, positions, table, inv, head_major=major)
        ws = torch.empty(pa.paged_attention_tree_workspace_bytes(B, hq, hkv, d, B * n, n, 1100), dtype=torch.uint8, device=DEV)
        wide = torch.cat([table, torch.full((B, 80), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
        out = pa.paged_attention_tree(k, v, qs, cu, n, mask, wide, lens, 1100, d ** -0.5, workspace=ws, head_major=major)
        pa.paged_tree_accept(k, v, cu, lens, n, table, path, ints([3, 3]), head_major=major)
        at = table.long().cpu()
        held = []
        for pool in (k, v):
            for b in range(B):
                t = torch.arange(ctx + n)
                pages, places = at[b, t // page].to(DEV), (t % page).to(DEV)
                held.append(torch.stack([pool[p, :, x] if major else pool[p, x] for p, x in zip(pages.tolist(), places.tolist())]).clone())
        results.append([turned.clone(), out.clone()] + held)
        del k, v
        torch.cuda.empty_cache()
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_rows_that_share_memory_are_refused(pa):  # noqa: F811
    """One token's row for all of them (a stride of 0) is not taken for a contiguous tensor, nor are rows that overlap."""
    k, v = (torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    at, inv = ints([0, 1, 2]), torch.ones(32, dtype=torch.float64, device=DEV)
    good = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    same = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device=DEV).expand(3, 2, 64)
    over = torch.zeros(400, dtype=torch.bfloat16, device=DEV).as_strided((3, 2, 64), (64, 64, 1))
    table = ints([[0, 1]])
    for bad in (same, over):
        for q, kn, vn, out in ((bad, good, good, None), (good, bad, good, None), (good, good, bad, None), (good, good, good, bad)):
            with pytest.raises(pa.PagedAttnError):
                pa.paged_rope_append(k, v, q, kn, vn, at, ints([0, 0, 0]), at, table, inv, q_out=out)
    pa.paged_rope_append(k, v, good, good, good, at, ints([0, 0, 0]), at, table, inv)


def test_another_stream_and_prepared_calls(pa):  # noqa: F811
    """Calls run on the stream that they are given or that is current, in its order, and take what their tensors hold then."""
    c = make_tree_call([1500, 90], [8, 3], 8, 2, 128, 16, torch.bfloat16, ancestors(4), seed=5)
    side = torch.cuda.Stream()
    spaces = [torch.empty(pa.paged_attention_tree_workspace_bytes(2, 8, 2, 128, 11, 8, 1500), dtype=torch.uint8, device=DEV)
              for _ in range(2)]
    outs = [torch.zeros_like(c["q"]) for _ in range(3)]
    q2 = c["q"].clone()
    args = (c["cu"], 8, c["mask"], c["table"], c["lens"], 1500, c["scale"])
    here = pa.prepare_attention_tree(c["k"], c["v"], c["q"], *args, out=outs[0], workspace=spaces[0])
    there = pa.prepare_attention_tree(c["k"], c["v"], q2, *args, out=outs[1], workspace=spaces[1], stream=side)
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):                                            # two calls at a time
        here()
        with torch.cuda.stream(side):
            q2.copy_(c["q"]).mul_(2.0)                            # (in the stream's order before the call)
        there()
    with torch.cuda.stream(side):
        pa.paged_attention_tree(c["k"], c["v"], q2, *args, out=outs[2], workspace=spaces[1])
    torch.cuda.current_stream().wait_stream(side)
    lse = run_tree(pa, c)[1]
    check_tree(c, outs[0], lse)
    assert torch.equal(outs[1], outs[2])
    c["scale"] *= 2.0
    check_tree(c, outs[1], run_tree(pa, c)[1])


def test_two_graphs_that_share_a_workspace(pa):  # noqa: F811
    """Captured calls of two shapes in one workspace, replayed in turn with eager calls between, on new values each time."""
    calls, ws = [], 0
    for seed, (lens, news, hq, hkv, d) in enumerate([([3000, 500], [8, 8], 8, 2, 128), ([1200] * 3, [40, 2, 9], 16, 4, 64)]):
        c = make_tree_call(lens, news, hq, hkv, d, 16, torch.bfloat16, any_mask(seed), seed=seed)
        ws = max(ws, pa.paged_attention_tree_workspace_bytes(len(lens), hq, hkv, d, sum(news), max(news), max(lens)))
        calls.append(c)
    ws = torch.full((ws,), 0xFF, dtype=torch.uint8, device=DEV)
    graphs = []
    for c in calls:
        out, lse = torch.zeros_like(c["q"]), torch.zeros(c["q"].shape[:2], device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pa.paged_attention_tree(c["k"], c["v"], c["q"], c["cu"], max(c["news"]), c["mask"], c["table"], c["lens"],
                                    max(c["host_lens"]), c["scale"], out=out, lse=lse, workspace=ws)
        graphs.append((graph, out, lse))
    for turn in range(4):
        for c in calls:
            c["q"].copy_(c["q"].roll(1, 0))
        for i in (0, 1, 1, 0):
            graph, out, lse = graphs[i]
            out.zero_(), lse.zero_()
            graph.replay()
            if turn % 2:
                torch.cuda.synchronize()
            got = out.clone(), lse.clone()
            want = run_tree(pa, calls[i])
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (turn, i)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float16, 64), (torch.bfloat16, 256), (torch.float32, 128)])
def test_values_that_are_not_finite_in_long_contexts(pa, dtype, d):  # noqa: F811
    """As with short ones: where a call is cut over workgroups and takes many rows, a NaN or an infinity in a drafted token's V row
    reaches its column of the queries that see the token, in the context all queries', and nothing else."""
    n, ctx, hq, hkv = 40, 2500, 8, 2
    for at, bad in ((7, float("nan")), (7, float("inf")), (-1300, -float("inf"))):
        c = make_tree_call([ctx + n, 1100], [n, 2], hq, hkv, d, 16, dtype, ancestors(9), seed=6)
        page, place = int(c["table"][0, (ctx + at) // 16]), (ctx + at) % 16
        c["v"][page, place, :, 3] = bad
        out, _ = run_tree(pa, c)
        sees = torch.from_numpy(c["masks"][0][:, at] if at >= 0 else np.ones(n, bool)).to(DEV)
        col = out[:n, :, 3].float()
        assert bool((col[sees].isnan() if bad != bad else col[sees] == bad).all())
        assert bool(col[~sees].isfinite().all()) and int(sees.sum()) > 0
        clean = out.clone()
        clean[:n, :, 3] = 0
        assert bool(clean.isfinite().all())
        row = 0
        for s, m in enumerate(c["news"]):
            k, v = (x.double().numpy() for x in c["seqs"][s])
            ref, _, wide = R.tree_attention(k, v, c["q"][row:row + m].double().cpu().numpy(), c["masks"][s], c["host_lens"][s] - m, c["scale"],
                                            spread=True)
            near = half_step(dtype) * (np.abs(ref) + 6 / 3 ** 0.5 * wide) + 3e-5 * np.abs(v).max()
            over = np.abs(out[row:row + m].double().cpu().numpy() - ref) - near
            if s == 0:
                over[:, :, 3][sees.cpu().numpy()] = 0
            assert (over <= 0).all(), (s, at, bad)
            row += m


def test_scores_of_the_lowest_value(pa):  # noqa: F811
    """A K row of the type's lowest values, whose scores overflow 32 bits to -inf: the key weighs nothing."""
    c = make_tree_call([300], [4], 4, 2, 64, 16, torch.bfloat16, lambda s, n: np.tril(np.ones((n, n))), seed=6)
    page, place = int(c["table"][0, 100 // 16]), 100 % 16
    c["k"][page, place] = torch.finfo(torch.bfloat16).min
    c["q"].copy_(c["q"].abs())                                    # (every score of that key is hugely negative)
    sk, sv = c["seqs"][0]
    keep = torch.arange(300) != 100
    c["seqs"] = [(sk[keep], sv[keep])]
    out, lse = run_tree(pa, c)
    check_tree(dict(c, host_lens=[299]), out, lse)


def test_plans_that_ask_for_the_impossible(pa):  # noqa: F811
    """Lengths whose sum passes 31 bits, and a request of all rows at once: refused on the device, state as it was."""
    P, B = 16, 3
    for ctx, new, MB in (([2 ** 31 - 5, 0, 3], [64, 1, 1], 8), ([0, 0, 0], [5, 5, 5], 2)):
        rows = 14
        table = torch.full((B, MB), -1, dtype=torch.int32, device=DEV)
        num, free, count = ints([0] * B), ints(range(8)), ints([8])
        p = pa.paged_plan_step(ints(ctx), ints(new), table, num, free, count, P, rows, parents=ints([-1] * rows))
        assert p.shortage.tolist()[1] > 0 and p.seq_lens.tolist() == ctx and p.cu_q_lens.tolist() == [0] * (B + 1)
        assert int(count) == 8 and num.tolist() == [0] * B and bool((table == -1).all())
