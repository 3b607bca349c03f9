"""A step's plan and release at their limits."""
import numpy as np
import pytest
import torch

from tests import step_reference as R
from tests.test_gpu_step import DEV, ancestors, bits, check_tree, ints, make_tree_call, pa  # noqa: F401

pytestmark = pytest.mark.gpu


def guarded(shape, dtype=torch.int32, guard=4096):
    """A tensor in the middle of a buffer of -77, and the two ends of that buffer."""
    n = int(np.prod(shape))
    buf = torch.full((n + 2 * guard,), -77, dtype=dtype, device=DEV)
    return buf[guard:guard + n].view(shape), (buf[:guard], buf[guard + n:])


@pytest.mark.parametrize("how", ["tree", None])
@pytest.mark.parametrize("ctx,new,rows", [
    ([0, 0, 0], [1 << 30, 1 << 30, 5], 20),                       # a sum of 2^31 + 5
    ([9, 0, 7, 1], [2 ** 31 - 10, 2 ** 31 - 1, 2 ** 31 - 8, 9], 150),   # each length within 31 bits, three times the sum over
    ([5, 6, 7, 8, 9], [3, 1 << 30, 2 ** 31 - 8, 2 ** 31 - 9, 4], 10),
    ([1] * 1500, [1 << 30] * 1500, 70),                           # 2^40
    ([3] * 300, [2] * 299 + [2 ** 31 - 4], 700),
])
def test_plans_whose_rows_pass_31_bits(pa, ctx, new, rows, how):  # noqa: F811
    """Refused on the device, with the state as it was, the rows that there are described and nothing written beyond them."""
    B, MB, P, words = len(ctx), 4, 16, 3
    table, num = torch.full((B, MB), -1, dtype=torch.int32, device=DEV), ints([0] * B)
    free, count = ints(range(8)), ints([8])
    outs, guards = {}, []
    for name, shape, dtype in (("seq_lens", (B,), torch.int32), ("cu_q_lens", (B + 1,), torch.int32), ("seq_ids", (rows,), torch.int32),
                               ("positions", (rows,), torch.int32), ("rope_positions", (rows,), torch.int32),
                               ("tree_mask", (rows, words), torch.int64), ("shortage", (2,), torch.int32)):
        outs[name], ends = guarded(shape, dtype)
        guards += ends
    parents = None if how is None else ints([max(i - 2, 0) for i in range(rows)])
    p = pa.paged_plan_step(ints(ctx), ints(new), table, num, free, count, P, rows, parents=parents, **outs)
    late = sum(-(-(c + n) // P) > MB or n > 64 * words for c, n in zip(ctx, new)) + sum(new) - rows
    need = sum(-(-(c + n) // P) for c, n in zip(ctx, new)) - 8
    assert p.shortage.tolist() == [min(need, 2 ** 31 - 1), min(late, 2 ** 31 - 1)]
    assert p.seq_lens.tolist() == ctx and p.cu_q_lens.tolist() == [0] * (B + 1)
    assert int(count) == 8 and num.tolist() == [0] * B and bool((table == -1).all())
    row, at = 0, dict(seq_ids=[], positions=[], rope_positions=[], tree_mask=[])
    for s, (c, n) in enumerate(zip(ctx, new)):
        masks, depths = [], []
        for i in range(min(n, rows - row)):
            up = i - 1 if how is None else max(row + i - 2, 0)
            up = up if 0 <= up < i else -1
            masks.append((masks[up] if up >= 0 else 0) | 1 << i)
            depths.append(depths[up] + 1 if up >= 0 else 0)
            at["seq_ids"].append(s), at["positions"].append(c + i), at["rope_positions"].append(c + depths[-1])
            at["tree_mask"].append([masks[-1] >> 64 * w & (1 << 64) - 1 for w in range(words)])
        row += len(masks)
    # (positions past 31 bits are negative)
    for name in ("seq_ids", "positions", "rope_positions"):
        assert getattr(p, name).tolist() == [x if x < 2 ** 31 else x - 2 ** 32 for x in at[name]] + [-1 if name != "rope_positions" else 0] * (rows - row)
    assert torch.equal(p.tree_mask, bits(np.array(at["tree_mask"] + [[0] * words] * (rows - row), dtype=np.uint64)))
    for g in guards:
        assert bool((g == -77).all())


@pytest.mark.parametrize("B,P,room", [(3, 16, 0), (3, 16, 4), (5, 1, 37), (40, 8, 11), (2500, 16, 700), (2500, 16, 0), (2500, 16, 10 ** 6)])
def test_pages_that_the_free_list_has_no_room_for_stay_mapped(pa, B, P, room):  # noqa: F811
    """`room` places are left: the last blocks get them, the first ones stay in their rows, and no page is lost.  A later call
    with room takes them."""
    rng = np.random.default_rng(B + room)
    MB = 9
    have, keep = rng.integers(0, MB + 1, B), rng.integers(0, (MB + 2) * P, B)
    table = np.full((B, MB), -1)
    perm = rng.permutation(int(have.sum()) + 5)
    live, perm = perm[:5].tolist(), perm[5:]
    at = 0
    for s in range(B):
        table[s, :have[s]] = perm[at:at + have[s]]
        at += have[s]
    back = [(s, b) for s in range(B) for b in range(-(-int(keep[s]) // P), int(have[s]))]
    room = min(room, len(back) + 2)
    stay = max(len(back) - room, 0)
    want_free = live + [int(table[s, b]) for s, b in back[stay:]][::-1]
    want_table, want_num = table.copy(), have.copy()
    for s, b in back[stay:]:
        want_table[s, b] = -1
        want_num[s] -= 1
    t_table, t_num, t_count, t_keep = ints(table), ints(have), ints([5]), ints(keep)
    t_free, ends = guarded((5 + room,))
    t_free[:5] = ints(live)
    pa.paged_release_blocks(t_keep, t_table, t_num, t_free, t_count, P)
    assert t_table.tolist() == want_table.tolist() and t_num.tolist() == want_num.tolist()
    assert int(t_count) == len(want_free) and t_free.tolist()[:len(want_free)] == want_free
    assert all(bool((g == -77).all()) for g in ends)
    wide = torch.cat([t_free, ints([0] * len(back))]) if len(back) else t_free
    pa.paged_release_blocks(t_keep, t_table, t_num, wide, t_count, P)
    assert t_num.tolist() == np.minimum(have, -(-keep // P)).tolist()
    assert sorted(wide.tolist()[:int(t_count)] + t_table[t_table >= 0].tolist()) == sorted(live + perm.tolist())


@pytest.mark.parametrize("dtype,d,max_q", [(torch.bfloat16, 128, 1 << 17), (torch.float32, 256, 1 << 15)])
def test_bounds_however_loose_are_taken(pa, dtype, d, max_q):  # noqa: F811
    """Bounds of millions of tokens on contexts of thousands: on the matrix cores while places and threads fit their counts, else on the
    portable kernel; the call is not refused."""
    from paper_2506_07311_amd import binding
    P, B = 1024, 4
    c = make_tree_call([3000, 40, 5, 1200], [6, 3, 5, 1], 8, 1, d, P, dtype, ancestors(3), seed=4, pad=2)
    for bound, kernel in ((1 << 21, "paged_attention_tree_mfma_kernel"), (1 << 22, "paged_attention_tree_%s_kernel" % ("mfma" if d == 128 else "generic")),
                          (1 << 25, "paged_attention_tree_generic_kernel")):
        table = torch.full((B, bound // P), -1, dtype=torch.int32, device=DEV)
        table[:, :c["table"].shape[1]] = c["table"]
        mask = torch.zeros((c["q"].shape[0], max_q // 64), dtype=torch.int64, device=DEV)
        mask[:, :1] = c["mask"]
        ws, ends = guarded((pa.paged_attention_tree_workspace_bytes(B, 8, 1, d, c["q"].shape[0], max_q, bound),), torch.int8)
        out, lse = torch.full_like(c["q"], 9.0), torch.full(c["q"].shape[:2], 7.0, device=DEV)
        binding.pa_profile_reset()
        binding.pa_profile_enable(True)
        try:
            pa.paged_attention_tree(c["k"], c["v"], c["q"], c["cu"], max_q, mask, table, c["lens"], bound, c["scale"], out=out, lse=lse,
                                    workspace=ws)
            assert binding.pa_profile_read(kernel)[0] == 1
        finally:
            binding.pa_profile_enable(False)
            binding.pa_profile_reset()
        check_tree(c, out, lse, f"{bound}")
        assert all(bool((g == -77).all()) for g in ends)


@pytest.mark.parametrize("parents", [False, True])
def test_a_plan_without_masks(pa, parents):  # noqa: F811
    """A prompt's tokens are more than a word of mask has bits; a program that attends causally asks for no masks."""
    ctx, new, P, rows = [100, 0, 5], [700, 1, 65], 16, 800
    table = torch.full((3, 60), -1, dtype=torch.int32, device=DEV)
    up = None if not parents else [max(i - 2, -1) for n in new for i in range(n)] + [-1] * (rows - sum(new))
    ref = R.plan(ctx, new, up, table.cpu().numpy(), [0] * 3, list(range(90)), P, rows, 64)
    p = pa.paged_plan_step(ints(ctx), ints(new), table, ints([0] * 3), ints(range(90)), ints([90]), P, rows,
                           parents=None if up is None else ints(up), mask_words=0)
    assert p.tree_mask is None and p.shortage.tolist() == [0, 0]
    for name in ("seq_lens", "cu_q_lens", "seq_ids", "positions", "rope_positions"):
        assert getattr(p, name).tolist() == list(ref[name]), name
    assert table.tolist() == ref["block_table"].tolist()


@pytest.mark.parametrize("B", [1025, 2500])
@pytest.mark.parametrize("short", [0, 1])
@pytest.mark.parametrize("how", ["tree", None])
def test_plans_and_releases_of_thousands_of_sequences(pa, B, short, how):  # noqa: F811
    """More sequences than the workgroup that counts has threads: rows, pages and what returns carry over from one block of them to
    the next, growth and release in each; once granted, once a page short."""
    rng = np.random.default_rng(B)
    P, words, pad = 16, 1, 9
    ctx, new = rng.integers(0, 60, B).tolist(), rng.integers(0, 20, B).tolist()
    before = [R.blocks(x, P) for x in ctx]
    MB = 6
    grow = sum(R.blocks(x + n, P) - k for x, n, k in zip(ctx, new, before))
    perm = rng.permutation(sum(before) + grow - short + 2 * (1 - short))
    table, at = np.full((B, MB), -1, np.int64), 0
    for s in range(B):
        table[s, :before[s]] = perm[at:at + before[s]]
        at += before[s]
    free, rows = perm[at:].tolist(), sum(new) + pad
    up = None if how is None else [max(0, i - int(rng.integers(1, 4))) if i else -1 for n in new for i in range(n)] + [-1] * pad
    ref = R.plan(ctx, new, up, table, before, free, P, rows, words)
    assert ref["shortage"] == [short, 0]
    t_table, t_num, t_free, t_count = ints(table), ints(before), ints(free + [-7] * (len(perm) - len(free))), ints([len(free)])
    p = pa.paged_plan_step(ints(ctx), ints(new), t_table, t_num, t_free, t_count, P, rows, parents=None if up is None else ints(up))
    for name in ("seq_lens", "cu_q_lens", "seq_ids", "positions", "rope_positions", "shortage"):
        assert getattr(p, name).tolist() == list(ref[name]), name
    assert torch.equal(p.tree_mask, bits(np.array(ref["tree_mask"], dtype=np.uint64).reshape(rows, words)))
    assert t_table.tolist() == ref["block_table"].tolist() and t_num.tolist() == ref["num_blocks"]
    assert t_free.tolist()[:int(t_count)] == ref["free"] and int(t_count) == len(ref["free"])
    for keep in (rng.integers(0, 60, B).tolist(), [0] * B):
        back = R.release(keep, t_table.cpu().numpy(), t_num.tolist(), t_free.tolist()[:int(t_count)], P)
        pa.paged_release_blocks(ints(keep), t_table, t_num, t_free, t_count, P)
        assert t_table.tolist() == back["block_table"].tolist() and t_num.tolist() == back["num_blocks"]
        assert t_free.tolist()[:int(t_count)] == [int(x) for x in back["free"]]
    assert sorted(t_free.tolist()[:int(t_count)]) == sorted(perm.tolist())
