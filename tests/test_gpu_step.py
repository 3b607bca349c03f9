"""A step of drafted tokens on the GPU against its definitions in 64 bits: plan and release of pages, rotary append, attention of
trees, acceptance, and all of them in a row."""
import numpy as np
import pytest
import torch

from tests import step_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pa():
    import paper_2506_07311_amd as pa_mod
    pa_mod.load_library()
    return pa_mod


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int64).tolist(), dtype=torch.int32, device=DEV)


def bits(masks):
    """[rows, words] Python integers of 64 bits -> int64."""
    return torch.from_numpy(np.array(masks, dtype=np.uint64).view(np.int64)).to(DEV)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- plan and release ----------------------------------------------------------------------------------------------

def random_parents(rng, new, wild):
    out = []
    for n in new:
        for i in range(n):
            out.append(int(rng.integers(-2, i + 3)) if wild else int(rng.integers(max(0, i - 5), i)) if i else -1)
    return out


PLAN_CASES = [  # ctx, new, page, parents (None, "tree", "wild"), spare rows, words, pages short, table columns to spare
    ([0], [1], 16, "tree", 0, 1, 0, 0),
    ([0], [0], 16, None, 3, 1, 0, 1),
    ([5, 0, 31, 16], [3, 0, 1, 64], 16, "tree", 0, 1, 0, 2),
    ([5, 0, 31, 16], [3, 0, 1, 64], 16, "wild", 5, 2, 0, 0),
    ([100, 7, 0], [65, 128, 200], 8, "tree", 0, 4, 0, 0),
    ([100, 7, 0], [65, 128, 200], 1, "wild", 1, 5, 0, 0),
    ([100, 7, 0], [65, 128, 200], 32, None, 0, 4, 0, 3),
    ([100, 7, 0], [65, 128, 200], 32, "tree", 0, 4, 1, 3),        # one page short
    ([100, 7, 0], [65, 128, 200], 32, "tree", 0, 3, 0, 3),        # a tree wider than the masks
    ([100, 7, 0], [65, 128, 200], 32, "tree", -1, 4, 0, 3),       # a row short
    ([100, 7, 0], [65, 128, 200], 32, "tree", 0, 4, 0, -1),       # a block too few in the table
    ("many", 3, 16, "tree", 7, 1, 0, 0),
    ("many", 700, 128, "tree", 0, 11, 0, 0),
]


@pytest.mark.parametrize("case", PLAN_CASES, ids=[str(i) for i in range(len(PLAN_CASES))])
def test_plan_and_release(pa, case):
    ctx, new, P, how, pad, words, short, columns = case
    rng = np.random.default_rng(11)
    if ctx == "many":                                             # more sequences than a workgroup has threads
        n = 300 if new == 3 else 20
        ctx, new = rng.integers(0, 500, n).tolist(), rng.integers(0, new + 1, n).tolist()
    B, rows = len(ctx), sum(new) + pad
    before = [R.blocks(c, P) for c in ctx]
    before[0] += 1 if B > 2 else 0                                # a block left over from an earlier step
    after = [max(R.blocks(c + n, P), k) for c, n, k in zip(ctx, new, before)]
    MB = max(max(after) + columns, max(before), 1)
    grow = sum(after) - sum(before)
    spare = max(grow - short, 0) if short else grow + 3
    perm = rng.permutation(sum(before) + spare)
    table, at = np.full((B, MB), -1, np.int64), 0
    for s in range(B):
        table[s, :before[s]] = perm[at:at + before[s]]
        at += before[s]
    free = perm[at:].tolist()
    parents = None if how is None else (random_parents(rng, new, how == "wild") + [-1] * max(pad, 0))[:rows]
    ref = R.plan(ctx, new, parents, table, before, free, P, rows, words)
    t_ctx, t_new, t_table, t_num = ints(ctx), ints(new), ints(table), ints(before)
    t_free, t_count = ints(free + [-7] * (sum(before) + 2)), ints([len(free)])
    plan = pa.paged_plan_step(t_ctx, t_new, t_table, t_num, t_free, t_count, P, rows,
                              parents=None if parents is None else ints(parents), mask_words=words)
    for name in ("seq_lens", "cu_q_lens", "seq_ids", "positions", "rope_positions", "shortage"):
        assert getattr(plan, name).tolist() == list(ref[name]), name
    assert torch.equal(plan.tree_mask, bits(np.array(ref["tree_mask"], dtype=np.uint64).reshape(rows, words)))
    assert t_table.tolist() == ref["block_table"].tolist() and t_num.tolist() == ref["num_blocks"]
    assert t_count.tolist() == [len(ref["free"])] and t_free.tolist()[:len(ref["free"])] == ref["free"]
    if short or ref["shortage"] != [0, 0]:
        assert ref["shortage"] != [0, 0] and t_table.tolist() == table.tolist()
    # back to the contexts, the same plan again (the same pages), then all of it back
    for keep in (ctx, [0] * B, [10 ** 6] * B):
        back = R.release(keep, t_table.cpu().numpy(), t_num.tolist(), t_free.tolist()[:int(t_count)], P)
        pa.paged_release_blocks(ints(keep), t_table, t_num, t_free, t_count, P)
        assert t_table.tolist() == back["block_table"].tolist() and t_num.tolist() == back["num_blocks"]
        assert t_free.tolist()[:int(t_count)] == [int(x) for x in back["free"]]
        if keep is ctx and ref["shortage"] == [0, 0] and all(b == R.blocks(c, P) for b, c in zip(before, ctx)):
            pa.paged_plan_step(t_ctx, t_new, t_table, t_num, t_free, t_count, P, rows,
                               parents=None if parents is None else ints(parents), mask_words=words)
            assert t_table.tolist() == ref["block_table"].tolist()
            pa.paged_release_blocks(ints(keep), t_table, t_num, t_free, t_count, P)
    assert sorted(t_free.tolist()[:int(t_count)]) == sorted(perm.tolist())


# ---- rotary append -------------------------------------------------------------------------------------------------

ROPE_CASES = [  # T, hq, hkv, d, rot, interleaved, page, head_major
    (1, 1, 1, 8, 8, False, 1, False),
    (5, 8, 2, 64, 64, False, 16, False),
    (5, 8, 2, 64, 64, True, 16, True),
    (130, 32, 8, 128, 128, False, 16, False),
    (131, 32, 8, 128, 128, True, 64, False),
    (37, 6, 2, 80, 32, True, 32, True),
    (37, 6, 2, 80, 20, False, 32, False),                         # halves that are no whole 16-byte pieces
    (37, 6, 2, 80, 36, True, 32, False),                          # nor a rotated part
    (9, 3, 3, 256, 256, False, 16, False),
    (9, 16, 8, 256, 64, True, 16, False),
    (33, 4, 4, 72, 2, False, 8, False),
    (33, 4, 4, 96, 0, False, 8, False),                           # nothing rotated
    (2100, 4, 1, 64, 32, False, 16, False),
]


def rope_tolerance(ref, x, dtype, mscale):
    """The result's rounding, and the products': sine and cosine within 2^-22 (their argument is a 32-bit half turn of at most 1),
    two products and a sum of 2^-24 each, of |x| + |y| <= 2 max |x|."""
    return half_step(dtype) * np.abs(ref) + mscale * 2.0 * float(np.abs(x).max()) * (2.0 ** -22 + 3 * 2.0 ** -24) + 1e-30


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("case", ROPE_CASES, ids=[str(i) for i in range(len(ROPE_CASES))])
def test_rope_append(pa, case, dtype):
    T, hq, hkv, d, rot, inter, P, head_major = case
    g = torch.Generator().manual_seed(3)
    B, MB = 3, 2 * (T // P + 2)
    rng = np.random.default_rng(5)
    seq = rng.integers(0, B, T)
    far = rng.integers(0, 1 << 20, T)                             # turned by positions far from where they are stored
    pos = np.zeros(T, np.int64)
    for s in range(B):
        pos[seq == s] = np.arange((seq == s).sum()) + 3
    dead = rng.random(T) < 0.2 if T > 1 else np.zeros(T, bool)
    pos[dead] = -1
    NP = B * MB + 1
    table = rng.permutation(NP)[:B * MB].reshape(B, MB)
    hole = table.copy()
    if T > 100:
        hole[1, 1] = -1                                           # an unmapped block: its rows are not stored
    q, k_new, v_new = (torch.randn(T, h, d, generator=g).to(dtype) for h in (hq, hkv, hkv))
    shape = (NP, hkv, P, d) if head_major else (NP, P, hkv, d)
    k0, v0 = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    mscale = 1.25
    inv = torch.from_numpy(10000.0 ** (-np.arange(rot // 2) * 2.0 / max(rot, 1)))
    # q, k and v as parts of one projection
    fused = torch.cat([q.flatten(1), k_new.flatten(1), v_new.flatten(1)], 1).to(DEV)
    fq, fk, fv = (x.view(T, -1, d) for x in fused.split([hq * d, hkv * d, hkv * d], 1))
    args = (ints(far), ints(seq), ints(pos), ints(hole), inv.to(DEV))
    ref_q = R.rope(q.double().numpy(), far, inv.numpy(), inter, mscale)
    ref_k = R.rope(k_new.double().numpy(), far, inv.numpy(), inter, mscale)
    ek, ev = k0.double().numpy(), v0.double().numpy()
    tk = half_step(dtype) * 0 * ek
    for t in range(T):
        if pos[t] < 0 or hole[seq[t], pos[t] // P] < 0:
            continue
        at = (hole[seq[t], pos[t] // P], slice(None), pos[t] % P) if head_major else (hole[seq[t], pos[t] // P], pos[t] % P)
        ek[at], ev[at] = ref_k[t], v_new[t].double().numpy()
        tk[at] = rope_tolerance(ref_k[t], k_new.double().numpy(), dtype, mscale)
    outs = []
    for form in range(3):                                         # contiguous; parts of a projection; q in place
        k, v = k0.to(DEV), v0.to(DEV)
        a, b, c = (fq, fk, fv) if form == 1 else (q.to(DEV), k_new.to(DEV), v_new.to(DEV))
        out = pa.paged_rope_append(k, v, a, b, c, *args, interleaved=inter, mscale=mscale, head_major=head_major,
                                   q_out=a if form == 2 else None)
        outs.append(out)
        got = out.double().cpu().numpy()
        assert (np.abs(got - ref_q) <= rope_tolerance(ref_q, q.double().numpy(), dtype, mscale)).all()
        if rot < d:
            assert torch.equal(out[..., rot:].cpu(), q[..., rot:])
        assert (np.abs(k.double().cpu().numpy() - ek) <= tk).all()
        assert np.array_equal(v.double().cpu().numpy(), ev)
        assert torch.equal(out, outs[0])
    # either part alone
    k, v = k0.to(DEV), v0.to(DEV)
    assert torch.equal(pa.paged_rope_append(k, v, q.to(DEV), None, None, args[0], None, None, None, args[4], interleaved=inter,
                                            mscale=mscale, head_major=head_major), outs[0])
    assert torch.equal(k.cpu(), k0) and torch.equal(v.cpu(), v0)
    assert pa.paged_rope_append(k, v, None, k_new.to(DEV), v_new.to(DEV), *args, interleaved=inter, mscale=mscale,
                                head_major=head_major) is None
    assert (np.abs(k.double().cpu().numpy() - ek) <= tk).all() and np.array_equal(v.double().cpu().numpy(), ev)


def test_rope_values_that_are_not_finite_stay_with_their_pair(pa):
    x = torch.randn(2, 4, 64).to(torch.bfloat16)
    x[0, 1, 3], x[0, 2, 40], x[1, 0, 63] = float("nan"), float("inf"), float("-inf")
    inv = torch.from_numpy(10000.0 ** (-np.arange(16) / 16.0))
    k = torch.zeros(4, 16, 4, 64, dtype=torch.bfloat16, device=DEV)
    out = pa.paged_rope_append(k, k.clone(), x.to(DEV), None, None, ints([7, 9]), None, None, None, inv.to(DEV)).cpu()
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 1, 3] = bad[0, 1, 19] = bad[0, 2, 40] = bad[1, 0, 63] = True
    assert torch.equal(~torch.isfinite(out), bad)
    assert out[0, 2, 40] == float("inf") and out[1, 0, 63] == float("-inf")


# ---- attention of trees --------------------------------------------------------------------------------------------

def make_tree_call(lens, news, hq, hkv, d, P, dtype, masks, head_major=False, seed=0, pad=0, poison=True):
    """Pools whose slots without a token hold NaN, random pages, and the call's tensors; masks: a function (s, n) -> [n, n]."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    B, rows = len(lens), sum(news) + pad
    nb = [R.blocks(n, P) for n in lens]
    NP = sum(nb) + 3
    perm, at = rng.permutation(NP), 0
    table = np.full((B, max(nb + [1]) + 1), -1)
    shape = (NP, hkv, P, d) if head_major else (NP, P, hkv, d)
    k, v = (torch.full(shape, float("nan") if poison else 0.5, dtype=dtype) for _ in range(2))
    seqs = []
    for s, n in enumerate(lens):
        table[s, :nb[s]] = perm[at:at + nb[s]]
        at += nb[s]
        sk, sv = (torch.randn(n, hkv, d, generator=g).to(dtype) for _ in range(2))
        pages, places = torch.from_numpy(table[s, np.arange(n) // P]), torch.arange(n) % P
        if head_major:
            k[pages, :, places], v[pages, :, places] = sk, sv
        else:
            k[pages, places], v[pages, places] = sk, sv
        seqs.append((sk, sv))
    q = torch.randn(rows, hq, d, generator=g).to(dtype)
    words = max(1, -(-max(news + [1]) // 64))
    mask_bits, per_seq = np.zeros((rows, words), np.uint64), []
    r = 0
    for s, n in enumerate(news):
        m = np.asarray(masks(s, n), bool).reshape(n, n)
        per_seq.append(m)
        for i in range(n):
            for t in np.nonzero(m[i])[0]:
                mask_bits[r, t // 64] |= np.uint64(1 << int(t % 64))
            for t in range(n, 64 * words):                        # bits behind the tokens: anything
                if rng.random() < 0.5:
                    mask_bits[r, t // 64] |= np.uint64(1 << int(t % 64))
            r += 1
    cu = np.concatenate([[0], np.cumsum(news)])
    return dict(k=k.to(DEV), v=v.to(DEV), q=q.to(DEV), cu=ints(cu), mask=bits(mask_bits), table=ints(table), lens=ints(lens),
                seqs=seqs, masks=per_seq, host_lens=lens, news=news, scale=d ** -0.5, head_major=head_major)


def run_tree(pa, c, max_len=None, **kw):
    lse = torch.full(c["q"].shape[:2], 7.0, dtype=torch.float32, device=DEV)
    out = torch.full_like(c["q"], 9.0)
    longest = max(c["host_lens"] + [0]) if max_len is None else max_len
    words = c["mask"].shape[1]
    ws = pa.paged_attention_tree_workspace_bytes(len(c["news"]), c["q"].shape[1], c["k"].shape[1 if c["head_major"] else 2],
                                                 c["q"].shape[2], c["q"].shape[0], max(c["news"] + [1]), longest)
    ws = torch.full((ws,), 0xFF, dtype=torch.uint8, device=DEV)   # NaN as float, -1 as int
    got = pa.paged_attention_tree(c["k"], c["v"], c["q"], c["cu"], max(c["news"] + [1]), c["mask"], c["table"], c["lens"], longest,
                                  c["scale"], out=out, lse=lse, workspace=ws, head_major=c["head_major"], **kw)
    assert got is out and words * 64 >= max(c["news"] + [1])
    return out, lse


def check_tree(c, out, lse, what="", bound=None):
    """Half a rounding step of the output; besides, of max |v| (a weighted mean's scale): softmax weights in two 16-bit terms
    (2^-17), their exponentials (scores below 16 in 32 bits: 16 * 2^-23), 32-bit sums and the final division, together below
    3e-5 for 16-bit inputs; with fp32 inputs scores of up to 256 products of 2^-24 each, 1e-5.  lse: scores as there.
    Calls with more than 64 rows (query, head of a group) for contexts of 256 keys and more take weights of 16 bits: each is off
    by up to half a step of itself, evenly and independently, a deviation of half a step / sqrt(3); six deviations of what
    that does to the output (two in 10^9 are beyond)."""
    dtype, row = c["q"].dtype, 0
    hkv = c["k"].shape[1 if c["head_major"] else 2]
    one_term = dtype != torch.float32 and max(c["news"]) * c["q"].shape[1] // hkv > 64 and (bound or max(c["host_lens"])) >= 256
    extra = 1e-5 if dtype == torch.float32 else 3e-5
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    q = c["q"].double().cpu().numpy()
    for s, n in enumerate(c["news"]):
        k, v = (x.double().numpy() for x in c["seqs"][s])
        ref, ref_lse, wide = R.tree_attention(k, v, q[row:row + n], c["masks"][s], c["host_lens"][s] - n, c["scale"], spread=True)
        vmax = np.abs(v).max() if v.size else 0.0
        o, l = got[row:row + n], got_lse[row:row + n]
        assert np.isfinite(o).all(), (what, s)
        over = np.abs(o - ref) - (half_step(dtype) * (np.abs(ref) + (6 / 3 ** 0.5 * wide if one_term else 0.0)) + extra * vmax)
        assert (over <= 0).all(), (what, s, float(over.max()))
        empty = np.isinf(ref_lse)
        assert (l[empty] == -np.inf).all() and (o[empty] == 0).all(), (what, s)
        assert (np.abs(l[~empty] - ref_lse[~empty]) <= 2e-5 + 2e-6 * np.abs(ref_lse[~empty])).all(), (what, s)
        row += n
    assert (got[row:] == 9.0).all() and (got_lse[row:] == 7.0).all(), f"{what}: rows behind the last sequence"


def ancestors(seed):
    def masks(s, n):
        rng = np.random.default_rng(seed + s)
        m = np.eye(n, dtype=bool)
        for i in range(1, n):
            m[i] |= m[int(rng.integers(max(0, i - 4), i))]
        return m
    return masks


def any_mask(seed):
    """Not ancestors: any bits, rows without any, keys after the query's own."""
    def masks(s, n):
        rng = np.random.default_rng(seed + s)
        m = rng.random((n, n)) < 0.3
        m[rng.random(n) < 0.3] = False
        return m
    return masks


TREE_SHAPES = [  # hq, hkv, d, page
    (8, 8, 64, 16), (32, 8, 128, 16), (16, 1, 128, 64), (12, 4, 128, 16), (8, 2, 256, 32), (4, 4, 256, 16), (6, 2, 80, 16),
    (10, 2, 96, 128), (4, 4, 112, 32), (3, 1, 40, 16), (4, 2, 72, 1), (8, 8, 128, 4), (40, 2, 64, 16), (64, 8, 128, 32),
]
LENS = [1, 15, 16, 17, 0, 40, 64, 65, 127, 129, 300, 517]
NEWS = [1, 15, 1, 16, 0, 5, 64, 33, 8, 65, 7, 2]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("shape", TREE_SHAPES, ids=lambda s: "hq%d-hkv%d-d%d-P%d" % s)
def test_tree_attention(pa, shape, dtype):
    """Contexts from none to several tiles, one to 65 drafted tokens, no tokens and no keys at all; pools of both orders; slots
    without a token hold NaN; two rows behind the last sequence."""
    hq, hkv, d, P = shape
    for masks, head_major in ((ancestors(1), False), (any_mask(2), True)):
        c = make_tree_call(LENS, NEWS, hq, hkv, d, P, dtype, masks, head_major, seed=d + hq, pad=2)
        out, lse = run_tree(pa, c)
        check_tree(c, out, lse, f"{shape} {dtype} {head_major}")
        again, lse2 = run_tree(pa, c)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("hq,hkv,d,lens,news", [
    (8, 2, 128, [5000], [1]), (8, 2, 128, [5000, 3, 2500], [16, 2, 40]), (4, 4, 64, [4097], [130]), (16, 2, 256, [2100, 1800], [64, 3]),
    (32, 4, 128, [3000, 0, 700], [5, 0, 64]), (5, 1, 128, [1500] * 9, [3] * 9), (8, 8, 96, [3000], [9])])
def test_tree_attention_on_longer_contexts(pa, hq, hkv, d, lens, news, dtype):
    """Contexts that are cut over workgroups, with a bound on them that is loose, too."""
    c = make_tree_call(lens, news, hq, hkv, d, 16, dtype, ancestors(5), seed=3)
    for bound in (None, 7 * max(lens)):
        if bound is not None:
            wide = torch.full((len(lens), R.blocks(bound, 16)), -1, dtype=torch.int32, device=DEV)
            wide[:, :c["table"].shape[1]] = c["table"]
            c["table"] = wide
        out, lse = run_tree(pa, c, max_len=bound)
        check_tree(c, out, lse, f"{lens} {news} {bound}", bound)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tree_attention_with_values_that_are_not_finite(pa, dtype):
    """A NaN or an infinity in the K or V row of a drafted token reaches the queries that see it, and no other; scores of the
    type's lowest size in places that a mask hides do nothing."""
    n, ctx, d = 12, 70, 64
    masks = ancestors(9)
    for where in ("k", "v"):
        for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min):
            c = make_tree_call([ctx + n], [n], 4, 2, d, 16, dtype, masks, seed=6)
            at = 4                                                # the drafted token that holds it
            page, place = int(c["table"][0, (ctx + at) // 16]), (ctx + at) % 16
            c[where][page, place, :, 3] = bad
            out, lse = run_tree(pa, c)
            sees = c["masks"][0][:, at]
            assert 0 < sees.sum() < n
            sk, sv = c["seqs"][0]
            clean = dict(c, seqs=[(sk, sv)])
            ref, ref_lse = R.tree_attention(sk.double().numpy(), sv.double().numpy(), c["q"].double().cpu().numpy(), c["masks"][0],
                                            ctx, c["scale"])
            o = out.double().cpu().numpy()
            assert clean and np.isfinite(o[~sees]).all()
            assert (np.abs(o - ref)[~sees] <= half_step(dtype) * np.abs(ref[~sees]) + 3e-5 * float(sv.abs().max())).all()
            if where == "v":
                col = out[:, :, 3].float()[torch.from_numpy(sees).to(DEV)]
                assert (col.isnan() if bad != bad else col == bad if np.isinf(bad) else col.abs() > 1e3).all()
                assert np.isfinite(np.delete(o, 3, axis=2)).all()
            elif bad != bad:
                assert np.isnan(o[sees]).all() and np.isnan(lse.cpu().numpy()[sees]).all()


def test_tree_attention_of_a_chain_is_causal_prefill(pa):
    """A chain of drafts is a causal chunk on top of the context: the same as paged_attention_prefill within the rounding of
    both outputs (half a step each) and of that kernel's weights, which it rounds to bf16 where there are many: each is off by at
    most 2^-8 of itself, so their weighted mean of v by at most 2^-8 max |v|."""
    lens, news = [300, 64, 1000, 7], [16, 64, 3, 7]
    c = make_tree_call(lens, news, 32, 8, 128, 16, torch.bfloat16, lambda s, n: np.tril(np.ones((n, n))), seed=8)
    out, lse = run_tree(pa, c)
    lse2 = torch.empty_like(lse)
    ref = pa.paged_attention_prefill(c["k"], c["v"], c["q"], c["cu"], max(news), c["table"], c["lens"], max(lens), c["scale"], True,
                                     lse=lse2)
    vmax = max(float(v.abs().max()) for _, v in c["seqs"])
    near = (out.float() - ref.float()).abs() <= 2.0 ** -7 * ref.float().abs() + 2.0 ** -8 * vmax
    assert bool(near.all()) and float((lse - lse2).abs().max()) <= 4e-5


# ---- acceptance ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("news,max_path,P,hkv,d", [
    ([1], 1, 16, 1, 8), ([5, 0, 64, 1], 64, 16, 8, 128), ([65, 200, 3], 200, 4, 2, 64), ([30, 30], 3, 32, 8, 256), ([300], 300, 1, 1, 64),
    ([12] * 70, 12, 16, 12, 80)])
def test_tree_accept(pa, news, max_path, P, hkv, d, dtype, head_major):
    rng = np.random.default_rng(sum(news) + P)
    g = torch.Generator().manual_seed(1)
    ctx = rng.integers(0, 90, len(news)).tolist()
    lens = [a + b for a, b in zip(ctx, news)]
    nb = [R.blocks(n, P) for n in lens]
    NP = sum(nb) + 2
    perm, at = rng.permutation(NP), 0
    table = np.full((len(news), max(nb) + 1), -1)
    for s in range(len(news)):
        table[s, :nb[s]] = perm[at:at + nb[s]]
        at += nb[s]
    shape = (NP, hkv, P, d) if head_major else (NP, P, hkv, d)
    k, v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    parents, tokens, targets = [], [], []
    for n in news:                                                # few different tokens: long paths, and children that agree
        parents.append([-1] + [int(rng.integers(max(0, i - 3), i)) for i in range(1, n)] if n else [])
        tokens.append(rng.integers(0, 2, n).tolist())
        targets.append(rng.integers(0, 2, n).tolist())
    ref = [R.accept(p, t, g_, max_path) for p, t, g_ in zip(parents, tokens, targets)]
    want = []
    for pool in (k, v):
        pool = pool.clone()
        for s, (path, _) in enumerate(ref):
            rows = []
            for i in path:
                t = ctx[s] + i
                rows.append((pool[table[s, t // P], :, t % P] if head_major else pool[table[s, t // P], t % P]).clone())
            for i, row in enumerate(rows):
                t = ctx[s] + i
                if head_major:
                    pool[table[s, t // P], :, t % P] = row
                else:
                    pool[table[s, t // P], t % P] = row
        want.append(pool)
    cu = ints(np.concatenate([[0], np.cumsum(news)]))
    flat = [ints(sum(x, []) + [5]) for x in (parents, tokens, targets)]
    gk, gv = k.to(DEV), v.to(DEV)
    path, path_lens = torch.full((len(news), max_path), 99, dtype=torch.int32, device=DEV), ints([77] * len(news))
    _, _, nxt, kept = pa.paged_tree_accept(gk, gv, cu, ints(lens), max(news), ints(table), path, path_lens, parents=flat[0],
                                           tokens=flat[1], targets=flat[2], head_major=head_major)
    assert path_lens.tolist() == [len(p) for p, _ in ref]
    assert path.tolist() == [p + [-1] * (max_path - len(p)) for p, _ in ref]
    assert nxt.tolist() == [t for _, t in ref] and kept.tolist() == [c + len(p) for c, (p, _) in zip(ctx, ref)]
    assert torch.equal(gk.cpu(), want[0]) and torch.equal(gv.cpu(), want[1])
    # another layer: the same path on its pools
    gk, gv = k.to(DEV), v.to(DEV)
    before = path.clone()
    _, _, nxt, kept2 = pa.paged_tree_accept(gk, gv, cu, ints(lens), max(news), ints(table), path, path_lens, head_major=head_major)
    assert nxt is None and torch.equal(path, before) and torch.equal(kept, kept2)
    assert torch.equal(gk.cpu(), want[0]) and torch.equal(gv.cpu(), want[1])


# ---- all of them in a row ------------------------------------------------------------------------------------------

class Step:
    """Two layers' caches and everything that a loop of steps keeps, for `B` sequences."""

    def __init__(self, pa, B, W, hq, hkv, d, P, dtype, MB, pages):
        self.pa, self.B, self.W, self.P, self.scale = pa, B, W, P, d ** -0.5
        self.caches = [tuple(torch.full((pages, P, hkv, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2)) for _ in range(2)]
        self.table = torch.full((B, MB), -1, dtype=torch.int32, device=DEV)
        self.num_blocks, self.ctx = ints([0] * B), ints([0] * B)
        self.free, self.count = ints(np.random.default_rng(0).permutation(pages)), ints([pages])
        self.inv = torch.from_numpy(10000.0 ** (-np.arange(d // 2) * 2.0 / d)).to(DEV)
        self.hq, self.hkv, self.d, self.dtype, self.MB = hq, hkv, d, dtype, MB
        rows = B * W
        self.new, self.parents = ints([0] * B), ints([-1] * rows)
        self.tokens, self.targets = ints([0] * rows), ints([0] * rows)
        self.qkv = [torch.zeros(rows, (hq + 2 * hkv) * d, dtype=dtype, device=DEV) for _ in range(2)]
        self.path, self.path_lens = ints(np.zeros((B, W))), ints([0] * B)
        self.next = ints([0] * B)
        self.outs = [torch.zeros(rows, hq, d, dtype=dtype, device=DEV) for _ in range(2)]
        self.lses = [torch.zeros(rows, hq, device=DEV) for _ in range(2)]
        self.plan = None

    def step(self):
        pa, hq, hkv, d = self.pa, self.hq, self.hkv, self.d
        rows = self.B * self.W
        self.plan = p = pa.paged_plan_step(self.ctx, self.new, self.table, self.num_blocks, self.free, self.count, self.P, rows,
                                           parents=self.parents)
        for layer, (k, v) in enumerate(self.caches):
            q, kn, vn = (x.view(rows, -1, d) for x in self.qkv[layer].split([hq * d, hkv * d, hkv * d], 1))
            q = pa.paged_rope_append(k, v, q, kn, vn, p.rope_positions, p.seq_ids, p.positions, self.table, self.inv)
            pa.paged_attention_tree(k, v, q, p.cu_q_lens, self.W, p.tree_mask, self.table, p.seq_lens, self.MB * self.P, self.scale,
                                    out=self.outs[layer], lse=self.lses[layer])
            found = dict(parents=self.parents, tokens=self.tokens, targets=self.targets, next_tokens=self.next) if layer == 0 else {}
            pa.paged_tree_accept(k, v, p.cu_q_lens, p.seq_lens, self.W, self.table, self.path, self.path_lens, kept_lens=self.ctx,
                                 **found)


def fill_step(st, rng, g, news):
    """Another step's requests: (parents, tokens, targets) per sequence and the layers' projections."""
    trees, flat = [], [[], [], []]
    for n in news:
        parents = [-1] + [int(rng.integers(max(0, i - 3), i)) for i in range(1, n)] if n else []
        tree = (parents, rng.integers(0, 2, n).tolist(), rng.integers(0, 2, n).tolist())
        trees.append(tree)
        for a, b in zip(flat, tree):
            a.extend(b)
    rows, total = st.B * st.W, sum(news)
    st.new.copy_(ints(news))
    for dst, x in zip((st.parents, st.tokens, st.targets), flat):
        dst.copy_(ints(x + [-1] * (rows - total)))
    host = [torch.randn(st.qkv[0].shape, generator=g).to(st.dtype) for _ in st.qkv]
    for dst, x in zip(st.qkv, host):
        dst.copy_(x)
    return trees, host


@pytest.mark.parametrize("captured", [False, True])
def test_steps_in_a_row(pa, captured):
    """Five steps of two layers against a model of the cache on the host that keeps what was accepted, turned by its place in the
    text: eager, and one captured graph replayed with the program's own work between."""
    rng, g = np.random.default_rng(21), torch.Generator().manual_seed(21)
    B, W, hq, hkv, d, P = 3, 9, 4, 2, 64, 16
    st = Step(pa, B, W, hq, hkv, d, P, torch.float32, 5, 13)
    kept = [[([], []) for _ in range(B)] for _ in range(2)]       # per layer, sequence: turned K rows, V rows
    graph = None
    if captured:
        st.step()                                                 # nothing drafted: allocations before the capture
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                st.step()
        torch.cuda.current_stream().wait_stream(side)
    for step, news in enumerate([[9, 4, 1], [3, 0, 9], [0, 0, 0], [9, 9, 9], [2, 7, 5]]):
        trees, host = fill_step(st, rng, g, news)
        if captured:
            graph.replay()
        else:
            st.step()
        torch.cuda.synchronize()
        assert st.plan.shortage.tolist() == [0, 0]
        row = 0
        paths = [R.accept(*t, W) for t in trees]
        for s, n in enumerate(news):
            parents = trees[s][0]
            m = np.eye(n, dtype=bool)
            for i in range(1, n):
                m[i] |= m[parents[i]]
            for layer in range(2):
                x = host[layer][row:row + n].double().numpy().reshape(n, hq + 2 * hkv, d)
                ks, vs = kept[layer][s]
                pos = len(ks) + m.sum(1) - 1 if n else np.zeros(0)
                turned = R.rope(x[:, :hq + hkv], pos, st.inv.cpu().numpy(), False, 1.0)
                k = np.array(ks + list(turned[:, hq:])).reshape(-1, hkv, d)
                v = np.array(vs + list(x[:, hq + hkv:])).reshape(-1, hkv, d)
                ref, ref_lse = R.tree_attention(k, v, turned[:, :hq], m, len(ks), st.scale)
                got = st.outs[layer][row:row + n].double().cpu().numpy()
                # 1e-5 of attention itself (check_tree) and, through the scores, what turned rows are off by
                assert (np.abs(got - ref) <= 4e-5 * max(1.0, np.abs(v).max() if n else 1.0)).all(), (step, s, layer)
                assert (np.abs(st.lses[layer][row:row + n].cpu().numpy() - ref_lse) <= 4e-5).all()
                for i in paths[s][0]:
                    ks.append(turned[i, hq:])
                    vs.append(x[i, hq + hkv:])
            assert int(st.ctx[s]) == len(kept[0][s][0])
            row += n
        assert st.next.tolist() == [t for _, t in paths] and st.path_lens.tolist() == [len(p) for p, _ in paths]
        # the cache holds what was accepted
        for layer, (k, v) in enumerate(st.caches):
            for s in range(B):
                for t, (rk, rv) in enumerate(zip(*kept[layer][s])):
                    page = int(st.table[s, t // P])
                    assert np.abs(k[page, t % P].double().cpu().numpy() - rk).max() <= 2e-6 * max(1.0, np.abs(rk).max())
                    assert np.array_equal(v[page, t % P].double().cpu().numpy(), rv)
    pa.paged_release_blocks(ints([0] * B), st.table, st.num_blocks, st.free, st.count, P)
    assert int(st.count) == 13 and sorted(st.free.tolist()) == list(range(13)) and (st.table == -1).all()
