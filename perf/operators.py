"""What a step of drafted tokens over the paged cache is timed on, operator by operator and as a whole.  `run` computes
the operators in elementary torch, or (`own`) as a user's program calls them, with the arguments marshalled once.

A case is a dict of plain values:
    kind        "plan"   slots, positions, masks and pages of a step from request lengths (behind the return of the
                         pages that the last step's drafts held)
                "rope"   rotary positions of q and of new K rows, K and V into their pages
                "tree"   attention of trees of drafted tokens over the cache
                "accept" drafts written as by "rope", then the accepted path found and its rows moved together
                "step"   all of these in the order of a serving loop
    dtype       "bf16", "fp16" or "fp32"
    batch, lo, hi, lens_seed   sequences; lengths of their contexts, log-uniform in [lo, hi], without the new tokens
    new, even   new tokens of a sequence: `new` of them each (even), or any number from 1 to `new`
    tree        0: each token follows the one before it; n: a token's parent is one of the n tokens before it
    pad         rows behind the last sequence (a captured step has room for more tokens than it gets)
    short       plan: the free list has this many pages too few (0: enough)
    hq, hkv, d, page           query heads, KV heads, head_dim, tokens per page
    rot, inter, scaling        leading elements of a head that are rotated; neighbours as pairs (else halves); positions
                               "none", "linear", "base", "parts" or "ramp" (see _frequencies)
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BASE = dict(kind="tree", dtype="bf16", batch=1, lo=2048, hi=2048, lens_seed=0, new=8, even=True, tree=4, pad=0, short=0,
            hq=32, hkv=8, d=128, page=16, rot=128, inter=False, scaling="none")


def _case(name=None, **kw):
    c = dict(BASE, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The smallest step: one user, five drafted tokens; launch and latency only.
        _case("plan_1x5", kind="plan", batch=1, new=5),
        # A full server: 512 requests with up to 64 drafts each, in a captured step with room to spare.
        _case("plan_512x64", kind="plan", batch=512, lo=64, hi=32768, lens_seed=4, new=64, even=False, pad=100),
        # Plain decoding: one new token for each of eight chats.
        _case("rope_8x1", kind="rope", batch=8, lo=128, hi=2048, lens_seed=1, new=1, tree=0),
        # A chunk of a long document's prompt, positions scaled for long contexts by parts.
        _case("rope_8192_of_131072", kind="rope", batch=1, lo=122880, hi=122880, new=8192, tree=0, scaling="parts"),
        # A model with heads of 80 that rotates two fifths of each in neighbours, fp16, odd prompt lengths.
        _case("rope_fp16_d80_part", kind="rope", dtype="fp16", batch=3, lo=1, hi=1, new=777, even=False, tree=0, hq=32, hkv=32,
              d=80, page=64, rot=32, inter=True),
        # The smallest attention: full precision, one sequence, five drafts.
        _case("tree_fp32_1x128", dtype="fp32", lo=128, hi=128, new=5, hq=8, hkv=8, d=64, rot=64),
        # Interactive serving: eight chats, 16 drafts each.
        _case("tree_8x16_128to2048", batch=8, lo=128, hi=2048, lens_seed=1, new=16),
        # A busy server: 64 sequences of all lengths with up to eight drafts.
        _case("tree_64x8_mixed", batch=64, lo=64, hi=32768, lens_seed=4, new=8, even=False),
        # Long documents: 16 sequences of 131072 tokens, 8.6 GB of K and V.
        _case("tree_16x16_131072", batch=16, lo=131056, hi=131056, new=16, hq=64),
        # Interactive serving behind its attention: what of 16 drafts stays.
        _case("accept_8x16", kind="accept", batch=8, lo=128, hi=2048, lens_seed=1, new=16),
        # A busy server with wide trees.
        _case("accept_256x64", kind="accept", batch=256, lo=64, hi=2048, lens_seed=5, new=64, even=False),
        # A whole step with wide trees at head_dim 256, positions interpolated.
        _case("step_fp16_d256_2x64", kind="step", dtype="fp16", batch=2, lo=2000, hi=4000, lens_seed=3, new=64, hq=16, hkv=8,
              d=256, page=32, rot=256, scaling="linear"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the ranges above."""
    kind = rng.choice(["plan", "rope", "rope", "tree", "tree", "tree", "tree", "accept", "step"])
    c = _case(kind=kind, lens_seed=rng.randrange(1 << 20), dtype=rng.choice(["bf16", "bf16", "fp16"]))
    c["hq"], c["hkv"] = rng.choice([(32, 8), (32, 8), (32, 32), (64, 8), (16, 8), (8, 1), (12, 4)])
    c["d"] = rng.choice([128, 128, 128, 64, 256, 80, 96])
    c["page"] = rng.choice([16, 16, 32, 64, 128])
    c["rot"] = rng.choice([c["d"], c["d"], c["d"] // 2, c["d"] // 4])
    c["inter"] = rng.random() < 0.4
    c["scaling"] = rng.choice(["none", "linear", "base", "parts", "ramp"])
    c["tree"] = rng.choice([0, 1, 2, 4, 8, 16])
    c["even"] = rng.random() < 0.4
    c["pad"] = rng.choice([0, 0, 0, 1, 33])
    c["new"] = _log(rng, 1, 64)
    c["hi"] = _log(rng, 100, 131072 if kind == "tree" else 32768)
    c["lo"] = rng.choice([c["hi"], max(1, c["hi"] // 2), max(1, c["hi"] // 30)])
    per_token = 4 * c["hkv"] * c["d"]                             # bytes of one token's K and V at 16 bits
    if kind == "plan":
        c["batch"] = _log(rng, 1, 512)
        c["short"] = rng.choice([0, 0, 0, 3])
    elif kind == "rope":
        c["tree"] = 0
        c["new"] = _log(rng, 1, 4096)
        c["batch"] = max(1, min(_log(rng, 1, 256), 16384 // c["new"]))
        c["lo"], c["hi"] = 1, rng.choice([1, 4000, 120000])
    else:
        c["batch"] = max(1, min(_log(rng, 1, 64), int(4e9 // (per_token * (c["hi"] + c["new"])))))
        if rng.random() < 0.15:
            c.update(dtype="fp32", d=rng.choice([64, 128]), batch=min(c["batch"], 8), hi=min(c["hi"], 2048))
            c["hq"], c["hkv"] = rng.choice([(8, 8), (32, 8)])
            c["lo"], c["rot"] = min(c["lo"], c["hi"]), c["d"]
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------

def _lengths(case):
    """(contexts, new tokens) of the case's sequences; the same for every seed."""
    rng = random.Random(900 + case["lens_seed"])
    ctx = [_log(rng, case["lo"], case["hi"]) for _ in range(case["batch"])]
    return ctx, [case["new"] if case["even"] else rng.randint(1, case["new"]) for _ in ctx]


def _frequencies(case):
    """Radians a position of each pair, and the factor on both coordinates: base^(-2 i / r), for contexts 8 times as long
    as the 8192 tokens the base was made for.  "linear": positions by that factor closer together.  "base": a larger base
    that does so for the slowest pair and nothing for the fastest.  "parts": only pairs slower than the old context / 1,
    none faster than the old context / 4, in between both.  "ramp": the same with a ramp over the pair's number, from
    the pair that turns 32 times in the old context to the one that turns once, coordinates lengthened by 0.1 ln 8 + 1."""
    r, base, factor, old, kind = case["rot"], 10000.0, 8.0, 8192.0, case["scaling"]
    i = np.arange(r // 2, dtype=np.float64)
    if kind == "base" and r > 2:
        base *= factor ** (r / (r - 2.0))
    f = base ** (-2.0 * i / r)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "parts":
        keep = np.clip((old * f / (2.0 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 1.0
    if kind == "ramp":
        lo, hi = (r * math.log(old / (2.0 * math.pi * turns)) / (2.0 * math.log(base)) for turns in (32.0, 1.0))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
        keep = 1.0 - np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _randn(shape, dtype, gen):
    """N(0, 1) in the storage type, drawn in pieces so that no fp32 copy of a large pool exists."""
    out = torch.empty(shape, dtype=dtype, device=DEVICE)
    step = max(1, (1 << 28) // max(1, math.prod(shape[1:])))
    for i in range(0, shape[0], step):
        out[i:i + step] = torch.randn((min(step, shape[0] - i),) + tuple(shape[1:]), generator=gen, device=DEVICE)
    return out


def _trees(case, new, seed):
    """parents [B, W] (-1: a root, and behind the sequence's tokens), drafted tokens and what the model would choose after each
    node: one of its children's tokens three times in four."""
    rng = np.random.default_rng(seed)
    B, W = len(new), max(new)
    i = np.arange(W)
    back = rng.integers(1, max(case["tree"], 1) + 1, (B, W)) if W > 1 else np.ones((B, W), np.int64)
    parents = np.where(i == 0, -1, np.maximum(i - back, 0)).astype(np.int32)
    tokens = rng.integers(0, 32000, (B, W)).astype(np.int32)
    targets = rng.integers(0, 32000, (B, W)).astype(np.int32)
    for c in rng.permutation(W - 1) + 1:                          # the last child written wins: any of them
        hit = rng.random(B) < 0.75
        targets[hit, parents[hit, c]] = tokens[hit, c]
    return parents, tokens, targets


def _inputs(case, seed):
    """What the program holds, plain torch and numpy."""
    ctx, new = _lengths(case)
    dtype, P, d = TORCH[case["dtype"]], case["page"], case["d"]
    B, W, kind = len(ctx), max(new), case["kind"]
    total = sum(new)
    rows = total + case["pad"]
    lens = [a + b for a, b in zip(ctx, new)]
    live = np.arange(W)[None, :] < np.array(new)[:, None]
    parents, tokens, targets = _trees(case, new, seed)
    words = -(-W // 64) if kind != "rope" else 0
    depth = np.zeros((B, W), np.int64)
    mask = np.zeros((B, W, max(words, 1)), np.uint64)
    if kind != "rope":
        b = np.arange(B)
        for i in range(W):
            if i:
                depth[:, i] = np.where(parents[:, i] >= 0, depth[b, parents[:, i]] + 1, 0)
                mask[:, i] = np.where(parents[:, i, None] >= 0, mask[b, parents[:, i]], 0)
            mask[:, i, i // 64] |= np.uint64(1 << (i % 64))
    else:
        depth[:] = np.arange(W)
    before, after = [-(-n // P) for n in ctx], [-(-n // P) for n in lens]
    planned = kind in ("plan", "step")
    # pages: a random permutation of a pool with a quarter more than in use; "rope" writes its tokens' blocks alone
    first = [n // P if kind == "rope" else 0 for n in ctx]
    mapped = before if planned else after
    used = sum(m - f for m, f in zip(mapped, first))
    grow = sum(after) - sum(before)
    spare = 0 if not planned else max(0, grow - case["short"]) if case["short"] else grow + 7
    pages = used + spare if planned else used + used // 4 + 1
    perm = np.random.default_rng(seed).permutation(pages).astype(np.int32)
    table = np.full((B, max(after) + 2), -1, dtype=np.int32)
    at = 0
    for s in range(B):
        table[s, first[s]:mapped[s]] = perm[at:at + mapped[s] - first[s]]
        at += mapped[s] - first[s]

    def ints(x):
        return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=np.int32))).to(DEVICE)

    def packed(x, fill):
        x = x[live].astype(np.int32)
        return ints(np.concatenate([x, np.full(case["pad"], fill, np.int32)]))

    t = dict(block_table=ints(table), ctx_lens=ints(ctx), new_lens=ints(new))
    if kind != "rope":
        t.update(parents=packed(parents, -1), tokens=packed(tokens, -1), targets=packed(targets, -1))
    if planned:
        free = np.zeros(pages, np.int32)
        free[:spare] = perm[used:]
        t.update(num_blocks=ints(before), free_pages=ints(free), free_count=ints([spare]))
        t.update(seq_lens=ints(np.zeros(B)), cu_q_lens=ints(np.zeros(B + 1)), shortage=ints([0, 0]))
        t.update({n: ints(np.zeros(rows)) for n in ("seq_ids", "positions", "rope_positions")})
        t["tree_mask"] = torch.zeros((rows, words), dtype=torch.int64, device=DEVICE)
    else:
        t.update(seq_lens=ints(lens), cu_q_lens=ints([0] + np.cumsum(new).tolist()))
        t["seq_ids"] = packed(np.broadcast_to(np.arange(B)[:, None], (B, W)), -1)
        t["positions"] = packed(np.array(ctx)[:, None] + np.arange(W), -1)
        t["rope_positions"] = packed(np.array(ctx)[:, None] + depth, 0)
        if words:
            m = np.concatenate([mask[live], np.zeros((case["pad"], words), np.uint64)])
            t["tree_mask"] = torch.from_numpy(m.view(np.int64)).to(DEVICE)
    if kind == "plan":
        return t
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    pool = (pages, P, case["hkv"], d)
    t["k_cache"], t["v_cache"] = _randn(pool, dtype, gen), _randn(pool, dtype, gen)
    t["q"] = _randn((rows, case["hq"], d), dtype, gen)
    if kind != "tree":
        t["k_new"], t["v_new"] = (_randn((rows, case["hkv"], d), dtype, gen) for _ in range(2))
        t["inv_freq"] = torch.from_numpy(_frequencies(case)[0]).to(DEVICE)
        t["q_out"] = torch.empty_like(t["q"])
    if kind in ("tree", "step"):
        t["out"] = torch.zeros_like(t["q"])
        t["lse"] = torch.zeros((rows, case["hq"]), dtype=torch.float32, device=DEVICE)
    if kind in ("accept", "step"):
        t["path"] = ints(np.zeros((B, W)))
        t.update({n: ints(np.zeros(B)) for n in ("path_lens", "next_tokens", "kept_lens")})
    return t


def prepare(case, seed):
    state = dict(case=case, t=_inputs(case, seed), width=max(_lengths(case)[1]),
                 longest=max(a + b for a, b in zip(*_lengths(case))), mscale=_frequencies(case)[1])
    if own:
        state["calls"] = _calls(state)
    return state


OUTPUTS = {
    "plan": ("seq_lens", "cu_q_lens", "seq_ids", "positions", "rope_positions", "tree_mask", "block_table", "num_blocks",
             "free_pages", "free_count", "shortage"),
    "rope": ("q_out", "k_cache", "v_cache"),
    "tree": ("out", "lse"),
    "accept": ("q_out", "k_cache", "v_cache", "path", "path_lens", "next_tokens", "kept_lens"),
    "step": ("block_table", "free_count", "rope_positions", "tree_mask", "q_out", "out", "lse", "k_cache", "v_cache", "path",
             "path_lens", "next_tokens", "kept_lens"),
}


def run(state):
    if own:
        for call in state["calls"]:
            call()
    else:
        kind, t = state["case"]["kind"], state["t"]
        if kind in ("plan", "step"):
            _release(state, t)
            _plan(state, t)
        if kind in ("rope", "accept", "step"):
            _rope(state, t)
        if kind in ("tree", "step"):
            _tree(state, t)
        if kind in ("accept", "step"):
            _accept(state, t)
    return {n: state["t"][n] for n in OUTPUTS[state["case"]["kind"]]}


# ---- as a user's program calls the framework ---------------------------------------------------------------------

def _calls(state):
    import paper_2506_07311_amd as pa
    case, t = state["case"], state["t"]
    kind, P = case["kind"], case["page"]
    calls = []
    if kind in ("plan", "step"):
        calls.append(pa.prepare_release_blocks(t["ctx_lens"], t["block_table"], t["num_blocks"], t["free_pages"], t["free_count"], P))
        calls.append(pa.prepare_plan_step(
            t["ctx_lens"], t["new_lens"], t["block_table"], t["num_blocks"], t["free_pages"], t["free_count"], P,
            t["seq_ids"].shape[0], parents=t["parents"], seq_lens=t["seq_lens"], cu_q_lens=t["cu_q_lens"], seq_ids=t["seq_ids"],
            positions=t["positions"], rope_positions=t["rope_positions"], tree_mask=t["tree_mask"], shortage=t["shortage"]))
    if kind in ("rope", "accept", "step"):
        calls.append(pa.prepare_rope_append(
            t["k_cache"], t["v_cache"], t["q"], t["k_new"], t["v_new"], t["rope_positions"], t["seq_ids"], t["positions"],
            t["block_table"], t["inv_freq"], interleaved=case["inter"], mscale=state["mscale"], q_out=t["q_out"]))
    if kind in ("tree", "step"):
        q = t["q_out"] if kind == "step" else t["q"]
        workspace = torch.empty(pa.paged_attention_tree_workspace_bytes(case["batch"], case["hq"], case["hkv"], case["d"], q.shape[0],
                                                                        state["width"], state["longest"]), dtype=torch.uint8, device=DEVICE)
        calls.append(pa.prepare_attention_tree(
            t["k_cache"], t["v_cache"], q, t["cu_q_lens"], state["width"], t["tree_mask"], t["block_table"], t["seq_lens"],
            state["longest"], case["d"] ** -0.5, out=t["out"], lse=t["lse"], workspace=workspace))
    if kind in ("accept", "step"):
        calls.append(pa.prepare_tree_accept(
            t["k_cache"], t["v_cache"], t["cu_q_lens"], t["seq_lens"], state["width"], t["block_table"], t["path"], t["path_lens"],
            parents=t["parents"], tokens=t["tokens"], targets=t["targets"], next_tokens=t["next_tokens"],
            kept_lens=t["kept_lens"]))
    return calls


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _release(state, t):
    """Blocks beyond the context go back to the end of the free list, so that the same plan takes them again."""
    P, table, n = state["case"]["page"], t["block_table"], t["num_blocks"]
    b = torch.arange(table.shape[1], device=DEVICE)[None, :]
    keep = (t["ctx_lens"] + P - 1) // P
    gone = (b >= keep[:, None]) & (b < n[:, None])
    total = gone.sum()
    at = t["free_count"] + total - gone.flatten().cumsum(0)
    at = torch.where(gone.flatten(), at, t["free_pages"].shape[0])
    free = torch.cat([t["free_pages"], t["free_count"]]).scatter(0, at, table.flatten())
    t["free_pages"].copy_(free[:-1])
    t["free_count"] += total
    table.masked_fill_(gone, -1)
    n.copy_(torch.minimum(n, keep))


def _plan(state, t):
    P, table, n, count = state["case"]["page"], t["block_table"], t["num_blocks"], t["free_count"]
    lens = t["ctx_lens"] + t["new_lens"]
    want = (lens + P - 1) // P
    b = torch.arange(table.shape[1], device=DEVICE)[None, :]
    take = (b >= n[:, None]) & (b < want[:, None])
    total = (want - n).clamp(min=0).sum()
    long = (want > table.shape[1]).sum()
    t["shortage"].copy_(torch.cat([(total - count).clamp(min=0), long[None]]))
    ok = (total <= count) & (long == 0)
    rank = (count - take.flatten().cumsum(0)).clamp(min=0, max=max(0, t["free_pages"].shape[0] - 1))
    page = t["free_pages"][rank].reshape(table.shape) if t["free_pages"].shape[0] else table
    table.copy_(torch.where(take & ok, page, table))
    n.copy_(torch.where(ok, torch.maximum(n, want), n))
    count -= torch.where(ok, total, 0)
    # rows: those of the request, whether it is granted or not
    cu = torch.cat([torch.zeros_like(count), t["new_lens"].cumsum(0)])
    r = torch.arange(t["seq_ids"].shape[0], device=DEVICE)
    live = r < cu[-1]
    s = torch.searchsorted(cu, r, right=True).clamp(max=lens.shape[0]) - 1
    i = r - cu[s]
    t["seq_ids"].copy_(torch.where(live, s, -1))
    t["positions"].copy_(torch.where(live, t["ctx_lens"][s] + i, -1))
    up = _ancestors(state, cu, t["parents"])
    above = up[s, i.clamp(max=up.shape[1] - 1)]                  # [rows, W]: the row's ancestors and itself
    t["rope_positions"].copy_(torch.where(live, t["ctx_lens"][s] + above.sum(1) - 1, 0))
    words = t["tree_mask"].shape[1]
    bits = torch.zeros((r.shape[0], 64 * words), dtype=torch.int64, device=DEVICE)
    bits[:, :above.shape[1]] = above & live[:, None]
    bits <<= torch.arange(64, device=DEVICE).repeat(words)
    t["tree_mask"].copy_(bits.reshape(-1, words, 64).sum(2))
    t["seq_lens"].copy_(torch.where(ok, lens, t["ctx_lens"]))
    t["cu_q_lens"].copy_(torch.where(ok, cu, 0))


def _ancestors(state, cu, parents):
    """[B, W, W]: token j of sequence s is token i or one of those that it follows."""
    W = state["width"]
    j = torch.arange(W, device=DEVICE)
    at = (cu[:-1, None] + j).clamp(max=parents.shape[0] - 1)
    up = torch.where(j < (cu[1:] - cu[:-1])[:, None], parents[at], -1)
    return _closure((up[:, :, None] == j).float() + torch.eye(W, device=DEVICE), W) > 0


def _closure(a, steps):
    return a if steps <= 1 else _closure((torch.bmm(a, a) > 0).float(), (steps + 1) // 2)


def _turned(case, x, angle, mscale):
    """x [rows, heads, d] with its leading elements turned by angle [rows, rot / 2], in 32 bits."""
    r = case["rot"]
    c, s = (angle.cos() * mscale).float()[:, None], (angle.sin() * mscale).float()[:, None]
    y = x.float()
    if case["inter"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _slots(state, t):
    """(page, place in it) of each row's token; behind the last row the first row's again."""
    P, p = state["case"]["page"], t["positions"]
    s, p = torch.where(p < 0, t["seq_ids"][0], t["seq_ids"]), torch.where(p < 0, p[0], p)
    return t["block_table"][s, p // P], p % P


def _rope(state, t):
    case = state["case"]
    angle = t["rope_positions"].double()[:, None] * t["inv_freq"]
    t["q_out"].copy_(_turned(case, t["q"], angle, state["mscale"]))
    pages, places = _slots(state, t)
    dead = (t["positions"] < 0)[:, None, None]
    k = _turned(case, t["k_new"], angle, state["mscale"])
    t["k_cache"][pages, places] = torch.where(dead, k[:1], k)
    t["v_cache"][pages, places] = torch.where(dead, t["v_new"][:1], t["v_new"])


def _tree(state, t):
    case, W, L, P = state["case"], state["width"], state["longest"], state["case"]["page"]
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    q_in = t["q_out"] if case["kind"] == "step" else t["q"]
    cu, lens = t["cu_q_lens"], t["seq_lens"]
    n = (cu[1:] - cu[:-1])[:, None]
    i = torch.arange(W, device=DEVICE)
    at = (cu[:-1, None] + i).clamp(max=q_in.shape[0] - 1)         # [B, W]: packed row of query i
    j = torch.arange(L, device=DEVICE)
    pages = t["block_table"][:, :-(-L // P)].clamp(min=0)
    # every sequence as long as the longest: [B, hkv, L, d]
    k = t["k_cache"][pages].flatten(1, 2)[:, :L].float().permute(0, 2, 3, 1).reshape(B * hkv, d, L).contiguous()
    q = q_in[at].float().reshape(B, W, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B * hkv, W * (hq // hkv), d)
    x = torch.bmm(q * d ** -0.5, k).reshape(B, hkv, W, hq // hkv, L)
    del k
    node = j[None, :] - (lens[:, None] - n)                       # [B, L]: number among the drafted tokens, < 0 in the context
    bit = node.clamp(min=0, max=64 * t["tree_mask"].shape[1] - 1)
    word = t["tree_mask"][at].gather(2, (bit // 64)[:, None, :].expand(B, W, L))
    seen = ((word >> (bit % 64)[:, None, :]) & 1 > 0) | (node < 0)[:, None, :]
    seen &= (j < lens[:, None])[:, None, :]
    del word
    x.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = t["v_cache"][pages].flatten(1, 2)[:, :L].float().permute(0, 2, 1, 3).reshape(B * hkv, L, d).contiguous()
    o = torch.bmm(x.reshape(B * hkv, -1, L), v).reshape(B, hkv, W, hq // hkv, d) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, W, hq)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, W, hq, d)
    # back to packed rows; those behind the last sequence stay as they were
    r = torch.arange(q_in.shape[0], device=DEVICE)
    s = torch.searchsorted(cu, r, right=True).clamp(max=B) - 1
    live = r < cu[-1]
    i = (r - cu[s]).clamp(max=W - 1)
    t["out"].copy_(torch.where(live[:, None, None], o[s, i].to(q_in.dtype), t["out"]))
    t["lse"].copy_(torch.where(live[:, None], lse[s, i], t["lse"]))


def _accept(state, t):
    W, P = state["width"], state["case"]["page"]
    cu, lens, table = t["cu_q_lens"], t["seq_lens"], t["block_table"]
    n = (cu[1:] - cu[:-1])[:, None]
    i = torch.arange(W, device=DEVICE)
    at = (cu[:-1, None] + i).clamp(max=t["tokens"].shape[0] - 1)
    live = i < n
    up = t["parents"][at]
    chosen = live & (up >= 0) & (t["tokens"][at] == t["targets"][at].gather(1, up.clamp(min=0).long()))
    # of a node's chosen children the first; a token stays if it and all that it follows are such, from the first token on
    same = (up[:, :, None] == up[:, None, :]) & chosen[:, None, :] & (i[None, :] < i[:, None])
    link = (chosen & ~same.any(2)) | (i == 0) & live
    stays = live & ~(_ancestors(state, cu, t["parents"]) & ~link[:, None, :]).any(2)
    count = stays.sum(1)
    path = torch.where(stays, i, W).sort(1).values
    path = torch.where(path < W, path, -1)
    t["path"].copy_(path)
    t["path_lens"].copy_(count)
    last = path.gather(1, (count - 1).clamp(min=0)[:, None]).clamp(min=0)
    t["next_tokens"].copy_(torch.where(count > 0, t["targets"][at].gather(1, last)[:, 0], -1))
    ctx = lens - n[:, 0]
    t["kept_lens"].copy_(ctx + count)
    # rows of the cache: all read, then all written; where there is nothing to move, the row of the first token onto itself
    b = torch.arange(lens.shape[0], device=DEVICE)[:, None]
    src = ctx[:, None] + path.clamp(min=0)
    dst = ctx[:, None] + torch.where(path >= 0, i, 0)
    first = ctx[:, None] + torch.where(count > 0, path[:, 0], 0)[:, None]
    src = torch.where(path >= 0, src, first)
    src, dst = src.clamp(min=0), dst.clamp(min=0)
    src_page, dst_page = table[b, src // P], table[b, dst // P]
    t["k_cache"][dst_page, dst % P] = t["k_cache"][src_page, src % P]
    t["v_cache"][dst_page, dst % P] = t["v_cache"][src_page, src % P]


# ---- what a pass has to do, and its results in 64 bits -------------------------------------------------------------

def work(case):
    ctx, new = _lengths(case)
    kind, P = case["kind"], case["page"]
    B, T, W = len(ctx), sum(new), max(new)
    e = 4 if case["dtype"] == "fp32" else 2
    row, words = case["hkv"] * case["d"] * e, -(-W // 64)
    bytes_ = flops = 0
    if kind in ("plan", "step"):
        pages = sum(-(-(a + b) // P) - -(-a // P) for a, b in zip(ctx, new))
        bytes_ += 4 * (6 * B + 4 * T) + 8 * words * T + 16 * pages
        flops += T
    if kind in ("rope", "accept", "step"):
        bytes_ += T * (2 * case["hq"] * case["d"] * e + 4 * row + 12) + 4 * case["rot"]
        flops += 3 * T * case["rot"] * (case["hq"] + case["hkv"])
    if kind in ("tree", "step"):
        seen = sum(n * b for n, b in zip(ctx, new)) + T          # at least: the context and the token itself
        bytes_ += 2 * row * (sum(ctx) + T) + T * (2 * case["hq"] * case["d"] * e + 4 * case["hq"] + 8 * words)
        flops += 4 * case["d"] * case["hq"] * seen
    if kind in ("accept", "step"):
        bytes_ += 12 * T + 4 * B * (W + 6) + 2 * 2 * row * B      # a moved row or so of each sequence
        flops += T
    return {"bytes": bytes_, "flops": flops}


def exact(case, seed):
    """In 64 bits, sequence by sequence; None for whole numbers."""
    kind = case["kind"]
    if kind == "plan":
        return None
    t = _inputs(case, seed)
    ctx, new = _lengths(case)
    parents, tokens, targets = _trees(case, new, seed)
    res = {n: None for n in OUTPUTS[kind]}
    P, hq, hkv, d = case["page"], case["hq"], case["hkv"], case["d"]
    G, first = hq // hkv, np.cumsum([0] + new)
    table = t["block_table"].cpu().numpy().copy()
    if kind == "step":                                            # the plan: pages from the end of the free list
        free = t["free_pages"].cpu().numpy()[:int(t["free_count"][0])].tolist()
        for s in range(len(ctx)):
            for b in range(-(-ctx[s] // P), -(-(ctx[s] + new[s]) // P)):
                table[s, b] = free.pop()
    follows = []                                                  # per sequence: node -> the nodes it follows, and itself
    for s in range(len(ctx)):
        m = np.eye(new[s], dtype=bool)
        if kind != "rope":
            for i in range(1, new[s]):
                m[i] |= m[parents[s, i]]
        follows.append(m)
    q = t["q"].double()
    k_cache, v_cache = t["k_cache"], t["v_cache"]
    if kind != "tree":
        f, mscale = _frequencies(case)
        k_cache, v_cache = k_cache.double(), v_cache.double()
        z_rows = []
        for s in range(len(ctx)):
            depth = np.arange(new[s]) if kind == "rope" else follows[s].sum(1) - 1
            z_rows.append(np.outer((ctx[s] + depth).astype(np.float64), f))
        z = np.concatenate(z_rows + [np.zeros((case["pad"], case["rot"] // 2))])
        z = torch.from_numpy(mscale * np.exp(1j * z)).to(DEVICE)[:, None]   # a pair as a complex number, turned by a product

        def spin(x):
            x, r = x.double(), case["rot"]
            lead = x[..., :r].unflatten(-1, (-1, 2) if case["inter"] else (2, -1))
            lead = lead if case["inter"] else lead.transpose(-1, -2)
            lead = torch.view_as_real(torch.view_as_complex(lead.contiguous()) * z)
            lead = lead if case["inter"] else lead.transpose(-1, -2)
            return torch.cat([lead.flatten(-2), x[..., r:]], -1)

        q, k_rows = spin(t["q"]), spin(t["k_new"])
        res["q_out"] = q
        for s in range(len(ctx)):
            pos = np.arange(ctx[s], ctx[s] + new[s])
            page, place = (torch.from_numpy(x).to(DEVICE) for x in (table[s, pos // P].astype(np.int64), pos % P))
            k_cache[page, place] = k_rows[first[s]:first[s + 1]]
            v_cache[page, place] = t["v_new"][first[s]:first[s + 1]].double()
    if kind in ("tree", "step"):
        out = torch.zeros(t["q"].shape, dtype=torch.float64, device=DEVICE)
        lse = torch.zeros(t["q"].shape[:2], dtype=torch.float64, device=DEVICE)
        # (q and K as the operator before it rounds them: what attention is given)
        dtype = t["q"].dtype
        q_in = q.to(dtype).double()
        for s in range(len(ctx)):
            n = ctx[s] + new[s]
            pages = torch.from_numpy(table[s, :-(-n // P)].astype(np.int64)).to(DEVICE)
            rows = slice(int(first[s]), int(first[s + 1]))
            hidden = torch.from_numpy(~follows[s]).to(DEVICE)
            for g in range(hkv):
                k = k_cache[pages, :, g].reshape(-1, d)[:n].to(dtype).double().t().contiguous()
                v = v_cache[pages, :, g].reshape(-1, d)[:n].double()
                for h in range(g * G, (g + 1) * G):
                    x = q_in[rows, h] @ k * d ** -0.5
                    x[:, ctx[s]:] = x[:, ctx[s]:].masked_fill(hidden, -math.inf)
                    lse[rows, h] = torch.logsumexp(x, dim=1)
                    out[rows, h] = torch.exp(x - lse[rows, h][:, None]) @ v
        res["out"], res["lse"] = out, lse
    if kind in ("accept", "step"):
        for s in range(len(ctx)):
            path = [0]
            while True:
                hits = [c for c in range(1, new[s]) if parents[s, c] == path[-1] and tokens[s, c] == targets[s, path[-1]]]
                if not hits:
                    break
                path.append(hits[0])
            src, dst = ctx[s] + np.array(path), ctx[s] + np.arange(len(path))
            page, place, to_page, to_place = (torch.from_numpy(x.astype(np.int64)).to(DEVICE)
                                              for x in (table[s, src // P], src % P, table[s, dst // P], dst % P))
            for c in (k_cache, v_cache):
                c[to_page, to_place] = c[page, place].clone()
    if kind != "tree":
        res["k_cache"], res["v_cache"] = k_cache, v_cache
    return res
