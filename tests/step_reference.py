"""A step of drafted tokens by its definitions, in Python integers and 64-bit numpy: what the GPU's operators are compared with."""
import numpy as np


def blocks(tokens, page):
    return -(-int(tokens) // page)


def plan(ctx, new, parents, table, num_blocks, free, page, max_rows, words):
    """paged_plan_step on copies; parents: packed list or None.  Returns a dict of everything the call writes (free: the
    stack's live part)."""
    table, num_blocks, free = np.array(table), list(num_blocks), list(free)
    B, MB = table.shape
    new = [max(int(n), 0) for n in new]
    need = sum(max(blocks(c + n, page) - k, 0) for c, n, k in zip(ctx, new, num_blocks))
    late = sum(blocks(c + n, page) > MB or n > 64 * words for c, n in zip(ctx, new)) + max(sum(new) - max_rows, 0)
    short = [max(need - len(free), 0), late]
    ok = short == [0, 0]
    res = dict(seq_ids=[], positions=[], rope_positions=[], tree_mask=[], shortage=short,
               seq_lens=[c + n if ok else c for c, n in zip(ctx, new)], cu_q_lens=[0] * (B + 1))
    for s in range(B):
        if ok:
            res["cu_q_lens"][s + 1] = res["cu_q_lens"][s] + new[s]
            while num_blocks[s] < blocks(ctx[s] + new[s], page):
                table[s, num_blocks[s]] = free.pop()
                num_blocks[s] += 1
        start = sum(new[:s])
        masks, depths = [], []
        for i in range(new[s]):
            up = i - 1 if parents is None else (int(parents[start + i]) if start + i < max_rows else -1)
            up = up if 0 <= up < i else -1
            masks.append((masks[up] if up >= 0 else 0) | 1 << i)
            depths.append(depths[up] + 1 if up >= 0 else 0)
            res["seq_ids"].append(s)
            res["positions"].append(ctx[s] + i)
            res["rope_positions"].append(ctx[s] + depths[-1])
            res["tree_mask"].append([masks[-1] >> (64 * w) & (1 << 64) - 1 for w in range(words)])
    for name, fill in (("seq_ids", -1), ("positions", -1), ("rope_positions", 0), ("tree_mask", [0] * words)):
        res[name] = (res[name] + [fill] * max_rows)[:max_rows]
    res.update(block_table=table, num_blocks=num_blocks, free=free)
    return res


def release(keep, table, num_blocks, free, page):
    table, num_blocks, free = np.array(table), list(num_blocks), list(free)
    back = []
    for s in range(len(keep)):
        for b in range(blocks(keep[s], page), num_blocks[s]):
            back.append(table[s, b])
            table[s, b] = -1
        num_blocks[s] = min(num_blocks[s], blocks(keep[s], page))
    return dict(block_table=table, num_blocks=num_blocks, free=free + back[::-1])


def rope(x, positions, inv_freq, interleaved, mscale):
    """x [T, heads, d] in 64 bits."""
    x = np.array(x, dtype=np.float64)
    r = 2 * len(inv_freq)
    z = mscale * np.exp(1j * np.outer(np.asarray(positions, np.float64), inv_freq))[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    y = (a + 1j * b) * z
    out = x.copy()
    if interleaved:
        out[..., 0:r:2], out[..., 1:r:2] = y.real, y.imag
    else:
        out[..., :r // 2], out[..., r // 2:r] = y.real, y.imag
    return out


def tree_attention(k, v, q, mask, ctx, scale, spread=False):
    """One sequence: k, v [len, hkv, d], q [n, hq, d], mask [n, n] (query, drafted key).  Returns out, lse; and with spread
    sqrt(sum p^2 v^2) / sum p, what independent relative errors of the weights p, of deviation 1, do to out."""
    n, hq, d = q.shape
    wide = np.zeros((n, hq, d))
    G = hq // k.shape[1]
    seen = np.concatenate([np.ones((n, ctx), bool), np.asarray(mask, bool)], 1)
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    for h in range(hq):
        for i in range(n):
            j = np.nonzero(seen[i])[0]
            if len(j) == 0:
                continue
            x = k[j, h // G] @ q[i, h] * scale
            m = x.max()
            p = np.exp(x - m)
            out[i, h] = p @ v[j, h // G] / p.sum()
            lse[i, h] = m + np.log(p.sum())
            wide[i, h] = np.sqrt(p ** 2 @ v[j, h // G] ** 2) / p.sum()
    return (out, lse, wide) if spread else (out, lse)


def accept(parents, tokens, targets, max_path):
    """One sequence's path and next token."""
    n = len(tokens)
    if n == 0:
        return [], -1
    path = [0]
    while len(path) < max_path:
        hits = [c for c in range(path[-1] + 1, n) if parents[c] == path[-1] and tokens[c] == targets[path[-1]]]
        if not hits:
            break
        path.append(hits[0])
    return path, targets[path[-1]]
