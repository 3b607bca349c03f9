"""Attention of drafted trees where its weights and sums could lose something: weights that have to cancel, one key far ahead of all
others, infinities in K behind a head_dim that no tile is as wide as, values near the type's largest."""
import numpy as np
import pytest
import torch

from tests import step_reference as R
from tests.test_gpu_step import any_mask, half_step, make_tree_call, pa, run_tree  # noqa: F401

pytestmark = pytest.mark.gpu


def put(c, which, s, keys, value):
    """K or V ("k", "v") rows of some keys of sequence s of a token-major call: on the device and in the reference's copy."""
    seq = c["seqs"][s][0 if which == "k" else 1]
    P, table = c[which].shape[1], c["table"][s].cpu()
    keys = torch.as_tensor(np.asarray(keys), dtype=torch.int64)
    seq[keys] = torch.as_tensor(value).to(seq.dtype)
    c[which][table[keys // P].long().to(c[which].device), (keys % P).to(c[which].device)] = seq[keys].to(c[which].device)


def reference(c):
    """Per sequence: its rows, out and lse in 64 bits, the largest |v|."""
    row = 0
    for s, n in enumerate(c["news"]):
        k, v = (x.double().numpy() for x in c["seqs"][s])
        q = c["q"][row:row + n].double().cpu().numpy()
        with np.errstate(invalid="ignore", over="ignore"):
            out, lse = R.tree_attention(k, v, q, c["masks"][s], c["host_lens"][s] - n, c["scale"])
        yield slice(row, row + n), out, lse, np.abs(v).max() if v.size else 0.0
        row += n


def causal(s, n):
    return np.tril(np.ones((n, n)))


def awkward(dtype, count):
    """Numbers a > 0 of the type's own whose e^-a is nearly as far from the type's values as can be."""
    found = []
    for a in torch.arange(0.2, 1.0, 1 / 512).to(dtype).unique().double().tolist():
        w = np.exp(-a)
        step = half_step(dtype) * 2.0 ** np.floor(np.log2(w))
        if abs(float(torch.tensor(w).to(dtype).double()) - w) > 0.8 * step:
            found.append(a)
    return found[::max(1, len(found) // count)][:count]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,G,lens,news,loose", [
    (128, 1, [300], [5], 0), (128, 2, [1040, 700], [40, 3], 0), (64, 4, [300, 280], [33, 7], 0), (128, 8, [640], [40], 0),
    (256, 2, [900], [64], 0), (96, 4, [2000], [20], 0), (128, 4, [200], [20], 4096)])
def test_weights_that_cancel(pa, d, G, lens, news, loose, dtype):  # noqa: F811
    """Half of the keys weigh 1, with v = 1, the others w, with v = the type's value next to -1 / w: what is left of the sum is
    about as large as a weight rounded to the type would be off by.  Weights are two terms: 2^-16 and better, with 32-bit sums
    3e-5 of max |v| together, as for any other call; also where the bound on contexts is loose (`loose`)."""
    a = awkward(dtype, 4)
    c = make_tree_call(lens, news, 4 * G, 4, d, 16, dtype, causal, seed=2)
    c["q"].fill_(1.0)
    c["scale"] = 1.0 / d
    for s, n in enumerate(lens):
        odd = torch.arange(n) % 2 == 1
        k, v = torch.zeros(n, 4, d), torch.ones(n, 4, d)
        for h, x in enumerate(a):
            k[odd, h], v[odd, h] = -x, -float(np.exp(x))
        put(c, "k", s, np.arange(n), k), put(c, "v", s, np.arange(n), v)
    if loose:
        wide = torch.full((len(lens), loose // 16), -1, dtype=torch.int32, device=c["q"].device)
        wide[:, :c["table"].shape[1]] = c["table"]
        c["table"] = wide
    out, lse = run_tree(pa, c, max_len=loose or None)
    for rows, ref, ref_lse, vmax in reference(c):
        over = np.abs(out[rows].double().cpu().numpy() - ref) - (half_step(dtype) * np.abs(ref) + 3e-5 * vmax)
        assert (over <= 0).all(), float(over.max())
        assert (np.abs(lse[rows].double().cpu().numpy() - ref_lse) <= 2e-5 + 2e-6 * np.abs(ref_lse)).all()


@pytest.mark.parametrize("n", [1, 8, 40])
@pytest.mark.parametrize("d", [64, 80, 128, 256])
@pytest.mark.parametrize("lead,at", [(12.0, 0), (17.0, 7000), (17.0, 3)])
def test_fp16_weights_far_below_the_largest_are_not_lost(pa, d, n, lead, at):  # noqa: F811
    """One key of 8000 leads all others by e^17: each of them weighs 2^-24.5 of it, together 3e-4, and the leading key's values are
    0.  A weight is kept to 2^-36 of the largest, 8000 of them to 8000 * 2^-36 of max |v| = 1; exponentials of scores up to 17
    and 32-bit sums to 2^-17 of the result; then fp16's half step."""
    length = 8000
    c = make_tree_call([length, 500], [n, 1], 8, 2, d, 16, torch.float16, causal, seed=3)
    c["q"].fill_(1.0)
    c["scale"] = 1.0
    for s, m in enumerate(c["host_lens"]):
        put(c, "k", s, np.arange(m), torch.zeros(m, 2, d)), put(c, "v", s, np.arange(m), torch.ones(m, 2, d))
        put(c, "k", s, [min(at, 400)] if s else [at], lead / d), put(c, "v", s, [min(at, 400)] if s else [at], 0.0)
    out, lse = run_tree(pa, c)
    for rows, ref, ref_lse, _ in reference(c):
        near = (2.0 ** -11 + 2.0 ** -17) * np.abs(ref) + length * 2.0 ** -36
        tiny = 2.0 ** -25                                         # (half a step of subnormal results)
        assert (np.abs(out[rows].double().cpu().numpy() - ref) <= np.maximum(near, tiny)).all()
        assert (np.abs(lse[rows].double().cpu().numpy() - ref_lse) <= 2e-5 + 2e-6 * np.abs(ref_lse)).all()


@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("dtype,d", [(t, d) for t in (torch.bfloat16, torch.float16) for d in (40, 64, 72, 80, 112, 128, 200, 256)] +
                         [(torch.float32, d) for d in (40, 64, 80, 200)])
@pytest.mark.parametrize("portable", [False, True])
def test_what_a_query_gets_that_sees_an_infinity_in_k(pa, portable, dtype, d, n):  # noqa: F811
    """Where the score is -inf the key weighs nothing; where it is inf the result is NaN, as e^(inf - inf) is.  Tiles are wider than
    most of these head_dims: what stands behind them must not meet the infinity."""
    from paper_2506_07311_amd import binding
    for length, at in ((90 + n, 70), (90 + n, 90), (1500 + n, 700)):
        c = make_tree_call([length, 65], [n, 2], 8, 2, d, 16, dtype, any_mask(5) if n > 1 else causal, seed=d)
        k = c["seqs"][0][0][at].clone()
        k[:, 3] = float("inf")
        put(c, "k", 0, [at], k[None])
        binding.pa_set_option("force_generic", 1 if portable else 0)
        try:
            out, lse = run_tree(pa, c)
        finally:
            binding.pa_set_option("force_generic", 0)
        for rows, ref, ref_lse, vmax in reference(c):
            got, got_lse = out[rows].double().cpu().numpy(), lse[rows].double().cpu().numpy()
            bad = np.isnan(ref)
            assert np.array_equal(np.isnan(got), bad) and np.array_equal(np.isnan(got_lse), np.isnan(ref_lse))
            assert rows.start > 0 or n == 1 or bad.any() and not bad.all()
            near = half_step(dtype) * np.abs(ref[~bad]) + 3e-5 * vmax
            assert (np.abs(got[~bad] - ref[~bad]) <= near).all()


@pytest.mark.parametrize("portable", [False, True])
@pytest.mark.parametrize("n", [1, 12, 70])
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 256), (torch.float32, 64),
                                     (torch.float32, 128), (torch.float32, 256)])
@pytest.mark.parametrize("length", [100, 3000])
def test_means_of_values_near_the_largest_are_finite(pa, length, dtype, d, n, portable):  # noqa: F811
    """A mean of finite values is finite, however many there are and although later keys outweigh the first ones by e^6.
    Values: 3e38 for all of a column, of either sign at random in the others."""
    from paper_2506_07311_amd import binding
    c = make_tree_call([length + n, 70], [n, 2], 8, 2, d, 16, dtype, causal, seed=5)
    g = torch.Generator().manual_seed(6)
    c["q"].fill_(1.0)
    c["scale"] = 1.0
    for s, m in enumerate(c["host_lens"]):
        k = torch.full((m, 2, d), 6.0 / d)
        k[:m // 3] = 0.0
        v = 3e38 * torch.randint(0, 2, (m, 2, d), generator=g).mul(2).sub(1)
        v[..., ::3] = 3e38
        v[..., 1::3] = -3e38
        put(c, "k", s, np.arange(m), k), put(c, "v", s, np.arange(m), v)
    binding.pa_set_option("force_generic", 1 if portable else 0)
    try:
        out, lse = run_tree(pa, c)
    finally:
        binding.pa_set_option("force_generic", 0)
    for rows, ref, ref_lse, vmax in reference(c):
        got = out[rows].double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got / vmax - ref / vmax) <= half_step(dtype) * np.abs(ref / vmax) + 3e-5).all()
        assert (np.abs(lse[rows].double().cpu().numpy() - ref_lse) <= 2e-5 + 2e-6 * np.abs(ref_lse)).all()
