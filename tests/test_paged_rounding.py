"""What the rounding of the probabilities to bf16 may cost in attention of many
tokens over a paged cache: O is a mean of values weighted by the rounded ones."""
import math

import pytest
import torch

from test_paged_attention import Case, run
from test_paged_scores import along

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


def weights(c, i, scale, causal=True):
    """Probabilities [n, hq, s] of sequence i in 64 bits, and each row's largest sum of a score's absolute products."""
    hq, hkv = c.heads
    n, s = c.new[i], c.keys[i]
    q = c.q[c.starts[i]: c.starts[i] + n].double()
    k = c.k[i].double().repeat_interleave(hq // hkv, 1)
    x = torch.einsum("nhd,shd->nhs", q, k) * scale
    if causal:
        x = x.masked_fill((torch.arange(s)[None] > (s - n + torch.arange(n))[:, None])[:, None], -math.inf)
    return torch.softmax(x, -1), torch.einsum("nhd,shd->nhs", q.abs(), k.abs()).amax(-1) * scale


def check_mean(c, out, scale, causal=True):
    """With weights p_i (1 + e_i), |e_i| <= e, the mean o' of the values is off their mean o under p by
    sum p_i e_i (v_i - o) / sum p_i (1 + e_i), so by at most e / (1 - e) sum p_i |v_i - o|.  e: 2^-8 of the rounding
    to bf16, and of the scores in fp32 (d) and the exponential (2^-20) as in check.  The fp32 sums of products
    and of weights have at most a rounding a key, 2^-24 of the sum of absolute products each."""
    for i, s in enumerate(c.keys):
        if not c.new[i]:
            continue
        p, size = weights(c, i, scale, causal)
        v = c.v[i].double().repeat_interleave(c.heads[0] // c.heads[1], 1)
        got = out[c.starts[i]: c.starts[i] + c.new[i]].double().cpu()
        ref = torch.einsum("nhs,shd->nhd", p, v)
        mag = torch.einsum("nhs,shd->nhd", p, v.abs())
        for j in range(c.new[i]):
            e = 2.0 ** -8 + 2 * ((c.D + 8) * 2.0 ** -24 * size[j] + 2.0 ** -20)
            spread = torch.einsum("hs,shd->hd", p[j], (v - ref[j]).abs())
            tol = (e / (1 - e))[:, None] * spread + 2 * s * 2.0 ** -24 * mag[j] + 2.0 ** -22 * ref[j].abs() + 1e-30
            worst = float(((got[j] - ref[j]).abs() / tol).max())
            assert worst <= 1, (i, j, worst)


# a key that dominates, at e^`by` over the rest of the row: 2^8.4, 2^11.7, 2^14.6 and 2^30 of them
@pytest.mark.parametrize("by", [5.83, 8.11, 10.12, 20.8])
@pytest.mark.parametrize("new,heads,D", [([130], (4, 1), 128), ([200], (2, 1), 64), ([90, 65], (8, 2), 64)])
def test_a_dominant_key(B, by, new, heads, D):
    """Its probability is rounded like the others, relative to a reference that does not follow it at once."""
    keys = [1500, 1100][:len(new)]
    c = along(B, new, keys, heads, D, lambda t: torch.where(t == 777, by, -6.0))
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out, _, scale = run(B, c, scale=1.0, dtype=torch.float32, **({} if ws is None else dict(workspace=ws)))
        check_mean(c, out, scale)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("new,keys,heads,D,causal", [
    ([70], [900], (4, 1), 128, True), ([300, 64], [300, 5000], (4, 2), 128, True), ([257], [700], (2, 1), 64, False),
    ([64, 40, 90], [1000, 40, 333], (16, 4), 64, True)])
def test_random_scores(B, new, keys, heads, D, fmt, causal):
    c = Case(B, new, keys, heads, D, 16, fmt, seed=41, spread=2.0)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out, _, scale = run(B, c, causal=causal, dtype=torch.float32, **({} if ws is None else dict(workspace=ws)))
        check_mean(c, out, scale, causal)


@pytest.mark.parametrize("new,keys,heads,D", [([150], [2500], (4, 1), 128), ([100, 128], [700, 128], (4, 2), 64)])
def test_equal_values(B, new, keys, heads, D):
    """Where every key has the same value, that value comes out, but for the fp32 sums."""
    c = Case(B, new, keys, heads, D, 64, "bf16", seed=42, spread=2.0)
    vc = torch.full_like(c.cache.v, 1.3)
    c.cache = B.PagedCache(c.cache.k, vc)
    c.v = [torch.full_like(v, 1.3) for v in c.v]
    out, _, _ = run(B, c, dtype=torch.float32)
    value = float(torch.tensor(1.3).bfloat16())
    # a rounding a key in each sum, the reciprocal and the product
    assert float((out[:sum(new)] - value).abs().max()) <= value * (2 * max(keys) + 8) * 2.0 ** -24
