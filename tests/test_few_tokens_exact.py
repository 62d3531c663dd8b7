"""Attention of one or a few tokens over a paged cache to fp32's error: the second
product takes each probability to 2^-16 of itself."""
import pytest
import torch

from test_paged_attention import Case, run
from test_paged_scores import SHAPES, along

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


def check_exact(c, out, scale, causal=True):
    """A probability is off by 2^-16 of itself (its bf16 leaves at most 2^-8, whose bf16 leaves 2^-8 of that), by its score's
    error as in check (twice, against the row's others) and by a few 2^-24 of the exponential; the fp32 sums of
    products and of probabilities have at most a rounding a key, 2^-24 of the sum of absolute products, and the parts and
    the quotient some more.  Then the output's own rounding."""
    ref, _, mag, size = c.reference(scale, causal)
    T = c.starts[-1]
    got = out[:T].double().cpu()
    d = (c.D + 8) * 2.0 ** -24 * size + 2.0 ** -20
    tol = (2.0 ** -16 + 2 * d + (2 * max(c.keys) + 32) * 2.0 ** -24)[..., None] * mag + 1e-30
    if out.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
    worst = float(((got - ref).abs() / tol).max())
    assert worst <= 1, worst


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,D", [((4, 1), 128), ((8, 8), 128), ((8, 2), 64), ((16, 1), 64)])
@pytest.mark.parametrize("new,keys", [([1], [1]), ([1, 1, 1], [31, 129, 700]), ([1], [5000]), ([2, 2, 1], [40, 5, 333]), ([0, 1], [9, 2600])])
def test_outputs(B, new, keys, heads, D, dtype, fmt):
    c = Case(B, new, keys, heads, D, 16, fmt, seed=60 + len(new), pad=1, spread=1.5)
    out, _, scale = run(B, c, dtype=dtype)
    check_exact(c, out, scale)


@pytest.mark.parametrize("new,keys,heads,D,fmt", [([8], [900], (4, 1), 128, "bf16"), ([16, 3], [400, 2000], (4, 1), 128, "mxfp8"),
                                                 ([7, 30], [7, 1500], (4, 2), 64, "bf16"), ([5], [20000], (4, 1), 64, "mxfp8")])
def test_several_tokens(B, new, keys, heads, D, fmt):
    c = Case(B, new, keys, heads, D, 64, fmt, seed=70, spread=2.0)
    for causal in (True, False):
        for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
            out, _, scale = run(B, c, causal=causal, dtype=torch.float32, **({} if ws is None else dict(workspace=ws)))
            check_exact(c, out, scale, causal)


@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_scores_along_the_keys(B, shape):
    """Probabilities that underflow beside their row's largest, many equal ones, maxima that move."""
    c = along(B, [1, 2], [1500, 1100], (4, 1), 128, SHAPES[shape])
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out, _, scale = run(B, c, scale=1.0, dtype=torch.float32, **({} if ws is None else dict(workspace=ws)))
        check_exact(c, out, scale)
