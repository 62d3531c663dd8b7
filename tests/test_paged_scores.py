"""Attention over a paged cache where the running softmax can go wrong: scores
that climb or fall along the keys, many equal ones, first pages that are none
before very low scores, and bad pages deep in a piece that is not split."""
import pytest
import torch

from test_paged_attention import Case, check, run
from test_paged_use import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


def along(B, new, keys, heads, D, shape, page=64, seed=20):
    """A case whose scores (in powers of e, of every row) are shape(t) at key t, plus those of small random parts:
    q's first 32 elements are 1, a key's are shape(t) / 32 (rounded to bf16)."""
    c = Case(B, new, keys, heads, D, page, "bf16", seed=seed, spread=0.25)
    c.q[..., :32] = 1.0
    kc = c.cache.k.cpu()
    for i, n in enumerate(keys):
        c.k[i][..., :32] = (shape(torch.arange(n, dtype=torch.float64)) / 32).bfloat16()[:, None, None]
        for j in range(-(-n // page)):
            m = min(page, n - j * page)
            kc[c.table[i, j], :, :m] = c.k[i][j * page: j * page + m].transpose(0, 1)
    c.cache = B.PagedCache(kc.cuda(), c.cache.v)
    return c


SHAPES = {
    "climbs": lambda t: t * 0.05,
    "climbs a power of e a key": lambda t: t * 1.0 - 1000,
    "steps up": lambda t: 11.0 * torch.floor(t / 100),
    "just under the step": lambda t: torch.where(t < 64, 0.0, 11.0),
    "equal": lambda t: t * 0,
    "falls": lambda t: 80 - t * 0.5,
    "one high": lambda t: torch.where(t == 777, 90.0, -90.0),
    "low": lambda t: t * 0 - 3000,
}


@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("new,heads,D", [([1, 1], (4, 1), 128), ([7], (4, 1), 128), ([150, 20], (4, 2), 128), ([200], (2, 1), 64)])
def test_scores_along_the_keys(B, shape, new, heads, D):
    keys = [1500, 1100][:len(new)]
    c = along(B, new, keys, heads, D, SHAPES[shape])
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out, lse, scale = run(B, c, scale=1.0, dtype=torch.float32, **({} if ws is None else dict(workspace=ws)))
        check(c, out, lse, scale, True)


@pytest.mark.parametrize("new,heads", [([1], (2, 1)), ([40], (8, 1))])
def test_many_equal_keys(B, new, heads):
    """A sum past 2^16 of probabilities of 1: 100000 keys, in one piece and in many."""
    c = along(B, new, [100000], heads, 64, SHAPES["equal"], page=256)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out, lse, scale = run(B, c, scale=1.0, dtype=torch.float32, **({} if ws is None else dict(workspace=ws)))
        check(c, out, lse, scale, True)


@pytest.mark.parametrize("bad", [1, 4, 7, 9])
@pytest.mark.parametrize("new,heads", [([1], (4, 1)), ([6], (4, 1)), ([100], (4, 1))])
def test_none_before_low_scores(B, bad, new, heads):
    """The first `bad` pages of 16 are none, what follows scores about e^-3000: no reference stays from where
    nothing was seen."""
    c = along(B, new, [400], heads, 128, SHAPES["low"], page=16)
    table = c.table.clone()
    table[0, :bad] = -1
    hidden = [torch.arange(400) < 16 * bad]
    c.batch = B.PagedBatch(i32(c.starts), i32([400]), table.cuda(), max_q=new[0], max_k=400)
    out, lse, scale = run(B, c, scale=1.0, dtype=torch.float32)
    check(c, out, lse, scale, True, hidden)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
def test_bad_pages_deep_in_one_piece(B, fmt, D, page):
    """9000 keys in one piece (140 tiles of 64, whose pages are looked up in groups), with bad pages around the
    groups' ends."""
    keys = 9000
    c = Case(B, [70], [keys], (4, 1), D, page, fmt, seed=21)
    table, hidden = c.table.clone(), torch.zeros(keys, dtype=torch.bool)
    for key in (64 * 59, 64 * 60, 64 * 61 + 16, 64 * 62, 64 * 63 + 48, 64 * 64, 64 * 65 + 32, 64 * 66, 64 * 67,
                64 * 125 + 16, 64 * 127, 64 * 128, 64 * 130 + 48, 64 * 139):
        j = key // page
        table[0, j] = c.cache.pages if key & 64 else -1
        hidden[j * page: j * page + page] = True
    c.batch = B.PagedBatch(i32(c.starts), i32([keys]), table.cuda(), max_q=70, max_k=keys)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out, lse, scale = run(B, c, **({} if ws is None else dict(workspace=ws)))
        check(c, out, lse, scale, True, [hidden])
