"""Calls of the most tokens that rope and the append take: 2^26, whose launches have
to stay within the 2^32 - 1 threads of a grid (one broadcast row stands for the
tokens, so that little memory is needed)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MOST = 1 << 26


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens", [MOST, MOST - 5])
def test_rope(B, tokens, interleaved):
    print(f"[rope] {tokens} tokens", flush=True)
    row = torch.randn(1, 1, 16, device="cuda").bfloat16()
    inv = torch.tensor([1.0, 0.5, 0.2, 0.1, 0.05, 0.02, 0.01, 0.001], device="cuda")
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    y = B.rope(row.expand(tokens, 1, 16), pos, inv, interleaved=interleaved)
    for part in (slice(0, 100), slice((1 << 24) - 50, (1 << 24) + 50), slice(tokens - 100, tokens)):
        n = part.stop - part.start
        assert torch.equal(y[part], B.rope(row.expand(n, 1, 16), pos[part].contiguous(), inv, interleaved=interleaved))
    # no token left out: a turn keeps the row's norm, but for the rounding (2^-8 of a value, so 2^-7 + 2^-16 of a square)
    norm = float(row.float().square().sum())
    for part in y.split(1 << 24):
        off = (part.float().square().sum((1, 2)) - norm).abs().max()
        assert float(off) <= norm * (2.0 ** -7 + 2.0 ** -15)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_append(B, fmt):
    """All but the last 37 tokens belong to a sequence without keys, so nothing of them is kept."""
    print(f"[append] {MOST} tokens, {fmt}", flush=True)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    row = torch.randn(1, 1, 64, device="cuda").bfloat16()
    cache, want = (B.PagedCache.empty(4, 16, 1, 64, fmt) for _ in range(2))
    names = ("k", "v") + (("k_scale", "v_scale") if fmt == "mxfp8" else ())
    for n in names:
        getattr(cache, n).fill_(7), getattr(want, n).fill_(7)
    inv, pos = torch.rand(32, device="cuda"), torch.arange(MOST, dtype=torch.int32, device="cuda")
    x = row.expand(MOST, 1, 64)
    B.kv_append(x, x, cache, B.PagedBatch(i32([0, MOST - 37, MOST]), i32([0, 37]), i32([[0, 0, 0], [3, 0, 2]])), pos=pos, inv_freq=inv)
    B.kv_append(x[:37], x[:37], want, B.PagedBatch(i32([0, 37]), i32([37]), i32([[3, 0, 2]])), pos=pos[MOST - 37:].contiguous(),
                inv_freq=inv)
    for n in names:
        assert torch.equal(getattr(cache, n), getattr(want, n)), n
