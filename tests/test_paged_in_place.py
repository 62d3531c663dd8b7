"""Attention over a paged cache into the rows of its queries."""
import pytest
import torch

from test_paged_refusals import FAKE, VALID, L, batch, cache, no_gpu, refused, rows  # noqa: F401  (L is a fixture)


@pytest.mark.parametrize("out,dtype,tokens,status", [
    (dict(token=8192), 0, 2, -1), (dict(head=256, token=4096 * 4), 0, 2, -1), (dict(token=4096), 1, 2, -1), (dict(token=4096), 1, 1, -1),
    (dict(token=4096), 0, 2, VALID), (dict(token=8192), 0, 1, VALID), (dict(token=8192, data=FAKE + (1 << 20)), 0, 2, VALID),
    (dict(token=8192, data=FAKE + (1 << 20)), 1, 2, VALID)])
def test_other_rows_in_the_place_of_the_queries_are_refused(L, out, dtype, tokens, status):  # noqa: F811
    if status == VALID:
        no_gpu()
    refused(L, L.lib().efq_attn_paged(rows(L, token=4096), 32, cache(L), batch(L, tokens=tokens), 0.1, 1, rows(L, **out), dtype, None,
                                      None, 0, None), status)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("heads,D", [((4, 1), 128), ((16, 2), 64)])
@pytest.mark.parametrize("new,keys,split", [
    ([1, 0, 3], [700, 5, 40], False), ([1, 1], [9000, 3000], True), ([40, 7], [500, 2000], True), ([130, 300], [200, 1000], False),
    ([90], [6000], True)])
def test_in_place(L, new, keys, split, heads, D, fmt):  # noqa: F811
    from test_paged_attention import Case
    c = Case(L, new, keys, heads, D, 16, fmt, seed=50, pad=2)
    print(f"[in place] {(new, keys, heads, D, fmt, split)}", flush=True)
    ws = None if split else torch.empty(0, dtype=torch.uint8, device="cuda")
    want = torch.empty(c.q.shape, dtype=torch.bfloat16, device="cuda")
    L.attn_paged(c.q.cuda(), c.cache, c.batch, out=want, workspace=ws)
    full = torch.randn(len(c.q), heads[0] + 2, D, generator=torch.Generator().manual_seed(51)).bfloat16().cuda()
    full[:, 1:-1] = c.q.cuda()
    keep, q = full.clone(), full[:, 1:-1]
    assert L.attn_paged(q, c.cache, c.batch, out=q, workspace=ws) is q
    n = c.starts[-1]
    keep[:n, 1:-1] = want[:n]                        # padding and the heads beside stay
    assert torch.equal(full, keep)
