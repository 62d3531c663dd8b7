"""What rope, kv_append and attn_paged refuse, before any HIP call (no kernel
runs), and the sizes of their scratch."""
import ctypes

import pytest
import torch

FAKE = 4096          # 16-byte aligned, never dereferenced


@pytest.fixture(scope="module")
def L():
    from paper_2609_09721_amd import binding
    binding.lib()
    return binding


def rows(L, data=FAKE, token=1024, head=128):
    return L.Rows(data, token, head)


def rotary(L, pairs=64, axes=1, inv=FAKE, axis=None, pos=FAKE):
    return L.Rotary(pairs, axes, 0, inv, axis, pos)


def cache(L, pages=8, page=16, heads=8, D=128, fmt=0, k=FAKE, v=FAKE, ks=None, vs=None):
    return L.Cache(pages, page, heads, D, fmt, k, v, ks, vs)


def batch(L, seqs=2, tokens=2, width=4, max_q=1, max_k=64, starts=FAKE, keys=FAKE, table=FAKE):
    return L.Batch(seqs, tokens, width, max_q, max_k, starts, keys, table)


VALID = -4           # EFQ_EHIP: past every check, where no GPU is


def no_gpu():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present: the call would run on these addresses")


def refused(L, rc, status):
    assert rc == status, L.lib().efq_strerror(rc).decode()
    assert L.lib().efq_strerror(rc).decode() not in ("", "ok")


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=-1), -1), (dict(heads=0), -1), (dict(heads=65537), -2), (dict(tokens=(1 << 26) + 1), -2),
    (dict(head_dim=0), -1), (dict(head_dim=72), -2), (dict(head_dim=528), -2), (dict(dtype=2), -1),
    (dict(x=dict(data=None)), -1), (dict(x=dict(data=4104)), -1), (dict(x=dict(token=1023)), -1), (dict(x=dict(head=-128)), -1),
    (dict(x=dict(token=1 << 33)), -1), (dict(y=dict(token=64)), -1), (dict(y=dict(head=64)), -1), (dict(y=dict(token=0)), -1),
    (dict(y=dict(token=512, head=128)), -1), (dict(y=dict(token=128, head=256)), -1),
    (dict(rot=dict(pairs=0)), -1), (dict(rot=dict(pairs=72)), -1), (dict(rot=dict(pairs=60)), -2), (dict(rot=dict(axes=0)), -1),
    (dict(rot=dict(inv=None)), -1), (dict(rot=dict(pos=None)), -1), (dict(rot=None), -1), (dict(), VALID),
    (dict(x=dict(token=0, head=0, data=FAKE + 65536)), VALID),    # a broadcast input
    (dict(x=dict(token=0, head=0)), -1), (dict(x=dict(token=2048)), -1), (dict(x=dict(token=2048), tokens=1), VALID),  # in place
    (dict(y=dict(token=128, head=128 * 5, data=FAKE + 65536)), VALID),      # heads outermost
    (dict(tokens=0, x=dict(data=None), y=dict(data=None)), 0)])
def test_rope(L, kw, status):
    if status == VALID:
        no_gpu()
    a = dict(tokens=5, heads=8, head_dim=128, dtype=0, x={}, y={}, rot={})
    a.update(kw)
    rot = None if a["rot"] is None else rotary(L, **a["rot"])
    rc = L.lib().efq_rope(rows(L, **a["x"]), rows(L, **a["y"]), a["tokens"], a["heads"], a["head_dim"], a["dtype"], rot, 0, None)
    assert rc == 0 if status == 0 else refused(L, rc, status) is None


CACHES = [(dict(pages=0), -1), (dict(heads=0), -1), (dict(D=96), -2), (dict(page=8), -2), (dict(page=48), -2), (dict(page=512), -2),
          (dict(fmt=2), -1), (dict(k=None), -1), (dict(v=4104), -1), (dict(fmt=1), -1), (dict(fmt=1, ks=FAKE, vs=4098), -1),
          (dict(fmt=1, ks=FAKE, vs=FAKE), VALID), (dict(page=256, D=64), VALID)]
BATCHES = [(dict(seqs=0), -1), (dict(seqs=(1 << 20) + 1), -2), (dict(width=0), -1), (dict(tokens=-1), -1), (dict(max_q=-1), -1),
           (dict(tokens=(1 << 26) + 1), -2), (dict(starts=None), -1), (dict(keys=None), -1), (dict(table=None), -1)]


@pytest.mark.parametrize("c,status", CACHES)
def test_caches(L, c, status):
    if status == VALID:
        no_gpu()
    D = c.get("D", 128)
    r = rows(L, token=32 * D, head=D)
    refused(L, L.lib().efq_kv_append(r, r, cache(L, **c), batch(L), None, None, 0, None, None), status)
    refused(L, L.lib().efq_attn_paged(r, 32 if c.get("heads") != 0 else 8, cache(L, **c), batch(L), 0.1, 1, r, 0, None, None, 0, None),
            status)
    if status != VALID:
        assert L.lib().efq_attn_paged_workspace_bytes(cache(L, **c), batch(L), 32) == 0


@pytest.mark.parametrize("b,status", BATCHES)
def test_batches(L, b, status):
    r = rows(L, token=4096)
    refused(L, L.lib().efq_kv_append(r, r, cache(L), batch(L, **b), None, None, 0, None, None), status)
    refused(L, L.lib().efq_attn_paged(r, 32, cache(L), batch(L, **b), 0.1, 1, r, 0, None, None, 0, None), status)


def test_append_arguments(L):
    lib, r, c, b = L.lib(), rows(L, token=4096), cache(L), batch(L)
    bad = rows(L, data=4098, token=4096)
    f = lambda k=r, v=r, rot=None, q=None, hq=0, o=None, bb=b: lib.efq_kv_append(k, v, c, bb, rot, q, hq, o, None)
    refused(L, f(k=None), -1)
    refused(L, f(v=bad), -1)
    refused(L, f(rot=rotary(L, pairs=72)), -1)
    refused(L, f(q=r, hq=0, o=r), -1)
    refused(L, f(hq=4), -1)                                          # heads without q
    refused(L, f(q=r, hq=32), -1)                                    # no q_out
    refused(L, f(q=r, hq=32, o=rows(L, token=2048)), -1)             # its rows overlap
    refused(L, f(q=r, hq=32, o=rows(L, token=8192)), -1)             # in place, but other strides
    refused(L, lib.efq_kv_append(r, r, None, b, None, None, 0, None, None), -1)
    refused(L, lib.efq_kv_append(r, r, c, None, None, None, 0, None, None), -1)
    assert f(k=None, v=None, bb=batch(L, tokens=0)) == 0


def test_attention_arguments(L):
    lib, r, c, b = L.lib(), rows(L, token=4096), cache(L), batch(L)
    f = lambda q=r, hq=32, bb=b, scale=0.1, o=r, dt=0, lse=None, ws=None, n=0: lib.efq_attn_paged(
        q, hq, c, bb, scale, 1, o, dt, lse, ws, n, None)
    for hq in (0, 4, 33, -8):
        refused(L, f(hq=hq), -1)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(L, f(scale=scale), -1)
    refused(L, f(q=None), -1)
    refused(L, f(o=None), -1)
    refused(L, f(o=rows(L, token=2048)), -1)
    refused(L, f(dt=5), -1)
    refused(L, f(lse=4098), -1)
    refused(L, f(n=64), -3)
    refused(L, f(ws=4104, n=64), -1)
    refused(L, f(bb=batch(L, tokens=1 << 24)), -2)
    assert f(q=None, o=None, bb=batch(L, tokens=0)) == 0
    if not torch.cuda.is_available():
        refused(L, f(), VALID)


def test_scratch_only_where_keys_are_split(L):
    w = lambda c={}, **b: int(L.lib().efq_attn_paged_workspace_bytes(cache(L, **c), batch(L, **b), 32))
    assert w(width=8192, max_k=131072) > 0                           # one token each, long contexts
    assert w(tokens=1, seqs=1, max_k=100, width=8192) == 0           # short
    assert w(tokens=0) == 0
    assert w(dict(heads=32), seqs=1024, tokens=1024, width=512, max_k=8000) == 0      # enough rows without
    # the hints are upper bounds only as far as they go: none means the table's width
    assert w(max_k=0, max_q=0, width=8192, tokens=2) == w(max_k=131072, max_q=1, width=8192, tokens=2)


def test_binding_refuses_tensors_off_the_gpu(L):
    x = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    pos = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        L.rope(x, pos, torch.ones(64))
    with pytest.raises(ValueError):
        L.rope(x.half(), pos, torch.ones(64))
    with pytest.raises(ValueError):
        L.PagedCache(torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        L.PagedBatch(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        L.PagedCache.empty(2, 16, 1, 64, "fp4")


@pytest.mark.gpu
def test_binding_refuses_tensors_that_do_not_fit(L):
    dev = dict(device="cuda")
    x = torch.zeros(4, 8, 128, dtype=torch.bfloat16, **dev)
    pos, inv = torch.zeros(4, dtype=torch.int32, **dev), torch.ones(64, **dev)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, **dev)
    c = L.PagedCache.empty(2, 16, 2, 128)
    b = L.PagedBatch(i32(2), i32(1), i32(1, 2))
    kv = x[:, :2]
    bad = [
        lambda: L.rope(x, pos.long(), inv), lambda: L.rope(x, pos[:3], inv), lambda: L.rope(x, pos, inv.double()),
        lambda: L.rope(x, i32(3, 4), inv), lambda: L.rope(x, i32(3, 4), inv, axis=i32(63)), lambda: L.rope(x.half(), pos, inv),
        lambda: L.rope(x.transpose(1, 2), pos, inv), lambda: L.rope(x, pos, inv, out=x[:, :4]), lambda: L.rope(x[0], pos, inv),
        lambda: L.rope(x, pos.cpu(), inv), lambda: L.rope(x, pos, inv, out=x.float()),
        lambda: L.PagedCache(c.k, c.v[:1]), lambda: L.PagedCache(c.k.view(torch.uint8), c.v.view(torch.uint8)),
        lambda: L.PagedCache(c.k, c.v, torch.zeros(2, 2, 16, 4, dtype=torch.uint8, **dev)),
        lambda: L.PagedBatch(i32(3), i32(1), i32(1, 2)), lambda: L.PagedBatch(i32(2), i32(1).long(), i32(1, 2)),
        lambda: L.PagedBatch(i32(2), i32(1), i32(2, 2)), lambda: L.PagedBatch(i32(2), i32(1), i32(1, 2).cpu()),
        lambda: L.kv_append(x, kv, c, b), lambda: L.kv_append(kv, kv[:2], c, b), lambda: L.kv_append(kv, kv, c, b, pos=pos),
        lambda: L.kv_append(kv, kv, c, b, q_out=x), lambda: L.kv_append(kv, kv, c, b, q=x, q_out=x[:, :4]),
        lambda: L.kv_append(kv.float(), kv, c, b), lambda: L.attn_paged(x[..., :64], c, b), lambda: L.attn_paged(x.float(), c, b),
        lambda: L.attn_paged(x, c, b, out=x.half()), lambda: L.attn_paged(x, c, b, out=x[:3]),
        lambda: L.attn_paged(x, c, b, lse=torch.zeros(4, 7, **dev)),
        lambda: L.attn_paged(x, c, b, workspace=torch.zeros(64, dtype=torch.uint8))]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            raise AssertionError(f"call {i} was accepted")
    with pytest.raises(L.EfqError):
        L.attn_paged(x[:, :7], c, b)                 # heads_q not a multiple of heads_kv
    with pytest.raises(L.EfqError):
        L.rope(x, pos, torch.ones(60, **dev))
