"""Rotary positions (one and several axes, both pairings, forward and gradient)
against 64 bits, and the append to a paged cache: the rotation it applies is
rope's bit for bit, the MXFP8 codes and scales are quant_qk's."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


def turned(x, pos, inv_freq, axis, interleaved, inverse=False):
    """rope in 64 bits on the CPU, and the sum of the absolute products of each value."""
    x, pos, f = x.double().cpu(), pos.double().cpu(), inv_freq.double().cpu()
    n = len(f)
    ax = torch.zeros(n, dtype=torch.long) if axis is None else axis.long().cpu()
    known = (ax >= 0) & (ax < len(pos))
    angle = torch.where(known, pos[ax.clamp(0, len(pos) - 1)].t(), torch.zeros(())) * f
    c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if inverse else 1)
    lo = torch.arange(n) * 2 if interleaved else torch.arange(n)
    hi = lo + 1 if interleaved else lo + n
    y, size = x.clone(), x.abs()
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    size[..., lo], size[..., hi] = a.abs() + b.abs(), a.abs() + b.abs()
    return y, size


def check_turned(got, x, *turn):
    """A turn is off by 2^-25 of itself in fp32 (2 pi 2^-25 of angle), the sine
    and cosine by 2 ulp, the two products by half a step each; then one
    rounding to the type (bf16 2^-8, fp32 2^-24)."""
    ref, size = turned(x, *turn)
    half = torch.finfo(x.dtype).eps / 2
    off = (got.double().cpu() - ref).abs()
    # entries behind the pairs pass unchanged
    R = 2 * len(turn[1])
    assert torch.equal(got[..., R:].cpu(), x[..., R:].cpu())
    tol = size * (math.pi * 2.0 ** -24 + 2 * 2.0 ** -23 + 2.0 ** -23) + half * ref.abs()
    assert bool((off <= tol + 1e-37).all()), float((off / (tol + 1e-37)).max())


def frequencies(n, axes, g):
    inv = (1e6 ** (-torch.arange(n, dtype=torch.float64) / n)).float()
    return inv.cuda(), None if axes == 1 else torch.randint(0, axes, (n,), generator=g, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,D,pairs,axes,far", [
    (1, 1, 64, 32, 1, 100), (3, 40, 128, 64, 3, 1 << 20), (333, 5, 128, 32, 1, 131072), (17, 2, 80, 40, 2, 5000),
    (4100, 3, 128, 64, 3, 40000), (2, 7, 512, 256, 1, (1 << 31) - 1), (8192, 1, 16, 8, 3, 1000)])
def test_rope(B, tokens, heads, D, pairs, axes, far, interleaved, dtype):
    print(f"[rope] {(tokens, heads, D, pairs, axes, far, interleaved, dtype)}", flush=True)
    g = torch.Generator().manual_seed(tokens + D)
    inv, axis = frequencies(pairs, axes, g)
    pos = torch.randint(-far, far, (axes, tokens), generator=g).int().cuda()
    full = torch.randn(tokens, heads + 3, D + 16, generator=g).to(dtype).cuda()
    x = full[:, 1:1 + heads, :D]                     # strided in tokens and heads
    keep = full.clone()
    y = B.rope(x, pos, inv, axis, interleaved)
    check_turned(y, x, pos, inv, axis, interleaved)
    dx = B.rope_bwd(x, pos, inv, axis, interleaved)
    check_turned(dx, x, pos, inv, axis, interleaved, True)
    assert torch.equal(full, keep)
    out = torch.full((tokens, heads + 1, D), 3.0, dtype=dtype, device="cuda")
    B.rope(x, pos, inv, axis, interleaved, out=out[:, 1:])
    assert torch.equal(out[:, 1:], y) and bool((out[:, 0] == 3).all())
    B.rope(x, pos, inv, axis, interleaved, out=x)    # in place
    assert torch.equal(x, y)
    keep[:, 1:1 + heads, :D] = y
    assert torch.equal(full, keep)


def test_rope_gradient_by_differences(B):
    """<dy, rope(x + e) - rope(x)> = <rope_bwd(dy), e>: linear in x, so exact up to fp32 rounding."""
    g = torch.Generator().manual_seed(3)
    inv, axis = frequencies(32, 3, g)
    pos = torch.randint(0, 5000, (3, 50), generator=g).int().cuda()
    x, e, dy = (torch.randn(50, 4, 128, generator=g).cuda() for _ in range(3))
    for interleaved in (False, True):
        f = lambda t: B.rope(t, pos, inv, axis, interleaved).double()
        left = float((dy.double() * (f(x + e) - f(x))).sum())
        right = float((B.rope_bwd(dy, pos, inv, axis, interleaved).double() * e.double()).sum())
        # 25600 products of values of order 1, each off by a few 2^-24: at most 25600 * 3 * 8 * 2^-24
        assert abs(left - right) <= 0.04 and abs(left) > 10


def test_rope_shapes(B):
    """[B, S, H, D] is [B * S, H, D]; one axis as [tokens]; unknown axes turn by nothing; no tokens."""
    g = torch.Generator().manual_seed(4)
    inv, _ = frequencies(64, 1, g)
    x = torch.randn(3, 5, 2, 128, generator=g).bfloat16().cuda()
    pos = torch.arange(15, dtype=torch.int32).cuda()
    y = B.rope(x, pos, inv)
    assert y.shape == x.shape and torch.equal(y.view(15, 2, 128), B.rope(x.view(15, 2, 128), pos[None], inv))
    one = x[:, :1]                                   # S = 1: the batch is the tokens
    assert torch.equal(B.rope(one, pos[:3] * 5, inv), y[:, :1])
    axis = torch.full((64,), 7, dtype=torch.int32).cuda()
    axis[3] = -1
    assert torch.equal(B.rope(x, pos, inv, axis), x)
    assert B.rope(x[:0], pos[:0], inv).shape == (0, 5, 2, 128)
    with pytest.raises(ValueError):
        B.rope(x[:, ::2], torch.arange(9, dtype=torch.int32).cuda(), inv)


# ------------------------------------------------------------------- append
def layout(new, keys, page, g, wide=1):
    used = [-(-k // page) for k in keys]
    pages = sum(used) + 3
    perm = torch.randperm(pages, generator=g).tolist()
    table = torch.full((len(keys), max(1, max(used)) + wide), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = torch.tensor(perm[at:at + n], dtype=torch.int32)
        at += n
    starts = torch.tensor([0] + new).cumsum(0).int()
    return pages, table, starts


def slots(new, keys, page, table):
    """(token, page, offset) of every new token that has a key."""
    t = 0
    for i, (n, s) in enumerate(zip(new, keys)):
        for j in range(n):
            at = s - n + j
            if at >= 0:
                yield t, int(table[i, at // page]), at % page
            t += 1


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("heads,D", [((4, 1), 128), ((3, 3), 64), ((32, 8), 128)])
@pytest.mark.parametrize("new,keys,page,interleaved,axes", [
    ([1], [1], 16, False, 1), ([1] * 70, [5 + 3 * i for i in range(70)], 16, True, 3), ([0, 40, 1, 7], [9, 41, 100, 3], 32, False, 3),
    ([513], [700], 64, False, 1), ([300, 5000], [300, 5001], 128, True, 1)])
def test_append(B, new, keys, page, interleaved, axes, heads, D, fmt):
    print(f"[append] {(len(new), sum(new), page, interleaved, axes, heads, D, fmt)}", flush=True)
    g = torch.Generator().manual_seed(sum(new) + D)
    hq, hkv = heads
    pages, table, starts = layout(new, keys, page, g)
    T = sum(new) + 2                                 # two padding tokens
    qkv = torch.randn(T, hq + 2 * hkv, D, generator=g)
    qkv *= torch.exp2(torch.randint(-9, 9, (T, hq + 2 * hkv, D // 32, 1), generator=g).float()).expand(-1, -1, -1, 32).flatten(-2)
    qkv = qkv.bfloat16().cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    inv, axis = frequencies(D // 2, axes, g)
    pos = torch.randint(0, 100000, (axes, T), generator=g).int().cuda()
    cache = B.PagedCache.empty(pages, page, hkv, D, fmt)
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if t is not None:
            t.fill_(3)
    batch = B.PagedBatch(starts.cuda(), torch.tensor(keys, dtype=torch.int32).cuda(), table.cuda())
    q_out = torch.full((T, hq, D), 5.0, dtype=torch.bfloat16, device="cuda")
    assert B.kv_append(k, v, cache, batch, q=q, q_out=q_out, pos=pos, inv_freq=inv, axis=axis,
                       interleaved=interleaved) is q_out
    turn = lambda t: B.rope(t, pos, inv, axis, interleaved)
    n = sum(new)
    assert torch.equal(q_out[:n], turn(q)[:n]) and bool((q_out[n:] == 5).all())
    kt, vt = turn(k), v.contiguous()
    where = list(slots(new, keys, page, table))
    tok, pg, off = (torch.tensor(x).cuda() for x in zip(*where))
    if fmt == "bf16":
        want = {"k": kt, "v": vt}
    else:
        (_, kh), (_, vh) = (B.quant_qk(t[None], t[None]) for t in (kt, vt))
        sh = B.Shape(1, T, T, hkv, hkv, D)
        import ctypes
        soff = B.lib().efq_khat_scale_offset(ctypes.byref(sh))
        want = {}
        for name, h in (("k", kh), ("v", vh)):
            c, e = B.qk8_natural(h, 1, hkv, T, D, soff)
            want[name], want[name + "_scale"] = c[0].transpose(0, 1), e[0].transpose(0, 1)
    for name, w in want.items():
        got = getattr(cache, name)
        untouched = torch.full_like(got, 3)
        untouched[pg, :, off] = w[tok]
        assert torch.equal(got, untouched), name


def test_append_without_positions_and_in_place(B):
    g = torch.Generator().manual_seed(8)
    pages, table, starts = layout([3, 2], [20, 2], 16, g)
    batch = B.PagedBatch(starts.cuda(), torch.tensor([20, 2], dtype=torch.int32).cuda(), table.cuda())
    k, v, q = (torch.randn(5, h, 128, generator=g).bfloat16().cuda() for h in (2, 2, 4))
    a, b = B.PagedCache.empty(pages, 16, 2, 128), B.PagedCache.empty(pages, 16, 2, 128)
    for t in (a.k, a.v, b.k, b.v):
        t.zero_()
    assert B.kv_append(k, v, a, batch) is None
    for t, p, o in slots([3, 2], [20, 2], 16, table):
        assert torch.equal(a.k[p, :, o], k[t]) and torch.equal(a.v[p, :, o], v[t])
    assert int((a.k != 0).any(-1).sum()) == 10
    inv, _ = frequencies(64, 1, g)
    pos = torch.arange(5, dtype=torch.int32).cuda()
    want = B.rope(q, pos, inv)
    assert B.kv_append(k, v, b, batch, q=q, q_out=q, pos=pos, inv_freq=inv) is q and torch.equal(q, want)
    copy = B.kv_append(k, v, b, batch, q=q)          # no positions: a copy
    assert torch.equal(copy, q) and copy.data_ptr() != q.data_ptr()


def test_append_lengths_out_of_range(B):
    """Pages that are none, more keys than the table holds, more new tokens than
    keys, starts that fall or leave the tokens: nothing outside the pages is
    written, and what is in range lands where it belongs."""
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(6, 1, 64, generator=g).bfloat16().cuda() for _ in range(2))

    def go(starts, keys, table, pages=2):
        guard = torch.zeros(pages + 2, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
        vg = torch.zeros_like(guard)
        cache = B.PagedCache(guard[1:-1], vg[1:-1])
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
        B.kv_append(k, v, cache, B.PagedBatch(i32(starts), i32(keys), i32(table)))
        torch.cuda.synchronize()
        assert not bool(guard[0].any()) and not bool(guard[-1].any())
        at = {}
        for p in range(pages):
            for o in range(16):
                if bool(cache.k[p, 0, o].any()):
                    t = [t for t in range(6) if torch.equal(cache.k[p, 0, o], k[t, 0])]
                    assert t and torch.equal(cache.v[p, 0, o], v[t[0], 0])
                    at[p, o] = t[0]
        return at

    assert go([0, 3, 6], [3, 17], [[1, -1], [0, 9]]) == {(1, 0): 0, (1, 1): 1, (1, 2): 2, (0, 14): 3, (0, 15): 4}
    assert go([0, 6], [2], [[0]]) == {(0, 0): 4, (0, 1): 5}            # four tokens before the first key
    assert go([0, 2], [1000], [[1]]) == {(1, 14): 0, (1, 15): 1}       # cut to the table's 16 keys
    assert go([0, 2], [-5], [[1]]) == {}
    assert go([-4, 4, 2, 900], [4, 1, 16], [[0], [1], [1]]) .keys() <= {(p, o) for p in range(2) for o in range(16)}


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,tokens", [(torch.bfloat16, 33000), (torch.float32, 17000)])
def test_rope_past_the_last_cache(B, dtype, tokens, interleaved):
    """An output of more than 256 MB, whose writes are streamed, is that of its parts, which are not."""
    x = torch.randn(tokens, 32, 128, device="cuda").to(dtype)
    pos = torch.randint(0, 100000, (tokens,), dtype=torch.int32, device="cuda")
    inv = (10000.0 ** (-torch.arange(64) / 64)).float().cuda()
    assert x.numel() * x.element_size() > 256 << 20
    whole = B.rope(x, pos, inv, interleaved=interleaved)
    for t in range(0, tokens, 7001):
        part = slice(t, t + 7001)
        assert torch.equal(whole[part], B.rope(x[part], pos[part].contiguous(), inv, interleaved=interleaved))
