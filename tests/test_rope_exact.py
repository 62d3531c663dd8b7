"""The turn of rope and of the append to its last rounding: sines and cosines are
those of 64 bits rounded once to fp32, so a turned value is the rounding of one
within three fp32 half steps of its products.  An fp32 angle or sine is further off."""
import math

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


def parts(pos, inv_freq, axis):
    """|angle| [tokens, pairs] in 64 bits, its cosine and sine."""
    ax = torch.zeros(len(inv_freq), dtype=torch.long) if axis is None else axis.long()
    angle = pos.double()[ax].t() * inv_freq.double()
    return angle.abs(), angle.cos(), angle.sin()


def turned(x, pos, inv_freq, axis, interleaved, trig=None):
    """(turned x, bound on what an fp32 evaluation is off by), of x on the CPU; trig: another cosine and sine.

    With c and s rounded once (2^-24 of each), u c - v s as fma(u, c, -(v s)) is off by 2^-24 (|u c| + |v s|) for
    these, 2^-24 |v s| for the product and 2^-24 of the result, at most |u c| + |v s|: 3 2^-24 (|u c| + |v s|) to
    first order, the rest below 2^-40.  The angle is off by 3 2^-53 of itself in the kernel (two products and 1 / 2 pi)
    and by 2^-53 here, which moves the result by that times |u| + |v|."""
    size, c, s = parts(pos, inv_freq, axis)
    if trig:
        c, s = trig
    c, s, size = c[:, None], s[:, None], size[:, None]
    n = len(inv_freq)
    lo = torch.arange(n) * 2 if interleaved else torch.arange(n)
    hi = lo + 1 if interleaved else lo + n
    x = x.double()
    y, tol = x.clone(), torch.zeros_like(x)
    u, v = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = u * c - v * s, v * c + u * s
    off = lambda a, b: 3.001 * 2.0 ** -24 * (a.abs() + b.abs()) + 4 * 2.0 ** -53 * size * (u.abs() + v.abs())
    tol[..., lo], tol[..., hi] = off(u * c, v * s), off(v * c, u * s)
    return y, tol


def within(got, y, tol):
    """got is the rounding of a value within tol of y: rounding is monotone."""
    dtype = got.dtype
    below, above = ((y + d).to(dtype) if dtype == torch.bfloat16 else y + d for d in (-tol, tol))
    return (got.double() >= below.double()) & (got.double() <= above.double())


def data(tokens, heads, D, pairs, axes, far, dtype, seed=7):
    g = torch.Generator().manual_seed(seed)
    inv = (1e6 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float()
    axis = None if axes == 1 else torch.randint(0, axes, (pairs,), generator=g, dtype=torch.int32)
    pos = torch.randint(-far, far, (axes, tokens), generator=g).int()
    return torch.randn(tokens, heads, D, generator=g).to(dtype), pos, inv, axis


CASES = [(33, 40, 128, 64, 3, 1 << 20), (700, 4, 128, 32, 1, 131072), (17, 9, 80, 40, 2, 5000), (400, 3, 64, 32, 1, (1 << 31) - 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_rope(B, case, interleaved, dtype):
    x, pos, inv, axis = data(*case, dtype)
    on = lambda t: None if t is None else t.cuda()
    for f, sign in ((B.rope, 1), (B.rope_bwd, -1)):
        got = f(x.cuda(), pos.cuda(), inv.cuda(), on(axis), interleaved).cpu()
        assert bool(within(got, *turned(x, pos * sign, inv, axis, interleaved)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens", [1, 60, 9000])
def test_appended_keys(B, tokens, interleaved):
    """The keys in a bf16 cache are those of 64 bits rounded once, in an MXFP8 one these rounded further."""
    from test_paged_attention import mxfp8
    x, pos, inv, axis = data(tokens, 2, 128, 64, 3, 100000, torch.bfloat16)
    v = torch.randn(x.shape, generator=torch.Generator().manual_seed(8)).bfloat16()
    pages = -(-tokens // 64)
    i32 = lambda t: torch.tensor(t, dtype=torch.int32).cuda()
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(9)).int()
    batch = B.PagedBatch(i32([0, tokens]), i32([tokens]), table[None].contiguous().cuda())
    caches = [B.PagedCache.empty(pages, 64, 2, 128, fmt) for fmt in ("bf16", "mxfp8")]
    for c in caches:
        B.kv_append(x.cuda(), v.cuda(), c, batch, pos=pos.cuda(), inv_freq=inv.cuda(), axis=axis.cuda(), interleaved=interleaved)
    rows = lambda t: t.cpu()[table.long()].transpose(1, 2).flatten(0, 1)[:tokens]      # [tokens, heads, ..]
    key = rows(caches[0].k)
    assert bool(within(key, *turned(x, pos, inv, axis, interleaved)).all())
    assert torch.equal(rows(caches[0].v), v)
    for name, t in (("k", key), ("v", v)):
        codes, scales, _ = mxfp8(t)
        assert torch.equal(rows(getattr(caches[1], name)), codes) and torch.equal(rows(getattr(caches[1], name + "_scale")), scales)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_the_bound_tells(case, interleaved):
    """On the CPU: the turn as the kernel forms it is within the bound; with the angle's last turn or the sine and cosine
    in fp32, planted here, fp32 values are not (few of these mistakes move a bf16 value)."""
    for dtype in (torch.bfloat16, torch.float32):
        x, pos, inv, axis = data(*case, dtype)
        y, tol = turned(x, pos, inv, axis, interleaved)
        n = len(inv)
        lo = torch.arange(n) * 2 if interleaved else torch.arange(n)
        hi = lo + 1 if interleaved else lo + n

        def in_fp32(c, s):
            z = x.float().clone()
            u, v = z[..., lo].clone(), z[..., hi].clone()
            fma = lambda a, b, t: (a.double() * b.double() + t.double()).float()     # one rounding (53 bits hold the product)
            z[..., lo], z[..., hi] = fma(u, c, -(v * s)), fma(v, c, u * s)
            return z.to(dtype)

        _, c, s = parts(pos, inv, axis)
        assert bool(within(in_fp32(c.float()[:, None], s.float()[:, None]), y, tol).all())
        if dtype == torch.bfloat16:
            continue
        turns = (pos.double()[torch.zeros(n, dtype=torch.long) if axis is None else axis.long()].t() * inv.double()) / (2 * math.pi)
        rest = (turns - turns.round()).float() * torch.tensor(2 * math.pi, dtype=torch.float32)      # fp32 angle of the last turn
        assert not bool(within(in_fp32(rest.cos()[:, None], rest.sin()[:, None]), y, tol).all())
        ulp = lambda t: t.float() * (1 + 2.0 ** -22)                                                  # a sine off by 2 ulp
        assert not bool(within(in_fp32(ulp(c)[:, None], ulp(s)[:, None]), y, tol).all())
