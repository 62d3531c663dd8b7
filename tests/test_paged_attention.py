"""Attention of new tokens over a paged cache against softmax attention in 64
bits: one token to chunks, ragged batches, odd lengths, both cache formats, and
what the cache may hold outside the sequences."""
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


def mxfp8(x):
    """(codes, scales) as bytes, and the values they stand for, of bf16 x [..., D]."""
    b = x.double().unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    k = torch.where(amax > 0, torch.frexp(amax)[1].double() - 9, -127.0).clamp_min(-127.0)
    y = (b * torch.exp2(-k)).clamp(-448, 448).float().to(torch.float8_e4m3fn)
    return (y.flatten(-2).view(torch.uint8), (k[..., 0] + 127).to(torch.uint8),
            (y.double() * torch.exp2(k)).flatten(-2))


class Case:
    """A batch with its keys laid into randomly ordered pages of a cache whose
    other slots hold `rest`."""

    def __init__(self, B, new, keys, heads, D, page, fmt, seed=0, rest=float("nan"), pad=0, wide=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        hq, hkv = heads
        self.new, self.keys, self.heads, self.D = new, keys, heads, D
        used = [-(-k // page) for k in keys]
        pages = sum(used) + 2
        width = max(1, max(used)) + wide
        self.k = [(torch.randn(n, hkv, D, generator=g) * spread).bfloat16() for n in keys]
        self.v = [torch.randn(n, hkv, D, generator=g).bfloat16() for n in keys]
        self.q = torch.randn(sum(new) + pad, hq, D, generator=g).bfloat16()
        perm = torch.randperm(pages, generator=g).tolist()
        table = torch.full((len(keys), width), -1, dtype=torch.int32)
        kc, vc = (torch.full((pages, hkv, page, D), rest).bfloat16() for _ in range(2))
        at = 0
        for i, n in enumerate(keys):
            for j in range(used[i]):
                table[i, j] = perm[at]
                m = min(page, n - j * page)
                kc[perm[at], :, :m] = self.k[i][j * page: j * page + m].transpose(0, 1)
                vc[perm[at], :, :m] = self.v[i][j * page: j * page + m].transpose(0, 1)
                at += 1
        self.table = table
        if fmt == "mxfp8":
            live = torch.isfinite(kc.float())
            (kq, ks, _), (vq, vs, _) = mxfp8(kc.nan_to_num(0)), mxfp8(vc.nan_to_num(0))
            if rest != rest:             # NaN codes and scales where no key lies
                kq[~live] = vq[~live] = 0x7F
                ks[~live[..., ::32]] = vs[~live[..., ::32]] = 0xFF
            self.cache = B.PagedCache(kq.cuda(), vq.cuda(), ks.cuda(), vs.cuda())
            self.k = [mxfp8(t)[2] for t in self.k]
            self.v = [mxfp8(t)[2] for t in self.v]
        else:
            self.cache = B.PagedCache(kc.cuda(), vc.cuda())
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        self.starts = starts
        self.batch = B.PagedBatch(torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor(keys, dtype=torch.int32).cuda(),
                                  table.cuda(), max_q=max(new), max_k=max(keys))

    def reference(self, scale, causal, hidden=None):
        """Per token (in 64 bits): output, log-sum-exp, sum p |v|, and the largest
        sum of a score's absolute products."""
        hq, hkv = self.heads
        T = self.starts[-1]
        out, mag = (torch.zeros(T, hq, self.D, dtype=torch.float64) for _ in range(2))
        lse = torch.full((T, hq), -math.inf, dtype=torch.float64)
        size = torch.zeros(T, hq, dtype=torch.float64)
        for i, (n, s) in enumerate(zip(self.new, self.keys)):
            if n == 0 or s == 0:
                continue
            rows = slice(self.starts[i], self.starts[i] + n)
            q = self.q[rows].double()
            k = self.k[i].double().repeat_interleave(hq // hkv, 1)
            v = self.v[i].double().repeat_interleave(hq // hkv, 1)
            x = torch.einsum("nhd,shd->nhs", q, k) * scale
            t = torch.arange(s)
            seen = torch.ones(n, s, dtype=torch.bool)
            if causal:
                seen = t[None] <= (s - n + torch.arange(n))[:, None]
            if hidden is not None:
                seen = seen & ~hidden[i][None, :s]
            x = x.masked_fill(~seen[:, None], -math.inf)
            lse[rows] = torch.logsumexp(x, -1)
            p = torch.softmax(x, -1).nan_to_num(0)
            out[rows] = torch.einsum("nhs,shd->nhd", p, v)
            mag[rows] = torch.einsum("nhs,shd->nhd", p, v.abs())
            size[rows] = torch.einsum("nhd,shd->nhs", q.abs(), k.abs()).amax(-1) * scale
        return out, lse, mag, size


def check(c, out, lse, scale, causal, hidden=None):
    """A score sums D products in fp32: off by at most D 2^-24 of its absolute
    products (d); exp2's argument and the exponential add a few 2^-23 of the
    score.  A probability is rounded to bf16 (2^-8), the sums are fp32."""
    T = c.starts[-1]
    ref, rl, mag, size = c.reference(scale, causal, hidden)
    got, gl = out[:T].double().cpu(), lse[:T].double().cpu()
    d = (c.D + 8) * 2.0 ** -24 * size + 2.0 ** -20
    empty = torch.isinf(rl)
    assert torch.equal(torch.isinf(gl), empty) and bool((gl[empty] < 0).all())
    assert bool((got[empty] == 0).all()) and bool(torch.isfinite(got).all())
    off = (gl - rl).abs()[~empty]
    assert bool((off <= (d + 2.0 ** -22 * rl.abs())[~empty]).all()), float(off.max())
    tol = (2.0 ** -8 + 2 * d)[..., None] * mag + 1e-30
    if out.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
    worst = float(((got - ref).abs() / tol).max())
    assert worst <= 1, worst
    # and the roundings are independent: their size on the whole is far below the bound's
    if mag.numel() > 4096:
        assert float((got - ref).norm() / ref.norm()) < 4e-3


HEADS = [(4, 1, 128), (8, 8, 128), (8, 2, 64), (16, 1, 64)]


def run(B, c, scale=None, causal=True, dtype=torch.bfloat16, **kw):
    T = len(c.q)
    out = torch.full((T, c.heads[0], c.D), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((T, c.heads[0]), 7.0, dtype=torch.float32, device="cuda")
    scale = c.D ** -0.5 if scale is None else scale
    print(f"[paged] new {c.new} keys {c.keys} heads {c.heads} D {c.D} page {c.cache.page_size} "
          f"fmt {c.cache.c.format} causal {causal}", flush=True)
    B.attn_paged(c.q.cuda(), c.cache, c.batch, scale=scale, causal=causal, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    T = c.starts[-1]
    assert bool((out[T:] == 7).all()) and bool((lse[T:] == 7).all())
    return out, lse, scale


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("new,keys,page", [
    ([1], [1], 16), ([1], [17], 16), ([1, 1, 1], [31, 128, 129], 32), ([1, 0, 1, 1], [700, 0, 0, 64], 64),
    ([1], [5000], 128), ([2, 5, 1], [40, 5, 333], 16), ([3], [3], 256), ([9, 4], [1000, 4], 16)])
def test_few_tokens(B, new, keys, page, heads, fmt):
    hq, hkv, D = heads
    c = Case(B, new, keys, (hq, hkv), D, page, fmt, seed=len(new) + keys[0], pad=2)
    out, lse, scale = run(B, c)
    check(c, out, lse, scale, True)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("new,keys,page", [
    ([64], [64], 16), ([65, 300], [65, 301], 64), ([100, 1, 0, 257], [1000, 77, 9, 300], 16),
    ([130], [2300], 128), ([300, 2], [299, 1], 32)])
def test_chunks(B, new, keys, page, heads, fmt):
    hq, hkv, D = heads
    c = Case(B, new, keys, (hq, hkv), D, page, fmt, seed=len(new) + keys[0], pad=3)
    out, lse, scale = run(B, c)
    check(c, out, lse, scale, True)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("new,keys", [([1, 3], [333, 40]), ([70, 200], [33, 1500])])
def test_every_key_seen(B, new, keys, fmt):
    c = Case(B, new, keys, (8, 2), 128, 16, fmt, seed=4)
    out, lse, scale = run(B, c, causal=False, dtype=torch.float32)
    check(c, out, lse, scale, False)


@pytest.mark.parametrize("new", [[1, 1], [200, 90]])
def test_large_scores(B, new):
    """Maxima that move all the time, probabilities that underflow."""
    c = Case(B, new, [900, 2000], (4, 2), 128, 64, "bf16", seed=5, spread=30.0)
    out, lse, scale = run(B, c, scale=0.3, dtype=torch.float32)
    check(c, out, lse, scale, True)
