"""The cache operators as a program uses them, and the calls their documentation
allows: a prompt fed in chunks and generated on, wrong hints, strided rows, calls
without scratch, bad pages and lengths, streams, captured graphs, long caches."""
import math

import pytest
import torch

from test_paged_attention import Case, check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_09721_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "no GPU"
    return binding


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def attention(q, k, v, scale):
    """Causal softmax attention of [S, H, D] in 64 bits on the CPU: output, log-sum-exp."""
    q, k, v = (t.double().cpu() for t in (q, k, v))
    k, v = (t.repeat_interleave(q.shape[1] // t.shape[1], 1) for t in (k, v))
    x = torch.einsum("nhd,shd->hns", q, k) * scale
    x = x.masked_fill(torch.ones(x.shape[1:], dtype=torch.bool).triu(1), -math.inf)
    return torch.einsum("hns,shd->nhd", torch.softmax(x, -1), v), torch.logsumexp(x, -1).t()


@pytest.mark.parametrize("fmt,steps", [("bf16", [70, 1, 130, 1, 1, 3]), ("mxfp8", [1, 200, 2, 1])])
def test_prompt_in_chunks_and_steps(B, fmt, steps):
    """Append and attend, several times: every token's output is that of attention over the whole sequence at once."""
    g = torch.Generator().manual_seed(1)
    hq, hkv, D, page, S = 8, 2, 128, 16, sum(steps)
    q, k, v = (torch.randn(2, S, h, D, generator=g).bfloat16().cuda() for h in (hq, hkv, hkv))
    inv = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    axis = (torch.arange(64) % 3).int().cuda()
    pos = torch.stack([torch.arange(S) // 9, torch.arange(S) % 9 // 3, torch.arange(S) % 3]).int().cuda()
    pages = -(-S // page)
    cache = B.PagedCache.empty(2 * pages, page, hkv, D, fmt)
    table = i32(torch.randperm(2 * pages, generator=g).view(2, pages).tolist())
    out = torch.empty(2, S, hq, D, device="cuda")
    lse = torch.empty(2, S, hq, device="cuda")
    at = 0
    for n in steps:
        batch = B.PagedBatch(i32([0, n, 2 * n]), i32([at + n, at + n]), table, max_q=n, max_k=at + n)
        part = lambda t: t[:, at:at + n].flatten(0, 1)
        where = pos[:, at:at + n].repeat(1, 2).contiguous()
        qr = B.kv_append(part(k), part(v), cache, batch, q=part(q), pos=where, inv_freq=inv, axis=axis)
        l = torch.empty(2 * n, hq, device="cuda")
        o = B.attn_paged(qr, cache, batch, lse=l)
        out[:, at:at + n], lse[:, at:at + n] = o.view(2, n, hq, D), l.view(2, n, hq)
        at += n
    for i in range(2):
        qt, kt = B.rope(q[i], pos, inv, axis), B.rope(k[i], pos, inv, axis)
        vt = v[i]
        if fmt == "mxfp8":
            from test_paged_attention import mxfp8
            kt, vt = mxfp8(kt.cpu())[2], mxfp8(vt.cpu())[2]
        ref, rl = attention(qt, kt, vt, D ** -0.5)
        # the probabilities' rounding (2^-8) and fp32 sums; |v| below 5.5 here
        assert float((out[i].double().cpu() - ref).abs().max()) <= 2.0 ** -8 * 5.5
        assert float((out[i].double().cpu() - ref).norm() / ref.norm()) < 3e-3
        assert float((lse[i].double().cpu() - rl).abs().max()) < 1e-4


@pytest.mark.parametrize("new,keys,max_q,max_k", [
    ([1, 9, 1], [300, 2000, 5], 1, 1), ([40, 300, 2], [40, 700, 3000], 1, 64), ([1, 1], [3000, 10], 500, 10 ** 6),
    ([200], [4000], 2, 100), ([3, 1, 90], [5000, 1, 90], 0, 0)])
@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("mxfp8", 64)])
def test_hints_change_no_result(B, new, keys, max_q, max_k, fmt, D):
    """max_q and max_k too small, too large or unknown: every row and key is still there."""
    c = Case(B, new, keys, (4, 1), D, 16, fmt, seed=11, wide=300)
    c.batch = B.PagedBatch(i32(c.starts), i32(keys), c.table.cuda(), max_q=max_q, max_k=max_k)
    out, lse, scale = run(B, c)
    check(c, out, lse, scale, True)


def test_strided_rows_and_outputs(B):
    """q a slice of a fused projection, out a slice of a wider buffer, bf16 and fp32."""
    for new, keys in (([1, 1, 1], [100, 3, 2600]), ([150, 2], [400, 60])):
        c = Case(B, new, keys, (8, 2), 128, 32, "bf16", seed=12)
        T = sum(new)
        fused = torch.randn(T, 12, 128).bfloat16().cuda()
        fused[:, 2:10] = c.q.cuda()
        for dtype in (torch.bfloat16, torch.float32):
            wide = torch.full((T, 11, 160), 9.0, dtype=dtype, device="cuda")
            lse = torch.empty(T, 8, device="cuda")
            B.attn_paged(fused[:, 2:10], c.cache, c.batch, out=wide[:, 3:, 16:144], lse=lse)
            check(c, wide[:, 3:, 16:144], lse, 128 ** -0.5, True)
            wide[:, 3:, 16:144] = 9.0
            assert bool((wide == 9).all())


@pytest.mark.parametrize("new,keys", [([1, 1], [5000, 9000]), ([20], [7000]), ([300, 64], [3000, 6000])])
def test_without_scratch_and_with_a_workspace(B, new, keys):
    c = Case(B, new, keys, (4, 1), 128, 64, "bf16", seed=13)
    n = B.attn_paged_workspace_bytes(c.cache, c.batch, len(c.q), 4)
    assert n > 0
    small = torch.zeros(n - 16, dtype=torch.uint8, device="cuda")
    for ws in (small[:0], small, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")):
        out, lse, scale = run(B, c, workspace=ws)
        check(c, out, lse, scale, True)
        again, _, _ = run(B, c, workspace=ws)
        assert torch.equal(out, again)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("new,keys", [([1, 2], [300, 2000]), ([130, 40], [900, 333])])
def test_pages_that_are_none(B, new, keys, fmt):
    """A page outside the cache holds nothing: its keys are not seen, wherever it lies in a tile; a sequence of
    nothing else gives 0 and -inf."""
    c = Case(B, new, keys, (4, 2), 128, 16, fmt, seed=14)
    table, hidden = c.table.clone(), []
    pages = c.cache.pages
    for i, s in enumerate(keys):
        h = torch.zeros(s, dtype=torch.bool)
        for j, bad in ((0, -1), (3, pages), (4, 2 ** 31 - 1), (10, -2 ** 31), ((s - 1) // 16, pages + 7)):
            if j * 16 < s:
                table[i, j] = bad
                h[16 * j: 16 * j + 16] = True
        hidden.append(h)
    c.batch = B.PagedBatch(i32(c.starts), i32(keys), table.cuda(), max_q=max(new), max_k=max(keys))
    out, lse, scale = run(B, c)
    check(c, out, lse, scale, True, hidden)
    c.batch = B.PagedBatch(i32(c.starts), i32(keys), torch.full_like(table, -1).cuda(), max_q=max(new), max_k=max(keys))
    out, lse, _ = run(B, c)
    assert bool((out[:sum(new)] == 0).all()) and bool(torch.isneginf(lse[:sum(new)]).all())


def test_lengths_out_of_range(B):
    """Lengths past the table are cut to it, negative ones are 0, starts are cut to the tokens."""
    for new, keys in (([1, 2], [64, 90]), ([100, 70], [64, 256])):
        c = Case(B, new, keys, (4, 2), 64, 16, "bf16", seed=15)
        T, w = sum(new), c.table.shape[1]
        full = [16 * w if k == max(keys) else k for k in keys]
        c2 = Case(B, new, full, (4, 2), 64, 16, "bf16", seed=15)
        c2.batch = B.PagedBatch(i32(c2.starts), i32([k if k != 16 * w else 2 ** 31 - 1 for k in full]), c2.table.cuda(),
                                max_q=max(new), max_k=16 * w)
        out, lse, scale = run(B, c2)
        check(c2, out, lse, scale, True)
        none = B.PagedBatch(i32(c.starts), i32([-3, -2 ** 31]), c.table.cuda(), max_q=max(new), max_k=max(keys))
        out = B.attn_paged(c.q.cuda(), c.cache, none)
        assert bool((out == 0).all())
        odd = B.PagedBatch(i32([-5, T + 1000, 2]), i32(keys), c.table.cuda())
        out = torch.full((T + 1, 4, 64), 5.0, device="cuda")
        B.attn_paged(torch.cat((c.q, c.q[:1])).cuda(), c.cache, odd, out=out)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(out).all())


def test_no_tokens(B):
    c = Case(B, [2], [10], (4, 1), 64, 16, "bf16")
    assert B.attn_paged(c.q[:0].cuda(), c.cache, c.batch).shape == (0, 4, 64)
    kv = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    assert B.kv_append(kv, kv, c.cache, c.batch) is None
    empty = Case(B, [0, 0], [5, 0], (4, 1), 64, 16, "bf16", pad=3)
    out, lse, _ = run(B, empty)                    # only padding: nothing is written (run checks it)


def test_many_sequences(B):
    """More sequences than one ballot looks at, some without tokens."""
    g = torch.Generator().manual_seed(16)
    new = [int(n) for n in torch.randint(0, 3, (150,), generator=g)]
    keys = [n + int(p) for n, p in zip(new, torch.randint(0, 90, (150,), generator=g))]
    for mq in (max(new), 0):
        c = Case(B, new, keys, (2, 1), 64, 16, "bf16", seed=17, pad=1)
        c.batch = B.PagedBatch(i32(c.starts), i32(keys), c.table.cuda(), max_q=mq, max_k=max(keys))
        out, lse, scale = run(B, c)
        check(c, out, lse, scale, True)


def test_another_stream(B):
    """On a stream that is not the current one, with scratch of that stream's."""
    c = Case(B, [1, 1], [3000, 9000], (4, 1), 128, 64, "bf16", seed=18)
    want, wl, scale = run(B, c)
    side = torch.cuda.Stream()
    q = c.q.cuda()
    out, lse = torch.zeros_like(want), torch.zeros_like(wl)
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        B.attn_paged(q, c.cache, c.batch, scale=scale, out=out, lse=lse, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want) and torch.equal(lse, wl)


def test_captured_step(B):
    """One generation step (append, attention) captured once and replayed as the sequences grow: lengths, positions
    and pages are read when it is replayed."""
    g = torch.Generator().manual_seed(19)
    hq, hkv, D, page, N, S = 8, 2, 128, 16, 3, 40
    inv = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    data = torch.randn(S, N, hq + 2 * hkv, D, generator=g).bfloat16().cuda()
    table = i32(torch.randperm(3 * N + 1, generator=g)[:3 * N].view(N, 3).tolist())
    x, pos, seq_k = torch.zeros_like(data[0]), i32([0] * N), i32([1] * N)
    start = i32(list(range(N + 1)))

    def step(cache, batch, x, pos, out):
        q = B.kv_append(x[:, hq:hq + hkv], x[:, hq + hkv:], cache, batch, q=x[:, :hq], pos=pos, inv_freq=inv)
        return B.attn_paged(q, cache, batch, out=out)

    caches = [B.PagedCache.empty(3 * N + 1, page, hkv, D) for _ in range(2)]
    for c in caches:
        c.k.zero_(), c.v.zero_()
    batch = B.PagedBatch(start, seq_k, table, max_q=1, max_k=48)
    out, eager = torch.empty(N, hq, D, device="cuda"), torch.empty(N, hq, D, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0], batch, x, pos, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], batch, x, pos, out)
    for t in range(S):
        x.copy_(data[t])
        pos.fill_(t)
        seq_k.fill_(t + 1)
        graph.replay()
        now = B.PagedBatch(start, i32([t + 1] * N), table, max_q=1, max_k=48)
        step(caches[1], now, data[t], i32([t] * N), eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), t
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)


def test_another_device_is_refused(B):
    """Tensors of another device than the current one: refused, not run on the wrong one."""
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    c = B.PagedCache.empty(2, 16, 1, 64)
    b = B.PagedBatch(i32([0, 2]), i32([2]), i32([[0]]))
    now = torch.cuda.current_device
    try:
        torch.cuda.current_device = lambda: 1
        for f in (lambda: B.attn_paged(x, c, b), lambda: B.kv_append(x[:, :1], x[:, :1], c, b),
                  lambda: B.rope(x, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda"))):
            with pytest.raises(ValueError):
                f()
    finally:
        torch.cuda.current_device = now


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_offsets_past_32_bits(B, fmt):
    """Pages beyond 4 GiB of a cache, written by the append and read by both kernels."""
    hkv, D, page = 8, 128, 256
    row = D * 2 if fmt == "bf16" else D
    pages = (1 << 32) // (hkv * page * row) + 40
    if torch.cuda.mem_get_info()[0] < 5 * pages * hkv * page * row:
        pytest.skip("needs 24 GB of device memory")
    cache = B.PagedCache.empty(pages, page, hkv, D, fmt)
    small = B.PagedCache.empty(3, page, hkv, D, fmt)
    far = [pages - 1, pages - 30, pages - 7]
    g = torch.Generator().manual_seed(20)
    k, v, q = (torch.randn(600, h, D, generator=g).bfloat16().cuda() for h in (hkv, hkv, 16))
    for n in (600, 1):
        batches = [B.PagedBatch(i32([0, n]), i32([600]), i32([t]), max_q=n, max_k=600) for t in (far, [0, 1, 2])]
        if n == 600:
            for c, b in zip((cache, small), batches):
                B.kv_append(k, v, c, b)
        a, b = (B.attn_paged(q[:n], c, b) for c, b in zip((cache, small), batches))
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    for i, p in enumerate(far):
        n = min(page, 600 - i * page)                # the slots behind them were never written
        assert torch.equal(cache.k[p, :, :n], small.k[i, :, :n]) and torch.equal(cache.v[p, :, :n], small.v[i, :, :n])


@pytest.mark.parametrize("heads,D", [((7, 1), 64), ((33, 3), 128), ((100, 4), 64), ((48, 1), 128), ((130, 2), 128), ((5, 5), 64)])
@pytest.mark.parametrize("new,keys", [([1, 1, 1], [90, 700, 1]), ([5, 1, 9], [300, 64, 9]), ([70, 33], [500, 40])])
def test_any_number_of_heads_to_a_key(B, heads, D, new, keys):
    c = Case(B, new, keys, heads, D, 32, "bf16", seed=30, pad=1)
    out, lse, scale = run(B, c)
    check(c, out, lse, scale, True)
