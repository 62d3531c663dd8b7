"""Sequences whose length or starts do not fit the page table or the call's tokens:
a new token is the key that its sequence's length and end say, so what the table has
no slot for is dropped and no key that is already there is written over."""
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


BIG = 2 ** 31 - 1


# starts, lengths, table -> (page, slot) of the tokens that are appended, page size 16, 6 tokens
@pytest.mark.parametrize("starts,keys,table,want", [
    ([0, 1], [17], [[1]], {}),                                             # just outgrown
    ([0, 3], [18], [[1]], {(1, 15): 0}),                                   # by two of its three tokens
    ([0, 2], [1000], [[1]], {}),
    ([0, 6], [BIG], [[1]], {}),
    ([0, 2, 6], [33, 20], [[2, 0], [1, 3]], {(0, 15): 0, (3, 0): 2, (3, 1): 3, (3, 2): 4, (3, 3): 5}),
    ([0, 9], [12], [[1]], {(1, 3 + t): t for t in range(6)}),              # three tokens more than the call has
    ([0, 2, 8], [16, 7], [[0], [1]], {(0, 14): 0, (0, 15): 1, (1, 1): 2, (1, 2): 3, (1, 3): 4, (1, 4): 5}),
    ([-3, 3, 6], [4, 3], [[0], [1]], {(0, 1): 0, (0, 2): 1, (0, 3): 2, (1, 0): 3, (1, 1): 4, (1, 2): 5}),
    # as before: bad pages, more tokens than keys, negative lengths
    ([0, 3, 6], [3, 17], [[1, -1], [0, 9]], {(1, 0): 0, (1, 1): 1, (1, 2): 2, (0, 14): 3, (0, 15): 4}),
    ([0, 6], [2], [[0]], {(0, 0): 4, (0, 1): 5}),
    ([0, 2], [-5], [[1]], {}),
])
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_append_keeps_the_keys_that_are_there(B, starts, keys, table, want, fmt):
    print(f"[append] {(starts, keys, table, fmt)}", flush=True)
    g = torch.Generator().manual_seed(len(want) + 1)
    k, v, old_k, old_v = (torch.randn(n, 2, 64, generator=g).bfloat16().cuda() for n in (6, 6, 96, 96))

    def cache():                             # six pages: the first and last are none of the call's
        c = B.PagedCache.empty(6, 16, 2, 64, fmt)
        B.kv_append(old_k, old_v, c, B.PagedBatch(i32([0, 96]), i32([96]), i32([[0, 1, 2, 3, 4, 5]])))
        return c

    parts = ("k", "v") + (("k_scale", "v_scale") if fmt == "mxfp8" else ())
    a, b = cache(), cache()
    inner = B.PagedCache(*(getattr(a, n)[1:-1] for n in parts))
    B.kv_append(k, v, inner, B.PagedBatch(i32(starts), i32(keys), i32(table)))
    new = B.PagedCache.empty(1, 16, 2, 64, fmt)            # the tokens side by side, as they are stored
    B.kv_append(k, v, new, B.PagedBatch(i32([0, 6]), i32([6]), i32([[0]])))
    for n in parts:
        expect = getattr(b, n)
        for (p, o), t in want.items():
            expect[p + 1, :, o] = getattr(new, n)[0, :, t]
        assert torch.equal(getattr(a, n), expect), n


class Placed(Case):
    """A case whose token j of a sequence sees its first `visible` keys."""

    def reference(self, scale, causal, hidden=None):
        hq, hkv = self.heads
        T = self.starts[-1]
        out, mag = (torch.zeros(T, hq, self.D, dtype=torch.float64) for _ in range(2))
        lse = torch.full((T, hq), -math.inf, dtype=torch.float64)
        size = torch.zeros(T, hq, dtype=torch.float64)
        for t, (i, n) in enumerate(self.visible):
            if n == 0:
                continue
            q = self.q[t].double()
            k, v = (x[i][:n].double().repeat_interleave(hq // hkv, 1) for x in (self.k, self.v))
            x = torch.einsum("hd,shd->hs", q, k) * scale
            lse[t] = torch.logsumexp(x, -1)
            p = torch.softmax(x, -1)
            out[t], mag[t] = torch.einsum("hs,shd->hd", p, v), torch.einsum("hs,shd->hd", p, v.abs())
            size[t] = torch.einsum("hd,shd->hs", q.abs(), k.abs()).amax(-1) * scale
        return out, lse, mag, size


# new tokens, the keys that the table holds, the lengths given
@pytest.mark.parametrize("new,held,given", [
    ([3, 1], [64, 32], [65, 40]), ([5], [1024], [1027]), ([2, 2], [48, 2048], [5000, 2049]),       # few tokens
    ([130, 40], [64, 256], [150, 257]), ([300], [1024], [1100]), ([70, 64], [48, 48], [100000, 20]),  # chunks
    ([90], [4096], [4100])])                                                                       # split keys
@pytest.mark.parametrize("heads,D,fmt", [((4, 1), 128, "bf16"), ((8, 2), 64, "mxfp8")])
def test_attention_ends_at_the_table(B, new, held, given, heads, D, fmt):
    c = Placed(B, new, held, heads, D, 16, fmt, seed=sum(new), pad=1)
    room = 16 * c.table.shape[1]
    c.visible = [(i, max(0, min(s - n + j + 1, room, h))) for i, (n, h, s) in enumerate(zip(new, held, given)) for j in range(n)]
    # a shorter sequence's table goes on with entries that are none
    c.batch = B.PagedBatch(i32(c.starts), i32(given), c.table.cuda(), max_q=max(new), max_k=max(held))
    out, lse, scale = run(B, c)
    check(c, out, lse, scale, True)


@pytest.mark.parametrize("new,keys,more", [([6], [100], 3), ([100], [150], 40), ([3], [2000], 1)])
def test_attention_of_a_sequence_with_more_tokens_than_the_call(B, new, keys, more):
    """The end past the call's tokens: these are the first of the sequence's new ones."""
    c = Placed(B, new, keys, (4, 2), 64, 16, "bf16", seed=3)
    c.visible = [(0, keys[0] - new[0] - more + j + 1) for j in range(new[0])]
    c.batch = B.PagedBatch(i32([0, new[0] + more]), i32(keys), c.table.cuda())
    out, lse, scale = run(B, c)
    check(c, out, lse, scale, True)


def test_a_sequence_that_outgrows_its_table(B):
    """One token a step past the table's 32 keys: the keys stay, and a step's output is that over them."""
    g = torch.Generator().manual_seed(5)
    data = torch.randn(40, 8, 64, generator=g).bfloat16().cuda()
    cache, table = B.PagedCache.empty(4, 16, 2, 64), i32([[3, 1]])
    kept = None
    for t in range(40):
        x = data[t:t + 1]
        batch = B.PagedBatch(i32([0, 1]), i32([t + 1]), table, max_q=1, max_k=32)
        B.kv_append(x[:, 4:6], x[:, 6:], cache, batch)
        out = B.attn_paged(x[:, :4], cache, batch)
        if t == 31:
            kept = cache.k[[3, 1]].clone(), cache.v[[3, 1]].clone()
        if t >= 32:
            assert torch.equal(cache.k[[3, 1]], kept[0]) and torch.equal(cache.v[[3, 1]], kept[1])
        whole = B.PagedBatch(i32([0, 1]), i32([min(t + 1, 32)]), table, max_q=1, max_k=32)
        assert torch.equal(out, B.attn_paged(x[:, :4], cache, whole))
