"""Where the outputs that a caller does not bring are allocated: in the memory pool
of the stream the call runs on, and kept while the current stream may use them.
Without a GPU the allocation and the library are replaced."""
import contextlib

import pytest
import torch


class OnGpu:
    """A CPU tensor that says it is on cuda:0."""

    is_cuda, device = True, "cuda:0"

    def __init__(self, t, log):
        self.t, self.log = t, log

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.log.append(("kept for", stream))


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


CURRENT, SIDE, WRAPPED = Stream(1), Stream(7), "wrapped 9"


@pytest.fixture
def B(monkeypatch):
    """The binding with a library that computes nothing; B.log has what is allocated, under which stream."""
    from paper_2609_09721_amd import binding
    real, now, log = torch.empty, [], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def empty(shape, dtype=None, device=None):
        shape = (shape,) if isinstance(shape, int) else tuple(shape)
        log.append(("allocated", now[-1] if now else None))
        return OnGpu(real(shape, dtype=dtype), log)

    class Library:
        def __getattr__(self, name):
            return lambda *a: log.append((name, None)) or (256 if name.endswith("_bytes") and "paged" not in name else 0)

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: f"wrapped {handle}")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: CURRENT)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1, raising=False)
    library = Library()
    monkeypatch.setattr(binding, "lib", lambda: library)
    monkeypatch.setattr(binding, "_scratch", lambda n, stream=None: None)
    monkeypatch.setattr(binding, "log", log, raising=False)
    return binding


class Handle:
    cuda_stream = 9


def gpu(B, shape, dtype=torch.bfloat16):
    return OnGpu(torch.zeros(shape, dtype=dtype), B.log)


def paged(B):
    cache = B.PagedCache(gpu(B, (2, 2, 16, 64)), gpu(B, (2, 2, 16, 64)))
    i32 = lambda *s: gpu(B, s, torch.int32)
    return cache, B.PagedBatch(i32(2), i32(1), i32(1, 2)), gpu(B, (3, 2, 64)), gpu(B, (3, 4, 64)), i32(3), gpu(B, (32,), torch.float32)


def calls(B):
    cache, batch, kv, q, pos, inv = paged(B)
    yield "rope", lambda **k: B.rope(q, pos, inv, **k)
    yield "rope_bwd", lambda **k: B.rope_bwd(q, pos, inv, **k)
    yield "kv_append", lambda **k: B.kv_append(kv, kv, cache, batch, q=q, **k)
    yield "attn_paged", lambda **k: B.attn_paged(q, cache, batch, **k)


def forward_calls(B):
    """The attention forward's functions, those of their kinds that allocate."""
    q, k = gpu(B, (1, 5, 4, 64)), gpu(B, (1, 5, 2, 64))
    sh, buf, f32 = B.Shape(1, 5, 5, 4, 2, 64), gpu(B, (64,), torch.uint8), gpu(B, (1, 5, 4, 64), torch.float32)
    yield "quant_v", lambda **a: B.quant_v(k, **a)
    yield "quant_qk", lambda **a: B.quant_qk(q, k, **a)
    yield "attn_fwd", lambda **a: B.attn_fwd(q, k, k, **a)
    yield "attn_fwd_vhat", lambda **a: B.attn_fwd_vhat(q, k, buf, **a)
    yield "efq_attn_fwd", lambda **a: B.efq_attn_fwd(q, k, k, **a)
    yield "efq_attn_fwd_expq", lambda **a: B.efq_attn_fwd_expq(q, k, k, **a)
    yield "attn_fwd_dump", lambda **a: B.attn_fwd_dump(q, k, buf, **a)
    yield "attn_fwd_qk8", lambda **a: B.attn_fwd_qk8(buf, buf, buf, sh, **a)
    yield "attn_fwd_qk8_dump", lambda **a: B.attn_fwd_qk8_dump(buf, buf, buf, sh, **a)
    yield "attn_fwd_lowbit", lambda **a: B.attn_fwd_lowbit(q, k, k, **a)
    yield "calibrate", lambda **a: B.calibrate(q, k, k, f32, [-3.0], [2.0], **a)
    yield "pgen", lambda **a: B.pgen(gpu(B, (2, 64), torch.float32), **a)
    yield "pgen_bench", lambda **a: B.pgen_bench(**a)
    yield "clock_probe", lambda **a: B.clock_probe(**a)


NAMES = ["rope", "rope_bwd", "kv_append", "attn_paged", "quant_v", "quant_qk", "attn_fwd", "attn_fwd_vhat", "efq_attn_fwd",
         "efq_attn_fwd_expq", "attn_fwd_dump", "attn_fwd_qk8", "attn_fwd_qk8_dump", "attn_fwd_lowbit", "calibrate", "pgen",
         "pgen_bench", "clock_probe"]


@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_in_the_pool_of_the_calls_stream(B, name):
    f = {**dict(calls(B)), **dict(forward_calls(B))}[name]
    for stream, pool, kept in ((None, None, False), (SIDE, SIDE, True), (CURRENT, None, False), (Handle(), WRAPPED, True)):
        del B.log[:]
        f(stream=stream)
        outputs = [x for x in B.log if x[0] == "allocated"]
        assert outputs and all(x == ("allocated", pool) for x in outputs), (name, B.log)
        assert [x for x in B.log if x[0] == "kept for"] == [("kept for", CURRENT)] * (len(outputs) if kept else 0)


def pool_of(t):
    """The stream handle whose memory pool t lies in."""
    at = t.data_ptr()
    return [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]


@pytest.mark.gpu
@pytest.mark.parametrize("handle", [False, True])
def test_another_stream_with_outputs_of_its_own(handle):
    """Outputs that the calls allocate, on a stream that is not the current one: its pool, and the same values."""
    from paper_2609_09721_amd import binding as B
    g = torch.Generator().manual_seed(6)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    x, kv = (torch.randn(40, h, 64, generator=g).bfloat16().cuda() for h in (8, 2))
    pos, inv = torch.arange(40, dtype=torch.int32).cuda(), torch.rand(32, generator=g).cuda()
    cache = B.PagedCache.empty(3, 16, 2, 64)
    batch = B.PagedBatch(i32([0, 40]), i32([40]), i32([[2, 0, 1]]), max_q=40, max_k=40)
    calls = [lambda **k: B.rope(x, pos, inv, **k), lambda **k: B.rope_bwd(x, pos, inv, **k),
             lambda **k: B.kv_append(kv, kv, cache, batch, q=x, pos=pos, inv_freq=inv, **k), lambda **k: B.attn_paged(x, cache, batch, **k)]
    want = [f() for f in calls]
    side = torch.cuda.Stream()

    class Raw:
        cuda_stream = side.cuda_stream

    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = [f(stream=Raw() if handle else side) for f in calls]
        torch.cuda.current_stream().wait_stream(side)
        for g, w in zip(got, want):
            assert pool_of(g) == [side.cuda_stream] and pool_of(w) != pool_of(g)
            assert torch.equal(g, w)
        del got
        side.wait_stream(torch.cuda.current_stream())


@pytest.mark.gpu
def test_captured_on_a_forked_stream():
    """Calls on a stream that a capture forks to, with outputs of their own; replays between eager calls."""
    from paper_2609_09721_amd import binding as B
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    x, kv = torch.zeros(40, 8, 64, device="cuda").bfloat16(), torch.zeros(40, 2, 64, device="cuda").bfloat16()
    pos, inv = torch.arange(40, dtype=torch.int32).cuda(), torch.rand(32).cuda()
    cache = B.PagedCache.empty(3, 16, 2, 64)
    batch = B.PagedBatch(i32([0, 40]), i32([40]), i32([[2, 0, 1]]), max_q=40, max_k=40)
    side = torch.cuda.Stream()

    def step(**k):
        q = B.kv_append(kv, kv, cache, batch, q=x, pos=pos, inv_freq=inv, **k)
        return B.attn_paged(B.rope(q, pos, inv, **k), cache, batch, **k)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = step(stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        x.copy_(torch.randn(x.shape)), kv.copy_(torch.randn(kv.shape))
        graph.replay()
        torch.cuda.synchronize()
        now = got.clone()
        assert torch.equal(now, step()), i
        torch.cuda.synchronize()
