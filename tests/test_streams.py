"""Calls on a stream of the caller's: memory that a call allocates by itself (workspace, outputs) comes from the pool of
the stream its kernels run on, so that no work queued elsewhere is given it while they run."""
import contextlib

import pytest
import torch

from paper_2606_04302_amd import ops
from paper_2606_04302_amd import workloads as W


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ops.lib()
    torch.cuda.init()


class _Library:
    """Stands in for the loaded library: sizes are 64 bytes, every call succeeds and notes its last argument."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_size"):
                return 64
            self.streams.append(args[-1])
            return 0
        return call


@pytest.mark.parametrize("name", ["prefill", "decode", "decode_shared", "combine", "materialize_k", "run_lazy",
                                  "run_materialized", "prefill_backward"])
def test_memory_is_allocated_for_the_stream_of_the_call(monkeypatch, name):
    """Every allocation of a call on a stream is made for that stream (host tensors and a stand-in library)."""
    stream, inside, made = 0x5EED0, [], []
    library = _Library()

    @contextlib.contextmanager
    def allocating_for(s):
        inside.append(s)
        yield
        inside.pop()

    def noted(fn):
        def alloc(*a, **kw):
            made.append(inside[-1] if inside else None)
            return fn(*a, **kw)
        return alloc

    w = W.tiny_rag_prefill(0)
    dw = ops.upload(w, "cpu")
    wd = W.rag_decode(seed=1, batch=2, hq=4, hkv=2, d=64, n_chunks=2, chunk_len=20, pool_chunks=3, tail_len=2, tail_cap=4)
    dd = ops.upload(wd, "cpu")
    cfg, dcfg = ops.config_of(w), ops.config_of(wd)
    shared = ops.upload_plan(ops.shared_decode_plan(dcfg, wd.chunks, wd.chunk_start), "cpu")
    back = ops.upload_backward_plan(ops.backward_plan(cfg, w.q_start, w.q_pos0, w.chunks, w.chunk_start), "cpu")
    part, lse = torch.zeros(2, 3, 64, dtype=torch.bfloat16), torch.zeros(w.total_q, w.num_q_heads)
    calls = {
        "prefill": lambda: ops.prefill(cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.pool, dw.chunks, dw.chunk_start,
                                       4, 8, stream=stream),
        "decode": lambda: ops.decode(dcfg, dd.q, dd.q_pos0, dd.pool, dd.pool, dd.chunks, dd.chunk_start, 8,
                                     stream=stream),
        "decode_shared": lambda: ops.decode_shared(dcfg, dd.q, dd.q_pos0, dd.pool, dd.pool, shared, stream=stream),
        "combine": lambda: ops.combine(part, torch.zeros(2, 3), stream=stream),
        "materialize_k": lambda: ops.materialize_k(cfg, dw.pool, dw.chunks, 4, 8, stream=stream),
        "run_lazy": lambda: ops.run_lazy(dd, dcfg, stream=stream),
        "run_materialized": lambda: ops.run_materialized(dd, dcfg, stream=stream),
        "prefill_backward": lambda: ops.prefill_backward(cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.pool, dw.chunks,
                                                         dw.chunk_start, dw.q, lse, dw.q, back, stream=stream),
    }
    monkeypatch.setattr(ops, "lib", lambda: library)
    monkeypatch.setattr(ops, "_dev", lambda *a: None)
    monkeypatch.setattr(ops, "_chunks", lambda *a: None)
    monkeypatch.setattr(ops, "_allocating_for", allocating_for)
    for fn in ("empty", "empty_like", "zeros_like"):
        monkeypatch.setattr(torch, fn, noted(getattr(torch, fn)))
    calls[name]()
    assert made and set(made) == {stream}
    assert library.streams and set(library.streams) == {stream}


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
@pytest.mark.parametrize("how", ["gone", "another"])
def test_current_stream_without_the_functions_that_are_not_public(monkeypatch, missing, how):
    class Public:
        cuda_stream = 0xC0FFEE

    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Public)
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.setattr(torch._C, name, lambda *a: 0, raising=False)
    assert ops._stream(None) == 0
    if how == "gone":
        monkeypatch.delattr(torch._C, missing)
    else:
        monkeypatch.setattr(torch._C, missing, lambda one, two, three: 0)
    assert ops._stream(None) == 0xC0FFEE
    assert ops._stream(5) == 5 and ops._stream(Public) == 0xC0FFEE


@pytest.mark.gpu
def test_the_current_streams_pointer_is_the_public_one(gpu):
    side = torch.cuda.Stream()
    assert ops._stream(None) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert ops._stream(None) == side.cuda_stream


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["pointer 0", "default stream", "side stream"])
def test_calls_that_allocate_take_any_stream(gpu, which):
    """The default stream has the pointer 0."""
    side = torch.cuda.Stream()
    stream = {"pointer 0": 0, "default stream": torch.cuda.default_stream(), "side stream": side}[which]
    w = W.custom(4, 8, 2, 128, 1.0e4, [dict(chunks=[(300, 0), (40, 300)], q_len=40, q_pos0=300)])
    dw = ops.upload(w)
    cfg = ops.config_of(w, num_splits=3)
    plan = ops.upload_backward_plan(ops.backward_plan(cfg, w.q_start, w.q_pos0, w.chunks, w.chunk_start))

    def call(s):
        out, lse = ops.run_lazy(dw, cfg, stream=s)
        grads = ops.prefill_backward(cfg, dw.q, dw.q_start, dw.q_pos0, dw.pool, dw.pool, dw.chunks, dw.chunk_start, out,
                                     lse, dw.q, plan, stream=s)
        both = ops.run_materialized(dw, cfg, stream=s)[0]
        return (out, lse, *grads, *both)

    want = call(None)
    torch.cuda.synchronize()
    got = call(stream)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_forward_calls_on_another_stream_keep_their_memory(gpu):
    """Split decode and prefill on a stream that is still busy, while the current stream allocates and fills memory of
    the sizes that the calls took: the same bits as on the current stream."""
    wd = W.rag_decode(seed=2, batch=3, hq=8, hkv=2, d=128, n_chunks=5, chunk_len=200, pool_chunks=7, tail_len=9,
                      tail_cap=16)
    wp = W.custom(3, 8, 2, 128, 1.0e4, [dict(chunks=[(2000, 0), (40, 2000)], q_len=40, q_pos0=2000)])
    side = torch.cuda.Stream()
    for w in (wd, wp):
        dw = ops.upload(w)
        cfg = ops.config_of(w, num_splits=7)
        if w.kind == "decode":
            nbytes = ops.decode_workspace_size(cfg, w.batch, w.max_kv_len)
        else:
            nbytes = ops.prefill_workspace_size(cfg, w.batch, w.total_q, w.max_q_len, w.max_kv_len)
        assert nbytes > 0
        want = ops.run_lazy(dw, cfg)
        torch.cuda.synchronize()
        big = torch.randn(4096, 4096, device="cuda")
        for stream in (side, side.cuda_stream):
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                for _ in range(8):
                    big @ big
            out, lse = ops.run_lazy(dw, cfg, stream=stream)
            over = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (nbytes, out.numel() * 2, nbytes)]
            side.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            del over
