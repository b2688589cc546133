"""Where the binding takes a call's scratch from (CPU: torch's stream and allocation calls are
recorded, nothing runs on a GPU)."""

import contextlib
import types

import pytest

import paper_2606_16317_amd as dsa


@pytest.fixture
def recorded(monkeypatch):
    torch = pytest.importorskip("torch")
    log = []

    @contextlib.contextmanager
    def on(stream):
        log.append(("stream", stream.cuda_stream, str(stream.device)))
        yield

    def empty(n, dtype, device):
        log.append(("empty", n, str(device)))
        return types.SimpleNamespace(data_ptr=lambda: 4096)

    def external(handle, device):
        return types.SimpleNamespace(cuda_stream=handle, device=device)

    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch, "empty", empty)
    return log


def test_scratch_belongs_to_the_device_of_the_launch(recorded):
    """Tensors on cuda:1: without a stream the kernels go to the current device's current
    stream, with one to that stream's device."""
    dsa._workspace(64, "cuda:1", None)
    assert recorded == [("empty", 64, "cuda")]
    recorded.clear()
    dsa._workspace(64, "cuda:1", types.SimpleNamespace(cuda_stream=7, device="cuda:0"))
    assert recorded == [("stream", 7, "cuda:0"), ("empty", 64, "cuda:0")]
    recorded.clear()
    dsa._workspace(64, "cuda:1", types.SimpleNamespace(cuda_stream=8))
    assert recorded == [("stream", 8, "cuda:1"), ("empty", 64, "cuda:1")]
    assert dsa._workspace(0, "cuda:1", None) is None


@pytest.mark.parametrize("stream", [None, types.SimpleNamespace(cuda_stream=7, device="cuda:0")])
def test_optional_scratch_is_left_out_under_capture_and_without_memory(recorded, monkeypatch,
                                                                       stream):
    torch = pytest.importorskip("torch")
    assert dsa._workspace(64, "cuda:0", stream, optional=True) is not None

    def full(*args, **kw):
        raise torch.cuda.OutOfMemoryError("full")

    with monkeypatch.context() as m:
        m.setattr(torch, "empty", full)
        assert dsa._workspace(64, "cuda:0", stream, optional=True) is None
        with pytest.raises(torch.cuda.OutOfMemoryError):
            dsa._workspace(64, "cuda:0", stream)
    recorded.clear()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    assert dsa._workspace(64, "cuda:0", stream, optional=True) is None
    assert not any(entry[0] == "empty" for entry in recorded)
    assert dsa._workspace(64, "cuda:0", stream) is not None     # what the call needs, it gets


@pytest.fixture
def pools(monkeypatch):
    """CPU tensors that pass for GPU ones, a library whose calls succeed, and a log of what is
    allocated in which stream's pool and whom it is recorded for."""
    torch = pytest.importorskip("torch")
    log, inside = [], ["current"]

    class Gpu(torch.Tensor):
        is_cuda = property(lambda self: True)

    @contextlib.contextmanager
    def on(stream):
        inside.append(stream.cuda_stream)
        yield
        inside.pop()

    def allocation(make):
        def call(*args, **kw):
            if kw.get("device") == "cuda":
                kw["device"] = "cpu"
            log.append(("pool", inside[-1]))
            return make(*args, **kw).as_subclass(Gpu)
        return call

    class Library:
        def __getattr__(self, name):
            return lambda *args: 256 if name.endswith("_bytes") else 0

    handle = lambda n, device=None: types.SimpleNamespace(cuda_stream=n, device=device)
    monkeypatch.setattr(torch, "empty", allocation(torch.empty))
    monkeypatch.setattr(torch, "empty_like", allocation(torch.empty_like))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", handle)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: handle(3))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 3, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda self, s: log.append(("used by", s.cuda_stream)))
    monkeypatch.setattr(dsa, "lib", lambda: Library())
    for size in (dsa.dsattn_attn_bwd_workspace_bytes, dsa.dsattn_bias_attn_workspace_bytes,
                 dsa.dsattn_bias_attn_bwd_workspace_bytes):
        size.cache_clear()
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype).as_subclass(Gpu)
    yield new, handle, log
    for size in (dsa.dsattn_attn_bwd_workspace_bytes, dsa.dsattn_bias_attn_workspace_bytes,
                 dsa.dsattn_bias_attn_bwd_workspace_bytes):
        size.cache_clear()


def calls(new):
    """(name, call, outputs that it makes, pieces of scratch) of every entry that makes outputs."""
    import torch

    q, lse = new(1, 2, 64, 128), new(1, 2, 64, dtype=torch.float32)
    table, bucket = new(4, 2, dtype=torch.float32), new(127, dtype=torch.int32)
    index = new(64, dtype=torch.int32)
    q8, s8 = new(1, 2, 64, 128, dtype=torch.uint8), new(1, 2, 64, 4, dtype=torch.uint8)
    return [
        ("bwd", lambda **kw: dsa.dsattn_attn_bwd(0, q, q, q, q, lse, q, **kw), 3, 1),
        ("bias", lambda **kw: dsa.dsattn_bias_attn_fwd(q, q, q, table, bucket, **kw), 1, 1),
        ("bias bwd", lambda **kw: dsa.dsattn_bias_attn_bwd(q, q, q, table, bucket, q, lse, q, **kw),
         4, 1),
        ("dynsparse", lambda **kw: dsa.dynsparse_attn_fwd(q, q, q, **kw), 1, 0),
        ("lambda", lambda **kw: dsa.dynsparse_attn_fwd_lambda(q, q, q, **kw), 1, 0),
        ("blasst", lambda **kw: dsa.blasst_attn_fwd(q, q, q, **kw), 1, 0),
        ("dense", lambda **kw: dsa.dense_attn_fwd(q, q, q, **kw), 1, 0),
        ("ex", lambda **kw: dsa.dsattn_attn_fwd_ex(0, 0.0, q, q, q, **kw), 1, 0),
        ("mxfp8", lambda **kw: dsa.dsattn_attn_fwd_mxfp8(0, 0.0, q8, s8, q8, s8, q, **kw), 1, 0),
        ("reordered", lambda **kw: dsa.dsattn_attn_fwd_reordered(0, 0.0, q, q, q, index, index, **kw),
         1, 1),
        ("noalloc", lambda **kw: dsa.dsattn_attn_fwd_reordered_noalloc(0, 0.0, q, q, q, index, index,
                                                                       **kw), 1, 0),
        ("gather", lambda **kw: dsa.dsattn_gather_rows(q, index, **kw), 1, 0),
        ("scatter", lambda **kw: dsa.dsattn_scatter_rows(q, index, **kw), 1, 0),
        ("quantize", lambda **kw: dsa.dsattn_quantize_mxfp8(q, **kw), 2, 0),
        ("key mean", lambda **kw: dsa.dsattn_key_mean(q, **kw), 1, 1),
    ]


def test_outputs_come_from_the_pool_of_the_stream(pools):
    """What a call on another stream makes belongs to that stream, and to the current one that may
    read it; without a stream, or on the current one, all is as torch has it."""
    new, handle, log = pools
    for name, call, outputs, scratch in calls(new):
        log.clear()
        call(stream=handle(7, "cpu"))
        assert log.count(("pool", 7)) == outputs + scratch, name
        assert log.count(("used by", 3)) == outputs, name
        assert len(log) == 2 * outputs + scratch, name
        log.clear()
        call(stream=handle(3, "cpu"))
        assert log == [("pool", 3)] * (outputs + scratch), name
        log.clear()
        call()
        assert log == [("pool", "current")] * (outputs + scratch), name
