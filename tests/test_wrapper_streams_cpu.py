"""What the op-level wrappers tell PyTorch's allocator when they are given a stream.

A block that was freed on one stream may still be read or written by that stream's queued
kernels, so memory for a call on another stream has to come from that stream; and what is
used on a stream that it does not come from has to be recorded there.  Looked at here with
host tensors that say they are CUDA ones and a library that does nothing: the race itself
would corrupt memory on a GPU."""
import contextlib
import types

import pytest
import torch

from paper_2608_10362_gb300 import engine

CURRENT, SIDE = types.SimpleNamespace(cuda_stream=1), types.SimpleNamespace(cuda_stream=2)


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0

    def record_stream(self, stream):
        LOG.append(("record", self.data_ptr(), stream))


LOG = []


def _t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def allocations(monkeypatch):
    """[(tensor, the stream that was current when it was made)]"""
    stack, made = [CURRENT], []

    @contextlib.contextmanager
    def stream(s):
        stack.append(s)
        yield
        stack.pop()

    def maker(real):
        def make(*size, **kw):
            t = real(*size, **kw).as_subclass(OnGpu)
            made.append((t, stack[-1]))
            return t
        return make

    class Library:
        memspec_int4_packed_bytes = staticmethod(lambda n, k: 1072)

        def __getattr__(self, name):
            return lambda *args: 0

    LOG.clear()
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stack[-1])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: CURRENT.cuda_stream, raising=False)
    monkeypatch.setattr(torch, "empty", maker(torch.empty))
    monkeypatch.setattr(torch, "zeros", maker(torch.zeros))
    monkeypatch.setattr(engine._lib, "load", Library)
    monkeypatch.setattr(engine, "_linear_scratch_bytes", lambda *a: 512)
    monkeypatch.setattr(engine, "_lora_scratch_bytes", lambda *a: 512)
    monkeypatch.setattr(engine, "_call_on", lambda dev, stream, fn, *args: 0)
    return made


BF = torch.bfloat16
CALLS = {   # name: (the call's tensors, the call)
    "linear": (lambda: [_t(2, 128, dtype=BF), _t(16, 128, dtype=BF)], lambda s, x, w: engine.op_linear(x, w, stream=s)),
    "linear_noalloc": (lambda: [_t(2, 128, dtype=BF), _t(16, 128, dtype=BF)],
                       lambda s, x, w: engine.op_linear_noalloc(x, w, stream=s)),
    "int4_pack": (lambda: [_t(16, 64, dtype=torch.uint8), _t(16, 1, dtype=BF), _t(16, 1, dtype=torch.uint8)],
                  lambda s, q, sc, z: engine.int4_pack(q, sc, z, stream=s)),
    "linear_int4": (lambda: [_t(2, 128, dtype=BF), _t(1072, dtype=torch.uint8)],
                    lambda s, x, p: engine.op_linear_int4(x, p, 16, stream=s)),
    "sample_filtered": (lambda: [_t(2, 40), _t(2), _t(2)],
                        lambda s, z, u, p: engine.op_sample_filtered(z, u, top_p=p, stream=s)),
    "filter_logits": (lambda: [_t(2, 40), _t(2, dtype=torch.int32)],
                      lambda s, z, k: engine.op_filter_logits(z, top_k=k, stream=s)),
    "lora": (lambda: [_t(2, 64, dtype=BF), _t(3, 8, 64, dtype=BF), _t(3, 32, 8, dtype=BF), _t(2, dtype=torch.int32),
                      _t(3), _t(3, dtype=torch.int32), _t(2, 32)],
             lambda s, *v: engine.op_lora(*v, stream=s)),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_comes_from_the_stream_of_the_call(allocations, name):
    tensors, call = CALLS[name]
    tensors = tensors()
    allocations.clear()
    out = call(SIDE, *tensors)
    assert allocations and all(s is SIDE for _, s in allocations)
    assert ("record", out.data_ptr(), CURRENT) in LOG     # the caller goes on with it there
    allocations.clear()
    LOG.clear()
    call(None, *tensors)
    assert allocations and all(s is CURRENT for _, s in allocations) and not LOG


@pytest.mark.parametrize("name", CALLS)
def test_the_callers_tensors_are_recorded_on_the_stream_of_the_call(allocations, name):
    tensors, call = CALLS[name]
    tensors = tensors()
    LOG.clear()
    call(SIDE, *tensors)
    used = [p for what, p, s in LOG if s is SIDE]
    assert all(t.data_ptr() in used for t in tensors)
