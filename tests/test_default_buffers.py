"""Buffers that a caller leaves to the binding come from the blocks of the stream
that the call goes to (no GPU needed: the library is replaced)."""

import contextlib

import pytest
import torch

from paper_2607_00501_amd import binding as B

F16, F32, I32 = torch.float16, torch.float32, torch.int32


class _Side:
    cuda_stream = 77


class _Library:
    """Answers 0 to everything, and 4096 to a query of bytes."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                args[-1]._obj.value = 4096
            else:
                self.streams.append(args[-1])
            return 0
        return call


def _z(*shape, dtype=I32):
    return torch.zeros(shape, dtype=dtype)


CALLS = {
    "qdec_argmax_rows": lambda s: B.qdec_argmax_rows(_z(3, 40, dtype=F32), stream=s),
    "qkv_plan": lambda s: B.qkv_plan(_z(2), _z(2), _z(2, 3), _z(5), _z(2), 16, 8, stream=s),
    "qkv_rope_append": lambda s: B.qkv_rope_append(
        _z(3, 128, dtype=F32), _z(3, 64, dtype=F32), _z(3, 64, dtype=F32), _z(3), _z(3, dtype=torch.int64),
        _z(9, 32, 2, dtype=F32), _z(2, 1, 16, 64, dtype=F16), _z(2, 1, 16, 64, dtype=F16), stream=s),
    "qattn_paged_f16": lambda s: B.qattn_paged_f16(
        _z(3, 2, 64, dtype=F16), _z(2, 1, 16, 64, dtype=F16), _z(2, 1, 16, 64, dtype=F16), _z(1, 2), _z(2), _z(1), 0.1,
        stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_buffers_come_from_the_stream_of_the_call(name, monkeypatch):
    current, taken, kept, library = [None], [], [], _Library()

    @contextlib.contextmanager
    def stream(s):
        before, current[0] = current[0], s or current[0]
        yield
        current[0] = before

    empty = torch.empty

    def counted(*args, **kwargs):
        t = empty(*args, **kwargs)
        taken.append((current[0], t.data_ptr()))
        return t

    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_tensors", lambda **named: None)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 11)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((s, t.data_ptr())))
    monkeypatch.setattr(torch, "empty", counted)
    side = _Side()
    out = CALLS[name](side)
    assert taken and all(s is side for s, _ in taken)
    assert library.streams == [77]
    # What the caller gets is held for the current stream, where it will be read.
    outs = [out] if isinstance(out, torch.Tensor) else [getattr(out, f) for f in out.__dataclass_fields__]
    assert kept == [("current", t.data_ptr()) for t in outs if t.numel()]
    del taken[:], kept[:], library.streams[:]
    CALLS[name](None)
    assert taken and all(s is None for s, _ in taken) and not kept and library.streams == [11]
