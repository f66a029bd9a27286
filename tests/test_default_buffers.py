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


def _weight(n, k, layout=B.LAYOUT_DEVICE):
    return B.QWeight(B.Q4_G32, layout, 1, n, k, _z(n * k // 2, dtype=torch.uint8), _z(n * k // 32, dtype=torch.int16))


def _x(*shape):
    return _z(*shape, dtype=F16)


W, CACHE = _weight(64, 64), (_x(1, 40, 64), _x(1, 40, 64))
OLDER = {
    "qm_quantise": lambda s: B.qm_quantise(_z(64, 64, dtype=F32), B.Q4_G32, stream=s),
    "qm_dequantise": lambda s: B.qm_dequantise(W, stream=s),
    "qm_repack": lambda s: B.qm_repack(W, B.LAYOUT_CANONICAL, stream=s),
    "qmatmul_gemv": lambda s: B.qmatmul_gemv(W, _x(64), stream=s),
    "qmatmul_gemv_grouped": lambda s: B.qmatmul_gemv_grouped([W, W], [_x(64), _x(64)], stream=s),
    "qmatmul_gemm": lambda s: B.qmatmul_gemm(W, _x(3, 64), stream=s),
    "qmatmul_gemm_grouped": lambda s: B.qmatmul_gemm_grouped([W, W], _x(3, 64), stream=s),
    "qmatmul_gemm_swiglu_f16": lambda s: B.qmatmul_gemm_swiglu_f16(W, W, _x(3, 64), stream=s),
    "qattn_decode": lambda s: B.qattn_decode(_x(2, 64), *CACHE, 7, 0.1, stream=s),
    "qattn_prefill": lambda s: B.qattn_prefill(_x(2, 3, 64), *CACHE, 0, 0.1, stream=s),
    "qattn_prefill_rows_f16": lambda s: B.qattn_prefill_rows_f16(_x(2, 3, 64), *CACHE, 0, 0.1, stream=s),
    "qdec_argmax": lambda s: B.qdec_argmax(_z(40, dtype=F32), stream=s),
    "qdec_cast_f16": lambda s: B.qdec_cast_f16(_z(40, dtype=F32), stream=s),
    "qmoe_route": lambda s: _fields(B.qmoe_route(_z(3, 8, dtype=F32), 2, stream=s)),
}


def _fields(r):
    return [t for t in (getattr(r, f) for f in r.__dataclass_fields__) if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("name", OLDER)
def test_buffers_of_the_other_calls_too(name, monkeypatch):
    current, taken, library = [None], [], _Library()

    @contextlib.contextmanager
    def stream(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    empty = torch.empty

    def counted(*args, **kwargs):
        taken.append(current[0])
        return empty(*args, **kwargs)

    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "qm_weight_bytes", lambda *args: (2048, 256))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    monkeypatch.setattr(torch, "empty", counted)
    side = _Side()
    OLDER[name](side)
    assert taken and all(s is side for s in taken)
    assert library.streams == [77]
