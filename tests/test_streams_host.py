"""Where the binding takes a call's own outputs from: the pool of the stream that
the call runs on.  On the host, over tensors that pass for device ones and a
library that records its calls."""
import contextlib

import pytest
import torch

from paper_1809_02697_amd import neo

under = [None]      # the streams entered by torch.cuda.stream
made = []           # the stream under which each output was made


class Device(torch.Tensor):
    is_cuda = True

    def _made(self, fill, shape, dtype):
        made.append(under[-1])
        return dev(torch.full(shape if isinstance(shape, tuple) else (shape,), fill, dtype=dtype))

    def new_empty(self, shape, dtype=None):
        return self._made(7, shape, dtype or self.dtype)

    def new_zeros(self, shape, dtype=None):
        return self._made(0, shape, dtype or self.dtype)


def dev(t):
    return t.as_subclass(Device)


class Stream:
    cuda_stream = 1234


class Library:
    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        def call(*args):
            self.streams.append(args[-1])
            return 0
        return call


@pytest.fixture()
def library(monkeypatch):
    L = Library()

    @contextlib.contextmanager
    def enter(s):
        under.append(s)
        yield
        under.pop()
    monkeypatch.setattr(neo, "lib", lambda: L)
    monkeypatch.setattr(torch.cuda, "stream", enter)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("stream", handle))
    neo._dtype(torch.float32)
    del made[:]
    return L


def f(*shape):
    return dev(torch.zeros(shape))


def i8(*shape):
    return dev(torch.zeros(shape, dtype=torch.int8))


def ints(*shape, dtype=torch.int32):
    return dev(torch.zeros(shape, dtype=dtype))


CACHE = tuple(i8(2, 1, 4, 16) for _ in "kv") + tuple(f(2, 1, 4) for _ in "kv")
CALLS = {
    "rmsnorm_int8": (lambda s: neo.rmsnorm_int8(f(4, 32), f(32), residual=f(4, 32), stream=s), 3),
    "quantize_tokens_int8": (lambda s: neo.quantize_tokens_int8(f(4, 32), gate=f(4, 32), stream=s), 2),
    "dequantize_tokens_int8": (lambda s: neo.dequantize_tokens_int8(i8(4, 32), f(4), 30, torch.float32, stream=s), 1),
    "matmul_int8": (lambda s: neo.matmul_int8(i8(4, 32), f(4), 32, i8(8, 32), f(8), 8, stream=s), 1),
    "kv_read_int8": (lambda s: neo.kv_read_int8(CACHE, ints(3, dtype=torch.int64), torch.float16, stream=s), 2),
    "attention_paged_int8": (lambda s: neo.attention_paged_int8(CACHE, f(2, 1, 16), ints(1, 2), ints(1), ints(2), 2, 8, stream=s), 1),
    "conv2d_blocked": (lambda s: neo.conv2d_blocked(f(1, 1, 4, 4, 16), 16, f(1, 1, 1, 1, 16, 16), 16, 1, 1, stream=s), 1),
    "conv2d_winograd": (lambda s: neo.conv2d_winograd(f(1, 1, 4, 4, 16), 16, f(1, 1, 16, 256), 16, stream=s), 1),
    "layout_transform": (lambda s: neo.layout_transform(f(1, 16, 4, 4), 0, 16, 1, 16, 4, 4, stream=s), 1),
    "pack_filter": (lambda s: neo.pack_filter(f(16, 16, 1, 1), stream=s), 1),
    "winograd_filter": (lambda s: neo.winograd_filter(f(16, 16, 3, 3), stream=s), 1),
    "quantize_int8": (lambda s: neo.quantize_int8(f(1, 1, 4, 4, 16), 16, 1.0, stream=s), 1),
    "pack_filter_int8": (lambda s: neo.pack_filter_int8(f(16, 16, 1, 1), stream=s), 2),
    "pack_dense_int8": (lambda s: neo.pack_dense_int8(f(8, 32), stream=s), 2),
    "quantize_rows_int8": (lambda s: neo.quantize_rows_int8(f(4, 32), 1.0, stream=s), 1),
    "dense_int8": (lambda s: neo.dense_int8(i8(4, 32), 32, i8(8, 32), f(8), 8, 1.0, y_scale=1.0, stream=s), 2),
}


@pytest.mark.parametrize("name", CALLS)
def test_outputs_come_from_the_calls_stream(library, name):
    call, outputs = CALLS[name]
    call(Stream())
    assert made == [("stream", 1234)] * outputs
    assert library.streams == [1234] and under == [None]


def test_outputs_of_a_call_on_the_current_stream(library, monkeypatch):
    monkeypatch.setattr(neo, "_stream", lambda s: 55)
    CALLS["matmul_int8"][0](None)
    assert made == [None] and library.streams == [55]
