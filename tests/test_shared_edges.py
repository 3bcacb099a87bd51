"""Calls of the operators of requests that share a prompt which the tests beside the
operators (test_shared_prompt) do not make: page tables that are columns of wider ones,
amplitudes of a rotation that float32 does not hold."""
import ctypes

import numpy as np
import pytest

from paper_1809_02697_amd import neo

from gpu_util import torch_cuda
from test_shared_prompt import _bits, _compacted, _layers, _tables, cuda
from test_token_ops import BAD_CACHES, F32, FAKE, ODD, U, _struct

gpu = pytest.mark.gpu
u = U["float32"]


@pytest.fixture(scope="module")
def torch():
    t = torch_cuda()
    neo.lib()
    return t


# ---- host ------------------------------------------------------------------------------

def test_closing_up_is_told_the_columns_of_its_table(monkeypatch):
    """A slice of a wider table: the call gets the slice's width beside the wide one's stride."""
    import torch
    told = []

    class Lib:
        def neo_kv_compact_columns(self, *a):
            told.append(a)
            return 0
    monkeypatch.setattr(neo, "lib", Lib)
    monkeypatch.setattr(neo, "_here", lambda *a: None)
    monkeypatch.setattr(neo, "_stream", lambda s: None)
    monkeypatch.setattr(neo, "_cache_ptrs", lambda *t: (0, 0, 0, 0))
    monkeypatch.setattr(neo, "_vec", lambda t, *a: 0)
    monkeypatch.setattr(neo, "_rows", lambda t, *a: (t.data_ptr(), t.stride(0)))
    cache = neo.kv_cache(4, 2, 16, 64, device="cpu")
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    wide = torch.zeros((3, 9), dtype=torch.int32)
    neo.kv_compact(cache, wide[:, 4:6], i32(3), i32(5), i32(4), 4)
    neo.kv_compact(cache, wide, i32(3), i32(5), i32(4), 4)
    assert [(a[4], a[5]) for a in told] == [(9, 2), (9, 9)]


def test_closing_up_within_columns_refusals():
    big = 4 * 2 * 16

    def call(c=None, layers=2, stride=big, table=FAKE, ts=8, pages=5, bases=FAKE, keep=FAKE, starts=FAKE, kept=5, seqs=2, most=4):
        return neo.lib().neo_kv_compact_columns(_struct() if c is None else c, layers, stride, table, ts, pages, bases, keep, starts, kept,
                                                seqs, most, None)
    for over, code in BAD_CACHES:
        assert call(_struct(**over)) == code and "neo_kv_compact_columns: cache" in neo.last_error(), over
    assert call(layers=-1) == -1 and call(stride=big - 1) == -2 and call(layers=1 << 17) == -4
    for over in (dict(table=None), dict(bases=None), dict(keep=None), dict(starts=None), dict(kept=-1), dict(seqs=-1), dict(most=-1)):
        assert call(**over) == -1, over
    for over in (dict(table=ODD), dict(bases=ODD), dict(keep=ODD), dict(starts=ODD)):
        assert call(**over) == -3, over
    assert call(ts=-1) == -2 and call(pages=-1) == -2 and call(pages=9) == -2 and call(ts=1 << 31, pages=1) == -4
    assert call(seqs=1, ts=0, pages=1 << 31) == -4
    assert call(pages=0, table=None) == 0 and call(kept=0, keep=None) == 0 and call(seqs=0, table=None) == 0


def test_an_amplitude_past_float32_is_refused():
    def call(amp):
        return neo.lib().neo_rotary(FAKE, 256, 64, 0, 4, 64, 64, 0, F32, FAKE, FAKE, amp, FAKE, 256, 64, None)
    assert call(3.4028234663852886e38) == 0 and call(-3.4028234663852886e38) == 0
    for amp in (3.5e38, -1e300, float("inf"), float("nan")):
        assert call(amp) == -1 and "amplitude" in neo.last_error(), amp


# ---- rotation --------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("amp", [1.2, 1.3465, 0.1, -7.3])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_sine_and_cosine_are_rounded_once(torch, layout, amp):
    """A pair (1, 0) becomes (A cos t, A sin t): in 64 bits within 2^-31 A (the series end below 7e-12
    and 2e-10, the angle's rounding below 2^-50 of an angle up to 2^20), rounded to float32 once (u)."""
    T, H, half = 700, 2, 24
    rng = np.random.default_rng(5)
    pos, f = rng.integers(0, 1 << 20, T), rng.uniform(0, 1, half)
    x = torch.zeros(T, H, 2 * half, device="cuda")
    a, b = (slice(0, half), slice(half, None)) if layout == "half" else (slice(0, None, 2), slice(1, None, 2))
    x[..., a] = 1
    t = pos.astype(np.float64)[:, None, None] * f
    got = [neo.rotary(x, cuda(pos), cuda(f), layout=layout, amplitude=amp)]
    cache = neo.kv_cache(T, 1, 1, 2 * half)
    got.append(neo.rotary_kv_write_int8(cache, x, x[:, :1], x[:, :1], torch.arange(T, device="cuda"), cuda(pos), cuda(f), layout=layout, amplitude=amp))
    for y in got:
        for part, want in ((a, amp * np.cos(t)), (b, amp * np.sin(t))):
            err = np.abs(y[..., part].double().cpu().numpy() - want)
            assert (err <= u * np.abs(want) * (1 + 2.0 ** -20) + 2.0 ** -30 * abs(amp)).all(), (err / np.abs(want)).max() / u


# ---- closing up ------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("first,end", [(0, 13), (3, 16), (5, 18)])
@pytest.mark.parametrize("rows", [slice(0, 3), slice(2, 3)])
@pytest.mark.parametrize("layers,H,page,D,tokens", [(2, 2, 4, 32, 30), (1, 3, 64, 128, 700), (3, 1, 64, 256, 700)])
def test_closing_up_looks_at_no_other_columns(torch, layers, H, page, D, tokens, rows, first, end):
    """Pages behind the slice's last column belong to others, and kept tokens point at them: they move
    nothing.  (Columns to the end of the wide table, so that the last row ends where the table does.)"""
    rng = np.random.default_rng(tokens + first)
    P, width = 80, end - first
    wide = rng.permutation(P)[:3 * 18].reshape(3, 18).astype(np.int32)
    table = wide[rows, first:end]
    have = _layers(torch, layers, P, H, page, D, 7)
    bases = [int(b) for b in rng.integers(0, 9, len(table))]
    keep = [sorted(rng.choice(np.arange(b, 18 * page), tokens if page > 4 else 30, replace=False).tolist()) for b in bases]
    assert any(k >= width * page for ks in keep for k in ks)
    want = _compacted(have, table, bases, keep)
    starts = np.concatenate([[0], np.cumsum([len(k) for k in keep])]).astype(np.int32)
    dev = tuple(cuda(a) for a in have)
    flat = np.array([x for k in keep for x in k], np.int32)
    neo.kv_compact(dev, cuda(wide)[rows, first:end], cuda(np.array(bases, np.int32)), cuda(flat), cuda(starts), max(len(k) for k in keep))
    assert all((_bits(a) == _bits(b)).all() for a, b in zip(dev, want))
    C = ctypes.c_void_p
    dev = tuple(cuda(a) for a in have)      # the entry for whole rows, of a table of its own
    args = [cuda(a) for a in (table, np.array(bases, np.int32), flat, starts)]
    struct = neo.KvCacheStruct(*(t.data_ptr() for t in dev), P, H, page, D)
    assert neo.lib().neo_kv_compact(ctypes.byref(struct), layers, P * H * page, C(args[0].data_ptr()), width, *(C(a.data_ptr()) for a in args[1:]),
                                    len(flat), len(bases), max(len(k) for k in keep), neo._stream()) == 0
    assert all((_bits(a) == _bits(b)).all() for a, b in zip(dev, want))
