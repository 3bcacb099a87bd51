"""Which keys the tokens of a chunk see (csrc/attention_keys.h), compiled for the
host and held against Python's unbounded integers: whatever lengths lie on the
device, the keys that are read stay below the caller's bound."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1809_02697_amd", "csrc")
SHIM = r"""
#include "attention_keys.h"
extern "C" int first(int pos, int window) { return neo::first_seen(pos, window); }
extern "C" void keys(int ctx, int all, int end, int t0, int t1, int window, int* r) { neo::seen_keys(ctx, all, end, t0, t1, window, r[0], r[1]); }
"""
TOP = 2 ** 31 - 1
WINDOWS = [0, 1, 2, 10, 64, 100, 5000, 1 << 30, TOP - 1, TOP]


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("keys")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "shim.so"),
                    str(d / "shim.cpp")], check=True, timeout=100)
    return ctypes.CDLL(str(d / "shim.so"))


def _check(host, ctx, all_, end, t0, t1, window):
    r = (ctypes.c_int * 2)()
    host.keys(ctx, all_, end, t0, t1, window, r)
    lo, hi = r
    what = dict(ctx=ctx, all=all_, end=end, t0=t0, t1=t1, window=window, lo=lo, hi=hi)
    assert 0 <= lo <= hi <= end, what
    p0, p1 = ctx - all_ + t0, ctx - all_ + t1
    # what the first and the last token see, cut at `end`; those between lie between
    seen = [(max(0, p + 1 - window) if window else 0, min(end, p + 1)) for p in (p0, p1)]
    seen = [(a, b) for a, b in seen if a < b]
    if seen:
        assert lo <= min(a for a, _ in seen) and hi >= max(b for _, b in seen), what
    assert lo == hi or (lo, hi) == (max(0, p0 + 1 - window) if window else 0, min(end, p1 + 1)), what


def test_first_seen(host):
    for pos in [-TOP, -300, -3, -1, 0, 1, 5, 63, 64, 4999, 5000, 1 << 30, TOP - 1, TOP]:
        for w in WINDOWS:
            assert host.first(pos, w) == (max(0, pos + 1 - w) if w and pos >= 0 else 0), (pos, w)


@pytest.mark.parametrize("window", WINDOWS)
def test_seen_keys(host, window):
    """Contexts within the bound, just and far above it; more new tokens than context."""
    for most in (0, 1, 15, 16, 64, 1000, 0x7fff0000):
        for ctx in (0, 1, 3, 15, 63, 64, 65, 100, 999, 1000, 1001, 1100, 5000, 1 << 30, 0x7fff0000, TOP):
            for all_ in (1, 2, 10, 40, 64, 300, 1 << 28):
                for t0 in {0, min(1, all_ - 1), all_ // 2, all_ - 1}:
                    for t1 in {t0, min(t0 + 15, all_ - 1), min(t0 + 255, all_ - 1)}:
                        _check(host, ctx, all_, min(ctx, most), t0, t1, window)


def test_seen_keys_at_random(host):
    r = random.Random(7)
    log = lambda: int(2 ** r.uniform(0, 31)) - 1  # noqa: E731
    for _ in range(20000):
        ctx, all_, most = log(), 1 + log() % (1 << 28), log()
        t0 = r.randrange(all_)
        _check(host, ctx, all_, min(ctx, most), t0, min(all_ - 1, t0 + r.randrange(256)), r.choice([0, 1 + log() % TOP]))
