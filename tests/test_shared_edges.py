"""Calls of the operators of requests that share a prompt which the tests beside the
operators (test_shared_prompt) do not make: page tables that are columns of wider ones,
amplitudes of a rotation that float32 does not hold, groups beside sequences that share
nothing and under windows.

Which table attention read is seen by a second one, in which all sequences of a group but
the first have pages outside the cache in place of the whole shared ones: it gives the
same bits where the shared tokens are read once, through the first one's, and others
where every sequence reads its own.  Tolerances are those of test_shared_prompt."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_1809_02697_amd import decoder, neo

from gpu_util import torch_cuda
from test_shared_prompt import SHARED, WHOLE, _attend, _bits, _compacted, _layers, _most, _shared, _tables, cuda
from test_token_ops import BAD_CACHES, F16, F32, FAKE, ODD, TYPES, U, _attention64, _attention_bound, _np, _rand, _struct

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1809_02697_amd", "csrc")

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


RULE = r"""
#include "attention_share.h"
extern "C" double saved(int64_t seqs, int64_t groups, int64_t rows, int64_t chunk, int64_t context, int64_t own, int64_t window) {
    return neo::saved_by_bounds(seqs, groups, rows, chunk, context, own, window);
}
extern "C" int worth(double saved, int heads, int dim) { return neo::worth_sharing(saved, heads, dim); }
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    at = tmp_path_factory.mktemp("rule")
    (at / "rule.cpp").write_text(RULE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(at / "rule.so"), str(at / "rule.cpp")], check=True)
    so = ctypes.CDLL(str(at / "rule.so"))
    so.saved.restype, so.saved.argtypes, so.worth.argtypes = ctypes.c_double, [ctypes.c_int64] * 7, [ctypes.c_double, ctypes.c_int, ctypes.c_int]
    return so


def test_whether_to_share(rule):
    """8 key/value heads of 128.  By the bounds where all sequences share alike, or told where they do not."""
    share = lambda saved: bool(rule.worth(saved, 8, 128))  # noqa: E731
    assert rule.saved(256, 1, 1024, 1, 32500, 500, 0) == 255 * 32000 == neo.shared_saving([0, 256], [32000])
    assert share(255 * 32000) and not share(0) and not share(-5)
    # one sequence that shares nothing, as long as the longest: the bounds say nothing of the others' prefix
    assert rule.saved(256, 2, 1024, 1, 32500, 32500, 0) == 0
    told = neo.shared_saving([0, 255, 256], [32000, 0])
    assert told == 254 * 32000 and share(told)
    # groups that differ; one of one sequence saves nothing whatever its prefix
    assert neo.shared_saving([0, 3, 4, 9], [1000, 700, 20]) == 2 * 1000 + 4 * 20
    # a window far shorter than the prefix: apart each sequence reads that much, together all of the prefix is multiplied
    for seqs, window, together in ((16, 1000, False), (256, 1000, False), (16, 8000, False), (256, 8000, True), (16, 16000, True), (256, 16000, True)):
        by_bounds = rule.saved(seqs, 1, seqs * 4, 1, 32500, 500, window)
        told = neo.shared_saving([0, seqs], [32000], window=window, heads=4)
        assert abs(by_bounds - told) <= 1 and share(told) == share(by_bounds) == together, (seqs, window)
    # one that is as long as the prefix or longer hides nothing of it
    assert rule.saved(7, 2, 28, 5, 500, 100, 396) == rule.saved(7, 2, 28, 5, 500, 100, 0) == 5 * 400
    assert neo.shared_saving([0, 7], [400], window=396, max_chunk=5) == neo.shared_saving([0, 7], [400]) == 6 * 400
    # sizes whose products leave 32 bits
    assert rule.saved(1 << 20, 1, 1 << 25, 1, 0x7fff0000, 0, 0) == ((1 << 20) - 1) * 0x7fff0000


def test_a_step_says_what_sharing_saves(rule):
    """255 sequences on 32,000 tokens beside an unrelated one of 32,500: as much as without it."""
    lone = list(range(1000, 1509))
    pages = [list(range(500)) + [2000 + 10 * b + i for i in range(8)] for b in range(255)]
    lengths = [32000 + b for b in range(255)]
    step = decoder.Step(pages + [lone], lengths + [32500], [1] * 256, 64, "cpu", decoder.shared_pages(pages + [lone], 64))
    assert step.saved == {"saved": 254 * 32000} and rule.worth(step.saved["saved"], 8, 128)
    one = decoder.Step(pages, lengths, [1] * 255, 64, "cpu", decoder.shared_pages(pages, 64))
    assert one.saved == {}
    # (one group: by the bounds)
    assert rule.saved(255, 1, 4 * 255, 1, one.max_context, one.max_own, 0) == 254 * 32000


def test_shared_attention_that_is_told_refusals():
    def call(c=None, q=FAKE, qt=256, T=3, Hq=4, dtype=F16, table=FAKE, ts=8, ctx=FAKE, st=FAKE, B=2, gs=FAKE, pl=FAKE, groups=1,
             n=2, group=3, most=100, own=50, saved=1 << 40, scale=0.125, window=0, out=FAKE, ot=256, oh=64):
        return neo.lib().neo_attention_shared_saving_int8(_struct() if c is None else c, q, qt, 64, T, Hq, dtype, table, ts, ctx, st, B, gs, pl,
                                                          groups, n, group, most, own, saved, scale, window, out, ot, oh, None)
    for over, code in BAD_CACHES:
        assert call(_struct(**over)) == code and "neo_attention_shared_saving_int8: cache" in neo.last_error(), over
    for name in ("q", "table", "ctx", "st", "out", "gs", "pl"):
        assert call(**{name: None}) == -1 and call(**{name: ODD}) == -3, name
    for name in ("T", "B", "n", "most", "window", "groups", "group", "own"):
        assert call(**{name: -1}) == -1 and call(**{name: -1}, saved=-1) == -1, name
    assert call(Hq=3) == -2 and call(qt=-1) == -1 and call(oh=63) == -2 and call(most=129) == -2 and call(groups=0) == -2 and call(groups=3) == -2
    assert call(scale=0.0) == -1 and call(T=1 << 29, n=1 << 29) == -4 and call(T=1 << 27, group=1 << 27) == -4
    assert call(T=0, q=None) == 0 and call(B=0, q=None) == 0 and call(n=0, q=None) == 0


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


KINDS = [  # layers, heads, page size, dim, sequences, entries of each, bound
    (1, 1, 16, 64, 2, 700, 700),       # chunks of 256 tokens
    (3, 90, 7, 32, 2, 600, 550),       # so many heads that none is split
    (1, 2, 16, 256, 3, 420, 333),      # an entry's bytes in four parts
    (2, 1, 10, 128, 1, 1100, 1099),    # in two
    (1, 3, 64, 240, 2, 300, 299),      # fifteen pieces, which are not split
]


@gpu
@pytest.mark.parametrize("case", range(len(KINDS)))
def test_closing_up_in_chunks_entries_of_any_kind(torch, case):
    """More entries than a chunk holds, which repeat, descend, lie at or below their place, past the table or in
    pages that do not exist, across the edges of chunks; a bound that ends inside a chunk, a base that is negative."""
    layers, H, page, D, B, n, most = KINDS[case]
    assert min(n, most) * D // 16 > 1024        # (the kernel that goes through them in chunks)
    rng = np.random.default_rng(case)
    need = -(-(2 * n) // page)
    P = B * need + 1
    table = _tables(rng, [need] * B, P)
    for row in table:                           # a tenth of the pages are nowhere
        row[rng.choice(need, need // 10, replace=False)] = rng.choice([-1, P, 2 ** 31 - 1])
    have = _layers(torch, layers, P, H, page, D, case)
    bases = [int(b) for b in rng.integers(0, 40, B)]
    if B > 2:
        bases[1] = -1
    keep = []
    for base in bases:
        i = np.arange(n)
        k = np.sort(rng.choice(2 * n, n, replace=False))                # most: from anywhere, in order
        k = np.where(rng.random(n) < 0.2, rng.integers(-50, 3 * n, n), k)
        k = np.where(rng.random(n) < 0.1, base + i, k)                  # where it is
        k[100:140] = 2 * n - 1                                          # one token many times
        k[200:290] = np.arange(200, 290)[::-1] + base + 95              # (descends past its own places)
        k[250:260] = 2 ** 31 - 1
        keep.append(k.tolist())
    want = _compacted(have, table, bases, [k[:most] for k in keep])
    starts = np.arange(B + 1, dtype=np.int32) * n
    for _ in range(2):
        dev = tuple(cuda(a) for a in have)
        neo.kv_compact(dev, cuda(table), cuda(np.array(bases, np.int32)), cuda(np.array(keep, np.int64).astype(np.int32).ravel()), cuda(starts), most)
        assert all((_bits(a) == _bits(b)).all() for a, b in zip(dev, want))


# ---- attention ---------------------------------------------------------------------------

MUCH = 1 << 40      # saved: enough to share whatever the sizes


def _blank(table, first, prefix, page):
    """The table in which sequences of a group but its first have no pages of the whole shared ones."""
    out = table.copy()
    for a, b, p in zip(first, first[1:], prefix):
        out[a + 1:b, :p // page] = -1
    return out


def _read(torch, dtype, groups, Hq, H, D, page, window=0, seed=0, **kw):
    """The call over the shared tables, held against 64 bits, and whether it read the first sequences' pages for all."""
    k, v, ks, vs, table, chunks, contexts, first, prefix = _shared(groups, H, D, page, seed)
    starts = np.concatenate([[0], np.cumsum(chunks)]).astype(np.int32)
    q = _rand(torch, (int(starts[-1]), Hq, D), dtype, seed + 1)
    ref, A, B = _attention64(q.double().numpy(), k, v, ks, vs, table, contexts, starts, D ** -0.5, window)
    args = [cuda(a) for a in (np.array(contexts, np.int32), starts, first, prefix)]
    run = lambda t: neo.attention_shared_int8((cuda(k), cuda(v), cuda(ks), cuda(vs)), q.cuda(), cuda(t), *args, max(chunks), _most(groups),  # noqa: E731
                                              max(contexts), window=window, **kw)
    got = run(table)
    bound = _attention_bound(ref, A, B, D, max(contexts), dtype) + 16 * u * A
    assert (np.abs(_np(got) - ref) <= bound).all()
    other = _blank(table, first, prefix, page)
    assert (other != table).any()
    return torch.equal(run(other), got)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", [i for i, (g, _, _, _, page, _) in enumerate(SHARED) if any(p >= page and len(s) > 1 for p, s in g)])
def test_sharing_goes_by_what_is_told(torch, case, dtype):
    """Windows among the cases."""
    groups, Hq, H, D, page, window = SHARED[case]
    assert _read(torch, dtype, groups, Hq, H, D, page, window, seed=case, saved=MUCH)
    assert not _read(torch, dtype, groups, Hq, H, D, page, window, seed=case, saved=0)
    assert not _read(torch, dtype, groups, Hq, H, D, page, window, seed=case, saved=-MUCH)


@gpu
@pytest.mark.parametrize("lone", [1, 800, 4100, 9000])
def test_a_group_beside_a_sequence_that_shares_nothing(torch, lone):
    """34 MB a prefix read once: told, the group's are, whatever the other's length; by the bounds not
    where that one is the longest."""
    groups = [(4000, [(1, 1 + b % 40) for b in range(40)]), (0, [(1, lone)])]
    own = max(lone, 40)
    told = neo.shared_saving([0, 40, 41], [4000, 0])
    assert _read(torch, "bfloat16", groups, 8, 8, 128, 16, seed=30, max_own=own, saved=told)
    if lone > 4000:
        assert not _read(torch, "bfloat16", groups, 8, 8, 128, 16, seed=30, max_own=own)


@gpu
@pytest.mark.parametrize("window,together", [(0, True), (200, False), (3000, True)])
def test_a_window_shorter_than_the_prefix_is_reckoned_with(torch, window, together):
    """By the bounds: 40 sequences that see 200 of 4000 shared tokens read less apart."""
    groups = [(4000, [(1, 1 + b % 40) for b in range(60)])]
    assert _read(torch, "float16", groups, 8, 8, 128, 16, window, seed=31, max_own=40) == together


@pytest.fixture
def watched(monkeypatch):
    """Of every call of attention over groups, whether it read the first sequences' pages for all."""
    was, seen = neo.attention_shared_int8, []

    def call(cache, q, table, contexts, starts, first, prefix, *rest, **kw):
        out = was(cache, q, table, contexts, starts, first, prefix, *rest, **kw)
        other = _blank(table.cpu().numpy(), first.tolist(), prefix.tolist(), cache[0].shape[-2])
        seen.append((was(cache, q, cuda(other), contexts, starts, first, prefix, *rest, **kw) == out).all().item())
        return out
    monkeypatch.setattr(neo, "attention_shared_int8", call)
    return seen


def _whole_pages(groups, page):
    return any(p >= page and sum(n > 0 for n, _ in s[1:]) for p, s in groups)


@gpu
@pytest.mark.parametrize("case", [i for i, (g, _, _, _, page, _) in enumerate(SHARED) if _whole_pages(g, page)])
def test_the_cases_of_shared_prompts_share(torch, watched, case):
    """Those of test_shared_prompt, whose bounds make sharing seem worth it; under a window the bounds
    do not (those share above, where they are told to)."""
    groups, Hq, H, D, page, window = SHARED[case]
    _attend(torch, "bfloat16", groups, Hq, H, D, page, window, seed=case)
    assert watched == [window == 0] * 2
    _attend(torch, "bfloat16", groups, Hq, H, D, page, window, seed=case, force=False)
    assert watched[2:] == [False] * 2


@gpu
@pytest.mark.parametrize("case", range(len(WHOLE)))
def test_the_cases_of_whole_units_share(torch, watched, case):
    groups, Hq, H, D, page, own = WHOLE[case]
    _attend(torch, "bfloat16", groups, Hq, H, D, page, seed=80 + case, max_own=own, force=case == 3)
    assert watched == [True] * 2
