"""The decoder's sequences that share pages: rotary positions, forks, tokens that
are dropped, pages that are given back, against the same network in 64 bits
with a cache of its own for every sequence.

Tolerance: as in test_decoder, a float32 row is within a few 10^-7 of 64 bits as long
as no value falls on the other side of the middle of two int8 steps, and off by
steps that later quantizations answer otherwise: every row within 5e-2.  There is no
bound of the median row: a key or value that fell so stays in the cache, and every later
row of its sequence, and of all sequences that share the token, reads it (with forks of
one prompt of 61 tokens, whose first row is off by such a step, all rows may be).  What
sharing itself adds is held exactly instead: forks give the bits that sequences apart
give which were fed the same tokens.
"""
import copy

import numpy as np
import pytest
import torch as cpu_torch

from paper_1809_02697_amd import decoder

from gpu_util import torch_cuda
from test_decoder import SHAPE, norm, q8

gpu = pytest.mark.gpu


# ---- host --------------------------------------------------------------------------------

def test_shared_pages():
    assert decoder.shared_pages([[1, 2], [3], []], 4) is None
    assert decoder.shared_pages([[], [1, 2, 3], [1, 2, 5, 6], [1, 4], [7], [8, 9], [8, 9]], 10) == ([0, 1, 4, 5, 7], [0, 10, 0, 20])
    assert decoder.shared_pages([[1], [1, 2]], 3) == ([0, 2], [3])
    assert decoder.shared_pages([[2], [2], [3], [3, 4]], 1) == ([0, 2, 4], [1, 1])


class _Host(decoder.Decoder):
    """A decoder without layers, whose copies of pages are written down."""

    def __init__(self, pages, page_size):
        self.page_size, self.device, self.free, self.users = page_size, "cpu", list(range(pages))[::-1], [0] * pages
        self.pages, self.lengths, self.at, self.copies, self.embed, self.layers, self.caches = [], [], [], [], cpu_torch.zeros(9, 8), [], []

    def _copy(self, src, dst, entries=None):
        if src:
            self.copies.append((list(src), list(dst), entries))

    def fill(self, sequence, n):
        while len(self.pages[sequence]) * self.page_size < n:
            self.pages[sequence].append(self._take())
        self.lengths[sequence], self.at[sequence] = n, list(range(n))


def test_pages_are_counted():
    d = _Host(8, 4)
    d.fill(d.add(), 10)
    assert d.pages == [[0, 1, 2]]
    assert d.fork(0, 2) == [1, 2]
    assert d.pages == [[0, 1, 2], [0, 1, 3], [0, 1, 4]] and d.copies == [([2, 2], [3, 4], [2, 2])] and d.users == [3, 3, 1, 1, 1, 0, 0, 0]
    d.drop(0)
    assert d.users == [2, 2, 0, 1, 1, 0, 0, 0] and set(d.free) == {2, 5, 6, 7} and d.pages[0] == []
    d.keep(1, range(6))                       # cut short: nothing moves, the page that is not full stays shared
    assert d.pages[1] == [0, 1] and d.lengths[1] == 6 and d.users[3] == 0 and len(d.copies) == 1
    d.drop(2)
    d.drop(1)
    assert sorted(d.free) == list(range(8)) and d.users == [0] * 8
    whole = d.add()
    d.fill(whole, 8)
    assert d.fork(whole) == [4] and d.pages[4] == d.pages[whole] and len(d.copies) == 1   # (no page that is not full: no copy)


def test_refusals_leave_the_decoder_as_it_was():
    d = _Host(3, 4)
    d.fill(d.add(), 10)
    before = copy.deepcopy((d.pages, d.lengths, d.users, d.free, d.at))
    for call, error in ((lambda: d.fork(0), RuntimeError), (lambda: d.keep(0, [0, 0]), ValueError), (lambda: d.keep(0, [10]), ValueError),
                        (lambda: d.keep(0, [3, 2]), ValueError), (lambda: d.keep(0, [-1, 2]), ValueError)):
        with pytest.raises(error):
            call()
        assert before == (d.pages, d.lengths, d.users, d.free, d.at)
    e = _Host(4, 4)
    e.fill(e.add(), 8)
    e.fork(0)
    e.fill(e.add(), 8)                        # no page is free
    before = copy.deepcopy((e.pages, e.lengths, e.users, e.free, e.at))
    e.lengths[1] = before[1][1] = 6           # (a page that is not full and shared: a token would need a copy of it)
    for call in (lambda: e.step([[], [1], []]), lambda: e.keep(0, [1, 2])):
        with pytest.raises(RuntimeError):
            call()
        assert before == (e.pages, e.lengths, e.users, e.free, e.at)


# ---- GPU ---------------------------------------------------------------------------------

class Reference:
    """One sequence in 64 bits: keys and values of every layer, and the tokens' positions."""

    def __init__(self, w, Hq, H, D, freqs=None):
        self.w = {k: v.double().cpu().numpy() for k, v in w.items() if k != "layers"}
        self.layers = [{k: (q8(v) if v.ndim == 2 else v) for k, v in ((k, t.double().cpu().numpy()) for k, t in lw.items())} for lw in w["layers"]]
        self.Hq, self.H, self.D, self.freqs = Hq, H, D, freqs
        self.k, self.v, self.at = [np.zeros((0, H, D)) for _ in self.layers], [np.zeros((0, H, D)) for _ in self.layers], []

    def turned(self, x, at):
        if self.freqs is None:
            return x
        t = np.array(at, np.float64)[:, None] * self.freqs
        c, s, half = np.cos(t)[:, None], np.sin(t)[:, None], len(self.freqs)
        a, b = x[..., :half], x[..., half:2 * half]
        return np.concatenate([a * c - b * s, b * c + a * s, x[..., 2 * half:]], -1)

    def feed(self, tokens):
        """The logits after the last of these tokens."""
        T, Hq, H, D = len(tokens), self.Hq, self.H, self.D
        first = self.at[-1] + 1 if self.at else 0
        new = list(range(first, first + T))
        before = len(self.at)
        self.at += new
        x, h = self.w["embed"][tokens], 0
        for i, p in enumerate(self.layers):
            h = h + x
            qkv = (q8(norm(h, p["norm1"])) @ p["qkv"].T).reshape(T, Hq + 2 * H, D)
            q = self.turned(qkv[:, :Hq], new)
            self.k[i] = np.concatenate([self.k[i], q8(self.turned(qkv[:, Hq:Hq + H], new))])
            self.v[i] = np.concatenate([self.v[i], q8(qkv[:, Hq + H:])])
            a = np.zeros((T, Hq, D))
            for j in range(Hq):
                s = q[:, j] @ self.k[i][:, j // (Hq // H)].T * D ** -0.5
                s[np.arange(before + T)[None] > before + np.arange(T)[:, None]] = -np.inf
                e = np.exp(s - s.max(1, keepdims=True))
                a[:, j] = e @ self.v[i][:, j // (Hq // H)] / e.sum(1, keepdims=True)
            h = h + q8(a.reshape(T, Hq * D)) @ p["out"].T
            gate, up = np.split(q8(norm(h, p["norm2"])) @ p["gate_up"].T, 2, 1)
            x = q8(up * gate / (1 + np.exp(-gate))) @ p["down"].T
        return (q8(norm(h + x, self.w["norm"])) @ q8(self.w["head"]).T)[-1]

    def keep(self, tokens):
        tokens = list(tokens)
        self.k, self.v, self.at = [k[tokens] for k in self.k], [v[tokens] for v in self.v], [self.at[t] for t in tokens]


@gpu
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("rotary", [True, False])
def test_forked_decoder_against_64_bits(rotary, page):
    torch = torch_cuda()
    from paper_1809_02697_amd import neo
    w = decoder.random_weights(2, 300, 96, inner=160, **SHAPE)
    freqs = neo.rotary_frequencies(24, scaling="linear", factor=2.0) if rotary else None
    d = decoder.Decoder(w, pages=120, page_size=page, dtype=torch.float32, freqs=freqs, **SHAPE)
    rng = np.random.default_rng(6)
    refs, offs = [], []

    def add():
        d.add()
        refs.append(Reference(w, SHAPE["q_heads"], SHAPE["kv_heads"], SHAPE["head_dim"], None if freqs is None else freqs.cpu().numpy()))

    def step(*new):
        tokens = [rng.integers(0, 300, n).tolist() for n in new]
        got = d.step(tokens).double().cpu().numpy()
        want = [r.feed(t) for r, t in zip(refs, tokens) if t]
        assert len(got) == len(want)
        offs.extend(np.linalg.norm(g - r) / np.linalg.norm(r) for g, r in zip(got, want))
        assert max(offs) <= 5e-2, offs

    def fork(i, n):
        assert d.fork(i, n) == list(range(len(refs), len(refs) + n))
        refs.extend(copy.deepcopy(refs[i]) for _ in range(n))

    def keep(i, tokens):
        d.keep(i, tokens)
        refs[i].keep(tokens)

    add()
    add()
    step(61, 9)
    step(1, 1)
    fork(0, 3)
    step(1, 0, 1, 7, 2)
    fork(3, 1)                                   # a fork of a fork, apart from its parent by the order of numbers
    step(1, 3, 1, 1, 0, 20)
    keep(2, list(range(58)))                     # back into the shared prompt
    keep(3, [t for t in range(d.lengths[3]) if t % 3])
    step(1, 1, 4, 1, 1, 1)
    keep(0, list(range(3, 30)))                  # in shared pages, which others still read
    step(2, 1, 1, 5, 1, 1)
    d.drop(4)
    refs[4] = Reference(w, SHAPE["q_heads"], SHAPE["kv_heads"], SHAPE["head_dim"], None if freqs is None else freqs.cpu().numpy())
    step(1, 1, 1, 1, 33, 1)
    for i in range(6):
        d.drop(i)
    assert sorted(d.free) == list(range(120))


@gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rotary", [True, False])
def test_forks_are_what_sequences_apart_are(rotary, dtype):
    """The same tokens in the same chunks, in forks and in sequences of their own: the same bits.  (Which kernel
    attends goes by the longest chunk of a call, so the sequences apart are fed beside one as long.)"""
    torch = torch_cuda()
    from paper_1809_02697_amd import neo
    w = decoder.random_weights(2, 300, 96, inner=160, **SHAPE)
    make = lambda: decoder.Decoder(w, pages=120, page_size=8, dtype=getattr(torch, dtype),  # noqa: E731
                                   freqs=neo.rotary_frequencies(32) if rotary else None, layout="interleaved", **SHAPE)
    d, apart = make(), make()
    rng = np.random.default_rng(7)
    history, numbers = [], []                    # of every sequence: its chunks and the longest beside each; its number apart

    def feed(tokens):
        """The logits of sequences apart, by number."""
        return apart.step([tokens.get(i, []) for i in range(len(apart.pages))])

    def new_apart(chunks):
        mine, beside = apart.add(), apart.add()
        numbers.append(mine)
        for c, longest in chunks:
            feed({mine: c, beside: [0] * longest})
        apart.drop(beside)

    def step(*new):
        tokens = [rng.integers(0, 300, n).tolist() for n in new]
        for h, t in zip(history, tokens):
            if t:
                h.append((t, max(new)))
        assert torch.equal(d.step(tokens), feed(dict(zip(numbers, tokens))))

    def fork(i, n):
        d.fork(i, n)
        for _ in range(n):
            history.append(list(history[i]))
            new_apart(history[i])
    for _ in range(2):
        d.add()
        numbers.append(apart.add())
        history.append([])
    step(45, 3)
    fork(0, 2)
    step(1, 1, 1, 5)
    fork(3, 1)
    fork(1, 1)
    for _ in range(9):                           # over the ends of pages
        step(1, 1, 1, 1, 1, 1)
    step(0, 2, 30, 0, 1, 1)
    d.keep(2, range(50))                         # back by whole tokens: as if they had never been
    assert d.at[2] == list(range(50))
    chunks = history[2][:6]
    assert sum(len(c) for c, _ in chunks) == 50
    new_apart(chunks)
    t = rng.integers(0, 300, 3).tolist()
    assert torch.equal(d.step([[], [], t, [], [], []]), feed({numbers[-1]: t}))


@gpu
def test_a_long_shared_prompt():
    """Sequences whose prompt is long enough to be read once for all: the same logits as of sequences apart,
    but for the order of sums (bfloat16 activations, whose roundings they may turn: 5e-2, as against 64 bits)."""
    torch = torch_cuda()
    from paper_1809_02697_amd import neo
    shape = dict(q_heads=16, kv_heads=8, head_dim=128)
    w = decoder.random_weights(1, 300, 256, inner=256, **shape)
    d = decoder.Decoder(w, pages=800, page_size=16, freqs=neo.rotary_frequencies(128), **shape)
    g = torch.Generator().manual_seed(3)
    prompt = torch.randint(300, (4000,), generator=g).tolist()
    d.add()
    d.step([prompt])
    forks = d.fork(0, 32)
    tokens = [[t % 300] for t in range(33)]
    calls = []
    was, paged = neo.attention_shared_int8, neo.attention_paged_int8
    neo.attention_shared_int8 = lambda *a, **k: calls.append(1) or was(*a, **k)
    try:
        one = d.step(tokens)
    finally:
        neo.attention_shared_int8 = was
    assert calls and forks == list(range(1, 33))
    for i in range(33):
        d.keep(i, range(4000))
    neo.attention_shared_int8 = lambda c, q, t, n, s, gs, p, chunk, group, most, own: paged(c, q, t, n, s, chunk, most)
    try:
        two = d.step(tokens)
    finally:
        neo.attention_shared_int8 = was
    off = (one - two).norm(dim=1) / two.norm(dim=1)
    assert off.max() <= 5e-2
