"""Which sequences a decoder's step puts into a group, and which pages it takes, on the host;
on the GPU that sequences which part in the middle of a page are what sequences apart are, and
that what a group has in common is read once, within the bound of attention (test_shared_prompt)."""
import random

import numpy as np
import pytest

from paper_1809_02697_amd import decoder

from gpu_util import torch_cuda
from test_decoder import SHAPE
from test_decoder_shared import _Host
from test_token_ops import U, _attention64, _attention_bound, _np

gpu = pytest.mark.gpu


class _Seen(Exception):
    pass


def _step(monkeypatch, d, tokens):
    """What a step of the decoder hands to the device: pages, lengths and groups of its sequences."""
    def step(pages, lengths, new, size, device, groups, rotary, positions):
        raise _Seen([list(p) for p in pages], lengths, new, groups)
    d.rotary = None
    monkeypatch.setattr(decoder, "Step", step)
    with pytest.raises(_Seen) as seen:
        d.step(tokens)
    return seen.value.args


def _saved(groups):
    first, prefix = groups
    return sum((b - a - 1) * p for a, b, p in zip(first, first[1:], prefix))


def test_one_that_left_early_does_not_part_the_others():
    """255 sequences on 500 pages and one that shares the first of them alone: before and behind them in order."""
    many = [list(range(500)) + [2000 + b] for b in range(255)]
    for early in (-1, 5000):
        pages = sorted(many + [[0, early, early + 1]])
        first, prefix = decoder.shared_pages(pages, 64)
        assert (first, prefix) == (([0, 1, 256], [0, 32000]) if early < 0 else ([0, 255, 256], [32000, 0]))
    # two prompts behind one system prompt; three that share that one alone stay beside them
    pages = sorted([[0, 1, 2, 3, 100 + b] for b in range(4)] + [[0, 10, 11, 12, 200 + b] for b in range(5)])
    assert decoder.shared_pages(pages, 1) == ([0, 4, 9], [4, 4])
    # where all save as much together, they stay together
    assert decoder.shared_pages([[0, 1, 2], [0, 1, 3], [0, 4]], 10) == ([0, 3], [10])
    assert decoder.shared_pages([[0, 1, 2, 5], [0, 1, 2, 6], [0, 4]], 10) == ([0, 2, 3], [30, 0])
    assert decoder.shared_pages([], 10) is None and decoder.shared_pages([[]], 10) is None and decoder.shared_pages([[1], [1]], 10) == ([0, 2], [10])
    # as deep as sequences are many
    deep = [list(range(k)) + [9000 + k] for k in range(1, 3000, 2)][::-1]
    assert _saved(decoder.shared_pages(deep, 1)) >= 1499 * 1


@pytest.mark.parametrize("seed", range(30))
def test_groups_hold_what_they_say_and_save_no_less_than_one_a_first_page(seed):
    r = random.Random(seed)
    pages, fresh = [[]], 1000
    for _ in range(r.randrange(1, 40)):
        old = r.choice(pages)
        p = old[:r.randrange(len(old) + 1)] if r.random() < 0.8 else []
        p = p + list(range(fresh, fresh + r.randrange(6)))
        fresh += 6
        pages.append(p)
    pages.sort()
    got = decoder.shared_pages(pages, 3)
    firsts = {}
    for p in pages:
        firsts.setdefault(p[0] if p else None, []).append(p)
    least = 0
    for k, ps in firsts.items():
        if k is not None:
            n = next((j for j, c in enumerate(zip(*ps)) if len(set(c)) > 1), min(map(len, ps)))
            least += (len(ps) - 1) * n * 3
    if got is None:
        assert least == 0
        return
    first, prefix = got
    assert first[0] == 0 and first[-1] == len(pages) and all(a < b for a, b in zip(first, first[1:])) and len(prefix) == len(first) - 1
    for a, b, n in zip(first, first[1:], prefix):
        assert n % 3 == 0 and all(p[:n // 3] == pages[a][:n // 3] and len(p) >= n // 3 for p in pages[a:b])
        assert n == 0 or b - a > 1
    assert _saved(got) >= least > 0 or least == 0


def test_a_sequence_without_new_tokens_lowers_nothing(monkeypatch):
    """A fork that went back to the first page and waits: the others' prefix is their own."""
    d = _Host(60, 4)
    d.fill(d.add(), 40)
    d.fork(0, 3)
    d.keep(2, range(6))
    pages, lengths, new, groups = _step(monkeypatch, d, [[1], [1, 1], [], [1]])
    assert groups == ([0, 3], [40]) and new == [1, 2, 1] and lengths == [40, 40, 40]
    assert all(p[:10] == list(range(10)) for p in pages)
    # all but one wait: nothing is shared, and no sequence is left out
    pages, lengths, new, groups = _step(monkeypatch, d, [[], [], [1], []])
    assert groups is None and new == [0, 0, 1, 0]


def test_dropping_an_early_token_leaves_the_others_their_prefix(monkeypatch):
    """(The pages behind it are copies then.)"""
    monkeypatch.setattr(decoder.neo, "kv_compact", lambda *a: None)
    d = _Host(100, 4)
    d.cache = None
    d.fill(d.add(), 80)
    d.fork(0, 5)
    d.keep(3, [t for t in range(80) if t != 6])
    assert d.pages[3][0] == 0 and d.pages[3][1] != 1
    pages, lengths, new, groups = _step(monkeypatch, d, [[1]] * 6)
    assert sorted(groups[1]) == [0, 80] and len(groups[0]) == 3


def test_the_last_holder_of_a_page_writes_the_page_itself(monkeypatch):
    """Two that share a page which is not full, one page free: one copy is enough."""
    d = _Host(3, 4)
    d.fill(d.add(), 8)
    d.fork(0)
    for i in range(2):
        d.keep(i, range(6))
    assert d.pages == [[0, 1], [0, 1]] and d.free == [2]
    _step(monkeypatch, d, [[1], [1]])
    assert d.copies == [([1], [2], None)] and d.pages == [[0, 2], [0, 1]] and d.users == [2, 1, 1] and d.free == []
    # with a third one that waits, both writers need a copy
    d = _Host(4, 4)
    d.fill(d.add(), 8)
    d.fork(0, 2)
    for i in range(3):
        d.keep(i, range(6))
    _step(monkeypatch, d, [[1], [], [1]])
    assert d.copies == [([1, 1], [2, 3], None)] and d.pages == [[0, 2], [0, 1], [0, 3]] and d.users == [3, 1, 1, 1]
    d = _Host(3, 4)
    d.fill(d.add(), 8)
    d.fork(0, 2)
    for i in range(3):
        d.keep(i, range(6))
    with pytest.raises(RuntimeError):
        d.step([[1], [], [1]])
    assert d.pages == [[0, 1]] * 3 and d.users == [3, 3, 0] and d.free == [2] and d.copies == []


def _closing(monkeypatch, d):
    """The tables and kept tokens of the decoder's calls that close up."""
    calls = []
    d.cache = None
    monkeypatch.setattr(decoder.neo, "kv_compact", lambda c, table, bases, keep, starts, most: calls.append((table.tolist(), bases.tolist(), keep.tolist())))
    return calls


def test_pages_that_a_sequence_gives_up_serve_its_copies(monkeypatch):
    """No page is free, the first is shared, and the last holds nothing that is kept."""
    d = _Host(4, 4)
    d.fill(d.add(), 4)
    d.fork(0)
    d.fill(0, 16)
    assert d.pages == [[0, 1, 2, 3], [0]] and d.free == []
    calls = _closing(monkeypatch, d)
    d.keep(0, [1, 2, 5, 6, 7])
    assert d.copies == [([0], [2], None)] and calls == [([[2, 1, 2, 3]], [0], [1, 2, 5, 6, 7])]
    assert d.pages == [[2, 1], [0]] and d.users == [1, 1, 1, 0] and d.free == [3] and d.at[0] == [1, 2, 5, 6, 7]
    # a page that something kept lies on is read when the tokens close up; one that others hold too is not free
    for first, second, kept in ((4, 16, [1, 5, 9, 12, 13]), (8, 8, [1, 2])):
        d = _Host(second // 4, 4)
        d.fill(d.add(), first)
        d.fork(0)
        d.fill(0, second)
        before = [list(p) for p in d.pages], list(d.users), list(d.free), list(d.lengths)
        with pytest.raises(RuntimeError):
            d.keep(0, kept)
        assert before == (d.pages, d.users, d.free, d.lengths) and d.copies == []


@gpu
@pytest.mark.parametrize("layers", [1, 3])
def test_sequences_that_part_in_the_middle_of_a_page(layers):
    """Three that share a page which is not full write into it in one step, in two copies and the page itself:
    the bits of sequences that shared nothing."""
    torch = torch_cuda()
    w = decoder.random_weights(layers, 300, 96, inner=160, **SHAPE)
    r = random.Random(5)
    prompt = [r.randrange(300) for _ in range(24)]
    make = lambda pages: decoder.Decoder(w, pages=pages, page_size=8, dtype=torch.float32, freqs=decoder.neo.rotary_frequencies(32), **SHAPE)  # noqa: E731
    d, apart = make(7), make(12)  # (two whole pages in common, three parted, two behind those)
    d.add()
    d.step([prompt])
    d.fork(0, 2)
    for _ in range(3):
        apart.add()
    apart.step([prompt] * 3)
    for x in (d, apart):
        for i in range(3):
            x.keep(i, range(21))
    for new in ([1, 2, 1], [2, 1, 2], [0, 3, 1]):
        tokens = [[r.randrange(300) for _ in range(n)] for n in new]
        assert torch.equal(d.step(tokens), apart.step(tokens))
    assert len({p[2] for p in d.pages}) == 3 and [p[:2] for p in d.pages] == [d.pages[0][:2]] * 3


@gpu
def test_a_full_cache_closes_up_into_pages_it_gives_up():
    torch = torch_cuda()
    w = decoder.random_weights(2, 300, 96, inner=160, **SHAPE)
    r = random.Random(6)
    head, tail = [r.randrange(300) for _ in range(8)], [r.randrange(300) for _ in range(24)]
    make = lambda pages: decoder.Decoder(w, pages=pages, page_size=8, dtype=torch.float32, freqs=decoder.neo.rotary_frequencies(32), **SHAPE)  # noqa: E731
    d, apart = make(4), make(6)
    d.add()
    d.step([head])
    d.fork(0)
    d.step([tail, []])
    assert d.free == []
    for _ in range(2):
        apart.add()
    apart.step([head, head])
    apart.step([tail, []])
    for x in (d, apart):
        x.keep(0, [0, 3, 4, 7, 9, 10, 15, 16, 18])
    assert len(d.free) == 1 and d.pages[1] != d.pages[0][:1]
    for tokens in ([[1, 2], []], [[3], []]):
        assert torch.equal(d.step(tokens), apart.step(tokens))
    d.drop(0)
    apart.drop(0)
    assert torch.equal(d.step([[], [4]]), apart.step([[], [4]]))       # what the fork reads is as it was


@gpu
@pytest.mark.parametrize("beside", [[], [4300], [1, 5000]])
def test_a_step_reads_a_long_prompt_once(monkeypatch, beside):
    """33 sequences on a prompt of 4000 tokens, of which one left it early and one waits, and others that share
    nothing, beside them: the pages of the first serve all of the group, and every output is within
    the bound of attention against 64 bits."""
    torch = torch_cuda()
    shape = dict(q_heads=16, kv_heads=8, head_dim=128)
    d = decoder.Decoder(decoder.random_weights(1, 300, 256, inner=256, **shape), pages=1500, page_size=16, dtype=torch.float32,
                        freqs=decoder.neo.rotary_frequencies(128), **shape)
    r = random.Random(8)
    text = lambda n: [r.randrange(300) for _ in range(n)]  # noqa: E731
    d.add()
    d.step([text(4000)])
    for n in beside:
        d.add()
        d.step([[]] * (len(d.pages) - 1) + [text(n)])
    forks = d.fork(0, 33)
    d.keep(forks[4], range(70))
    d.step([[]] * forks[4] + [text(40)] + [[]] * (len(d.pages) - forks[4] - 1))
    d.keep(forks[9], range(30))             # (it waits)
    was, seen = decoder.neo.attention_shared_int8, []

    def call(cache, q, table, contexts, starts, first, prefix, *rest, **kw):
        out = was(cache, q, table, contexts, starts, first, prefix, *rest, **kw)
        f, p, other = first.tolist(), prefix.tolist(), table.clone()
        for a, b, n in zip(f, f[1:], p):
            other[a + 1:b, :n // 16] = -1
        same = torch.equal(was(cache, q, other, contexts, starts, first, prefix, *rest, **kw), out)
        k, v, ks, vs = (t.cpu().numpy() for t in cache)
        ctx = contexts.tolist()
        ref, A, B = _attention64(q.double().cpu().numpy(), k, v, ks, vs, table.cpu().numpy(), ctx, starts.tolist(), 128 ** -0.5, 0)
        within = np.abs(_np(out) - ref) <= _attention_bound(ref, A, B, 128, max(ctx), "float32") + 16 * U["float32"] * A
        seen.append((same, within.all(), sorted(zip(p, (b - a for a, b in zip(f, f[1:]))))))
        return out
    monkeypatch.setattr(decoder.neo, "attention_shared_int8", call)
    for i in range(3):
        tokens = [text(1) for _ in d.pages]
        tokens[forks[9]] = []
        d.step(tokens)
        same, within, groups = seen[i]
        assert same and within and groups == sorted([(4000, 32), (0, 1)] + [(0, 1)] * len(beside))
