"""A decoder of transformer layers on the integer path: what the token operators
of ``neo`` are for, put together the way a serving program uses them.

A layer (weights int8 with a scale per channel, activations int8 with a scale
per token, keys and values int8 in a paged cache):

    q8 = rmsnorm_int8(delta + h)            residual addition, norm, quantization
    q, k, v = matmul_int8(q8, w_qkv)
    kv_write_int8(cache, k, v)
    a = attention_paged_int8(cache, q)
    delta = matmul_int8(quantize_tokens_int8(a), w_out)
    q8 = rmsnorm_int8(delta + h)
    gate, up = matmul_int8(q8, w_gate_up)
    delta = matmul_int8(quantize_tokens_int8(up, gate=gate), w_down)

``Decoder.step`` takes any number of new tokens of each sequence: whole
prompts, chunks of them, or one token each.  Positions enter through the causal
order alone, or with ``freqs`` through rotary positions, queries and keys turned on
their way to the attention and the cache (rotary_kv_write_int8).

Sequences may share pages: ``fork`` gives copies of a sequence that hold its whole
pages in common and a copy of the last one, and a step reads what neighbours
share once for all of them (attention_shared_int8).  ``keep`` drops tokens of a
sequence and closes up the others, ``drop`` gives its pages back.

    python -m paper_1809_02697_amd.decoder      # a small decoder: prompts, then tokens
"""
from __future__ import annotations

import torch

from . import neo


class Linear:
    """A dense layer without bias: float32 weights [out][in] on the device, held as int8 rows."""

    def __init__(self, w):
        self.out, self.inp = w.shape
        self.rows, self.scale = neo.pack_dense_int8(w.contiguous())

    def __call__(self, q, scale, dtype):
        return neo.matmul_int8(q, scale, self.inp, self.rows, self.scale, self.out, dtype=dtype)


class Layer:
    def __init__(self, w, q_heads, kv_heads, head_dim):
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.norm1, self.norm2 = w["norm1"], w["norm2"]
        self.qkv, self.out = Linear(w["qkv"]), Linear(w["out"])
        self.gate_up, self.down = Linear(w["gate_up"]), Linear(w["down"])

    def __call__(self, x, h, cache, step):
        """x: the last sublayer's output; h: the residual stream before it (None at the first).
        Returns both for the next layer."""
        T, dtype, D = x.shape[0], x.dtype, self.head_dim
        q8, s, h2 = neo.rmsnorm_int8(x, self.norm1, residual=h, h=h)
        h = x if h2 is None else h2
        qkv = self.qkv(q8, s, dtype).view(T, self.q_heads + 2 * self.kv_heads, D)
        q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
        if step.rotary is None:
            neo.kv_write_int8(cache, k, v, step.slots)
        else:
            q = neo.rotary_kv_write_int8(cache, q, k, v, step.slots, step.positions, **step.rotary, q_out=q)
        if step.prefix_lens is None:
            a = neo.attention_paged_int8(cache, q, step.table, step.contexts, step.starts, step.max_chunk, step.max_context)
        else:
            a = neo.attention_shared_int8(cache, q, step.table, step.contexts, step.starts, step.group_starts, step.prefix_lens,
                                          step.max_chunk, step.max_group, step.max_context, step.max_own, **step.saved)
        x = self.out(*neo.quantize_tokens_int8(a.view(T, self.q_heads * D)), dtype)
        q8, s, h = neo.rmsnorm_int8(x, self.norm2, residual=h)
        both = self.gate_up(q8, s, dtype)
        F = both.shape[1] // 2
        return self.down(*neo.quantize_tokens_int8(both[:, F:], gate=both[:, :F]), dtype), h


class Step:
    """Where one call's tokens stand: cache slots of the new ones, page table, lengths; with groups
    (their starts and shared tokens, from ``shared_pages``) what neighbouring sequences have in common,
    with rotary (freqs, layout, amplitude) the new tokens' positions."""

    def __init__(self, pages, lengths, new, page_size, device, groups=None, rotary=None, positions=None):
        slots, contexts = [], []
        for p, n, m in zip(pages, lengths, new):
            slots += [p[t // page_size] * page_size + t % page_size for t in range(n, n + m)]
            contexts.append(n + m)
        starts = [0]
        for m in new:
            starts.append(starts[-1] + m)
        most = max(1, max(len(p) for p in pages))
        table = [p + [-1] * (most - len(p)) for p in pages]
        ints = lambda v, t=torch.int32: torch.tensor(v, dtype=t, device=device)  # noqa: E731
        self.slots, self.table, self.contexts, self.starts = ints(slots, torch.int64), ints(table), ints(contexts), ints(starts)
        self.max_chunk, self.max_context = max(new), max(contexts)
        self.ends = [s - 1 for s in starts[1:]]
        self.last = ints([s for s, m in zip(self.ends, new) if m], torch.int64)
        self.rotary = rotary
        self.positions = None if rotary is None else ints(positions, torch.int64)
        self.prefix_lens = None
        if groups:
            first, prefix = groups
            self.group_starts, self.prefix_lens = ints(first), ints(prefix)
            self.max_group = max(starts[b] - starts[a] for a, b in zip(first, first[1:]))
            self.max_own = max(c - p for a, b, p in zip(first, first[1:], prefix) for c in contexts[a:b])
            # (a single group's prefix is max_context - max_own)
            self.saved = {} if len(prefix) == 1 else {"saved": neo.shared_saving(first, prefix)}


def _alike(a, b):
    """How many pages two lists begin with in common."""
    same, differ = 0, min(len(a), len(b)) + 1  # so many are alike, so many are not (or not there)
    step = differ - 1
    while differ - same > 1:
        if a[same:same + step] == b[same:same + step]:
            same += step
        else:
            differ = same + step
        step = (differ - same) // 2
    return same


def shared_pages(pages, page_size):
    """Of sequences in the order of their pages: groups that begin with the same ones, as (starts of the groups
    and the number of sequences, tokens that each group's sequences have in common); None if none do.  Sequences
    that have more in common than their neighbours have with them are a group of their own where that saves more
    reading: those on one long prompt, say, beside one that left it early."""
    part = None    # the last closed stretch: its first sequence, the pages that it saves, its groups (first sequence, pages)
    around = []    # stretches that go on: pages in common, and the same three of their closed parts
    for i, p in enumerate(pages):
        part = i, 0, [(i, 0)]
        alike = _alike(p, pages[i + 1]) if i + 1 < len(pages) else -1
        while around and around[-1][0] > alike:
            n, first, saved, groups = around.pop()
            saved, groups, whole = saved + part[1], groups + part[2], (i - first) * n
            part = (first, whole, [(first, n)]) if n and whole >= saved else (first, saved, groups)
        if around and around[-1][0] == alike:
            around[-1][2] += part[1]
            around[-1][3] += part[2]
        elif alike >= 0:
            around.append([alike, *part])
    if part is None or part[1] == 0:
        return None
    return [first for first, _ in part[2]] + [len(pages)], [n * page_size for _, n in part[2]]


class Decoder:
    """weights: {"embed": [vocab][width], "norm": [width], "head": [vocab][width],
    "layers": [{"norm1", "qkv", "out", "norm2", "gate_up", "down"}, ...]}, float32 on the device.
    freqs, layout, amplitude: rotary positions (neo.rotary), none without freqs."""

    def __init__(self, weights, q_heads, kv_heads, head_dim, pages, page_size=64, dtype=torch.bfloat16, freqs=None, layout="half",
                 amplitude=1.0):
        self.embed, self.norm, self.head = weights["embed"].to(dtype), weights["norm"], Linear(weights["head"])
        self.layers = [Layer(w, q_heads, kv_heads, head_dim) for w in weights["layers"]]
        device = weights["embed"].device
        self.cache = neo.kv_cache(pages, kv_heads, page_size, head_dim, device, layers=len(self.layers))
        self.caches = [neo.kv_layer(self.cache, i) for i in range(len(self.layers))]
        self.rotary = None if freqs is None else dict(freqs=freqs, layout=layout, amplitude=amplitude)
        self.page_size, self.dtype, self.device = page_size, dtype, device
        self.free = list(range(pages))[::-1]
        self.users = [0] * pages                   # sequences that hold a page
        self.pages, self.lengths, self.at = [], [], []  # of a sequence: pages, tokens, the tokens' positions

    def add(self):
        """A new, empty sequence; its number."""
        self.pages.append([])
        self.lengths.append(0)
        self.at.append([])
        return len(self.pages) - 1

    def _take(self):
        page = self.free.pop()
        self.users[page] = 1
        return page

    def _release(self, pages):
        for page in pages:
            self.users[page] -= 1
            if self.users[page] == 0:
                self.free.append(page)

    def _copy(self, src, dst, entries=None):
        if src:
            ints = lambda v: torch.tensor(v, dtype=torch.int32, device=self.device)  # noqa: E731
            neo.kv_copy_pages(self.cache, ints(src), ints(dst), None if entries is None else ints(entries))

    def fork(self, sequence, copies=1):
        """Sequences that go on from where this one is; their numbers.  Its whole pages are shared, what
        is on the last one is copied."""
        whole, rest = divmod(self.lengths[sequence], self.page_size)
        if rest and copies > len(self.free):
            raise RuntimeError("the cache has no page left")
        new = [self._take() for _ in range(copies)] if rest else []
        if rest:
            self._copy([self.pages[sequence][whole]] * copies, new, [rest] * copies)
        for i in range(copies):
            for page in self.pages[sequence][:whole]:
                self.users[page] += 1
            self.pages.append(self.pages[sequence][:whole] + new[i:i + 1])
            self.lengths.append(self.lengths[sequence])
            self.at.append(list(self.at[sequence]))
        return list(range(len(self.pages) - copies, len(self.pages)))

    def drop(self, sequence):
        """Gives a sequence's pages back; its number stays, for an empty one."""
        self._release(self.pages[sequence])
        self.pages[sequence], self.lengths[sequence], self.at[sequence] = [], 0, []

    def keep(self, sequence, tokens):
        """Drops a sequence's cached tokens but these (their places, ascending), which close up and stay as
        they are, turned for the positions that they had; the next token's follows the last one's."""
        tokens, pages, size = list(tokens), self.pages[sequence], self.page_size
        if not all(a < b for a, b in zip([-1] + tokens, tokens + [self.lengths[sequence]])):
            raise ValueError("tokens must be places of cached tokens, ascending")
        base = next((i for i, t in enumerate(tokens) if i != t), len(tokens))
        end = -(-len(tokens) // size)
        # pages that others hold too are written in a copy
        copied = [i for i in range(base // size, end) if self.users[pages[i]] > 1] if base < len(tokens) else []
        # (pages behind the last one that nothing kept lies on, and that no other holds, may serve)
        short, kept = len(copied) - len(self.free), {t // size for t in tokens}
        spare = [i for i in range(end, len(pages)) if i not in kept and self.users[pages[i]] == 1][:max(short, 0)]
        if short > len(spare):
            raise RuntimeError("the cache has no page left")
        self._release(pages[i] for i in spare)
        new = [self._take() for _ in copied]
        self._copy([pages[i] for i in copied], new)
        self._release(pages[i] for i in copied)
        for i, page in zip(copied, new):
            pages[i] = page
        if base < len(tokens):
            ints = lambda v: torch.tensor(v, dtype=torch.int32, device=self.device)  # noqa: E731
            neo.kv_compact(self.cache, ints([pages]), ints([base]), ints(tokens[base:]), ints([0, len(tokens) - base]), len(tokens) - base)
        self._release(pages[i] for i in range(end, len(pages)) if i not in spare)
        self.pages[sequence], self.lengths[sequence] = pages[:end], len(tokens)
        self.at[sequence] = [self.at[sequence][t] for t in tokens]

    def step(self, tokens):
        """tokens: for every sequence the list of its new tokens (maybe empty).  Returns the
        logits [sequences with new tokens][vocab] (float32) after the last of each.  A call that is
        refused leaves the decoder as it was."""
        new = [len(t) for t in tokens]
        if len(tokens) != len(self.pages) or not any(new):
            raise ValueError("one list of tokens a sequence, and at least one token")
        if not all(0 <= t < len(self.embed) for s in tokens for t in s):  # (looked up on the device it ends the process)
            raise ValueError(f"a token outside the vocabulary of {len(self.embed)}")
        size = self.page_size
        need = [-(-(n + m) // size) - len(p) for p, n, m in zip(self.pages, self.lengths, new)]
        # a page that is not full is written in a copy while others hold it too (the last of them writes the page itself)
        copied, holders = [], {}
        for i, (p, n, m) in enumerate(zip(self.pages, self.lengths, new)):
            if m and n % size:
                page = p[n // size]
                if holders.setdefault(page, self.users[page]) > 1:
                    copied.append(i)
                    holders[page] -= 1
        if sum(need) + len(copied) > len(self.free):
            raise RuntimeError("the cache has no page left")
        shared = [self.pages[i][self.lengths[i] // size] for i in copied]
        for i in copied:
            self.pages[i][self.lengths[i] // size] = self._take()
        self._copy(shared, [self.pages[i][self.lengths[i] // size] for i in copied])
        self._release(shared)
        for p, n in zip(self.pages, need):
            p += [self._take() for _ in range(n)]
        # sequences that begin with the same pages side by side, those without new tokens left out
        order, groups = list(range(len(new))), None
        if any(n > 1 for n in self.users):
            alike = sorted((i for i in order if new[i]), key=self.pages.__getitem__)
            groups = shared_pages([self.pages[i] for i in alike], size)
            order = alike if groups else order
        places = [range(a[-1] + 1 if a else 0, (a[-1] + 1 if a else 0) + m) for a, m in zip(self.at, new)]
        step = Step([self.pages[i] for i in order], [self.lengths[i] for i in order], [new[i] for i in order], size, self.device,
                    groups, self.rotary, [t for i in order for t in places[i]])
        x = self.embed[torch.tensor([t for i in order for t in tokens[i]], device=self.device)]
        h = None
        for layer, cache in zip(self.layers, self.caches):
            x, h = layer(x, h, cache, step)
        self.lengths = [n + m for n, m in zip(self.lengths, new)]
        for a, p in zip(self.at, places):
            a += p
        last = step.last
        if groups:
            ends = dict(zip(order, step.ends))
            last = torch.tensor([ends[i] for i, m in enumerate(new) if m], device=self.device)
        q8, s, _ = neo.rmsnorm_int8(x[last], self.norm, residual=h[last], h=False)
        return self.head(q8, s, torch.float32)


def random_weights(layers, vocab, width, q_heads, kv_heads, head_dim, inner, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    mat = lambda o, i: (torch.randn(o, i, generator=g) / i ** 0.5).to(device)  # noqa: E731
    gain = lambda: (torch.rand(width, generator=g) + 0.5).to(device)  # noqa: E731
    return {"embed": mat(vocab, width) * width ** 0.5, "norm": gain(), "head": mat(vocab, width),
            "layers": [{"norm1": gain(), "qkv": mat((q_heads + 2 * kv_heads) * head_dim, width),
                        "out": mat(width, q_heads * head_dim), "norm2": gain(), "gate_up": mat(2 * inner, width),
                        "down": mat(width, inner)} for _ in range(layers)]}


def main():
    import time
    shape = dict(q_heads=16, kv_heads=4, head_dim=128)
    d = Decoder(random_weights(4, 8192, 2048, inner=8192, **shape), pages=256, freqs=neo.rotary_frequencies(128), **shape)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(8192, (n,), generator=g).tolist() for n in (700, 33, 1, 256)]
    for _ in prompts:
        d.add()
    logits = d.step([p[:256] for p in prompts])           # the long prompt in chunks
    tokens = logits.argmax(1).tolist()
    while d.lengths[0] < 700:
        tokens[0] = d.step([prompts[0][d.lengths[0]:d.lengths[0] + 256], [], [], []]).argmax(1).item()
    torch.cuda.synchronize()
    t0, out = time.perf_counter(), [[t] for t in tokens]
    for _ in range(32):
        tokens = d.step([[t] for t in tokens]).argmax(1).tolist()
        for o, t in zip(out, tokens):
            o.append(t)
    print(f"32 tokens of each of 4 sequences in {(time.perf_counter() - t0) * 1e3:.1f} ms")
    for i, o in enumerate(out):
        print(f"sequence {i} ({len(prompts[i])} tokens of prompt):", *o[:12], "...")
    forks = d.fork(0, 3)                                   # four ways on from the long prompt
    logits = d.step([[tokens[0]], [], [], []] + [[t] for t in (1, 2, 3)])
    for i, t in zip([0] + forks, logits.argmax(1).tolist()):
        print(f"sequence {i} goes on with", t)
    d.keep(forks[0], range(d.lengths[forks[0]] - 5))       # one goes back five tokens
    for i in forks[1:]:
        d.drop(i)
    print("and from five tokens before:", d.step([[]] * 4 + [[5], [], []]).argmax(1).item())


if __name__ == "__main__":
    main()
