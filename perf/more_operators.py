"""The calls whose speed is measured of the operators for requests that share a prompt:
positions for queries and keys, pages that fork and close up, attention over a
prefix that many sequences have in common.

A case is a dict of plain values.  ``kind`` names the operator:

``rotary``   pairs of a head's values turned by an angle that grows with the token's
             position (``neo.rotary``)
``write``    the same for queries and keys of new tokens, the keys and values quantized
             into a paged cache as they come (``neo.rotary_kv_write_int8``), and the new
             tokens' entries read back (``neo.kv_read_int8``)
``copy``     pages of every layer's cache copied, whole or their first entries: a
             sequence forks (``neo.kv_copy_pages``)
``compact``  the tokens of a sequence that are kept close up, in every layer's cache
             (``neo.kv_compact``)
``attn``     causal attention of the newest tokens of sequences whose first tokens are
             the same for a group of them (``neo.attention_shared_int8``)

Rotation: pair i of a head's first ``rot`` values is (x[i], x[i + rot / 2]) in the layout
"half" and (x[2 i], x[2 i + 1]) in "interleaved"; it becomes (a cos t - b sin t, b cos t +
a sin t) times an amplitude, t = position * frequency[i].  The other values stay.

The cache and its quantization are those of ``neo.kv_write_int8``: int8 [pages][kv
heads][page size][head dim], float32 scales [pages][kv heads][page size], s = max|x| / 127
over a token's head, q = clamp(round_half_even(x / s), -127, 127).
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # queries and keys of one token of a single stream being decoded
        dict(name="rotary_token", kind="rotary", tokens=1, heads=40, dim=128, rot=128, layout="half", scaled="none",
             far=32000, dtype="bf16"),
        # a float32 network that turns part of heads of an odd size, at positions far out
        dict(name="rotary_odd", kind="rotary", tokens=777, heads=5, dim=90, rot=50, layout="interleaved", scaled="linear",
             far=1 << 30, dtype="f32"),
        # queries and keys of long prompts, frequencies stretched for long contexts
        dict(name="rotary_prompt", kind="rotary", tokens=16384, heads=40, dim=128, rot=128, layout="half", scaled="turns",
             far=131072, dtype="bf16"),
        # one token of each of 64 sequences
        dict(name="write_tokens", kind="write", tokens=64, q_heads=32, heads=8, dim=128, rot=128, layout="half",
             scaled="base", far=65536, page=64, pages=2048, dtype="bf16", out="bf16"),
        # a prompt, half of each head turned, in pairs of neighbours
        dict(name="write_prompt", kind="write", tokens=16000, q_heads=32, heads=8, dim=128, rot=64, layout="interleaved",
             scaled="none", far=16000, page=16, pages=1100, dtype="f16", out="f16"),
        # one sequence forks eight times in 16 layers: its last page, which is not full, is copied for each
        dict(name="fork_tails", kind="copy", pairs=8, layers=16, heads=8, dim=128, page=16, pages=512, partly=True),
        # pages moved together in 16 layers, whole
        dict(name="copy_pages", kind="copy", pairs=256, layers=16, heads=8, dim=128, page=64, pages=600, partly=False),
        # the accepted ones of up to eight proposed tokens of each of 32 sequences, 16 layers
        dict(name="compact_tree", kind="compact", seqs=32, base=4000, tokens=8, keep=0.5, layers=16, heads=8, dim=128,
             page=16, lens=1),
        # half of the tokens of four long sequences are dropped, eight layers
        dict(name="compact_long", kind="compact", seqs=4, base=64, tokens=12000, keep=0.5, layers=8, heads=8, dim=128,
             page=64, lens=2),
        # a few short sequences in two groups, float32, pages of ten tokens
        dict(name="shared_short", kind="attn", groups=2, seqs=6, chunk=3, prefix=300, fresh=40, heads=12, kv_heads=4,
             dim=64, page=10, window=0, dtype="f32", lens=3),
        # the next tokens of 16 sequences of four prompts
        dict(name="shared_chunk", kind="attn", groups=4, seqs=16, chunk=128, prefix=8000, fresh=1000, heads=32, kv_heads=8,
             dim=128, page=64, window=0, dtype="f16", lens=4),
        # 256 sequences decode a token each over one prompt of 32,000 tokens
        dict(name="shared_decode", kind="attn", groups=1, seqs=256, chunk=1, prefix=32000, fresh=500, heads=32, kv_heads=8,
             dim=128, page=64, window=0, dtype="bf16", lens=5),
    ]


def _log(rng, lo, hi):
    """A size, spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    kind = rng.choice(["rotary", "write", "copy", "compact", "attn", "attn"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if kind in ("rotary", "write"):
        # (the cache takes heads of whole 16 values)
        dim = rng.choice([64, 80, 96, 128, 256] if kind == "write" else [48, 64, 80, 90, 128, 200, 256])
        rot = rng.choice([dim // 2 * 2, dim // 2 * 2, dim // 4 * 2, 2 * rng.randint(1, dim // 2)])
        case = dict(kind=kind, dim=dim, rot=rot, layout=rng.choice(["half", "interleaved"]),
                    scaled=rng.choice(["none", "linear", "base", "turns"]), far=_log(rng, 1000, 1 << 30), dtype=dtype)
        most = 16384 * 40 * 128 // (2 if dtype == "f32" else 1)
        if kind == "rotary":
            case["heads"] = _log(rng, 1, 64)
            case["tokens"] = _log(rng, 1, max(1, min(16384, most // (case["heads"] * dim))))
            return case
        heads, page = rng.choice([1, 2, 4, 8, 16]), rng.choice([10, 16, 64, 128])
        group = rng.choice([1, 2, 4, 5, 8])
        tokens = _log(rng, 1, max(1, min(16000, most // (heads * (group + 2) * dim))))
        return dict(case, q_heads=heads * group, heads=heads, tokens=tokens, page=page, pages=-(-tokens // page) + _log(rng, 1, 200),
                    out="f16" if dtype == "f32" else dtype)
    if kind in ("copy", "compact"):
        heads, dim, page, layers = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 128, 256]), rng.choice([10, 16, 64, 128]), _log(rng, 1, 32)
        most = 256 * 64 * 16 * 8 * 128 // (heads * dim * layers)  # tokens, of all sequences or pages
        if kind == "copy":
            pairs = _log(rng, 1, max(1, min(2048, most // page)))
            return dict(kind=kind, pairs=pairs, layers=layers, heads=heads, dim=dim, page=page, pages=2 * pairs + _log(rng, 1, 100),
                        partly=rng.random() < 0.5)
        seqs = _log(rng, 1, 64)
        tokens = _log(rng, 1, max(1, min(20000, most // seqs // 2)))
        return dict(kind=kind, seqs=seqs, base=_log(rng, 1, max(1, min(4000, most // seqs // 2))), tokens=tokens,
                    keep=rng.choice([0.05, 0.5, 0.95]), layers=layers, heads=heads, dim=dim, page=page, lens=rng.randrange(1 << 20))
    kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8])
    dim, page = rng.choice([64, 80, 128, 256]), rng.choice([10, 16, 64, 128])
    seqs = _log(rng, 2, 256)
    groups = rng.choice([1, 1, max(1, seqs // 8), rng.randint(1, max(1, seqs // 2))])
    chunk = 1 if rng.random() < 0.6 else _log(rng, 2, 128)
    # (the padded scores and the padded keys stay below those of the largest listed cases)
    while seqs * chunk * kv * group > 64 * 1024:
        chunk = -(-chunk // 2)
    rows = seqs * chunk * kv * group * max(dim, 128) // 128
    prefix = _log(rng, 16, max(16, min(32000, 32000 * 256 * 32 // rows, 32000 * 8 * 128 * 8 // (groups * kv * dim))))
    fresh = _log(rng, chunk, max(chunk, min(2000, 256 * 500 * 8 * 128 // (seqs * kv * dim), 256 * 500 * 32 * 8 // rows)))
    return dict(kind="attn", groups=groups, seqs=seqs, chunk=chunk, prefix=prefix, fresh=fresh, heads=kv * group, kv_heads=kv,
                dim=dim, page=page, window=rng.choice([0, 0, 0, max(1, (prefix + fresh) // 2)]), dtype=dtype, lens=rng.randrange(1 << 20))


def _frequencies(case):
    """Radians a position, and the amplitude: as given, every one divided by the factor, the
    base raised, or divided only where a pair turns few times in the context first trained on."""
    rot, base, factor = case["rot"], 10000.0, 16.0
    if case["scaled"] == "base" and rot > 2:
        base *= factor ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if case["scaled"] == "linear":
        return [v / factor for v in f], 1.0
    if case["scaled"] == "turns":
        low, high, context = 1.0, 32.0, 4096
        stay = [min(1.0, max(0.0, (context * v / (2 * math.pi) - low) / (high - low))) for v in f]
        return [v * (s + (1 - s) / factor) for v, s in zip(f, stay)], 1 + 0.1 * math.log(factor)
    return f, 1.0


def _kept(case):
    """Of every sequence: its unchanged tokens, and which of those behind them are kept."""
    r = random.Random(case["lens"])
    bases, keep = [], []
    for _ in range(case["seqs"]):
        base = r.randint(0, case["base"])
        bases.append(base)
        keep.append([base + i for i in range(case["tokens"]) if r.random() < case["keep"]])
    return bases, keep


def _lens(case):
    """Of every group: how many sequences, and the shared tokens; of every sequence: its new
    tokens, and those behind the shared ones (the new ones among them)."""
    r = random.Random(case["lens"])
    cuts = sorted(r.sample(range(1, case["seqs"]), case["groups"] - 1))
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [case["seqs"]])]
    prefix = [case["prefix"]] + [_log(r, max(1, case["prefix"] // 4), case["prefix"]) for _ in sizes[1:]]
    new, fresh = [], []
    for b in range(case["seqs"]):
        new.append(case["chunk"] if b == 0 or case["chunk"] == 1 else r.randint(0, case["chunk"]))
        fresh.append(case["fresh"] if b == 0 else _log(r, max(1, new[-1], case["fresh"] // 32), case["fresh"]))
    return sizes, prefix, new, fresh


def _cache(g, layers, pages, heads, page, dim):
    """Keys, values and their scales of all layers."""
    return [torch.randint(-127, 128, (layers, pages, heads, page, dim), device=DEV, generator=g, dtype=torch.int8) for _ in "kv"] + \
        [torch.rand(layers, pages, heads, page, device=DEV, generator=g) * 0.02 + 0.01 for _ in "kv"]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 29)
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    st = dict(case)
    kind, page = case["kind"], case.get("page")
    if kind in ("rotary", "write"):
        t, T, D = TYPES[case["dtype"]], case["tokens"], case["dim"]
        f, st["amplitude"] = _frequencies(case)
        st["freqs"] = torch.tensor(f, dtype=torch.float64, device=DEV)
        first = torch.randint(0, max(1, case["far"] - T), (1,), device=DEV, generator=g)
        st["positions"] = first + torch.arange(T, device=DEV)
        if kind == "rotary":  # queries and keys in front of the values, as one projection writes them
            H = case["heads"]
            st["x"] = normal(T, (H + 2) * D).to(t).view(T, H + 2, D)[:, :H]
            return st
        Hq, H, P = case["q_heads"], case["heads"], case["pages"]
        qkv = normal(T, Hq + 2 * H, D).to(t)
        st["q"], st["k"], st["v"] = qkv.split([Hq, H, H], 1)
        st["cache"] = tuple(c[0] for c in _cache(g, 1, P, H, page, D))
        st["slots"] = torch.randperm(P * page, device=DEV, generator=g)[:T].contiguous()
        return st
    if kind == "copy":
        st["all"] = _cache(g, case["layers"], case["pages"], case["heads"], page, case["dim"])
        n, order = case["pairs"], torch.randperm(case["pages"], device=DEV, generator=g).to(torch.int32)
        # a fork's copies come from one page; moved pages each have their own
        st["src"] = order[:1].repeat(n) if case["partly"] else order[:n].contiguous()
        st["dst"] = order[n:2 * n].contiguous()
        st["entries"] = torch.randint(1, page + 1, (n,), device=DEV, generator=g, dtype=torch.int32) if case["partly"] else None
    elif kind == "compact":
        bases, keep = _kept(case)
        need = [-(-(b + case["tokens"]) // page) for b in bases]
        P = sum(need)
        st["all"] = _cache(g, case["layers"], P, case["heads"], page, case["dim"])
        st["table"] = _table(g, need, P)
        starts = [0]
        for k in keep:
            starts.append(starts[-1] + len(k))
        st.update(bases=ints(bases), keep=ints([i for k in keep for i in k]), starts=ints(starts), most=max(len(k) for k in keep))
    if kind in ("copy", "compact"):
        return st
    sizes, prefix, new, fresh = _lens(case)
    B, H, D = case["seqs"], case["kv_heads"], case["dim"]
    of = [i for i, n in enumerate(sizes) for _ in range(n)]
    first = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    # whole pages of the prefix are the first sequence's; the others hold a copy of what is left of it
    need = [-(-(prefix[of[b]] + fresh[b]) // page) for b in range(B)]
    mine = [n if b == first[of[b]] else n - prefix[of[b]] // page for b, n in enumerate(need)]
    P = sum(mine) + 1
    k, v, ks, vs = (c[0] for c in _cache(g, 1, P, H, page, D))
    k, v = ((torch.randn(c.shape, device=DEV, generator=g) * 35).round_().clamp_(-127, 127).to(torch.int8) for c in (k, v))
    table = torch.zeros(B, max(need), dtype=torch.int32)
    order, at = torch.randperm(P, device=DEV, generator=g).to(torch.int32).cpu(), 0
    for b in range(B):
        whole = 0 if b == first[of[b]] else prefix[of[b]] // page
        table[b, :whole] = table[first[of[b]], :whole]
        table[b, whole:need[b]] = order[at:at + mine[b]]
        at += mine[b]
    table = table.to(DEV)
    for i, p in enumerate(prefix):
        if p % page and sizes[i] > 1:
            a, b = table[first[i], p // page], table[first[i] + 1:first[i + 1], p // page].long()
            for c in (k, v, ks, vs):
                c[b, :, :p % page] = c[a, :, :p % page]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    st.update(cache=(k, v, ks, vs), table=table, contexts=ints([prefix[of[b]] + fresh[b] for b in range(B)]), starts=ints(starts),
              group_starts=ints(first), prefix_lens=ints(prefix), q=normal(starts[-1], case["heads"], D).to(TYPES[case["dtype"]]),
              max_chunk=max(new), max_group=max(starts[b] - starts[a] for a, b in zip(first, first[1:])), max_prefix=max(prefix),
              max_own=max(fresh), max_context=max(prefix[of[b]] + fresh[b] for b in range(B)), scale=D ** -0.5)
    return st


def _table(g, need, pages):
    """Page tables of sequences that have `need` pages each, in any order."""
    order, at = torch.randperm(pages, device=DEV, generator=g).to(torch.int32).cpu(), 0
    table = torch.zeros(len(need), max(need), dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table.to(DEV)


def run(st):
    if own:
        return _own(st)
    return {"rotary": _plain_rotary, "write": _plain_write, "copy": _plain_copy, "compact": _plain_compact, "attn": _plain_attn}[st["kind"]](st)


# ---- the framework's operators ---------------------------------------------------------

def _own(st):
    from paper_1809_02697_amd import neo
    if st["kind"] == "rotary":
        return neo.rotary(st["x"], st["positions"], st["freqs"], layout=st["layout"], amplitude=st["amplitude"])
    if st["kind"] == "write":
        q = neo.rotary_kv_write_int8(st["cache"], st["q"], st["k"], st["v"], st["slots"], st["positions"], st["freqs"],
                                     layout=st["layout"], amplitude=st["amplitude"])
        return (q, *neo.kv_read_int8(st["cache"], st["slots"], TYPES[st["out"]]))
    if st["kind"] == "copy":
        neo.kv_copy_pages(st["all"], st["src"], st["dst"], entries=st["entries"])
        return st["all"]
    if st["kind"] == "compact":
        neo.kv_compact(st["all"], st["table"], st["bases"], st["keep"], st["starts"], st["most"])
        return st["all"]
    return neo.attention_shared_int8(st["cache"], st["q"], st["table"], st["contexts"], st["starts"], st["group_starts"],
                                     st["prefix_lens"], st["max_chunk"], st["max_group"], st["max_context"], st["max_own"],
                                     scale=st["scale"], window=st["window"])


# ---- the same in elementary operations, 32 bits (64 for the angles) --------------------

def _turned(st, x):
    rot = st["rot"]
    t = st["positions"].double()[:, None] * st["freqs"]
    c, s = ((f(t) * st["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    y = x.float().clone()
    if st["layout"] == "half":
        a, b = x[..., :rot // 2].float(), x[..., rot // 2:rot].float()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., 0:rot:2].float(), x[..., 1:rot:2].float()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, b * c + a * s
    return y


def _plain_rotary(st):
    return _turned(st, st["x"]).to(TYPES[st["dtype"]])


def _quantize(x):
    """int8 values (as float32) and scales of the rows along x's last axis."""
    most = x.abs().amax(-1, keepdim=True)
    s = most / torch.full_like(most, 127.0)
    s = torch.where(most == 0, torch.ones_like(s), s)
    return (x / s).round().clamp(-127, 127), s


def _plain_write(st):
    kc, vc, ks, vs = st["cache"]
    p, o = st["slots"] // st["page"], st["slots"] % st["page"]
    k, sk = _quantize(_turned(st, st["k"]))
    v, sv = _quantize(st["v"].float())
    kc[p, :, o], vc[p, :, o] = k.to(torch.int8), v.to(torch.int8)
    ks[p, :, o], vs[p, :, o] = sk[..., 0], sv[..., 0]
    back = [(c[p, :, o].float() * s[p, :, o][..., None]).to(TYPES[st["out"]]) for c, s in ((kc, ks), (vc, vs))]
    return (_turned(st, st["q"]).to(TYPES[st["dtype"]]), *back)


def _plain_copy(st):
    src, dst, n = st["src"].long(), st["dst"].long(), st["entries"]
    k, v, ks, vs = st["all"]
    if n is None:
        k[:, dst], v[:, dst], ks[:, dst], vs[:, dst] = k[:, src], v[:, src], ks[:, src], vs[:, src]
    else:
        there = (torch.arange(st["page"], device=DEV) < n[:, None])[:, None]
        k[:, dst], v[:, dst] = (torch.where(there[..., None], c[:, src], c[:, dst]) for c in (k, v))
        ks[:, dst], vs[:, dst] = (torch.where(there, c[:, src], c[:, dst]) for c in (ks, vs))
    return st["all"]


def _plain_compact(st):
    starts, page, table = st["starts"].long(), st["page"], st["table"].long()
    i = torch.arange(st["keep"].numel(), device=DEV)
    b = torch.searchsorted(starts[1:].contiguous(), i, right=True)
    src, dst = st["keep"].long(), st["bases"].long()[b] + i - starts[b]
    p, o, pn, on = table[b, src // page], src % page, table[b, dst // page], dst % page
    k, v, ks, vs = st["all"]
    k[:, pn, :, on], v[:, pn, :, on] = k[:, p, :, o], v[:, p, :, o]
    ks[:, pn, :, on], vs[:, pn, :, on] = ks[:, p, :, o], vs[:, p, :, o]
    return st["all"]


def _part(q, keys, values, seen, scale):
    """Maximum, sum and weighted values of q [b][H][G][n][D] over keys and values [b][H][L][D]."""
    b, H, G, n, D = q.shape
    s = torch.matmul(q.reshape(b, H, G * n, D), keys.transpose(2, 3).contiguous()).view(b, H, G, n, -1) * scale
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    return top, s.sum(-1, keepdim=True), torch.matmul(s.view(b, H, G * n, -1), values).view(b, H, G, n, D)


def _plain_attn(st):
    kc, vc, ks, vs = st["cache"]
    q, table, ctx, starts = st["q"], st["table"].long(), st["contexts"].long(), st["starts"].long()
    gs, plen, page, w = st["group_starts"].long(), st["prefix_lens"].long(), st["page"], st["window"]
    B, (T, Hq, D), H = table.shape[0], q.shape, kc.shape[1]
    G, n = Hq // H, st["max_chunk"]
    # a token's position, a sequence's group
    t = torch.arange(T, device=DEV)
    seq = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    pos = ctx[seq] - starts[seq + 1] + t
    shared = plen[torch.searchsorted(gs[1:].contiguous(), torch.arange(B, device=DEV), right=True)]

    def padded(first, end, most):
        at = first[:, None] + torch.arange(most, device=DEV)
        real, at = at < end[:, None], at.clamp(max=T - 1)
        return q.float()[at].view(-1, most, H, G, D).permute(0, 2, 3, 1, 4), pos[at][..., None], real

    def packed(parts, real):  # in the order of the tokens
        return [x.permute(0, 3, 1, 2, 4)[real] for x in parts]

    def sight(j, pos):
        return (j <= pos) & (j > pos - w) if w else j <= pos

    # the shared tokens, for all of a group's queries
    L = st["max_prefix"]
    pages = table[gs[:-1], :-(-L // page)]
    keys, values = ((c[pages].float() * s[pages][..., None]).permute(0, 2, 1, 3, 4).reshape(len(plen), H, -1, D)[:, :, :L] for c, s in ((kc, ks), (vc, vs)))
    qs, at, real = padded(starts[gs[:-1]], starts[gs[1:]], st["max_group"])
    j = torch.arange(L, device=DEV)
    parts = packed(_part(qs, keys, values, sight(j, at) & (j < plen[:, None, None]), st["scale"]), real)
    # every sequence's own
    j = shared[:, None] + torch.arange(st["max_own"], device=DEV)
    p, o = table.gather(1, (j // page).clamp(max=table.shape[1] - 1)), j % page
    keys, values = ((c[p, :, o].float() * s[p, :, o][..., None]).transpose(1, 2).contiguous() for c, s in ((kc, ks), (vc, vs)))
    qs, at, real = padded(starts[:-1], starts[1:], n)
    mine = packed(_part(qs, keys, values, sight(j[:, None], at) & (j < ctx[:, None])[:, None], st["scale"]), real)
    top = torch.maximum(parts[0], mine[0])
    a, b = (torch.exp(x - top) for x in (parts[0], mine[0]))
    return ((parts[2] * a + mine[2] * b) / (parts[1] * a + mine[1] * b)).view(T, Hq, D).to(TYPES[st["dtype"]])


# ---- what a pass cannot do without -----------------------------------------------------

def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}
    kind = case["kind"]
    if kind == "rotary":
        n = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * size[case["dtype"]] + 8 * (case["tokens"] + case["rot"] // 2), "flops": 6 * case["tokens"] * case["heads"] * case["rot"] // 2}
    if kind == "write":
        n, heads, e = case["tokens"] * case["dim"], case["heads"], size[case["dtype"]]
        # (the entries are written and read back)
        entries = 2 * case["tokens"] * heads * (case["dim"] + 4)
        return {"bytes": 2 * n * case["q_heads"] * e + 2 * n * heads * (e + size[case["out"]]) + 2 * entries + 32 * case["tokens"],
                "flops": 3 * case["tokens"] * (case["q_heads"] + heads) * case["rot"] + 12 * n * heads}
    if kind == "copy":
        # (what the first entries come to is drawn: half a page and a half entry on average)
        each = (case["page"] + 1) / 2 if case["partly"] else case["page"]
        return {"bytes": int((1 if case["partly"] else 2) * case["pairs"] * each * case["layers"] * case["heads"] * 2 * (case["dim"] + 4)) + 8 * case["pairs"], "flops": 0}
    if kind == "compact":
        bases, keep = _kept(case)
        moved = sum(k != b + i for b, ks in zip(bases, keep) for i, k in enumerate(ks))
        return {"bytes": 2 * moved * case["layers"] * case["heads"] * 2 * (case["dim"] + 4) + 4 * sum(len(k) for k in keep) + 64, "flops": 0}
    sizes, prefix, new, fresh = _lens(case)
    of = [i for i, n in enumerate(sizes) for _ in range(n)]
    H, Hq, D, w = case["kv_heads"], case["heads"], case["dim"], case["window"]
    pairs, read, low = 0, 0, list(prefix)
    for b in range(case["seqs"]):
        p = prefix[of[b]]
        c, n = p + fresh[b], new[b]
        if not n:
            continue
        pairs += sum(min(x + 1, w) if w else x + 1 for x in range(c - n, c))
        first = max(0, c - n + 1 - w) if w else 0
        read += c - max(p, first)
        low[of[b]] = min(low[of[b]], first)
    read += sum(p - x for p, x in zip(prefix, low))
    return {"bytes": 2 * read * H * (D + 4) + 2 * sum(new) * Hq * D * size[case["dtype"]], "flops": 4 * D * Hq * pairs}


# ---- the definitions, in 64 bits -------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("rotary", "write"):
        rot = case["rot"]
        # rows of the rotation's matrix: value j goes with its partner and the pair's frequency
        j = torch.arange(rot, device=DEV)
        if case["layout"] == "half":
            mate, pair, sign = (j + rot // 2) % rot, j % (rot // 2), torch.where(j < rot // 2, -1.0, 1.0)
        else:
            mate, pair, sign = j ^ 1, j // 2, torch.where(j % 2 == 0, -1.0, 1.0)
        z = torch.polar(torch.full_like(st["freqs"], st["amplitude"]).expand(case["tokens"], -1).contiguous(),
                        st["positions"].double()[:, None] * st["freqs"])

        def turned(x):
            x = x.double()
            y = x[..., :rot] * z.real[:, pair][:, None] + x[..., mate] * (z.imag[:, pair] * sign.double())[:, None]
            return torch.cat([y, x[..., rot:]], -1)

        if case["kind"] == "rotary":
            return turned(st["x"])
        return turned(st["q"]), _steps(turned(st["k"])), _steps(st["v"].double())
    if case["kind"] == "copy":
        out = []
        for c in st["all"][2:]:
            new = c.double()
            for i, (a, b) in enumerate(zip(st["src"].tolist(), st["dst"].tolist())):
                n = case["page"] if st["entries"] is None else int(st["entries"][i])
                new[:, b, :, :n] = c[:, a, :, :n].double()
            out.append(new)
        return [None, None] + out
    if case["kind"] == "compact":
        bases, keep = _kept(case)
        page, table, out = case["page"], st["table"].long(), []
        for c in st["all"][2:]:
            new = c.double()
            for b, (base, ks) in enumerate(zip(bases, keep)):
                pages = table[b, :-(-(base + case["tokens"]) // page)]
                # [layers][heads][tokens] of the sequence, in order
                line = c[:, pages].double().transpose(1, 2).reshape(case["layers"], case["heads"], -1)
                line[:, :, base:base + len(ks)] = line[:, :, torch.tensor(ks, dtype=torch.long, device=DEV)]
                new[:, pages] = line.view(case["layers"], case["heads"], len(pages), page).transpose(1, 2)
            out.append(new)
        return [None, None] + out
    # every sequence over all of its own table
    sizes, prefix, new, fresh = _lens(case)
    of = [i for i, n in enumerate(sizes) for _ in range(n)]
    H, D, page, w = case["kv_heads"], case["dim"], case["page"], case["window"]
    G, out, at = case["heads"] // H, [], 0
    for b, n in enumerate(new):
        if not n:
            continue
        c = prefix[of[b]] + fresh[b]
        pages = st["table"][b, :-(-c // page)].long()
        keys, values = ((x[pages].double() * s[pages].double()[..., None]).transpose(0, 1).reshape(H, -1, D)[:, :c] for x, s in zip(st["cache"][:2], st["cache"][2:]))
        far = torch.arange(c, device=DEV)[None] - torch.arange(c - n, c, device=DEV)[:, None]
        dark = (far > 0) | (far <= -w) if w else far > 0
        rows = torch.empty(n, H, G, D, device=DEV, dtype=torch.float64)
        for h in range(H):
            s = st["q"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, D) @ keys[h].t().contiguous() * st["scale"]
            s = s.view(n, G, c).masked_fill_(dark[:, None], -math.inf)
            rows[:, h] = (torch.softmax(s, -1).view(n * G, c) @ values[h]).view(n, G, D)
        out.append(rows.reshape(n, H * G, D))
        at += n
    return torch.cat(out) if out else torch.zeros(0, H * G, D, device=DEV, dtype=torch.float64)


def _steps(x):
    """What the rows of x become when each is held in int8 with a scale."""
    s = x.abs().amax(-1, keepdim=True) / 127
    s = torch.where(s > 0, s, torch.ones_like(s))
    return torch.clamp(torch.round(x / s), -127, 127) * s
