"""The calls whose speed is measured of the token operators: the integer path of a
transformer layer, from its norm to the attention over an int8 cache.

A case is a dict of plain values.  ``kind`` names the operator:

``norm``   residual addition, root-mean-square norm and quantization to int8 rows
           with one scale per token (``neo.rmsnorm_int8``); returns the residual
           stream and the values that the int8 rows stand for
``matmul`` int8 rows with one scale per token times int8 weight rows with one scale
           per output channel (``neo.matmul_int8``).  ``source`` says what the
           caller has: int8 rows (as the norm writes them), float rows that are
           quantized first, or a gated pair up * silu(gate) that is quantized
           first (``neo.quantize_tokens_int8``)
``cache``  new keys and values quantized into a paged cache as they are written
           (``neo.kv_write_int8``), and tokens of the cache read back
           (``neo.kv_read_int8``)
``attn``   causal attention of the last tokens of every sequence over its paged
           int8 cache (``neo.attention_paged_int8``)

Quantization is symmetric: s = max|x| / 127 over a row (1 for a row of zeros),
q = clamp(round_half_even(x / s), -127, 127).  int8 rows are padded with zero
bytes to a multiple of 16.  The cache holds int8 [pages][kv heads][page
size][head dim] and float32 scales [pages][kv heads][page size], for keys and
for values; a sequence's token t lies at entry t % page_size of the page
page_table[seq][t // page_size].
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of a single stream being decoded
        dict(name="norm_token", kind="norm", rows=1, cols=4096, dtype="bf16", out="bf16"),
        # a long prompt of a wide model
        dict(name="norm_prompt", kind="norm", rows=8192, cols=8192, dtype="bf16", out="bf16"),
        # a float32 network of an odd width
        dict(name="norm_odd", kind="norm", rows=777, cols=2049, dtype="f32", out="f16"),
        # a projection of one token: the weights are read once, for one row
        dict(name="matmul_token", kind="matmul", source="float", M=1, K=4096, N=8192, dtype="bf16", out="bf16", bias=False),
        # the way down of a gated MLP for a batch of sequences being decoded
        dict(name="matmul_batch", kind="matmul", source="gate", M=96, K=16384, N=4096, dtype="f16", out="f16", bias=False),
        # a dense layer with a bias at sizes that fill no tile, out in float32
        dict(name="matmul_odd", kind="matmul", source="int8", M=1003, K=2049, N=1001, dtype="f32", out="f32", bias=True),
        # a projection of a long prompt, from the rows that the norm wrote
        dict(name="matmul_prompt", kind="matmul", source="int8", M=8192, K=8192, N=8192, dtype="bf16", out="bf16", bias=False),
        # one token of each of 32 sequences, written and read back
        dict(name="cache_tokens", kind="cache", new=32, read=32, heads=8, dim=128, page=16, pages=4096, dtype="bf16", out="bf16"),
        # a prompt written, and a longer context read back in float16
        dict(name="cache_prompt", kind="cache", new=16000, read=60000, heads=8, dim=128, page=64, pages=1024, dtype="f16", out="f16"),
        # a few short sequences with no to seven new tokens, float32, pages of ten tokens
        dict(name="attn_short", kind="attn", seqs=5, chunk=7, context=700, ragged=True, heads=12, kv_heads=4, dim=64,
             page=10, window=0, dtype="f32", lens=1),
        # 32 sequences decode a token each over contexts of up to 32,000 tokens
        dict(name="attn_decode", kind="attn", seqs=32, chunk=1, context=32000, ragged=True, heads=32, kv_heads=8,
             dim=128, page=64, window=0, dtype="bf16", lens=2),
        # the next chunk of one long prompt
        dict(name="attn_chunk", kind="attn", seqs=1, chunk=2048, context=32768, ragged=False, heads=32, kv_heads=8,
             dim=128, page=128, window=0, dtype="bf16", lens=3),
    ]


def _log(rng, lo, hi):
    """A size, spread over its logarithm (1536 and 3072 are left out)."""
    n = max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))
    return n - 1 if n in (1536, 3072) else n


def _width(rng, lo, hi):
    """A width; half of them multiples of 64."""
    n = _log(rng, lo, hi)
    if rng.random() < 0.5:
        n = -(-n // 64) * 64
    return n + 64 if n in (1536, 3072) else n


def draw(rng):
    kind = rng.choice(["norm", "matmul", "cache", "attn"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if kind == "norm":
        cols = _width(rng, 64, 16384)
        rows = _log(rng, 1, max(1, min(16384, 8192 * 8192 // cols // (2 if dtype == "f32" else 1))))
        return dict(kind=kind, rows=rows, cols=cols, dtype=dtype, out=dtype if dtype != "f32" else "f16")
    if kind == "matmul":
        K, N = _width(rng, 64, 16384), _width(rng, 64, 16384)
        M = _log(rng, 1, max(1, min(8192, 8192 ** 3 // (K * N))))
        source = rng.choice(["int8", "float", "gate"])
        # (what is quantized from float32 comes out in float16: a step of the
        # int8 values lies far above float32's rounding)
        out = "f16" if dtype == "f32" and source != "int8" else dtype
        return dict(kind=kind, source=source, M=M, K=K, N=N, dtype=dtype, out=out, bias=rng.random() < 0.3)
    if kind == "cache":
        heads, dim, page = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 80, 128, 256]), rng.choice([10, 16, 64, 128])
        read = _log(rng, 1, max(1, 60000 * 8 * 128 // (heads * dim) // (2 if dtype == "f32" else 1)))
        new = _log(rng, 1, max(1, min(16000 * 8 * 128 // (heads * dim), read)))
        return dict(kind=kind, new=new, read=read, heads=heads, dim=dim, page=page, pages=-(-read // page) + 3, dtype=dtype,
                    out="f16" if dtype == "f32" else dtype)
    kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8])
    dim, page = rng.choice([64, 80, 128, 256]), rng.choice([10, 16, 64, 128])
    seqs = _log(rng, 1, 64)
    chunk = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
    # (the padded scores and the padded cache stay below those of the largest listed cases)
    most = min(32768, 32 * 32000 * 8 * 128 // (seqs * kv * dim), 2048 * 32768 * 32 * 128 // (seqs * chunk * kv * group * max(dim, 128)))
    while most < 16:
        chunk = max(1, chunk // 2)
        most = min(32768, 32 * 32000 * 8 * 128 // (seqs * kv * dim), 2048 * 32768 * 32 * 128 // (seqs * chunk * kv * group * max(dim, 128)))
    context = _log(rng, 16, most)
    return dict(kind="attn", seqs=seqs, chunk=min(chunk, context), context=context, ragged=rng.random() < 0.7, heads=kv * group,
                kv_heads=kv, dim=dim, page=page, window=rng.choice([0, 0, max(1, context // 3)]), dtype=dtype, lens=rng.randrange(1 << 20))


def _lens(case):
    """New tokens and context length (the new ones among it) of every sequence."""
    r = random.Random(case["lens"])
    chunks, contexts = [], []
    for i in range(case["seqs"]):
        if case["ragged"] and i:
            contexts.append(_log(r, max(1, case["context"] // 32), case["context"]))
            chunks.append(min(contexts[-1], 1 if case["chunk"] == 1 else r.randint(0, case["chunk"])))
        else:
            contexts.append(case["context"])
            chunks.append(case["chunk"])
    return chunks, contexts


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 17)
    t = TYPES[case["dtype"]]
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    st = dict(case)
    if case["kind"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # a residual stream of a few large channels, as deep layers have
        big = torch.where(torch.rand(cols, device=DEV, generator=g) < 0.005, 20.0, 1.0)
        st.update(x=normal(rows, cols).to(t), res=(normal(rows, cols) * big * 2).to(t),
                  gamma=torch.rand(cols, device=DEV, generator=g) + 0.5, eps=1e-5)
    elif case["kind"] == "matmul":
        M, K, N = case["M"], case["K"], case["N"]
        w = torch.zeros(N, -(-K // 16) * 16, device=DEV, dtype=torch.int8)
        w[:, :K] = torch.randint(-127, 128, (N, K), device=DEV, generator=g, dtype=torch.int8)
        st.update(w=w, w_scale=(torch.rand(N, device=DEV, generator=g) + 0.5) / (73 * math.sqrt(K)))
        st["b"] = normal(N) * 0.1 if case["bias"] else None
        if case["source"] == "int8":
            x = torch.zeros(M, -(-K // 16) * 16, device=DEV, dtype=torch.int8)
            x[:, :K] = (normal(M, K) * 30).round_().clamp_(-127, 127)
            st.update(x=x, x_scale=torch.rand(M, device=DEV, generator=g) * 0.02 + 0.02)
        elif case["source"] == "float":
            st["x"] = (normal(M, K) * (torch.rand(M, 1, device=DEV, generator=g) + 0.5)).to(t)
        else:  # the gate's and the up projection's outputs, side by side as one product writes them
            st["x"] = normal(M, 2 * K).to(t)
    elif case["kind"] == "cache":
        H, D, P, page = case["heads"], case["dim"], case["pages"], case["page"]
        st["cache"] = tuple(torch.randint(-127, 128, (P, H, page, D), device=DEV, generator=g, dtype=torch.int8) for _ in "kv") + \
            tuple(torch.rand(P, H, page, device=DEV, generator=g) * 0.02 + 0.01 for _ in "kv")
        # k and v as parts of one projection's output
        qkv = normal(case["new"], 5 * H * D).to(t)
        st["k"] = qkv[:, 3 * H * D:4 * H * D].view(-1, H, D)
        st["v"] = qkv[:, 4 * H * D:].view(-1, H, D)
        where = torch.randperm(P, device=DEV, generator=g)[:-(-case["read"] // page)]
        slots = (where[:, None] * page + torch.arange(page, device=DEV)).reshape(-1)[:case["read"]].contiguous()
        st.update(slots=slots[case["read"] - case["new"]:].contiguous(), read_slots=slots)
    else:
        chunks, contexts = _lens(case)
        B, H, D, page = case["seqs"], case["kv_heads"], case["dim"], case["page"]
        need = [-(-n // page) for n in contexts]
        P = sum(need) + 1
        st["cache"] = tuple((torch.randn(P, H, page, D, device=DEV, generator=g) * 35).round_().clamp_(-127, 127).to(torch.int8) for _ in "kv") + \
            tuple(torch.rand(P, H, page, device=DEV, generator=g) * 0.03 + 0.01 for _ in "kv")
        order = torch.randperm(P, device=DEV, generator=g).to(torch.int32).cpu()
        table = torch.zeros(B, max(need), dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        starts = [0]
        for n in chunks:
            starts.append(starts[-1] + n)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
        st.update(q=normal(starts[-1], case["heads"], D).to(t), table=table.to(DEV), contexts=ints(contexts),
                  starts=ints(starts), max_chunk=max(chunks), max_context=max(contexts), scale=D ** -0.5)
    return st


def run(st):
    if own:
        return _own(st)
    return {"norm": _plain_norm, "matmul": _plain_matmul, "cache": _plain_cache, "attn": _plain_attn}[st["kind"]](st)


# ---- the framework's operators ---------------------------------------------------------

def _own(st):
    from paper_1809_02697_amd import neo
    if st["kind"] == "norm":
        q, scale, h = neo.rmsnorm_int8(st["x"], st["gamma"], st["eps"], residual=st["res"])
        return h, neo.dequantize_tokens_int8(q, scale, st["cols"], TYPES[st["out"]])
    if st["kind"] == "matmul":
        K, N, x = st["K"], st["N"], st["x"]
        if st["source"] == "int8":
            q, scale = x, st["x_scale"]
        elif st["source"] == "float":
            q, scale = neo.quantize_tokens_int8(x)
        else:
            q, scale = neo.quantize_tokens_int8(x[:, K:], gate=x[:, :K])
        return neo.matmul_int8(q, scale, K, st["w"], st["w_scale"], N, bias=st["b"], dtype=TYPES[st["out"]])
    if st["kind"] == "cache":
        neo.kv_write_int8(st["cache"], st["k"], st["v"], st["slots"])
        return neo.kv_read_int8(st["cache"], st["read_slots"], TYPES[st["out"]])
    return neo.attention_paged_int8(st["cache"], st["q"], st["table"], st["contexts"], st["starts"], st["max_chunk"],
                                    st["max_context"], scale=st["scale"], window=st["window"])


# ---- the same in elementary operations, 32 bits ----------------------------------------

def _quantize(x):
    """int8 values (as float32) and scales of the rows along x's last axis."""
    most = x.abs().amax(-1, keepdim=True)
    s = most / torch.full_like(most, 127.0)
    s = torch.where(most == 0, torch.ones_like(s), s)
    return (x / s).round().clamp(-127, 127), s


def _plain_norm(st):
    h = st["x"].float() + st["res"].float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + st["eps"]) * st["gamma"]
    q, s = _quantize(y)
    return h.to(TYPES[st["dtype"]]), (q * s).to(TYPES[st["out"]])


def _plain_matmul(st):
    K, x = st["K"], st["x"]
    if st["source"] == "int8":
        q, s = x[:, :K].float(), st["x_scale"][:, None]
    elif st["source"] == "float":
        q, s = _quantize(x.float())
    else:
        gate = x[:, :K].float()
        q, s = _quantize(x[:, K:].float() * (gate / (1 + torch.exp(-gate))))
    y = torch.matmul(q, st["w"][:, :K].float().t()) * s * st["w_scale"]
    if st["b"] is not None:
        y = y + st["b"]
    return y.to(TYPES[st["out"]])


def _plain_cache(st):
    kc, vc, ks, vs = st["cache"]
    page, t = st["page"], TYPES[st["out"]]
    p, o = st["slots"] // page, st["slots"] % page
    k, sk = _quantize(st["k"].float())
    v, sv = _quantize(st["v"].float())
    kc[p, :, o], vc[p, :, o] = k.to(torch.int8), v.to(torch.int8)
    ks[p, :, o], vs[p, :, o] = sk[..., 0], sv[..., 0]
    p, o = st["read_slots"] // page, st["read_slots"] % page
    return (kc[p, :, o].float() * ks[p, :, o][..., None]).to(t), (vc[p, :, o].float() * vs[p, :, o][..., None]).to(t)


def _plain_attn(st):
    kc, vc, ks, vs = st["cache"]
    q, table, ctx, starts = st["q"], st["table"].long(), st["contexts"].long(), st["starts"].long()
    B, (T, Hq, D), H, page, n = table.shape[0], q.shape, kc.shape[1], st["page"], st["max_chunk"]
    G, L = Hq // H, table.shape[1] * page
    i, j = torch.arange(n, device=DEV), torch.arange(L, device=DEV)
    at = starts[:-1, None] + i
    real = at < starts[1:, None]
    # [B][H][G * n][D] queries of a padded chunk, [B][H][L][D] keys and values
    qs = q.float()[at.clamp(max=T - 1)].view(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    keys, values = ((c[table].float() * s[table][..., None]).permute(0, 2, 1, 3, 4).reshape(B, H, L, D) for c, s in ((kc, ks), (vc, vs)))
    scores = torch.matmul(qs, keys.transpose(2, 3).contiguous()).view(B, H, G, n, L) * st["scale"]
    pos = (ctx - (starts[1:] - starts[:-1]))[:, None] + i
    seen = (j <= pos[..., None]) & (j < ctx[:, None, None]) & (pos[..., None] >= 0)
    if st["window"]:
        seen &= j > pos[..., None] - st["window"]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(B, H, G * n, L), values).view(B, H, G, n, D) / torch.where(total == 0, torch.ones_like(total), total)
    return out.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)[real].to(TYPES[st["dtype"]])


# ---- what a pass cannot do without -----------------------------------------------------

def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}
    e, o = size[case["dtype"]], size[case.get("out", case["dtype"])]
    if case["kind"] == "norm":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (3 * e + o) + 4 * case["cols"], "flops": 8 * n}
    if case["kind"] == "matmul":
        M, K, N = case["M"], case["K"], case["N"]
        each = {"int8": 1, "float": e, "gate": 2 * e}[case["source"]]
        return {"bytes": M * K * each + N * K + M * N * o + 4 * N, "flops": 2 * M * N * K}
    if case["kind"] == "cache":
        n, each = case["heads"] * case["dim"], case["heads"] * 4
        return {"bytes": 2 * (case["new"] * (n * (e + 1) + each + 4) + case["read"] * (n * (o + 1) + each + 4)), "flops": 6 * n * case["new"] + 2 * n * case["read"]}
    chunks, contexts = _lens(case)
    H, Hq, D, w = case["kv_heads"], case["heads"], case["dim"], case["window"]
    pairs, read = 0, 0
    for n, c in zip(chunks, contexts):
        if not n:
            continue
        pairs += sum(min(p + 1, w) if w else p + 1 for p in range(c - n, c))
        read += c - max(0, c - n + 1 - w) if w else c
    return {"bytes": 2 * read * H * (D + 4) + 2 * sum(chunks) * Hq * D * e, "flops": 4 * D * Hq * pairs}


# ---- the definitions, in 64 bits -------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "norm":
        h = st["x"].double() + st["res"].double()
        y = h / ((h ** 2).sum(1, keepdim=True) / case["cols"] + st["eps"]).sqrt() * st["gamma"].double()
        return h, _steps(y)
    if case["kind"] == "matmul":
        x, K = st["x"].double(), case["K"]
        if case["source"] == "int8":
            x = x[:, :K] * st["x_scale"].double()[:, None]
        elif case["source"] == "float":
            x = _steps(x)
        else:
            x = _steps(x[:, K:] * x[:, :K] * torch.sigmoid(x[:, :K]))
        y = x @ (st["w"][:, :K].double() * st["w_scale"].double()[:, None]).t().contiguous()
        return y if st["b"] is None else y + st["b"].double()
    if case["kind"] == "cache":
        out = []
        new = case["read"] - case["new"]
        for c, s, x in zip(st["cache"][:2], st["cache"][2:], (st["k"], st["v"])):
            c = (c.double() * s.double()[..., None]).transpose(1, 2).reshape(-1, case["heads"], case["dim"])
            out.append(torch.cat([c[st["read_slots"][:new]], _steps(x.double())]))
        return tuple(out)
    chunks, contexts = _lens(case)
    H, D, page = case["kv_heads"], case["dim"], case["page"]
    G = case["heads"] // H
    out, at = [], 0
    for b, (n, c) in enumerate(zip(chunks, contexts)):
        if not n:
            continue
        pages = st["table"][b, :-(-c // page)].long()
        keys, values = ((x[pages].double() * s[pages].double()[..., None]).transpose(0, 1).reshape(H, -1, D)[:, :c] for x, s in zip(st["cache"][:2], st["cache"][2:]))
        rows = torch.empty(n, H, G, D, device=DEV, dtype=torch.float64)
        far = torch.arange(c, device=DEV)[None] - torch.arange(c - n, c, device=DEV)[:, None]
        dark = (far > 0) | (far <= -case["window"]) if case["window"] else far > 0
        for h in range(H):
            for r in range(G):
                s = st["q"][at:at + n, h * G + r].double() @ keys[h].t().contiguous() * st["scale"]
                rows[:, h, r] = torch.softmax(s.masked_fill(dark, -math.inf), 1) @ values[h]
        out.append(rows.reshape(n, H * G, D))
        at += n
    return torch.cat(out) if out else torch.zeros(0, H * G, D, device=DEV, dtype=torch.float64)


def _steps(x):
    """What the rows of x become when each is held in int8 with a scale."""
    s = x.abs().amax(-1, keepdim=True) / 127
    s = torch.where(s > 0, s, torch.ones_like(s))
    return torch.clamp(torch.round(x / s), -127, 127) * s
