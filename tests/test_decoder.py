"""The decoder of paper_1809_02697_amd.decoder (norm, products, cache and
attention of the token operators run together) against the same network in 64
bits, with every quantization of the interface in its place.

Tolerance: where no value lies within float32's rounding of the middle of two
int8 steps (all rows but one in some dozens), float32 gives the 64-bit logits to
a few 10^-7: the median row is within 1e-5.  A value on the other side of such
a middle moves one step, 1/127 of its row's largest, and later quantizations
answer with steps of their own: such a row is off by 1 or 2 % of its norm (a
float32 evaluation in numpy is so too), and within 5e-2.  bfloat16 rounds every
activation to 2^-9, twelve roundings deep in two layers: within 5e-2.
"""
import numpy as np
import pytest

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu
SHAPE = dict(q_heads=6, kv_heads=2, head_dim=32)


def q8(x):
    """The values that rows quantized to int8 stand for."""
    top = np.abs(x).max(-1, keepdims=True)
    s = np.where(top == 0, 1, top / 127)
    return np.clip(np.rint(x / s), -127, 127) * s


def norm(x, g):
    return x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-5) * g


def reference(w, tokens, Hq, H, D):
    """Logits after every token of one sequence."""
    n = {k: v.double().cpu().numpy() for k, v in w.items() if k != "layers"}
    x = n["embed"][tokens]
    T = len(tokens)
    h = np.zeros_like(x)
    for lw in w["layers"]:
        p = {k: v.double().cpu().numpy() for k, v in lw.items()}
        mat = {k: q8(p[k]) for k in ("qkv", "out", "gate_up", "down")}
        h = h + x
        qkv = (q8(norm(h, p["norm1"])) @ mat["qkv"].T).reshape(T, Hq + 2 * H, D)
        q, k, v = qkv[:, :Hq], q8(qkv[:, Hq:Hq + H]), q8(qkv[:, Hq + H:])
        a = np.zeros((T, Hq, D))
        for i in range(Hq):
            s = q[:, i] @ k[:, i // (Hq // H)].T * D ** -0.5
            s[np.triu_indices(T, 1)] = -np.inf
            e = np.exp(s - s.max(1, keepdims=True))
            a[:, i] = e @ v[:, i // (Hq // H)] / e.sum(1, keepdims=True)
        h = h + q8(a.reshape(T, Hq * D)) @ mat["out"].T
        both = q8(norm(h, p["norm2"])) @ mat["gate_up"].T
        gate, up = np.split(both, 2, 1)
        x = q8(up * gate / (1 + np.exp(-gate))) @ mat["down"].T
    return q8(norm(h + x, n["norm"])) @ q8(n["head"]).T


@pytest.mark.parametrize("dtype,median", [("float32", 1e-5), ("bfloat16", 5e-2)])
@pytest.mark.parametrize("page", [16, 5])
def test_decoder_against_64_bits(dtype, median, page):
    torch = torch_cuda()
    from paper_1809_02697_amd import decoder
    w = decoder.random_weights(2, 300, 96, inner=160, **SHAPE)
    rng = np.random.default_rng(5)
    seqs = [rng.integers(0, 300, n) for n in (1, 9, 61, 140)]
    d = decoder.Decoder(w, pages=80, page_size=page, dtype=getattr(torch, dtype), **SHAPE)
    for _ in seqs:
        d.add()
    refs = [reference(w, s, SHAPE["q_heads"], SHAPE["kv_heads"], SHAPE["head_dim"]) for s in seqs]
    at = [0] * len(seqs)
    offs = []
    steps = [[1, 4, 30, 0], [0, 4, 1, 133], [0, 1, 30, 1], [0, 0, 0, 6]]   # chunks, single tokens, none
    for new in steps:
        logits = d.step([s[a:a + m].tolist() for s, a, m in zip(seqs, at, new)]).double().cpu().numpy()
        at = [a + m for a, m in zip(at, new)]
        row = 0
        for r, a, m in zip(refs, at, new):
            if m:
                off = np.linalg.norm(logits[row] - r[a - 1]) / np.linalg.norm(r[a - 1])
                assert off <= 5e-2, (new, row, off)
                offs.append(off)
                row += 1
        assert row == len(logits)
    assert np.median(offs) <= median, offs


def test_decoder_runs_out_of_pages():
    torch_cuda()
    from paper_1809_02697_amd import decoder
    d = decoder.Decoder(decoder.random_weights(1, 20, 32, inner=32, q_heads=2, kv_heads=1, head_dim=16), 2, 1, 16, pages=2, page_size=4)
    d.add()
    with pytest.raises(RuntimeError):
        d.step([[1] * 9])
    with pytest.raises(ValueError):
        d.step([[]])


def test_layer_in_a_graph():
    """A layer's step captured and replayed: every replay gives the eager bits,
    with eager work and synchronizations between them."""
    torch = torch_cuda()
    from paper_1809_02697_amd import decoder, neo
    w = decoder.random_weights(1, 50, 256, inner=512, **SHAPE)
    d = decoder.Decoder(w, pages=64, page_size=16, **SHAPE)
    layer, cache = d.layers[0], d.caches[0]
    step = decoder.Step([list(range(60)), [60, 61]], [900, 20], [1, 3], 16, "cuda")
    g = torch.Generator().manual_seed(3)
    k = torch.randn(900, 2, 32, generator=g).cuda()
    neo.kv_write_int8(cache, k, k.flip(0).contiguous(), torch.arange(900, device="cuda"))
    xs = [torch.randn(4, 256, generator=g).bfloat16().cuda() for _ in range(4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # (the workspaces of this stream grow here)
        eager = [tuple(t.clone() for t in layer(x, None, cache, step)) for x in xs]
        buf = xs[0].clone()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = layer(buf, None, cache, step)
    for _ in range(3):
        for x, e in zip(xs, eager):
            buf.copy_(x)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, e))
            torch.ones(1000, device="cuda").sum().item()
