"""The decoder layer of examples/decode_layer.py, all operators together, against the oracles.

The reference rounds where the layer does (fp16 before each GEMV, fp16 queries, cache rows and
attention output) and computes in 64 bits between. Each of these roundings differs from the layer's
only where a value lies at a rounding's edge, by 2^-11 of it; the GEMVs are within 1e-4 of their
terms' sum. Six such points follow one another, each passed on with a gain of a few at most
(softmax, silu, norms): the bound taken is 1e-2 of the update's 2-norm.
"""
import importlib.util
import os

import numpy as np
import pytest

import oracle
from oracle import decoder as od

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decode_layer", os.path.join(ROOT, "examples", "decode_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def linear(w, x):
    p = w.problem
    y, _ = oracle.gemv(x.astype(np.float16).view(np.uint16), p.T, p.alpha, p.v, p.salient_idx, p.residual_vals,
                       p.residual_idx)
    return y


def reference(layer, h, q_len, ctx, seqs):
    """The step in 64 bits; seqs: each sequence's (k, v) rows so far, extended here."""
    dim = layer.dim
    cos, sin = layer.cos.cpu().numpy(), layer.sin.cpu().numpy()
    pos = od.token_positions(q_len, ctx)
    heads = lambda y: y.reshape(len(y), -1, dim)  # noqa: E731
    h = h.astype(np.float64)
    _, x = od.norm(h, layer.norm_attn.double().cpu().numpy())
    q = od.prepare_heads(heads(linear(layer.wq, x)), pos, cos=cos, sin=sin).astype(np.float16)
    k = od.prepare_heads(heads(linear(layer.wk, x)), pos, cos=cos, sin=sin).astype(np.float16).astype(np.float64)
    v = heads(linear(layer.wv, x)).astype(np.float16).astype(np.float64)
    t = 0
    for s, n in enumerate(q_len):
        for side, new in ((0, k), (1, v)):
            seqs[s][side] = np.concatenate((seqs[s][side], new[t:t + n]))
        t += n
    a, _, _ = od.attention(q, [s[0] for s in seqs], [s[1] for s in seqs], q_len, ctx, dim ** -0.5)
    h, x = od.norm(h, layer.norm_mlp.double().cpu().numpy(), y=linear(layer.wo, a.reshape(len(a), -1)),
                   res_scale=layer.scale)
    g, u = linear(layer.wg, x) * layer.scale, linear(layer.wu, x)
    h, _ = od.norm(h, y=linear(layer.wd, g / (1 + np.exp(-g)) * u * layer.scale), res_scale=layer.scale)
    return h


def test_decoder_layer_steps_follow_the_oracle(example):
    layer = example.DecoderLayer(hidden=512, q_heads=4, kv_heads=2, dim=64, inner=1024, fmt="f16", page=16, max_seqs=3,
                                 max_context=80, seed=3)
    rng = np.random.default_rng(4)
    seqs = [[np.zeros((0, 2, 64)), np.zeros((0, 2, 64))] for _ in range(3)]
    ctx = [0, 0, 0]
    for q_len in ([5, 8, 3], [1, 1, 1], [4, 1, 2], [1, 1, 1]):  # small chunks, decode steps, drafted tokens
        ctx = [c + n for c, n in zip(ctx, q_len)]
        h = rng.standard_normal((sum(q_len), 512)).astype(np.float32)
        got = layer.step(torch.from_numpy(h).cuda(), layer.batch(q_len, ctx)).double().cpu().numpy()
        want = reference(layer, h, q_len, ctx, seqs)
        off = np.linalg.norm(got - want) / np.linalg.norm(want - h)
        assert off <= 1e-2, (q_len, off)


@pytest.mark.parametrize("fmt", ["f16", "fp8", "fp4"])
def test_decoder_layer_in_a_graph_gives_the_same(example, fmt):
    layer = example.DecoderLayer(hidden=512, q_heads=8, kv_heads=2, dim=128, inner=1024, fmt=fmt, page=32, max_seqs=1,
                                 max_context=96, seed=5)
    prompt = layer.batch([70], [70])
    k, v = (torch.randn(70, 256, device="cuda") for _ in range(2))
    example.qt.qtea_kv_append(layer.cache, prompt, k, v)
    start = torch.randn(1, 512, device="cuda")
    batch = layer.batch([1], [71])
    plain = []
    h = start.clone()
    for _ in range(3):
        plain.append(layer.step(h, batch).clone())
        batch.ctx_len += 1
    stream, h = torch.cuda.Stream(), start.clone()
    batch.ctx_len.fill_(71)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        layer.step(h, batch)  # the first call on a stream makes its workspace
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            layer.step(h, batch)
        h.copy_(start)
        for want in plain:
            graph.replay()
            assert torch.equal(h, want)
            batch.ctx_len += 1
    torch.cuda.synchronize()
