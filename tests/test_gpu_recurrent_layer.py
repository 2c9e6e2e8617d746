"""A recurrent layer's operators together, as the example runs them, beside the
layers that keep a cache: against the same layers in plain fp32, and tokens one
by one against tokens at once."""
import os
import sys

import pytest
import torch

from paper_2609_31938_amd import tokens

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def model(**kw):
    from stream_layer import WorldModel
    args = dict(channels=256, heads=4, kv_heads=2, layers=2, H=8, W=12, latent=32, max_frames=4, recurrent=1)
    return WorldModel(**dict(args, **kw))


def plain(m, x):
    """Predictions of the whole sequence in fp32, token by token in the
    recurrence, weights as they are stored, nothing else rounded."""
    def rms(v, g):
        return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * g

    def lin(v, w):
        return v @ (w.w.float() * w.scale[:, None]).t().contiguous()

    n = x.shape[0]
    h = lin(x.float(), m.embed)
    for layer in m.layers:
        q, k, v = lin(rms(h, layer.pre_a), layer.qkv).view(n, -1, layer.dim).split([layer.kv_heads, layer.kv_heads, layer.heads], 1)
        G = layer.heads // layer.kv_heads
        q, k = q.repeat_interleave(G, 1), k.repeat_interleave(G, 1)
        S, a = torch.zeros(layer.heads, layer.dim, layer.dim, device="cuda"), torch.empty_like(v)
        for t in range(n):
            S = layer.log_decay.exp()[:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
            a[t] = (q[t][:, :, None] * S).sum(1) * layer.dim ** -0.5
        h = h + lin(a.reshape(n, -1), layer.out)
        z = lin(rms(h, layer.pre_f), layer.gate_up)
        half = z.shape[1] // 2
        h = h + lin(torch.nn.functional.silu(z[:, :half]) * z[:, half:], layer.down)
    return lin(rms(h, m.last), m.head)


def relative(a, b):
    return float((a.float() - b.float()).norm() / b.float().norm())


def test_layers_match_plain_fp32():
    """Each of the 8-bit steps errs by about its step over sqrt(12): rows of
    products 1 / 127 of a row's largest value (some 3.5 of its root mean square,
    some 10 after a gate's product), hence 0.8% to 2.3%.  A dozen of them in
    sequence, independent, stay below 10%."""
    m = model()
    x = torch.randn(40, 128, device="cuda").bfloat16()
    assert relative(m.tokens(x, causal=True), plain(m, x)) < 0.1


@pytest.mark.parametrize("recurrent", [1, 2])
def test_tokens_one_by_one_match_tokens_at_once(recurrent):
    """The same sums in another order, and rounded activations that differ by a
    step here and there: far less than the steps themselves."""
    x = torch.randn(40, 128, device="cuda").bfloat16()
    whole = model(recurrent=recurrent).tokens(x, causal=True)
    m = model(recurrent=recurrent)
    steps = torch.cat([m.tokens(x[i:i + 1], causal=True) for i in range(40)])
    assert relative(steps, whole) < 0.03


def test_frames_with_both_memories():
    """A frame after another: the states move on, and a stream that begins anew
    begins at zero."""
    m = model(layers=3, recurrent=3, window_frames=2)
    assert isinstance(m.layers[2].states, tokens.StateCache) and isinstance(m.layers[0].cache, tokens.KVCache)
    first = torch.randn(m.per_frame, 128, device="cuda").bfloat16()
    x, states, outs = first, [], []
    for _ in range(3):
        x, y = m.frame(x)
        assert y.shape == (1, 96, 1, 8, 12) and y.isfinite().all()
        states.append(m.layers[2].states.state.clone())
        outs.append(x)
    assert not torch.equal(states[0], states[1]) and states[2].isfinite().all()
    m.length.zero_()
    again, _ = m.frame(first)
    assert torch.equal(again, outs[0]) and torch.equal(m.layers[2].states.state, states[0])


def test_a_step_captured_and_replayed():
    """One token through the layers as a graph, replayed along a stream."""
    m, e = model(recurrent=2), model(recurrent=2)
    x = torch.randn(1, 128, device="cuda").bfloat16()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m.tokens(x, causal=True)
    torch.cuda.synchronize()
    m.length.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m.tokens(x, causal=True)
    m.length.zero_()
    for i in range(5):
        x.copy_(torch.randn(1, 128, device="cuda"))
        graph.replay()
        want = e.tokens(x, causal=True)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
    assert torch.equal(m.layers[1].states.state, e.layers[1].states.state)
