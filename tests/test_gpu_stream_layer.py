"""The token operators together, as the example runs them: layers over a stream
with their caches, against the same layers in plain fp32, and tokens one by one
against tokens at once."""
import os
import sys

import pytest
import torch

from paper_2609_31938_amd import tokens

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def model(**kw):
    from stream_layer import WorldModel
    args = dict(channels=256, heads=4, kv_heads=2, layers=2, H=8, W=12, latent=32, max_frames=4)
    return WorldModel(**dict(args, **kw))


def plain(m, x):
    """Causal predictions of the whole sequence in fp32, weights as they are
    stored, nothing else rounded."""
    def rms(v, g):
        return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * g

    def lin(v, w):
        return v @ (w.w.float() * w.scale[:, None]).t().contiguous()

    n = x.shape[0]
    cos, sin = (t[:n, None] for t in m.angles)

    def turn(v):
        half = v.shape[-1] // 2
        a, b = v[..., :half], v[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    h = lin(x.float(), m.embed)
    hidden = torch.ones(n, n, device="cuda").triu(1).bool()
    for layer in m.layers:
        G = layer.heads // layer.kv_heads
        q, k, v = lin(rms(h, layer.pre_a), layer.qkv).view(n, -1, layer.dim).split([layer.heads, layer.kv_heads, layer.kv_heads], 1)
        q, k = turn(q).transpose(0, 1), turn(k).repeat_interleave(G, 1).transpose(0, 1)
        v = v.repeat_interleave(G, 1).transpose(0, 1).contiguous()
        s = q @ k.transpose(1, 2).contiguous() * layer.dim ** -0.5
        a = s.masked_fill(hidden, float("-inf")).softmax(-1) @ v
        y = lin(a.transpose(0, 1).reshape(n, -1), layer.out)
        h = h + layer.gate_a.float() * rms(y, layer.post_a)
        y = lin(torch.nn.functional.silu(lin(rms(h, layer.pre_f), layer.up)), layer.down)
        h = h + layer.gate_f.float() * rms(y, layer.post_f)
    return lin(rms(h, m.last), m.head)


def relative(a, b):
    return float((a.float() - b.float()).norm() / b.float().norm())


def test_layers_match_plain_fp32():
    """Each of the 8-bit steps errs by about its step over sqrt(12): rows of
    products 1 / 127 of a row's largest value (some 3.5 of its root mean
    square) hence 0.8%, keys and values 2^-4 / sqrt(12) / 1.4 of a value, 1.3%.
    A dozen of them in sequence, independent, stay below 10%."""
    m = model()
    x = torch.randn(40, 128, device="cuda").bfloat16()
    assert relative(m.tokens(x, causal=True), plain(m, x)) < 0.1


def test_tokens_one_by_one_match_tokens_at_once():
    """The same sums in another order, and rounded activations that differ by a
    step here and there: far less than the steps themselves."""
    x = torch.randn(40, 128, device="cuda").bfloat16()
    whole = model().tokens(x, causal=True)
    m = model()
    steps = torch.cat([m.tokens(x[i:i + 1], causal=True) for i in range(40)])
    assert relative(steps, whole) < 0.03


def test_frames_are_decoded_with_their_caches():
    m = model(window_frames=2)
    x = torch.randn(m.per_frame, 128, device="cuda").bfloat16()
    seen = []
    for _ in range(3):
        x, y = m.frame(x)
        assert y.shape == (1, 96, 1, 8, 12) and y.isfinite().all()
        seen.append(y)
    assert not torch.equal(seen[0], seen[1])
    assert int(m.length) == 3 * m.per_frame
    k = m.layers[0].cache.k[:int(m.length) // 64].float()
    assert k.isfinite().all() and isinstance(m.layers[0].cache, tokens.KVCache)
