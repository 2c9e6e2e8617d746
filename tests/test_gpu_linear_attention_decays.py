"""Linear attention with decays at the ends of their range: above 0, where states
grow, and so fast that a weight is next to nothing in fp32."""
import numpy as np
import pytest
import torch

from paper_2609_31938_amd import c3c, tokens
import layer_ref
import token_ref as ref
from test_gpu_linear_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,old", [([1, 1], [4, 0]), ([4, 2], [4, 0]), ([70, 33], [3, 0]), ([300, 1], [2, 2])])
@pytest.mark.parametrize("rate", [0.02, 0.5])
def test_decays_of_both_signs(dtype, new, old, rate):
    """Taken as they come, as long as their sums stay below 87: over 32 tokens,
    and where sequences are split over a part of one."""
    c = Case(new, old, 2, 2, 64, 64, dtype)
    c.g = rate * ref.randn(9, *c.g.shape)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[3], [60]])
def test_growing_states(dtype, new):
    """All decays above 0: a state that only grows."""
    c = Case(new, [3], 2, 2, 32, 48, dtype)
    c.g = c.g.abs() + 0.1
    c.check(c.run())


@pytest.mark.parametrize("rate", [80.0, 86.0, 88.0, 95.0, 103.0, 105.0, 1e4])
@pytest.mark.parametrize("new", [[1], [2, 5], [6], [40]])
def test_next_to_nothing(rate, new):
    """Weights below 2^-126 count as 0: large states keep what larger weights leave
    of them, and nothing is left where there is less."""
    c = Case(new, [3] * len(new), 2, 2, 32, 32, "f32", rate=0.0)
    c.state = c.state * 2.0 ** 100
    at = 0
    for n in new:  # the first token of each
        c.g[at] = -rate
        at += n
    out, state = c.run()
    q, k, v, g, S = (ref.f64(x) for x in (c.q, c.k, c.v, c.g, c.state))
    at = 0
    for b, n in enumerate(new):
        rows, s = slice(at, at + n), int(c.slot[b])
        want, end, so, se = layer_ref.linear_attention(q[rows], k[rows], v[rows], g[rows], S[s], 32 ** -0.5)
        lost = 2.0 ** -126 * np.abs(S[s])
        through = 32 ** -0.5 * np.einsum("thk,hkv->thv", np.abs(q[rows]), lost)
        ref.assert_within(out[rows], want, layer_ref.attention_tolerance("f32", want, so, n, 32) + through, b)
        ref.assert_within(state[s], end, layer_ref.state_tolerance(n, se) + lost, ("state", b))
        at += n
