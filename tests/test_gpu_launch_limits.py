"""Calls of more workgroups than one launch takes (2^32 threads): the rows on
both sides of that limit, against calls of those rows alone."""
import pytest
import torch

from paper_2609_31938_amd import c3c, tokens
import token_ref as ref

pytestmark = pytest.mark.gpu

MANY = (1 << 26) + 77  # rows of a wave each: 2^32 threads are 2^26 of them


def ends(T, n=301):
    """Slices of rows: the first, those around 2^25 and 2^26, the last."""
    return [slice(0, n), slice((1 << 25) - n, (1 << 25) + n), slice((1 << 26) - n, T)]


@pytest.mark.parametrize("rows", [1, 1 << 25])
def test_norm_gate(rows):
    C, ctx = 4, c3c.Context()
    g = torch.Generator(device="cuda").manual_seed(3)
    h, y = (torch.randn(MANY, C, generator=g, device="cuda").bfloat16() for _ in range(2))
    gate = torch.randn(-(-MANY // rows), C, generator=g, device="cuda").bfloat16()
    post, pre = (1 + 0.3 * ref.randn(s, C) for s in (1, 2))
    got = tokens.norm_gate(ctx, h, y, gate, post=post, pre=pre, rows_per_gate=rows)
    for s in ends(MANY):
        group = gate[torch.arange(s.start, s.stop, device="cuda") // rows]
        want = tokens.norm_gate(ctx, h[s], y[s], group, post=post, pre=pre, rows_per_gate=1)
        assert all(torch.equal(a[s], b) for a, b in zip(got, want)), s


def test_quantize_rows():
    C, ctx = 5, c3c.Context()
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(MANY, C, generator=g, device="cuda").bfloat16()
    q, s = tokens.quantize_rows(ctx, x)
    for at in ends(MANY):
        qw, sw = tokens.quantize_rows(ctx, x[at])
        assert torch.equal(q[at], qw) and torch.equal(s[at], sw), at
