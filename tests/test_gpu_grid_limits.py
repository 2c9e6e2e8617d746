"""Convolutions of more workgroups than a launch takes (2^32 threads): refused
or computed, never left undone without an error."""
import pytest
import torch

from paper_2609_31938_amd import c3c, inputs

pytestmark = pytest.mark.gpu

MANY = (1 << 24) + 40  # frames of one pixel, a workgroup of 256 threads each


@pytest.mark.parametrize("dtype,kw", [("bf16", dict(Kh=3, Kw=3)), ("f32", dict(Kh=3, Kw=3)), ("bf16", dict(Kh=1, Kw=1)),
                                      ("f32", dict(Kh=1, Kw=1))])
def test_streams_of_too_many_frames(dtype, kw):
    spec = inputs.spec(N=1, Ci=4, Co=4, T=MANY, Tc=2, H=1, W=1, has_bias=0, **kw)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    ctx = c3c.Context()
    x = torch.ones(1, 4, MANY, 1, 1, dtype=dt, device="cuda")
    cache = torch.ones(1, 4, 2, 1, 1, dtype=dt, device="cuda")
    w = torch.ones(4, 4, 3, spec["Kh"], spec["Kw"], dtype=dt, device="cuda")
    wpack = c3c.weight_repack(ctx, spec, w)
    y = torch.full((1, 4, MANY, 1, 1), 7.0, dtype=dt, device="cuda")
    try:
        c3c.conv3d_causal_cached(ctx, spec, x, cache, w, wpack, None, y=y)
    except c3c.C3CError as e:
        assert e.status == c3c.E_DEVICE and (y == 7).all()  # nothing was launched
    else:
        assert (y == 12).all()


def test_block_form_of_too_many_frames():
    spec = inputs.spec(N=1, Ci=4, Co=4, T=MANY, Tc=2, H=1, W=1, has_bias=0)
    ctx = c3c.Context()
    x = torch.ones(1, 4, MANY, 1, 1, dtype=torch.bfloat16, device="cuda")
    cache = torch.ones(1, 4, 2, 1, 1, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(4, 4, 3, 3, 3, dtype=torch.bfloat16, device="cuda")
    gamma, beta = torch.ones(4, device="cuda"), torch.zeros(4, device="cuda")
    ctx.set_workspace(torch.empty(c3c.block_workspace_bytes(spec), dtype=torch.uint8, device="cuda"))
    with pytest.raises(c3c.C3CError) as e:
        c3c.conv3d_causal_cached_block(ctx, spec, x, cache, w, c3c.weight_repack(ctx, spec, w), None, gamma, beta, 1e-6)
    assert e.value.status == c3c.E_DEVICE
