"""Norms, gate and residual, and 8-bit rows, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2609_31938_amd import c3c, tokens
import token_ref as ref

pytestmark = pytest.mark.gpu


def case(dtype, T, C, rows, seed=1):
    dt = ref.TORCH[dtype]
    g = -(-T // rows)
    return dict(h=ref.randn(seed, T, C).to(dt), y=(2 * ref.randn(seed + 1, T, C)).to(dt),
                gate=ref.randn(seed + 2, g, C).to(dt), post=1 + 0.3 * ref.randn(seed + 3, C),
                pre=1 + 0.3 * ref.randn(seed + 4, C))


def tolerances(dtype, h, u, hs, us):
    """Rounding at the output; fp32 arithmetic of some 16 operations and the
    sums over a row, whose partial sums are at most 40 deep: 64 roundings."""
    one, two = ref.UNIT[dtype], 64 * ref.EPS32
    return one * np.abs(h) + two * hs + ref.TINY[dtype], None if u is None else one * np.abs(u) + 2 * two * us + ref.TINY[dtype]


SHAPES = [(1, 1, 1), (1, 4096, 1), (3, 7, 2), (5, 64, 5), (130, 512, 1), (9, 513, 4), (33, 1024, 7), (2, 1531, 1),
          (300, 2000, 100), (7, 5120, 3), (2, 9001, 2), (3, 33000, 1), (2, 40001, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C,rows", SHAPES)
def test_matches_64_bits(dtype, T, C, rows):
    c, ctx = case(dtype, T, C, rows), c3c.Context()
    h, u = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], post=c["post"], pre=c["pre"], alpha=0.75, eps=1e-5,
                            rows_per_gate=rows)
    rh, ru, hs, us = ref.norm_gate(c["h"], c["y"], c["gate"], c["post"], c["pre"], 0.75, np.float32(1e-5), rows)
    th, tu = tolerances(dtype, rh, ru, hs, us)
    ref.assert_within(h, rh, th, "h")
    ref.assert_within(u, ru, tu, "u")


@pytest.mark.parametrize("C", [96, 1000, 20000, 40001])
@pytest.mark.parametrize("parts", ["no_post", "no_gate", "neither", "no_y", "no_pre"])
def test_omissions(C, parts):
    c, ctx = case("bf16", 6, C, 6), c3c.Context()
    if parts in ("no_post", "neither", "no_y"):
        c["post"] = None
    if parts in ("no_gate", "neither", "no_y"):
        c["gate"] = None
    if parts == "no_y":
        c["y"] = None
    if parts == "no_pre":
        c["pre"] = None
    h, u = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], post=c["post"], pre=c["pre"], alpha=-1.5, rows_per_gate=6)
    rh, ru, hs, us = ref.norm_gate(c["h"], c["y"], c["gate"], c["post"], c["pre"], -1.5, np.float32(1e-6), 6)
    th, tu = tolerances("bf16", rh, ru, hs, us)
    ref.assert_within(h, rh, th, "h")
    assert (u is None) == (parts == "no_pre")
    if u is not None:
        ref.assert_within(u, ru, tu, "u")


@pytest.mark.parametrize("C", [100, 3000, 33001])
def test_in_place(C):
    c, ctx = case("bf16", 5, C, 2), c3c.Context()
    args = dict(post=c["post"], pre=c["pre"], rows_per_gate=2)
    h, u = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], **args)
    h2, u2 = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], h_out=c["h"], **args)
    assert h2 is c["h"] and torch.equal(h, h2) and torch.equal(u, u2)


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_any_alignment(offset):
    """Tensors that begin at any element: the same bits as aligned ones."""
    c, ctx = case("bf16", 4, 777, 2), c3c.Context()

    def move(t):
        b = torch.empty(t.numel() + 8, dtype=t.dtype, device=t.device)
        v = b[offset:offset + t.numel()].view(t.shape)
        v.copy_(t)
        return v

    h, u = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], post=c["post"], pre=c["pre"], rows_per_gate=2)
    m = {k: move(t) for k, t in c.items()}
    h2, u2 = tokens.norm_gate(ctx, m["h"], m["y"], m["gate"], post=m["post"], pre=m["pre"], rows_per_gate=2,
                              h_out=move(h), u=move(u))
    assert torch.equal(h, h2) and torch.equal(u, u2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [40, 1531, 5120, 40000])
def test_8_bit_output(dtype, C):
    """The 8-bit rows stand for u within half a step and u's own error."""
    c, ctx = case(dtype, 5, C, 1), c3c.Context()
    c["h"][3] = 0
    c["y"][3] = 0
    h, q, s = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], post=c["post"], pre=c["pre"], quantize=True)
    _, ru, _, us = ref.norm_gate(c["h"], c["y"], c["gate"], c["post"], c["pre"], 1.0, np.float32(1e-6), 1)
    top = np.abs(ru).max(1)
    err = 2 * 64 * ref.EPS32 * us
    ref.assert_within(s, top / 127, 2 * ref.EPS32 * top / 127 + err.max(1) / 127, "scale")
    ref.assert_within(ref.f64(q) * ref.f64(s)[:, None], ru, 0.5001 * top[:, None] / 127 + 2 * err + 1e-30, "codes")
    assert (q[3] == 0).all() and s[3] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,C,ld", [(1, 1, 1), (3, 17, 17), (5, 1000, 1003), (70, 4096, 4096), (2, 33001, 33001)])
def test_quantize_rows(dtype, T, C, ld):
    x = ref.randn(7, T, ld).to(ref.TORCH[dtype])[:, :C]
    x[T // 2, C // 2] = 100
    q, s = tokens.quantize_rows(c3c.Context(), x)
    rq, rs = ref.quantize(x)
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s.cpu().numpy(), rs)


def test_quantize_rows_of_zeros_and_of_what_is_not_finite():
    x = ref.randn(8, 6, 300)
    x[0] = 0
    x[1, 5] = float("inf")
    x[2, 299] = float("nan")
    x[3] = 1e-45           # the scale rounds to 0
    x[4] *= 1e38 / x[4].abs().max()
    q, s = tokens.quantize_rows(c3c.Context(), x)
    rq, rs = ref.quantize(x)
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s.cpu().numpy(), rs, equal_nan=True)


def test_nan_stays_in_its_row():
    c, ctx = case("f32", 4, 200, 4), c3c.Context()
    c["y"][1, 3] = float("nan")
    h, q, s = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], post=c["post"], pre=c["pre"], rows_per_gate=4, quantize=True)
    assert h[1].isnan().all() and s[1].isnan() and (q[1] == 0).all()
    keep = [0, 2, 3]
    assert h[keep].isfinite().all() and s[keep].isfinite().all()


def test_no_tokens_and_other_stream():
    ctx = c3c.Context()
    h, u = tokens.norm_gate(ctx, torch.empty(0, 64, device="cuda"), pre=torch.ones(64, device="cuda"))
    assert h.shape == u.shape == (0, 64)
    c = case("bf16", 100, 1024, 10)
    args = dict(post=c["post"], pre=c["pre"], rows_per_gate=10)
    want = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], **args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = tokens.norm_gate(ctx, c["h"], c["y"], c["gate"], **args)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
