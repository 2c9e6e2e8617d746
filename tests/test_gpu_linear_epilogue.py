"""8-bit products with an epilogue, and gated ones, against exact integer sums
and functions in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2609_31938_amd import c3c, tokens
import layer_ref
import token_ref as ref

pytestmark = pytest.mark.gpu

ACTS = ["none", "silu", "gelu", "gelu_tanh"]
DTYPES = ["bf16", "f16", "f32"]
SHAPES = [(1, 1, 1), (1, 64, 128), (3, 33, 1000), (4, 40, 4096), (5, 130, 96), (17, 100, 160), (33, 65, 100), (64, 257, 513),
          (65, 129, 2048), (128, 128, 16), (200, 77, 4000), (333, 777, 1111), (1000, 1024, 272), (2049, 2049, 400)]


def context(n):
    ctx = c3c.Context()
    if n:
        ctx.set_workspace(torch.empty(n, dtype=torch.uint8, device="cuda"))
    return ctx


def weights(N, K, seed=3):
    """Products of about one with activations of about one."""
    g = torch.Generator().manual_seed(seed)
    w = torch.randint(-127, 128, (N, K), generator=g, dtype=torch.int8).cuda()
    return w, ((0.5 + torch.rand(N, generator=g)) / (73 * K ** 0.5)).cuda(), torch.randn(N, generator=g).cuda()


def epilogue_call(M, N, K, xd, yd, act="none", bias=True, residual=False, rows=0, alpha=0.9, in_place=False, ws=None, ld=None):
    """Runs the call and checks it."""
    x = ref.randn(5, M, ld or K)[:, :K]
    q, s = layer_ref.quantize(x) if xd == "i8" else (None, None)
    if xd != "i8":
        x = x.to(ref.TORCH[xd])
        q, s = layer_ref.quantize(x)
        xs = None
    else:
        x, xs = torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda()
    w, wscale, b = weights(N, K)
    b = b if bias else None
    res = (3 * ref.randn(6, M, N)).to(ref.TORCH[yd]) if residual else None
    gate = ref.randn(7, -(-M // rows), N).to(ref.TORCH[yd]) if rows else None
    n = tokens.linear_i8_workspace_bytes(M, N, K, xd, yd, ld_x=ld) if ws is None else ws
    z, err = layer_ref.product(q, s, w, wscale, b)
    want, tol = layer_ref.epilogue(z, err, act, None if gate is None else ref.f64(gate)[np.arange(M) // rows],
                                   None if res is None else ref.f64(res), alpha, yd)
    y = tokens.linear_i8(context(n), x, w, wscale, b, x_scale=xs, out_dtype=yd, out=res if in_place else None, act=act,
                         residual=res, gate=gate, alpha=alpha, rows_per_gate=rows or 1)
    ref.assert_within(y, want, tol)
    return y


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_activation_gate_and_residual(act, dtype, M, N, K):
    epilogue_call(M, N, K, dtype, dtype, act, residual=True, rows=3)


@pytest.mark.parametrize("act,residual,rows,bias", [("silu", False, 0, True), ("none", True, 0, False), ("none", False, 1, True),
                                                    ("gelu", False, 1000, False), ("gelu_tanh", True, 0, True),
                                                    ("silu", False, 1 << 40, True)])
@pytest.mark.parametrize("M,N,K", [(2, 50, 300), (30, 64, 64), (100, 300, 2000), (300, 515, 1024)])
@pytest.mark.parametrize("xd", ["i8", "bf16"])
def test_each_part_alone(act, residual, rows, bias, M, N, K, xd):
    epilogue_call(M, N, K, xd, "bf16", act, bias, residual, rows)


@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (20, 100, 100), (100, 300, 9000), (300, 300, 513), (2100, 2050, 256)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_onto_the_residual_itself(M, N, K, dtype):
    kw = dict(act="silu", residual=True, rows=7)
    assert torch.equal(epilogue_call(M, N, K, dtype, dtype, **kw), epilogue_call(M, N, K, dtype, dtype, in_place=True, **kw))


def test_split_and_unsplit_give_the_same_bits():
    M, N, K = 100, 300, 9000
    rows = M * 9008 + 4096
    assert tokens.linear_i8_workspace_bytes(M, N, K) > rows
    kw = dict(act="gelu", residual=True, rows=10)
    assert torch.equal(epilogue_call(M, N, K, "bf16", "bf16", **kw), epilogue_call(M, N, K, "bf16", "bf16", ws=rows, **kw))


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [(4200, 4100, 256), (4200, 4128, 95), (2100, 2050, 128)])
@pytest.mark.parametrize("rows", [0, 1, 300, 5000])
def test_large_tiles_onto_a_residual(act, dtype, M, N, K, rows):
    """Tiles of 256 and 128, whole ones and the last; tokens of a tile under one
    row of gates, and under several."""
    kw = dict(act=act, residual=True, rows=rows)
    assert torch.equal(epilogue_call(M, N, K, "i8", dtype, **kw), epilogue_call(M, N, K, "i8", dtype, in_place=True, **kw))


@pytest.mark.parametrize("M,N,K,ld", [(40, 130, 97, 99), (70, 130, 97, 99), (300, 257, 96, 112)])
def test_strided_rows(M, N, K, ld):
    epilogue_call(M, N, K, "f16", "f32", "silu", residual=True, ld=ld)


def test_no_epilogue_is_the_plain_product():
    x = ref.randn(5, 70, 100).bfloat16()
    w, ws, b = weights(33, 100)
    ctx = context(tokens.linear_i8_workspace_bytes(70, 33, 100))
    want = tokens.linear_i8(ctx, x, w, ws, b)
    d, e = tokens.LinearDesc(70, 33, 100, 100, 1, 1), tokens._Epilogue(None, None, 1, 1.0, 0)
    y = torch.empty_like(want)
    st = c3c.lib.c3c_linear_i8_epilogue(ctx._h, tokens.C.byref(d), tokens.C.byref(e), x.data_ptr(), None, w.data_ptr(),
                                        ws.data_ptr(), b.data_ptr(), y.data_ptr(), None)
    torch.cuda.synchronize()
    assert st == c3c.OK and torch.equal(y, want)


def test_nan_and_infinities_stay_where_they_are():
    M, N, K = 80, 40, 64
    x, (w, ws, b) = ref.randn(5, M, K), weights(N, K)
    res, gate = ref.randn(6, M, N), ref.randn(7, 4, N)
    x[3, 5], res[7, 9], gate[2, 4] = float("nan"), float("inf"), float("nan")
    ctx = context(tokens.linear_i8_workspace_bytes(M, N, K, "f32", "f32"))
    y = tokens.linear_i8(ctx, x, w, ws, b, act="gelu_tanh", residual=res, gate=gate, rows_per_gate=20)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[3], bad[7, 9], bad[40:60, 4] = True, True, True
    assert torch.equal(~y.isfinite(), bad) and y[7, 9] == float("inf")


# ---------------------------------------------------------------- gated

def gated_call(M, N, K, xd, yd, act="silu", bias=True, ws=None, ld=None):
    x = ref.randn(5, M, ld or K)[:, :K]
    if xd == "i8":
        q, s = layer_ref.quantize(x)
        x, xs = torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda()
    else:
        x, xs = x.to(ref.TORCH[xd]), None
        q, s = layer_ref.quantize(x)
    w, wscale, b = weights(2 * N, K)
    b = b if bias else None
    z, err = layer_ref.product(q, s, w, wscale, b)
    a, rel, off = layer_ref.act(z[:, :N], act)
    up = z[:, N:]
    want = a * up
    ea = (1.2 * err[:, :N] if act != "none" else err[:, :N]) + np.abs(a) * rel + off
    tol = ref.UNIT[yd] * np.abs(want) + np.abs(up) * ea + np.abs(a) * err[:, N:] + ea * err[:, N:] + ref.EPS32 * np.abs(want) + ref.TINY[yd]
    n = tokens.gated_linear_i8_workspace_bytes(M, N, K, xd, yd, ld_x=ld) if ws is None else ws
    y = tokens.gated_linear_i8(context(n), x, w, wscale, b, x_scale=xs, out_dtype=yd, act=act)
    ref.assert_within(y, want, tol)
    return y


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gated(act, dtype, M, N, K):
    gated_call(M, N, K, dtype, dtype, act)


@pytest.mark.parametrize("yd", DTYPES)
@pytest.mark.parametrize("M,N,K,ld", [(1, 48, 100, 100), (5, 48, 96, 112), (40, 130, 97, 99), (70, 130, 97, 99), (600, 515, 1024, 1024),
                                      (2100, 1030, 128, 128), (4200, 2050, 256, 256), (4200, 2064, 95, 95)])
def test_gated_8_bit_activations(yd, M, N, K, ld):
    gated_call(M, N, K, "i8", yd, bias=False, ld=ld)


def test_gated_split_and_unsplit_give_the_same_bits():
    M, N, K = 100, 150, 9000
    rows = M * 9008 + 4096
    assert tokens.gated_linear_i8_workspace_bytes(M, N, K) > rows
    assert torch.equal(gated_call(M, N, K, "bf16", "bf16"), gated_call(M, N, K, "bf16", "bf16", ws=rows))


@pytest.mark.parametrize("M", [3, 20, 100, 3000])
def test_gated_halves_are_those_of_plain_products(M):
    """Without an activation, the product of two plain products in fp32, to a rounding."""
    N, K = 1100, 304
    x, (w, ws, b) = ref.randn(5, M, K).bfloat16(), weights(2 * N, K)
    ctx = context(tokens.gated_linear_i8_workspace_bytes(M, N, K, "i8"))
    x, xs = tokens.quantize_rows(ctx, x)
    got = tokens.gated_linear_i8(ctx, x, w, ws, b, x_scale=xs, act="none", out_dtype="f32")
    a, u = (tokens.linear_i8(ctx, x, w[s], ws[s], b[s], x_scale=xs, out_dtype="f32") for s in (slice(0, N), slice(N, 2 * N)))
    assert torch.equal(got, a * u)


@pytest.mark.parametrize("M", [2, 200])
def test_captured_and_replayed(M):
    """An epilogue onto its own residual, and a gated product, in a graph."""
    N, K = 130, 256
    x, res = ref.randn(1, M, K).bfloat16(), ref.randn(2, M, K).bfloat16()
    (w, ws, b), (w2, ws2, _) = weights(2 * N, K), weights(K, N)
    ctxs = [context(1 << 24) for _ in range(2)]

    def step(ctx, r):
        u = tokens.gated_linear_i8(ctx, x, w, ws, b)
        return tokens.linear_i8(ctx, u, w2, ws2, residual=r, out=r)

    mine, eager = res.clone(), res.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(ctxs[0], res.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ctxs[0], mine)
    for _ in range(4):
        x.copy_(x.roll(1, 0))
        graph.replay()
        step(ctxs[1], eager)
        torch.cuda.synchronize()
        assert torch.equal(mine, eager)


def test_gated_large_offsets():
    """y past 2^32 bytes, rows of x past 2^31 bytes."""
    M, N, K = 140000, 16384, 16400
    x = torch.zeros(M, K, dtype=torch.int8, device="cuda")
    x[-300:] = torch.randint(-127, 128, (300, K), dtype=torch.int8).cuda()
    s = torch.ones(M, device="cuda")
    w, ws, _ = weights(2 * N, K)
    y = tokens.gated_linear_i8(c3c.Context(), x, w, ws, x_scale=s, act="silu")
    want = tokens.gated_linear_i8(c3c.Context(), x[-300:], w, ws, x_scale=s[-300:], act="silu")
    assert torch.equal(y[-300:], want) and (y[0] == 0).all()


@pytest.mark.parametrize("M", [3, 50])
@pytest.mark.parametrize("dtype", DTYPES)
def test_codes_next_to_a_half(M, dtype):
    """Values whose quotient by the rounded scale falls on the other side of a half
    take the code of the true quotient: identity weights give the codes back."""
    K = 1024
    g = torch.Generator().manual_seed(8)
    top = (1 + torch.rand(M, 1, generator=g)).to(ref.TORCH[dtype]).double()
    k = torch.randint(-126, 126, (M, K), generator=g).double() + 0.5
    x = (top * k / 127).to(ref.TORCH[dtype])
    x[:, 0] = top[:, 0].to(x.dtype)
    x = x.cuda()
    w, one = torch.eye(K, dtype=torch.int8, device="cuda"), torch.ones(K, device="cuda")
    ctx = context(tokens.linear_i8_workspace_bytes(M, K, K, dtype, "f32"))
    y = tokens.linear_i8(ctx, x, w, one, out_dtype="f32", gate=torch.ones(1, K, device="cuda"), rows_per_gate=M)
    q, s = layer_ref.quantize(x)
    assert np.array_equal(y.cpu().numpy(), q.astype(np.float32) * s[:, None])


def test_no_rows():
    w, ws, _ = weights(24, 48)
    assert tokens.gated_linear_i8(c3c.Context(), torch.empty(0, 48, device="cuda"), w, ws).shape == (0, 12)
    assert tokens.linear_i8(c3c.Context(), torch.empty(0, 48, device="cuda"), w, ws, act="silu").shape == (0, 24)
