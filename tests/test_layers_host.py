"""Host-side checks of a recurrent layer's operators that need no GPU: exports,
structure layouts, workspace queries, and refusals, which are all decided
before any device access (fake device addresses; skipped where a GPU is
present so that a validation bug could never become a launch)."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2609_31938_amd import c3c, tokens

no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer argument tests run on CPU-only hosts")
lib = c3c.lib
NAMES = ["c3c_linear_attention_workspace_bytes", "c3c_linear_attention", "c3c_linear_i8_epilogue",
         "c3c_gated_linear_i8_workspace_bytes", "c3c_gated_linear_i8"]
P = 1 << 26  # fake addresses, far apart


def at(i):
    return P * (i + 1)


def refused(status, ctx, word):
    assert status == c3c.E_INVAL
    assert word in ctx.last_error, ctx.last_error


def test_every_declared_symbol_is_exported_and_bound():
    text = open(os.path.join(os.path.dirname(c3c.HEADER), "c3c_layers.h")).read()
    assert sorted(re.findall(r"^int\s+(c3c_\w+)\s*\(", text, re.M)) == sorted(NAMES)
    for n in NAMES:
        assert getattr(lib, n).argtypes, n
    acts = dict(re.findall(r"C3C_ACT_(\w+) = (\d+)", text))
    assert {k.lower(): int(v) for k, v in acts.items()} == tokens.ACTS


def test_structures_match_the_header():
    assert C.sizeof(tokens._StateDesc) == 5 * 8
    assert C.sizeof(tokens._Epilogue) == 3 * 8 + 2 * 4


# ---------------------------------------------------------------- linear attention

def states(slots=4, heads=4, dim_k=64, dim_v=32, state=at(10)):
    return tokens._StateDesc(state, slots, heads, dim_k, dim_v)


def batch(B=2, T=40, max_new=30, max_len=50, cu=at(11), lens=at(12)):
    return tokens._BatchDesc(None, cu, lens, B, 0, T, max_new, max_len)


@no_gpu
def test_attention_refusals():
    ctx = c3c.Context()

    def call(s=states(), b=batch(), slot=at(13), dt=1, qkh=2, q=at(0), ldq=128, k=at(1), ldk=128, v=at(2), ldv=128, g=at(3),
             ldg=4, scale=0.1, out=at(4)):
        return lib.c3c_linear_attention(ctx._h, C.byref(s), C.byref(b), slot, dt, qkh, q, ldq, k, ldk, v, ldv, g, ldg, scale,
                                        out, None)

    for kw, word in ((dict(s=states(dim_k=72)), "dim_k"), (dict(s=states(dim_k=272)), "dim_k"), (dict(s=states(dim_v=8)), "dim_v"),
                     (dict(s=states(dim_v=0)), "dim_v"), (dict(s=states(heads=0)), "heads"), (dict(s=states(slots=-1)), "slots"),
                     (dict(s=states(heads=65536, dim_k=16, dim_v=16)), "65535"), (dict(b=batch(B=65536)), "65535"),
                     (dict(s=states(slots=(1 << 31) - 1)), "2^40"), (dict(s=states(state=None)), "NULL"),
                     (dict(s=states(state=at(10) + 2)), "aligned"), (dict(b=batch(B=-1)), "B and T"), (dict(b=batch(T=-1)), "B and T"),
                     (dict(b=batch(T=1 << 31)), "B and T"), (dict(b=batch(max_new=0)), "max_new"), (dict(b=batch(max_new=-1)), "max_new"),
                     (dict(b=batch(B=0)), "no sequence"), (dict(b=batch(cu=None)), "NULL"), (dict(b=batch(lens=None)), "NULL"),
                     (dict(dt=16), "dtype"), (dict(qkh=0), "divide"), (dict(qkh=3), "divide"), (dict(qkh=8), "divide"),
                     (dict(ldq=127), "stride"), (dict(ldk=127), "stride"), (dict(ldv=127), "stride"), (dict(ldv=1 << 23), "stride"),
                     (dict(ldg=3), "ld_decay"), (dict(ldg=-1), "ld_decay"), (dict(scale=float("inf")), "scale"),
                     (dict(scale=float("nan")), "scale"), (dict(q=None), "NULL"), (dict(k=None), "NULL"), (dict(v=None), "NULL"),
                     (dict(g=None), "NULL"), (dict(out=None), "NULL"), (dict(q=at(0) + 1), "aligned"), (dict(g=at(3) + 2), "aligned"),
                     (dict(out=at(0)), "overlaps"), (dict(out=at(2)), "overlaps"), (dict(out=at(10)), "overlap"),
                     (dict(k=at(10)), "overlaps"), (dict(slot=at(10) + 4), "overlaps")):
        refused(call(**kw), ctx, word)
    assert lib.c3c_linear_attention(None, *[None] * 3, 1, 1, *[None, 0] * 4, 1.0, None, None) == c3c.E_INVAL
    refused(lib.c3c_linear_attention(ctx._h, None, None, None, 1, 1, *[None, 0] * 4, 1.0, None, None), ctx, "NULL")
    assert lib.c3c_ctx_set_workspace(ctx._h, at(1), 4096) == c3c.OK
    refused(call(), ctx, "workspace overlaps")


def test_attention_workspace():
    n = C.c_size_t()

    def query(s, b, qkh=1, dt=1):
        return lib.c3c_linear_attention_workspace_bytes(C.byref(s), C.byref(b), dt, qkh, C.byref(n))

    # few heads of a long sequence are split: a state, and a factor, for each part
    assert query(states(), batch(B=1, T=5000, max_new=5000)) == c3c.OK
    assert n.value > 0 and n.value % (4 * (64 * 32 + 1) * 4) == 0
    # single and drafted tokens are not, nor heads and sequences that fill the device
    for b in (batch(T=2, max_new=1), batch(T=32, max_new=16)):
        assert query(states(), b) == c3c.OK and n.value == 0
    assert query(states(heads=64), batch(B=64, T=64000, max_new=1000)) == c3c.OK and n.value == 0
    # a bound on the new tokens that says nothing asks for no more than all tokens do
    assert query(states(), batch(B=2, T=5000, max_new=(1 << 31) - 1)) == c3c.OK
    loose = n.value
    assert query(states(), batch(B=2, T=5000, max_new=5000)) == c3c.OK and n.value == loose
    assert query(states(), batch(), qkh=3) == c3c.E_INVAL
    assert query(states(dim_k=20), batch()) == c3c.E_INVAL
    assert query(states(), batch(), dt=7) == c3c.E_INVAL


# ---------------------------------------------------------------- products

def desc(M=4, N=8, K=16, ld=16, xd=1, yd=1):
    return tokens.LinearDesc(M, N, K, ld, xd, yd)


@no_gpu
def test_epilogue_refusals():
    ctx = c3c.Context()

    def call(d=desc(), act=1, alpha=1.0, rows=1, gate=at(6), res=at(7), x=at(0), xs=None, w=at(1), ws=at(2), b=at(3), y=at(4)):
        return lib.c3c_linear_i8_epilogue(ctx._h, C.byref(d), C.byref(tokens._Epilogue(gate, res, rows, alpha, act)), x, xs, w,
                                          ws, b, y, None)

    for kw, word in ((dict(d=desc(M=-1)), "M must"), (dict(d=desc(K=131072, ld=131072)), "overflow"), (dict(d=desc(xd=9)), "x_dtype"),
                     (dict(act=4), "act"), (dict(act=-1), "act"), (dict(alpha=float("nan")), "alpha"), (dict(alpha=float("inf")), "alpha"),
                     (dict(rows=0), "rows_per_gate"), (dict(rows=-3), "rows_per_gate"), (dict(x=None), "NULL"), (dict(y=None), "NULL"),
                     (dict(gate=at(6) + 1), "aligned"), (dict(res=at(7) + 1), "aligned"), (dict(res=at(4) + 2), "overlaps"),
                     (dict(gate=at(4)), "overlaps"), (dict(y=at(0)), "overlaps"), (dict(), "workspace"),
                     (dict(res=at(4)), "workspace is smaller")):
        refused(call(**kw), ctx, word)
    assert lib.c3c_linear_i8_epilogue(None, *[None] * 9) == c3c.E_INVAL
    refused(lib.c3c_linear_i8_epilogue(ctx._h, None, *[None] * 8), ctx, "NULL")
    d = desc()
    refused(lib.c3c_linear_i8_epilogue(ctx._h, C.byref(d), *[None] * 8), ctx, "epilogue is NULL")
    assert lib.c3c_ctx_set_workspace(ctx._h, at(7), 4096) == c3c.OK
    refused(call(), ctx, "workspace overlaps")


@no_gpu
def test_gated_refusals():
    ctx = c3c.Context()

    def call(d=desc(), act=1, x=at(0), xs=None, w=at(1), ws=at(2), b=at(3), y=at(4)):
        return lib.c3c_gated_linear_i8(ctx._h, C.byref(d), act, x, xs, w, ws, b, y, None)

    for kw, word in ((dict(d=desc(N=0)), "M must"), (dict(d=desc(N=1 << 30)), "2 N"), (dict(d=desc(N=1 << 29, K=4096, ld=4096)), "2^40"),
                     (dict(d=desc(ld=15)), "ld_x"), (dict(act=9), "act"), (dict(d=desc(xd=16)), "x_scale"), (dict(w=None), "NULL"),
                     (dict(y=at(1) + 130), "overlaps"), (dict(y=at(1) + 255 - 1), "overlaps"), (dict(), "workspace")):
        refused(call(**kw), ctx, word)
    assert lib.c3c_gated_linear_i8(None, None, 1, *[None] * 7) == c3c.E_INVAL
    refused(lib.c3c_gated_linear_i8(ctx._h, None, 1, *[None] * 7), ctx, "NULL")


def test_gated_workspace():
    """That of a product with all 2 N rows of weights."""
    for M, N, K, xd in ((1, 4096, 4096, "i8"), (7, 100, 100, "bf16"), (100, 300, 9000, "f16"), (333, 777, 1111, "f32"), (0, 5, 5, "f32")):
        assert tokens.gated_linear_i8_workspace_bytes(M, N, K, xd) == tokens.linear_i8_workspace_bytes(M, 2 * N, K, xd)
    for M, N, K in ((-1, 4, 4), (1, 0, 4), (1, 1 << 30, 4)):
        with pytest.raises(c3c.C3CError):
            tokens.gated_linear_i8_workspace_bytes(M, N, K)


def test_binding_checks(monkeypatch):
    monkeypatch.setattr(tokens, "_device", lambda: -1)  # a CPU tensor's device
    ctx, x = c3c.Context(), torch.zeros(4, 16)
    w, ws = torch.zeros(6, 16, dtype=torch.int8), torch.zeros(6)
    with pytest.raises(ValueError, match="act is"):
        tokens.gated_linear_i8(ctx, x, w, ws, act="tanh")
    with pytest.raises(ValueError, match="two halves"):
        tokens.gated_linear_i8(ctx, x, w[:5], ws)
    with pytest.raises(ValueError, match="device tensor"):
        tokens.linear_i8(ctx, x, w, ws, act="silu")
    with pytest.raises(ValueError, match="slots"):
        tokens.StateCache(torch.zeros(2, 3, 16))
    with pytest.raises(ValueError, match="dtype"):
        tokens.StateCache(torch.zeros(2, 3, 16, 16, dtype=torch.bfloat16))
    s = tokens.StateCache.__new__(tokens.StateCache)
    s.heads, s.dim_k, s.dim_v = 2, 16, 16
    with pytest.raises(ValueError, match="k has shape"):
        tokens.linear_attention(ctx, s, None, *(Fake(torch.zeros(3, h, 16)) for h in (2, 1, 2)), torch.zeros(2))
    with pytest.raises(ValueError, match="heads of a token"):
        tokens.linear_attention(ctx, s, None, Fake(torch.zeros(3, 16, 2).transpose(1, 2)), *[Fake(torch.zeros(3, 2, 16))] * 2, torch.zeros(2))
    for g in (torch.zeros(3), torch.zeros(4, 2), torch.zeros(3, 2, dtype=torch.float64)):
        with pytest.raises(ValueError, match="log_decay|device"):
            tokens.linear_attention(ctx, s, None, *[Fake(torch.zeros(3, 2, 16))] * 3, g)


class Fake:
    """A CPU tensor that says it is on the device (never used as an address)."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return True if name == "is_cuda" else getattr(self.t, name)


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(tokens, "_device", lambda: 1)
    x = Fake(torch.zeros(4, 16))
    w, ws = torch.zeros(6, 16, dtype=torch.int8), torch.zeros(6)
    with pytest.raises(ValueError, match="current one is 1"):
        tokens.gated_linear_i8(c3c.Context(), x, w, ws)
    with pytest.raises(ValueError, match="current one is 1"):
        tokens.linear_attention(c3c.Context(), None, None, x, x, x, None)
