"""Host-side checks of the token operators that need no GPU: exports,
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
NAMES = ["c3c_quantize_rows", "c3c_linear_i8_workspace_bytes", "c3c_linear_i8", "c3c_norm_gate", "c3c_kv_append",
         "c3c_paged_attention_workspace_bytes", "c3c_paged_attention"]


def test_every_declared_symbol_is_exported_and_bound():
    text = open(os.path.join(os.path.dirname(c3c.HEADER), "c3c_tokens.h")).read()
    assert sorted(re.findall(r"^int\s+(c3c_\w+)\s*\(", text, re.M)) == sorted(NAMES)
    for n in NAMES:
        assert getattr(lib, n).argtypes, n


def test_structures_match_the_header():
    assert C.sizeof(tokens.LinearDesc) == 4 * 8 + 2 * 4
    assert C.sizeof(tokens.NormDesc) == 3 * 8 + 4 * 4
    assert C.sizeof(tokens._CacheDesc) == 8 * 8
    assert C.sizeof(tokens._BatchDesc) == 8 * 8
    assert C.sizeof(tokens._RopeDesc) == 5 * 8 + 2 * 4


def test_linear_workspace():
    """Nothing for 8-bit rows of an unsplit call; padded rows and scales for float ones."""
    assert tokens.linear_i8_workspace_bytes(1, 4096, 4096, "i8") == 0
    for M, K in ((1, 100), (7, 4096), (64, 33)):
        rows = M * (-(-K // 16) * 16)
        need = -(-rows // 256) * 256 + -(-M * 4 // 256) * 256
        assert tokens.linear_i8_workspace_bytes(M, 4096, K, "f16") == need
    assert tokens.linear_i8_workspace_bytes(0, 64, 64) == 0
    for M, N, K in ((-1, 4, 4), (1, 0, 4), (1, 4, 0), (1, 4, 131072), (1 << 31, 4, 4)):
        with pytest.raises(c3c.C3CError):
            tokens.linear_i8_workspace_bytes(M, N, K)


P = 1 << 20  # fake addresses, far apart


def at(i):
    return P * (i + 1)


def refused(status, ctx, word):
    assert status == c3c.E_INVAL
    assert word in ctx.last_error, ctx.last_error


@no_gpu
def test_linear_refusals():
    ctx = c3c.Context()

    def call(M=4, N=8, K=16, ld=16, xd=1, yd=1, x=at(0), xs=None, w=at(1), ws=at(2), b=at(3), y=at(4)):
        return lib.c3c_linear_i8(ctx._h, C.byref(tokens.LinearDesc(M, N, K, ld, xd, yd)), x, xs, w, ws, b, y, None)

    for kw, word in ((dict(M=-1), "M must"), (dict(N=0), "M must"), (dict(K=0), "M must"), (dict(K=131072, ld=131072), "overflow"),
                     (dict(ld=15), "ld_x"), (dict(xd=9), "x_dtype"), (dict(yd=16), "y_dtype"), (dict(xd=16), "x_scale"),
                     (dict(xs=at(5)), "x_scale"), (dict(x=None), "NULL"), (dict(w=None), "NULL"), (dict(ws=None), "NULL"),
                     (dict(y=None), "NULL"), (dict(y=at(0)), "overlaps"), (dict(y=at(1) + 8), "overlaps"),
                     (dict(x=at(0) + 1), "aligned"), (dict(y=at(4) + 1), "aligned"), (dict(), "workspace"),
                     (dict(M=1 << 31), "2^31"), (dict(M=(1 << 31) - 1, ld=1 << 30), "2^40")):
        refused(call(**kw), ctx, word)
    assert lib.c3c_linear_i8(None, None, *[None] * 7) == c3c.E_INVAL
    refused(lib.c3c_linear_i8(ctx._h, None, *[None] * 7), ctx, "NULL")
    # a workspace that overlaps a tensor
    assert lib.c3c_ctx_set_workspace(ctx._h, at(1), 4096) == c3c.OK
    refused(call(), ctx, "workspace overlaps")


@no_gpu
def test_quantize_refusals():
    ctx = c3c.Context()

    def call(T=4, n=8, ld=8, dt=1, x=at(0), q=at(1), s=at(2)):
        return lib.c3c_quantize_rows(ctx._h, T, n, ld, dt, x, q, s, None)

    for kw, word in ((dict(T=-1), "T must"), (dict(n=0), "T must"), (dict(ld=7), "T must"), (dict(dt=16), "dtype"),
                     (dict(x=None), "NULL"), (dict(q=None), "NULL"), (dict(s=None), "NULL"), (dict(q=at(0)), "overlaps"),
                     (dict(s=at(1)), "overlap"), (dict(s=at(2) + 2), "aligned")):
        refused(call(**kw), ctx, word)


@no_gpu
def test_norm_refusals():
    ctx = c3c.Context()

    def call(T=4, n=8, rows=1, alpha=1.0, eps=1e-6, dt=1, h=at(0), y=at(1), gate=at(2), post=at(3), pre=at(4), ho=at(5),
             u=at(6), uq=None, us=None):
        return lib.c3c_norm_gate(ctx._h, C.byref(tokens.NormDesc(T, n, rows, alpha, eps, dt, 0)), h, y, gate, post, pre,
                                 ho, u, uq, us, None)

    for kw, word in ((dict(T=-1), "T must"), (dict(n=0), "T must"), (dict(rows=0), "rows_per_gate"), (dict(dt=0), "dtype"),
                     (dict(alpha=float("inf")), "finite"), (dict(eps=-1.0), "finite"), (dict(eps=float("nan")), "finite"),
                     (dict(y=None), "post and gate"), (dict(u=None), "goes with pre"), (dict(pre=None), "goes with pre"),
                     (dict(uq=at(7)), "together"), (dict(us=at(7)), "together"), (dict(h=None), "h is NULL"),
                     (dict(pre=None, u=None, ho=None), "no output"), (dict(ho=at(1)), "overlaps an input"),
                     (dict(u=at(0)), "overlaps an input"), (dict(ho=at(0) + 2), "overlaps an input"),
                     (dict(u=at(5)), "two outputs"), (dict(gate=at(2) + 1), "aligned")):
        refused(call(**kw), ctx, word)


def cache(pages=4, heads=2, page=32, dim=64, k=at(10), v=at(11), ks=at(12), vs=at(13)):
    return tokens._CacheDesc(k, v, ks, vs, pages, heads, page, dim)


def batch(B=2, cols=3, T=4, max_new=2, max_len=50, table=at(14), cu=at(15), lens=at(16)):
    return tokens._BatchDesc(table, cu, lens, B, cols, T, max_new, max_len)


SHARED = [(dict(c=cache(page=24)), "page"), (dict(c=cache(page=8)), "page"), (dict(c=cache(dim=72)), "dim"),
          (dict(c=cache(dim=272)), "dim"), (dict(c=cache(heads=0)), "heads"), (dict(c=cache(pages=-1)), "pages"),
          (dict(c=cache(k=at(10) + 8)), "aligned"), (dict(c=cache(v=None)), "NULL"), (dict(c=cache(ks=None)), "NULL"),
          (dict(c=cache(pages=1 << 30, page=1 << 20)), "2^40"), (dict(b=batch(B=-1)), "B, T"), (dict(b=batch(max_new=0)), "max_new"),
          (dict(b=batch(B=0)), "no sequence"), (dict(b=batch(max_len=-1)), "max_len"), (dict(b=batch(table=None)), "NULL"),
          (dict(b=batch(cu=None)), "NULL"), (dict(b=batch(lens=None)), "NULL"), (dict(dt=16), "dtype")]


@no_gpu
def test_append_refusals():
    ctx = c3c.Context()

    def call(c=cache(), b=batch(), r=None, dt=1, qh=4, q=at(0), ldq=256, k=at(1), ldk=128, v=at(2), ldv=128, qo=at(3)):
        return lib.c3c_kv_append(ctx._h, C.byref(c), C.byref(b), None if r is None else C.byref(r), dt, qh, q, ldq, k, ldk,
                                 v, ldv, qo, None)

    def rope(rot=64, rows=50, pairs=0, cos=at(5), sin=at(6), pos=None):
        return tokens._RopeDesc(cos, sin, pos, rows, rot, pairs, 0)

    for kw, word in SHARED + [
            (dict(qh=0), "q_heads"), (dict(ldq=255), "stride"), (dict(ldk=127), "stride"), (dict(ldv=127), "stride"),
            (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(qo=None), "together"), (dict(q=None), "together"),
            (dict(qo=at(0), ldq=300), "in place"), (dict(qo=at(1)), "overlaps"), (dict(k=at(10)), "overlaps"),
            (dict(c=cache(v=at(10))), "two outputs"), (dict(k=at(1) + 1), "aligned"), (dict(r=rope(rot=3)), "rot"),
            (dict(r=rope(rot=66)), "rot"), (dict(r=rope(pairs=2)), "pairs"), (dict(r=rope(rows=0)), "empty"),
            (dict(r=rope(cos=None)), "NULL"), (dict(r=rope(sin=None)), "NULL")]:
        refused(call(**kw), ctx, word)
    assert lib.c3c_kv_append(ctx._h, None, None, None, 1, 1, *[None, 0] * 3, None, None) == c3c.E_INVAL


@no_gpu
def test_attention_refusals():
    ctx = c3c.Context()

    def call(c=cache(), b=batch(), dt=1, qh=4, q=at(0), ldq=256, scale=0.1, causal=1, window=0, out=at(3), lse=at(4)):
        return lib.c3c_paged_attention(ctx._h, C.byref(c), C.byref(b), dt, qh, q, ldq, scale, causal, window, out, lse, None)

    for kw, word in SHARED + [
            (dict(qh=3), "divide"), (dict(qh=0), "q_heads"), (dict(ldq=255), "ld_q"), (dict(q=None), "NULL"),
            (dict(out=None), "NULL"), (dict(scale=0.0), "scale"), (dict(scale=float("inf")), "scale"),
            (dict(scale=float("nan")), "scale"), (dict(causal=2), "causal"), (dict(window=-1), "window"),
            (dict(out=at(0)), "overlaps"), (dict(lse=at(3)), "two outputs"), (dict(lse=at(4) + 2), "aligned")]:
        refused(call(**kw), ctx, word)
    assert lib.c3c_ctx_set_workspace(ctx._h, at(10), 4096) == c3c.OK
    refused(call(), ctx, "workspace overlaps")


def test_attention_workspace():
    n = C.c_size_t()

    def query(c, b, qh=8, causal=1, window=0):
        return lib.c3c_paged_attention_workspace_bytes(C.byref(c), C.byref(b), 1, qh, causal, window, C.byref(n))

    big = cache(pages=100, heads=2, page=32, dim=64)
    # one token of one long sequence splits, and its partial rows are whole
    assert query(big, batch(B=1, cols=200, T=1, max_new=1, max_len=6400)) == c3c.OK
    assert n.value > 0 and n.value % (8 * (64 + 2) * 4) == 0
    # a short one does not, nor do more queries than the device has room for
    assert query(big, batch(B=1, cols=200, T=1, max_new=1, max_len=64)) == c3c.OK and n.value == 0
    assert query(big, batch(B=64, cols=200, T=1 << 17, max_new=2048, max_len=6400)) == c3c.OK and n.value == 0
    assert query(big, batch(), qh=7) == c3c.E_INVAL
    assert query(big, batch(), window=-1) == c3c.E_INVAL


def test_binding_checks():
    with pytest.raises(ValueError, match="multiple"):
        tokens.KVCache.empty(2, 1, 24, 64, device="cpu")
    x = torch.zeros(4, 16)
    with pytest.raises(ValueError, match="contiguous rows"):
        tokens.quantize_rows(c3c.Context(), x.t())
    with pytest.raises(ValueError, match="dtype"):
        tokens.norm_gate(c3c.Context(), x.double())
    with pytest.raises(ValueError, match="device tensor"):
        tokens.norm_gate(c3c.Context(), x, pre=torch.ones(16))


@no_gpu
def test_grid_limits_are_refused():
    ctx = c3c.Context()
    for c, b, qh in ((cache(), batch(B=65536, cols=1, T=65536, max_new=1), 4), (cache(heads=65536, dim=16), batch(), 65536),
                     (cache(heads=2, dim=16), batch(), 65536)):
        st = lib.c3c_paged_attention(ctx._h, C.byref(c), C.byref(b), 1, qh, at(0), 1 << 22, 0.1, 1, 0, at(3), None, None)
        refused(st, ctx, "65535")


def test_angles_come_in_pairs():
    c = tokens.KVCache.__new__(tokens.KVCache)
    c.heads, c.dim = 1, 16
    with pytest.raises(ValueError, match="go together"):
        x = torch.zeros(1, 1, 16)
        tokens.kv_append(c3c.Context(), c, None, x, x, cos=torch.zeros(1, 8))
