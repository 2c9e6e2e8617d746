"""What attention's arithmetic holds of a probability and of a value, against
64 bits and bounds that follow from it:

* a probability p (relative to the row's largest) enters the second product as
  2^7 p in 1 (bf16), 2 (f16) or 3 (f32) f16 terms: relative 2^-11, 2^-22 or
  2^-33, and absolute 2^-25 / 2^7 = 2^-32, half the spacing of f16 below its
  normal range;
* where a block's value scale is 2^d, d > 15, below the largest that the call's
  queries see, 2^(15 - d) goes to the probability: absolute 2^(d - 47).

fp32 around it: the score's sum of D products (as in token_ref), the
exponential and its argument, the sum and the reciprocal."""
import numpy as np
import pytest
import torch

from paper_2609_31938_amd import tokens
import token_ref as ref
from test_gpu_paged_attention import context, make

pytestmark = pytest.mark.gpu

TERMS = {"bf16": 2.0 ** -11, "f16": 2.0 ** -22, "f32": 2.0 ** -33}
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # of an output, relative (half a spacing)


def expected(dtype, cache, table, cu, lens, new, q, scale, causal, window=0):
    """Per sequence (rows, out, bound): the definition in 64 bits."""
    pages, D, nb = ref.Pages(cache), cache.dim, cache.page // 16
    for b, length in enumerate(lens):
        rows = slice(int(cu[b]), int(cu[b + 1]))
        k, v, ok = pages.values(list(table[b]), length)
        n, G = rows.stop - rows.start, q.shape[1] // cache.heads
        qs = ref.f64(q[rows])
        j, out, bound = np.arange(len(k)), np.zeros(qs.shape), np.zeros(qs.shape)
        e = np.zeros((len(k), cache.heads))  # exponents of the tokens' value scales
        for t in np.flatnonzero(ok):
            e[t] = np.log2(pages.vs[table[b, t // cache.page], :, t % cache.page // 16])
        first = max(0, length - n - window + 1) if window else 0
        seen = ok & (j >= first)
        for h in range(q.shape[1]):
            kv = h // G
            deep = np.maximum(e[seen, kv].max() - e[:, kv] - 15, 0) if seen.any() else e[:, kv]
            for i in range(n):
                p = length - n + i
                see = ok & ((j <= p) if causal else True) & ((j > p - window) if window else True)
                if not see.any():
                    continue
                kk, vv = k[see, kv], np.abs(v[see, kv])
                s = kk @ qs[i, h] * scale
                w = np.exp(s - s.max())
                total = w.sum()
                out[i, h] = w @ v[see, kv] / total
                size = (np.abs(kk) @ np.abs(qs[i, h])).max() * scale
                score = ref.EPS32 * ((D / 8 + 8) * size + 4 * (1.5 * np.abs(s).max() + 1))
                relative = TERMS[dtype] + 2 * score + (16 + len(s) / 16) * ref.EPS32
                floor = 2.0 ** -32 * 2.0 ** deep[see]
                bound[i, h] = (relative * (w @ vv) + floor @ vv) / total + ROUND[dtype] * np.abs(out[i, h]) + ref.TINY[dtype]
        yield rows, out, bound


def check(dtype, cache, batch, table, cu, lens, new, Hq, scale=None, causal=True, window=0, seed=2):
    D = cache.dim
    q = ref.randn(seed, int(cu[-1]), Hq, D).to(ref.TORCH[dtype])
    scale = np.float32(D ** -0.5 if scale is None else scale)
    out = tokens.paged_attention(context(cache, q, batch, causal, window), cache, batch, q, causal=causal, window=window,
                                 scale=float(scale))
    for rows, want, bound in expected(dtype, cache, table, cu, lens, new, q, float(scale), causal, window):
        ref.assert_within(out[rows], want, bound, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [1, 6, 130])
@pytest.mark.parametrize("page", [16, 64])
def test_probabilities_hold_their_bits(dtype, new, page):
    """Two tokens of nearly equal probability and opposite values: an output is
    their difference, which shows the rounding of each."""
    D = 64
    sequences = 1 if new > 1 else 40
    lens = [2] * sequences
    cache, batch, table, cu = make([new] * sequences, lens, 2, D, page)
    v = cache.v.view(torch.uint8)
    v[..., 1] = v[..., 0] ^ 0x80
    check(dtype, cache, batch, table, cu, lens, [new] * sequences, 16, scale=2e-3, causal=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [10, 15, 18, 24, 30, 36, 44])
@pytest.mark.parametrize("new,page", [(1, 16), (3, 64), (40, 16), (40, 64)])
def test_value_scales_far_apart(dtype, d, new, page):
    """Blocks whose value scale lies 2^d below another's, whose own values are
    zeros: the output is what is held of the small ones."""
    lens = [120]
    cache, batch, table, cu = make([new], lens, 2, 64, page)
    for blk in range(8):
        at = (table[0, blk * 16 // page], slice(None), blk * 16 % page // 16)
        big = blk in (1, 4)
        cache.v_scale[at] = 2.0 ** (3 if big else 3 - d)
        if big:
            cache.v.view(torch.uint8)[at] = 0
    check(dtype, cache, batch, table, cu, lens, [new], 4)
    check(dtype, cache, batch, table, cu, lens, [new], 4, causal=False, window=50)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,page", [(1, 16), (40, 64)])
def test_value_scales_that_rise_and_fall(dtype, new, page):
    """A scale of its own for every block, from 2^-100 to 2^60, in both orders."""
    lens = [16 * 20]
    for sign in (1, -1):
        cache, batch, table, cu = make([new], lens, 1, 64, page)
        for blk in range(20):
            cache.v_scale[table[0, blk * 16 // page], :, blk * 16 % page // 16] = 2.0 ** (-20 + sign * 8 * (blk - 10))
        check(dtype, cache, batch, table, cu, lens, [new], 2)
