"""Attention over a cache whose unseen blocks hold anything, scales included:
blocks past a sequence's end that a page never had written, and blocks in
front of a window."""
import numpy as np
import pytest
import torch

from paper_2609_31938_amd import tokens
import token_ref as ref
from test_gpu_paged_attention import check, context, make

pytestmark = pytest.mark.gpu

JUNK = {"nan": 0x7FC00000, "inf": 0x7F800000, "huge": 0x71800000, "ones": 0xFFFFFFFF, "negative": 0xF1800000}


def poison(cache, table, new, lens, window, bits):
    """Fills the scales, and the codes with NaN, of every block of 16 tokens
    that no query of the call sees."""
    nb = cache.page // 16
    seen = np.zeros(cache.k_scale.shape, bool)
    for b, (n, length) in enumerate(zip(new, lens)):
        first = max(0, length - n - window + 1) if window else 0
        for p in range(first, length):
            seen[table[b, p // cache.page], :, p % cache.page // 16] = True
    free = torch.from_numpy(~seen).cuda()
    assert free.any()
    for t in (cache.k_scale, cache.v_scale):
        t.view(torch.int32)[free] = bits - (1 << 32) if bits >> 31 else bits
    k, v = cache.k.view(torch.uint8), cache.v.view(torch.uint8)
    k.view(k.shape[0], k.shape[1], nb, 16, -1)[free] = 0x7F
    v[free] = 0xFF


def run(dtype, new, lens, Hq, Hkv, D, page, causal, window, bits, seed=1):
    cache, batch, table, cu = make(new, lens, Hkv, D, page, seed)
    poison(cache, table, new, lens, window, bits)
    q = ref.randn(seed, int(cu[-1]), Hq, D).to(ref.TORCH[dtype])
    lse = torch.empty(q.shape[:2], device="cuda")
    out = tokens.paged_attention(context(cache, q, batch, causal, window), cache, batch, q, causal=causal, window=window,
                                 lse=lse)
    check(dtype, cache, table, cu, lens, q, out, lse, D ** -0.5, causal, window)


@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("page", [16, 48, 64, 128])
@pytest.mark.parametrize("new,lens", [([1, 1], [100, 17]), ([40, 3], [100, 70]), ([130], [330])])
def test_blocks_past_the_end(junk, page, new, lens):
    run("bf16", new, lens, 4, 2, 64, page, True, 0, JUNK[junk])


@pytest.mark.parametrize("junk", JUNK)
@pytest.mark.parametrize("page", [16, 48, 64, 128])
@pytest.mark.parametrize("new,lens,window", [([1, 1], [300, 200], 50), ([20, 40], [300, 200], 33), ([130], [400], 17)])
@pytest.mark.parametrize("causal", [True, False])
def test_blocks_before_a_window(junk, page, new, lens, window, causal):
    run("bf16", new, lens, 4, 2, 64, page, causal, window, JUNK[junk])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", [80, 96, 128, 192, 256])
@pytest.mark.parametrize("page", [48, 64])
@pytest.mark.parametrize("new", [2, 50])
def test_every_form_of_the_kernels(dtype, D, page, new):
    """Head sizes with and without padding, each type, few and many queries."""
    run(dtype, [new], [150], 4, 2, D, page, True, 0, JUNK["nan"])
    run(dtype, [new], [230], 4, 2, D, page, True, 40, JUNK["inf"])
