"""Windows, evicted pages and NaN with pages of whole 64-token tiles, whose
kernels find their tiles another way than those of smaller pages, and mixtures
of everything at random."""
import numpy as np
import pytest
import torch

from paper_2609_31938_amd import tokens
import token_ref as ref
from test_gpu_attention_scales import JUNK, poison
from test_gpu_paged_attention import check, context, make

pytestmark = pytest.mark.gpu


def attend(dtype, cache, batch, table, cu, lens, Hq, causal, window, seed=2):
    q = ref.randn(seed, int(cu[-1]), Hq, cache.dim).to(ref.TORCH[dtype])
    lse = torch.empty(q.shape[:2], device="cuda")
    out = tokens.paged_attention(context(cache, q, batch, causal, window), cache, batch, q, causal=causal, window=window,
                                 lse=lse)
    check(dtype, cache, table, cu, lens, q, out, lse, cache.dim ** -0.5, causal, window)


@pytest.mark.parametrize("page", [64, 128, 192])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [1, 63, 64, 130, 5000])
@pytest.mark.parametrize("new,lens", [([1, 1], [400, 3]), ([90, 10], [700, 500]), ([200], [200])])
def test_windows(page, causal, window, new, lens):
    cache, batch, table, cu = make(new, lens, 2, 64, page)
    attend("bf16", cache, batch, table, cu, lens, 4, causal, window)


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("new", [1, 30, 300])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 150)])
@pytest.mark.parametrize("lost", [[0], [1, 2], [0, 1, 2, 3, 4, 5, 6], [6]])
def test_evicted_pages(page, new, causal, window, lost):
    lens = [800]
    cache, batch, table, cu = make([new], lens, 2, 96, page)
    lost = [c for c in lost if c < table.shape[1]]
    table[0, lost] = [-1 if c % 2 else 1 << 20 for c in lost]
    batch.table.copy_(torch.from_numpy(table))
    attend("f16", cache, batch, table, cu, lens, 4, causal, window)


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("D", [64, 80])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 40), (False, 40)])
@pytest.mark.parametrize("where", [[150, 299], [205, 170, 171], [3], [63, 64, 127, 128]])
def test_nan_codes(page, D, causal, window, where):
    """A NaN key makes the rows that see it NaN, a NaN value one channel."""
    lens = [300]
    cache, batch, table, cu = make([100], lens, 1, D, page)
    for i, p in enumerate(where):
        pg, at = table[0, p // page], p % page
        if i % 2 == 0:
            cache.v.view(torch.uint8)[pg, 0, at // 16, 5 + 3 * i, at % 16] = 0xFF
        else:
            cache.k.view(torch.uint8)[pg, 0, at, 9] = 0x7F
    attend("bf16", cache, batch, table, cu, lens, 2, causal, window)


@pytest.mark.parametrize("seed", range(60))
def test_mixtures(seed):
    """Ragged sequences, among them empty ones, of any form, with evicted pages
    and junk wherever no query looks."""
    rng = np.random.default_rng(seed)
    dtype = ["bf16", "f16", "f32"][seed % 3]
    Hkv, G = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 5, 8]))
    D, page = int(rng.choice([16, 64, 80, 128, 144, 192, 256])), int(rng.choice([16, 48, 64, 128]))
    B = int(rng.integers(1, 5))
    most = int(rng.choice([1, 3, 20, 90]))
    new = [int(rng.integers(0, most + 1)) for _ in range(B)]
    new[0] = max(new[0], 1)
    lens = [n + int(rng.integers(0, 400)) for n in new]
    causal, window = bool(rng.integers(0, 2)), int(rng.choice([0, 0, 1, 17, 100]))
    cache, batch, table, cu = make(new, lens, Hkv, D, page, seed)
    poison(cache, table, new, lens, window, list(JUNK.values())[seed % 5])
    for b in range(B):
        if rng.integers(0, 3) == 0:
            table[b, int(rng.integers(0, table.shape[1]))] = -1
    batch.table.copy_(torch.from_numpy(table))
    attend(dtype, cache, batch, table, cu, lens, G * Hkv, causal, window, seed)
