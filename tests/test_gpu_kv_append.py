"""Rotation and the paged 8-bit cache's append, against the plain form."""
import numpy as np
import pytest
import torch

from paper_2609_31938_amd import c3c, tokens
import token_ref as ref

pytestmark = pytest.mark.gpu


def make(new, old, Hkv, D, page, seed=1, extra_cols=1):
    """A cache with junk in it, and a batch whose pages are scattered."""
    rng = np.random.default_rng(seed)
    used = [-(-(n + o) // page) for n, o in zip(new, old)]
    pages, cols = sum(used) + 3, max(used) + extra_cols
    order = rng.permutation(pages)
    table = np.full((len(new), cols), -1, np.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    cache = tokens.KVCache.empty(pages, Hkv, page, D)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 120, t.shape, dtype=np.uint8)))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.from_numpy(2.0 ** rng.integers(-12, -4, t.shape)))
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    lens = np.array([n + o for n, o in zip(new, old)], np.int32)
    batch = tokens.Batch(torch.from_numpy(table).cuda(), torch.from_numpy(cu).cuda(), torch.from_numpy(lens).cuda(),
                         max_new=max(new), max_len=max(int(lens.max()), 0))
    return cache, batch, table, cu, lens


def angles(rows, half, seed=5):
    a = 6.28 * torch.rand(rows, half, generator=torch.Generator().manual_seed(seed))
    return a.cos().cuda(), a.sin().cuda()


def plain(pages, table, cu, lens, q, k, v, cos, sin, pos, pairs):
    """Appends to the host copy; returns the rotated queries (fp32 values)."""
    n32 = lambda t: ref.f64(t).astype(np.float32)  # noqa: E731
    q, k, v = n32(q), n32(k).copy(), n32(v)
    rq = q.copy()
    for b in range(len(lens)):
        start = int(lens[b]) - (cu[b + 1] - cu[b])
        for i, t in enumerate(range(cu[b], cu[b + 1])):
            if cos is not None:
                at = start + i if pos is None else int(pos[t])
                c, s = cos.cpu().numpy(), sin.cpu().numpy()
                rq[t], k[t] = ref.rotate(q[t], c, s, at, pairs), ref.rotate(k[t], c, s, at, pairs)
        pages.append(list(table[b]), start, k[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]])
    return rq, k


def same(cache, pages):
    got = ref.Pages(cache)
    t = ref.e4m3_table()
    assert np.array_equal(got.ks, pages.ks) and np.array_equal(got.vs, pages.vs)
    for a, b in ((got.k, pages.k), (got.v, pages.v)):
        assert np.array_equal(t[a], t[b], equal_nan=True), np.argwhere(t[a] != t[b])[:5]


def run(dtype, new, old, Hq, Hkv, D, page, rot, pairs, use_pos=False, seed=1, scale=1.0):
    cache, batch, table, cu, lens = make(new, old, Hkv, D, page, seed)
    T = int(cu[-1])
    dt = ref.TORCH[dtype]
    # one projection's output, and rows of different sizes so that scales grow
    qkv = ref.randn(seed, T, (Hq + 2 * Hkv) * D) * scale * torch.exp(ref.randn(seed + 1, T, 1))
    q, k, v = qkv.to(dt).view(T, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
    cos, sin = angles(int(lens.max()) + 1, rot // 2) if rot else (None, None)
    pos = torch.randperm(T).int().cuda() % (int(lens.max()) + 1) if use_pos else None
    pages = ref.Pages(cache)
    rq, rk = plain(pages, table, cu, lens, q, k, v, cos, sin, pos, pairs)
    got = tokens.kv_append(c3c.Context(), cache, batch, k, v, q=q, cos=cos, sin=sin, pos=pos, pairs=pairs)
    assert torch.equal(got.cpu(), torch.from_numpy(rq).to(dt))
    same(cache, pages)
    return cache, table, cu, lens, rk, v


CASES = [
    # new, earlier, Hq, Hkv, D, page, rot
    ([1], [0], 1, 1, 16, 16, 16), ([1, 1, 1], [15, 16, 37], 4, 2, 64, 16, 64), ([5, 0, 40], [3, 20, 64], 6, 2, 80, 32, 40),
    ([17], [31], 3, 3, 128, 64, 128), ([2, 100], [7, 1], 8, 1, 256, 48, 128), ([1] * 20, list(range(20)), 5, 5, 96, 32, 2),
    ([33, 16, 15], [0, 0, 16], 2, 1, 240, 16, 240), ([4], [60], 12, 12, 128, 64, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pairs", ["half", "next"])
@pytest.mark.parametrize("new,old,Hq,Hkv,D,page,rot", CASES)
def test_matches_the_plain_form(dtype, pairs, new, old, Hq, Hkv, D, page, rot):
    run(dtype, new, old, Hq, Hkv, D, page, rot, pairs)


def test_positions_given():
    run("bf16", [9, 3], [0, 30], 4, 2, 64, 16, 32, "half", use_pos=True)


@pytest.mark.parametrize("scale", [1e-30, 1e-38, 1e30])
def test_far_magnitudes(scale):
    run("f32", [20], [5], 2, 1, 32, 16, 16, "next", scale=scale)


def test_codes_are_within_half_a_step_of_64_bits():
    """Against the rotation in 64 bits: half an e4m3 step (2^-4 of the value,
    2^-10 of the scale below the normal range) and the fp32 rotation's error."""
    new, old, Hkv, D = [40], [0], 2, 64
    cache, batch, table, cu, lens = make(new, old, Hkv, D, 32)
    k, v = ref.randn(1, 40, Hkv, D), ref.randn(2, 40, Hkv, D)
    cos, sin = angles(40, 32)
    tokens.kv_append(c3c.Context(), cache, batch, k, v, cos=cos, sin=sin)
    c, s, x = ref.f64(cos)[:, None], ref.f64(sin)[:, None], ref.f64(k)
    a, b = x[..., :32], x[..., 32:]
    want = np.concatenate([a * c - b * s, b * c + a * s], -1)
    size = np.concatenate([np.abs(a * c) + np.abs(b * s)] * 2, -1) + np.concatenate([np.abs(b * c) + np.abs(a * s)] * 2, -1)
    p = ref.Pages(cache)
    gk, gv, ok = p.values(list(table[0]), 40)
    assert ok.all()
    blocks = np.array([[p.ks[table[0, t // 32], h, t % 32 // 16] for h in range(Hkv)] for t in range(40)])[..., None]
    ref.assert_within(gk, want, np.abs(want) / 16 + blocks * 2.0 ** -10 + 4 * ref.EPS32 * size, "k")
    assert np.all(blocks * 448 >= np.abs(gk))


def test_token_by_token_equals_at_once():
    """Appends of one token reach the scales of one append of all, and the
    same codes but for those that were rounded twice below the normal range."""
    n, Hkv, D = 50, 2, 64
    k = (ref.randn(1, n, Hkv, D) * torch.exp(ref.randn(3, n, 1, 1))).to(torch.bfloat16)
    v = ref.randn(2, n, Hkv, D).to(torch.bfloat16)
    ctx = c3c.Context()
    whole, batch, table, _, _ = make([n], [0], Hkv, D, 32)
    steps, _, _, _, _ = make([n], [0], Hkv, D, 32)
    tokens.kv_append(ctx, whole, batch, k, v)
    cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    one = tokens.Batch(batch.table, cu, lens, max_new=1, max_len=n)
    for t in range(n):
        lens.fill_(t + 1)
        tokens.kv_append(ctx, steps, one, k[t:t + 1], v[t:t + 1])
    a, b = ref.Pages(whole), ref.Pages(steps)
    used = table[0, :2]
    assert np.array_equal(a.ks[used[0]], b.ks[used[0]]) and np.array_equal(a.vs[used[0]], b.vs[used[0]])
    for x, y in zip(a.values(list(table[0]), n)[:2], b.values(list(table[0]), n)[:2]):
        top = np.abs(x).max()
        assert np.all(np.abs(x - y) <= top * 2.0 ** -17), np.abs(x - y).max()


def test_what_is_not_finite_stays_alone():
    cache, batch, table, cu, lens = make([10], [4], 1, 32, 16)
    k, v = ref.randn(1, 10, 1, 32), ref.randn(2, 10, 1, 32)
    k[2, 0, 5], k[3, 0, 6], v[4, 0, 7] = float("nan"), float("inf"), float("-inf")
    pages = ref.Pages(cache)
    plain(pages, table, cu, lens, k, k, v, None, None, None, "half")
    tokens.kv_append(c3c.Context(), cache, batch, k, v)
    same(cache, pages)
    gk, gv, _ = ref.Pages(cache).values(list(table[0]), 14)
    assert np.isnan(gk).sum() == 2 and np.isnan(gv).sum() == 1


def test_places_without_a_page_and_rows_out_of_range():
    """Evicted pages, a table that is too short, lengths that are too short,
    rows past the tensors and positions past the angle table."""
    cache, batch, table, cu, lens = make([40, 6, 5], [0, 0, 20], 2, 32, 16, extra_cols=0)
    table[0, 1] = -1            # evicted
    table[2, 1] = 1 << 30       # no such page
    lens[0] = 70                # its last tokens lie past the table's columns
    lens[1] = 3                 # fewer than its new tokens: places -3 .. 2
    T = int(cu[-1])
    cu[3] = T + 100             # cut off
    batch.table.copy_(torch.from_numpy(table))
    batch.lens.copy_(torch.from_numpy(lens))
    batch.cu.copy_(torch.from_numpy(cu))
    cu[3] = T
    q, k, v = ref.randn(1, T, 4, 32), ref.randn(2, T, 2, 32), ref.randn(3, T, 2, 32)
    cos, sin = angles(24, 8)
    pages = ref.Pages(cache)
    rq, _ = plain(pages, table, cu, lens, q, k, v, cos, sin, None, "half")
    got = tokens.kv_append(c3c.Context(), cache, batch, k, v, q=q, cos=cos, sin=sin)
    assert np.array_equal(ref.f64(got), rq, equal_nan=True) and got.isnan().any()
    same(cache, pages)


def test_in_place_queries_and_odd_strides():
    cache, batch, table, cu, lens = make([7], [0], 2, 48, 16)
    cos, sin = angles(7, 24)
    wide = ref.randn(1, 7, 4 * 48 + 4 * 48 + 1).to(torch.bfloat16)
    q, k, v = (wide[:, a:b].unflatten(1, (-1, 48)) for a, b in ((1, 193), (193, 289), (289, 385)))
    ctx = c3c.Context()
    want = tokens.kv_append(ctx, cache, batch, k, v, q=q, cos=cos, sin=sin)
    a = ref.Pages(cache)
    other = tokens.KVCache.empty(*[cache.k.shape[i] for i in (0, 1, 2, 3)])
    mine = q.contiguous()
    got = tokens.kv_append(ctx, other, batch, k.contiguous(), v.contiguous(), q=mine, cos=cos, sin=sin, q_out=mine)
    assert got is mine and torch.equal(got, want)
    b = ref.Pages(other)
    for x, y in zip(a.values(list(table[0]), 7), b.values(list(table[0]), 7)):
        assert np.array_equal(x, y)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 codes: the last page."""
    Hkv, page, D = 8, 64, 128
    P = (1 << 32) // (Hkv * page * D) + 2
    nb = page // 16
    cache = tokens.KVCache(*(torch.empty(s, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                             for s in ((P, Hkv, page, D), (P, Hkv, nb, D, 16))),
                           *(torch.ones(P, Hkv, nb, device="cuda") for _ in range(2)))
    small = tokens.KVCache.empty(1, Hkv, page, D)
    k, v = ref.randn(1, 20, Hkv, D), ref.randn(2, 20, Hkv, D)
    ctx = c3c.Context()
    i32 = dict(dtype=torch.int32, device="cuda")
    for c, last in ((cache, P - 1), (small, 0)):
        b = tokens.Batch(torch.tensor([[last]], **i32), torch.tensor([0, 20], **i32), torch.tensor([20], **i32),
                         max_new=20, max_len=20)
        tokens.kv_append(ctx, c, b, k, v)
    assert torch.equal(cache.k[-1, :, :20].view(torch.uint8), small.k[0, :, :20].view(torch.uint8))
    assert torch.equal(cache.v[-1, :, 0].view(torch.uint8), small.v[0, :, 0].view(torch.uint8))
    assert torch.equal(cache.k_scale[-1, :, :2], small.k_scale[0, :, :2])


def test_no_tokens():
    cache, batch, _, _, _ = make([1], [0], 1, 16, 16)
    empty = torch.empty(0, 1, 16, device="cuda")
    assert tokens.kv_append(c3c.Context(), cache, batch, empty, empty, q=empty).shape == (0, 1, 16)
