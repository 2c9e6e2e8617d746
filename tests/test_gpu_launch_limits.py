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


@pytest.mark.parametrize("x_dtype", ["i8", "bf16"])
def test_linear_of_few_tokens(x_dtype):
    """Output channels by 16 a workgroup of 256 threads: more than 2^28."""
    N, K, ctx = (1 << 28) + 33, 8, c3c.Context()
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda")
    ws = torch.rand(N, device="cuda")
    x = torch.randint(-127, 128, (1, K), device="cuda")
    x, xs = (x.to(torch.int8), torch.ones(1, device="cuda")) if x_dtype == "i8" else (x.bfloat16(), None)
    ctx.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
    y = tokens.linear_i8(ctx, x, w, ws, x_scale=xs)
    for s in (slice(0, 301), slice((1 << 27) - 300, (1 << 27) + 300), slice((1 << 28) - 300, N)):
        assert torch.equal(y[:, s], tokens.linear_i8(ctx, x, w[s], ws[s], x_scale=xs)), s


def test_linear_of_many_tokens():
    """256 tokens a workgroup of 512 threads: 2^31 - 1."""
    M, ctx = (1 << 31) - 1, c3c.Context()
    x = torch.randint(-127, 128, (M, 1), dtype=torch.int8, device="cuda")
    s = torch.full((M,), 0.25, device="cuda")
    w, ws = torch.full((1, 1), 3, dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda")
    y = tokens.linear_i8(ctx, x, w, ws, x_scale=s)
    for at in (slice(0, 999), slice((1 << 30) - 999, (1 << 30) + 999), slice(M - 999, M)):
        assert torch.equal(y[at], (x[at].float() * 0.75).bfloat16()), at


def cache_and_batch(new, old, max_new, Hkv=2, D=16, page=16):
    """A cache of junk in order of pages, and a batch with this bound."""
    lens = [n + o for n, o in zip(new, old)]
    used = [-(-n // page) for n in lens]
    table = torch.full((len(new), max(used)), -1, dtype=torch.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = torch.arange(at, at + u)
        at += u
    cache = tokens.KVCache.empty(at, Hkv, page, D)
    for i, t in enumerate((cache.k, cache.v)):
        t.view(torch.uint8).copy_(torch.randint(0, 120, t.shape, generator=torch.Generator().manual_seed(i)).to(torch.uint8))
    cu = torch.tensor([0] + new).cumsum(0).int()
    return cache, tokens.Batch(table.cuda(), cu.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), max_new=max_new,
                               max_len=max(lens))


@pytest.mark.parametrize("bound", [(1 << 28) - 20, 1 << 28, (1 << 31) - 1])
def test_append_with_a_loose_bound(bound):
    """max_new only says that no sequence has more new tokens."""
    new, old = [40, 1, 7], [3, 20, 0]
    k, v, q = (ref.randn(s, 48, h, 16).bfloat16() for s, h in ((1, 2), (2, 2), (3, 4)))
    results = []
    for m in (40, bound):
        cache, batch = cache_and_batch(new, old, m)
        got = tokens.kv_append(c3c.Context(), cache, batch, k, v, q=q)
        results.append([got] + [t.view(torch.uint8) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("bound", [1 << 28, (1 << 31) - 1])
@pytest.mark.parametrize("window", [0, 20])
def test_attention_with_a_loose_bound(bound, window):
    new, old = [40, 1, 7], [3, 200, 0]
    q, results = ref.randn(1, 48, 4, 16).bfloat16(), []
    for m in (40, bound):
        cache, batch = cache_and_batch(new, old, m)
        results.append(tokens.paged_attention(c3c.Context(), cache, batch, q, window=window))
        assert tokens.paged_attention_workspace_bytes(cache, q, batch, window=window) < 1 << 24
    assert torch.equal(*results)


def test_attention_of_many_workgroups():
    """5000 sequences, one of 31000 new tokens: 5000 x 16 heads x 243 tiles of
    128 columns, 2^24 and more workgroups of 256 threads."""
    long, B, H, D = 31000, 5000, 16, 16
    new, old = [long] + [1] * (B - 1), [0] + [5 + b % 90 for b in range(B - 1)]
    cache, batch = cache_and_batch(new, old, long, Hkv=H)
    q = ref.randn(1, long + B - 1, H, D).bfloat16()
    ctx = c3c.Context()
    got = tokens.paged_attention(ctx, cache, batch, q)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    one = tokens.Batch(batch.table[:1].contiguous(), batch.cu[:2].contiguous(), batch.lens[:1].contiguous(),
                       max_new=long, max_len=long)
    assert torch.equal(got[:long], tokens.paged_attention(ctx, cache, one, q[:long].contiguous()))
    for b in (1, 900, 2000, B - 200):  # a hundred single tokens, as chunk calls take them
        cu = torch.cat([zero, torch.arange(1, 101, dtype=torch.int32, device="cuda")])
        part = tokens.Batch(batch.table[b:b + 100].contiguous(), cu, batch.lens[b:b + 100].contiguous(), max_new=100, max_len=100)
        rows = slice(long + b - 1, long + b + 99)
        assert torch.equal(got[rows], tokens.paged_attention(ctx, cache, part, q[rows].contiguous())), b
