"""A recurrent layer's operators on two streams at once, each with a context, a
workspace and states of its own, and other inputs: kernels that last longer than
the host's work for them, several in turn, which overlap in time (checked), give
the bits that they give one stream after the other."""
import pytest
import torch

from paper_2609_31938_amd import c3c, tokens

pytestmark = pytest.mark.gpu

ROUNDS = 6


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


class Attention:
    """A prompt in ROUNDS pieces; the state goes from one to the next."""

    def __init__(self, seed, T=12000, H=8, D=128):
        self.q, self.k, self.v = (rand(seed + i, T, H, D).bfloat16() for i in range(3))
        self.g = -0.02 * rand(seed + 3, T, H).abs()
        self.first = rand(seed + 4, 1, H, D, D)
        cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        self.batch = tokens.Batch(torch.empty(1, 0, dtype=torch.int32, device="cuda"), cu, cu[1:] + 1, max_new=T, max_len=T + 1)
        self.bytes = tokens.linear_attention_workspace_bytes(tokens.StateCache(self.first), self.batch, self.q)
        assert self.bytes > 0, "the sequence is not split"

    def begin(self):
        self.states = tokens.StateCache(self.first.clone())
        self.out = [torch.empty_like(self.v) for _ in range(ROUNDS)]

    def step(self, ctx, i, stream):
        tokens.linear_attention(ctx, self.states, self.batch, self.q, self.k, self.v, self.g, out=self.out[i], stream=stream)

    def results(self):
        return self.out + [self.states.state]


class Products:
    """A gated block onto its residual, ROUNDS times: the rows of both products
    are quantised in the workspace, and copied there as they are odd."""

    def __init__(self, seed, M=4000, K=1111, N=1300):
        self.x = rand(seed, M, K).bfloat16()
        self.w, self.w2 = (torch.randint(-127, 128, s, generator=torch.Generator(device="cuda").manual_seed(seed + 1), dtype=torch.int8,
                                         device="cuda") for s in ((2 * N, K), (K, N)))
        self.ws, self.ws2 = (torch.full((n,), 1 / (73 * m ** 0.5), device="cuda") for n, m in ((2 * N, K), (K, N)))
        self.bytes = max(tokens.gated_linear_i8_workspace_bytes(M, N, K), tokens.linear_i8_workspace_bytes(M, K, N))
        self.shape = (M, N)

    def begin(self):
        self.h = [self.x.clone() for _ in range(ROUNDS)]
        self.u = torch.empty(self.shape, dtype=torch.bfloat16, device="cuda")

    def step(self, ctx, i, stream):
        tokens.gated_linear_i8(ctx, self.h[i], self.w, self.ws, out=self.u, stream=stream)
        tokens.linear_i8(ctx, self.u, self.w2, self.ws2, residual=self.h[i], out=self.h[i], act="silu", stream=stream)

    def results(self):
        return self.h


@pytest.mark.parametrize("make", [Attention, Products])
def test_two_streams_at_once(make):
    jobs, ctxs, streams = [make(10), make(20)], [], []
    for j in jobs:
        ctxs.append(c3c.Context())
        ctxs[-1].set_workspace(torch.empty(j.bytes, dtype=torch.uint8, device="cuda"))
        streams.append(torch.cuda.Stream())
    want = []
    for j, ctx, s in zip(jobs, ctxs, streams):
        j.begin()
        torch.cuda.synchronize()
        for i in range(ROUNDS):
            j.step(ctx, i, s)
        torch.cuda.synchronize()
        want.append([t.clone() for t in j.results()])
        j.begin()
    assert not torch.equal(want[0][0], want[1][0])
    first, last = ([torch.cuda.Event(enable_timing=True) for _ in jobs] for _ in range(2))
    torch.cuda.synchronize()
    for i in range(ROUNDS):
        for n, (j, ctx, s) in enumerate(zip(jobs, ctxs, streams)):
            if i == 0:
                first[n].record(s)
            j.step(ctx, i, s)
    for e, s in zip(last, streams):
        e.record(s)
    torch.cuda.synchronize()
    assert first[1].elapsed_time(last[0]) > 0 and first[0].elapsed_time(last[1]) > 0, "the streams did not overlap"
    for j, w in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(j.results(), w))
