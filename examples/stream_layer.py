"""A small streaming world model: causal transformer layers that make one latent
frame after another, and a cached causal Conv3D layer that decodes them.

Every frame's tokens run through the layers in one call each (a frame sees
itself and the frames that its window still holds), or token by token; the
layers keep keys and values in paged 8-bit caches, the decoder keeps its last
two frames.  Every n-th layer may be a recurrent one (--recurrent n), which
remembers the stream in a state of constant size and sees it token by token.
Weights and inputs are synthetic.

    python examples/stream_layer.py [--frames 6] [--channels 1536] [--layers 2] [--recurrent 0]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_31938_amd import c3c, inputs, tokens  # noqa: E402

PAGE = 64


class Weights:
    """8-bit weights (N, K) with a scale for every output channel."""

    def __init__(self, ctx, gen, N, K):
        w = torch.randn(N, K, generator=gen, device="cuda") / K ** 0.5
        self.w, self.scale = tokens.quantize_rows(ctx, w)

    def __call__(self, ctx, x, x_scale=None, **epilogue):
        return tokens.linear_i8(ctx, x, self.w, self.scale, x_scale=x_scale, out_dtype="bf16", **epilogue)


class Layer:
    """Attention and a feed-forward block, each between norms."""

    def __init__(self, ctx, gen, channels, heads, kv_heads, pages):
        self.heads, self.kv_heads, self.dim = heads, kv_heads, channels // heads
        self.qkv = Weights(ctx, gen, (heads + 2 * kv_heads) * self.dim, channels)
        self.out = Weights(ctx, gen, channels, channels)
        self.up = Weights(ctx, gen, 4 * channels, channels)
        self.down = Weights(ctx, gen, channels, 4 * channels)
        self.cache = tokens.KVCache.empty(pages, kv_heads, PAGE, self.dim)
        self.products = self.qkv, self.out, self.up, self.down

        def gain():
            return 1 + 0.1 * torch.randn(channels, generator=gen, device="cuda")

        self.pre_a, self.post_a, self.pre_f, self.post_f = gain(), gain(), gain(), gain()
        # one row of gates for the whole stream (a layer scale)
        self.gate_a, self.gate_f = (0.3 * torch.randn(1, channels, generator=gen, device="cuda").bfloat16()
                                    for _ in range(2))

    def workspace(self, T, batch, window):
        """Bytes that the calls of T tokens ask for."""
        q = torch.empty(T, self.heads, self.dim, dtype=torch.bfloat16, device="cuda")
        return [tokens.paged_attention_workspace_bytes(self.cache, q, batch, causal, window) for causal in (False, True)]

    def __call__(self, ctx, h, x, x_scale, batch, angles, causal, window, pre_next):
        """h (T, channels): the residual stream; x, x_scale: the layer's input
        after its norm, as 8-bit rows.  Returns h and the next layer's input."""
        T = h.shape[0]
        qkv = self.qkv(ctx, x, x_scale).view(T, self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        q = tokens.kv_append(ctx, self.cache, batch, k, v, q=q, cos=angles[0], sin=angles[1])
        a = tokens.paged_attention(ctx, self.cache, batch, q, causal=causal, window=window)
        y = self.out(ctx, a.view(T, -1))
        h, x, x_scale = tokens.norm_gate(ctx, h, y, self.gate_a, post=self.post_a, pre=self.pre_f, rows_per_gate=T,
                                         quantize=True)
        y = self.down(ctx, torch.nn.functional.silu(self.up(ctx, x, x_scale)))
        return tokens.norm_gate(ctx, h, y, self.gate_f, post=self.post_f, pre=pre_next, rows_per_gate=T, quantize=True)


class RecurrentLayer:
    """Linear attention with a decay for each head and a gated feed-forward block,
    each added to the residual stream by its last product."""

    def __init__(self, ctx, gen, channels, heads, kv_heads):
        self.heads, self.kv_heads, self.dim = heads, kv_heads, channels // heads
        # heads share queries and keys in groups
        self.qkv = Weights(ctx, gen, (heads + 2 * kv_heads) * self.dim, channels)
        self.out = Weights(ctx, gen, channels, channels)
        self.gate_up = Weights(ctx, gen, 2 * 3 * channels, channels)
        self.down = Weights(ctx, gen, channels, 3 * channels)
        self.products = self.qkv, self.out, self.down
        self.states = tokens.StateCache.empty(1, heads, self.dim, self.dim)
        # a head forgets half of what it holds within some 20 to 600 tokens
        self.log_decay = torch.log1p(-torch.exp2(-5 - 5 * torch.arange(heads, device="cuda") / heads))
        self.pre_a, self.pre_f = (1 + 0.1 * torch.randn(channels, generator=gen, device="cuda") for _ in range(2))

    def workspace(self, T, batch, window):
        q = torch.empty(T, self.kv_heads, self.dim, dtype=torch.bfloat16, device="cuda")
        return [tokens.linear_attention_workspace_bytes(self.states, batch, q),
                tokens.gated_linear_i8_workspace_bytes(T, self.gate_up.w.shape[0] // 2, self.gate_up.w.shape[1], "i8")]

    def __call__(self, ctx, h, x, x_scale, batch, angles, causal, window, pre_next):
        T = h.shape[0]
        qkv = self.qkv(ctx, x, x_scale).view(T, 2 * self.kv_heads + self.heads, self.dim)
        q, k, v = qkv.split([self.kv_heads, self.kv_heads, self.heads], 1)
        a = tokens.linear_attention(ctx, self.states, batch, q, k, v, self.log_decay)
        h = self.out(ctx, a.view(T, -1), residual=h, out=h)
        _, x, x_scale = tokens.norm_gate(ctx, h, pre=self.pre_f, h_out=h, quantize=True)
        u = tokens.gated_linear_i8(ctx, x, self.gate_up.w, self.gate_up.scale, x_scale=x_scale, out_dtype="bf16", act="silu")
        h = self.down(ctx, u, residual=h, out=h)
        return tokens.norm_gate(ctx, h, pre=pre_next, h_out=h, quantize=True)


class WorldModel:
    """`layers` layers over frames of H x W latent pixels in 2 x 2 patches, every
    `recurrent`-th of them a recurrent one (0: none), and the decoder's first
    convolution."""

    def __init__(self, channels=1536, heads=12, kv_heads=4, layers=2, H=60, W=104, latent=32, max_frames=8,
                 window_frames=0, seed=0, recurrent=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx = c3c.Context()
        self.H, self.W, self.latent, self.per_frame = H, W, latent, H // 2 * (W // 2)
        self.max_len = max_frames * self.per_frame
        cols = -(-self.max_len // PAGE)
        self.layers = [RecurrentLayer(self.ctx, gen, channels, heads, kv_heads) if recurrent and i % recurrent == recurrent - 1
                       else Layer(self.ctx, gen, channels, heads, kv_heads, cols) for i in range(layers)]
        self.embed = Weights(self.ctx, gen, channels, 4 * latent)
        self.head = Weights(self.ctx, gen, 4 * latent, channels)
        self.last = torch.ones(channels, device="cuda")
        self.window = window_frames * self.per_frame
        dim = channels // heads
        freq = 10000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
        angle = torch.arange(self.max_len, device="cuda", dtype=torch.float64)[:, None] * freq
        self.angles = angle.cos().float(), angle.sin().float()
        # one stream: its pages in order; the batch is updated in place
        self.table = torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
        self.length = torch.zeros(1, dtype=torch.int32, device="cuda")
        self._batches = {}
        # the decoder: one cached causal 3x3x3 convolution
        self.spec = inputs.spec(N=1, Ci=latent, Co=96, T=1, Tc=2, H=H, W=W)
        self.w, self.b = inputs.layer_tensors(self.spec, "bf16", 1, 0, "cuda")
        self.wpack = c3c.weight_repack(self.ctx, self.spec, self.w)
        self.frames = torch.zeros(1, latent, 2, H, W, dtype=torch.bfloat16, device="cuda")
        self._bytes = 0

    def _batch(self, T):
        if T not in self._batches:
            cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
            batch = tokens.Batch(self.table, cu, self.length, max_new=T, max_len=self.max_len)
            # the largest workspace that a call of T tokens asks for
            need = [n for layer in self.layers for n in layer.workspace(T, batch, self.window)]
            for m in [m for x in self.layers for m in x.products] + [self.embed, self.head]:
                need.append(tokens.linear_i8_workspace_bytes(T, *m.w.shape))
            need.append(c3c.workspace_bytes(self.spec, "bf16"))
            self._batches[T] = batch, max(need)
        batch, need = self._batches[T]
        if need > self._bytes:
            self.ctx.set_workspace(torch.empty(need, dtype=torch.uint8, device="cuda"))
            self._bytes = need
        return batch

    def tokens(self, x, causal):
        """The next tokens of the stream, x (T, 4 latent): their predictions."""
        ctx, batch = self.ctx, self._batch(x.shape[0])
        self.length.add_(x.shape[0])
        h = self.embed(ctx, x)
        _, u, s = tokens.norm_gate(ctx, h, pre=self.layers[0].pre_a, h_out=h, quantize=True)
        for i, layer in enumerate(self.layers):
            after = self.layers[i + 1].pre_a if i + 1 < len(self.layers) else self.last
            h, u, s = layer(ctx, h, u, s, batch, self.angles, causal, self.window, after)
        return self.head(ctx, u, s)

    def frame(self, x):
        """The next frame: its tokens' predictions, decoded with the frames before."""
        H, W, c = self.H // 2, self.W // 2, self.latent
        p = self.tokens(x, causal=False)
        z = p.view(1, H, W, 2, 2, c).permute(0, 5, 1, 3, 2, 4).reshape(1, c, 1, self.H, self.W)
        y, self.frames = c3c.conv3d_causal_cached(self.ctx, self.spec, z, self.frames, self.w, self.wpack, self.b)
        return p, y


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--frames", type=int, default=6)
    ap.add_argument("--channels", type=int, default=1536)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--recurrent", type=int, default=0)
    a = ap.parse_args()
    model = WorldModel(channels=a.channels, heads=a.channels // 128, kv_heads=max(1, a.channels // 384), layers=a.layers,
                       max_frames=a.frames + 1, window_frames=4, recurrent=a.recurrent)
    x = torch.randn(model.per_frame, 4 * model.latent, device="cuda").bfloat16()
    for f in range(a.frames):
        torch.cuda.synchronize()
        t = time.perf_counter()
        x, y = model.frame(x)
        torch.cuda.synchronize()
        print(f"frame {f}: {model.per_frame} tokens, {1e3 * (time.perf_counter() - t):.2f} ms, "
              f"decoded {tuple(y.shape)}, finite {bool(y.isfinite().all())}", flush=True)
    for i in range(3):
        torch.cuda.synchronize()
        t = time.perf_counter()
        model.tokens(x[i:i + 1], causal=True)
        torch.cuda.synchronize()
        print(f"one token: {1e3 * (time.perf_counter() - t):.2f} ms", flush=True)


if __name__ == "__main__":
    main()
