"""Performance cases of the token operators: one call each, through the public binding.

The token operators are those of one layer of a causal transformer over the
stream whose chunks the cached Conv3D layers decode.  Every case carries a
``kind``:

  norm     norm after a block, gate, scaled residual and norm before the next
           block, in one call
  linear   matrix product in 8-bit integers, with a scale for every token and
           every output channel; the activations come as floats (the call
           quantises them) or, with ``pre``, as 8-bit codes with their scales
  append   rotation of queries and keys, and keys and values into a paged
           cache held in 8 bits
  attend   attention over that cache

The cache holds e4m3 codes with one power-of-two scale for every block of 16
tokens and every head:

  k codes [pages][Hkv][page][D]              scales [pages][Hkv][page / 16]
  v codes [pages][Hkv][page / 16][D][16]     scales [pages][Hkv][page / 16]

Sequences are ragged: sequence b has ``new`` tokens in this call, the last of
the ``len`` tokens that its pages hold after it.  Sizes are generic, or those
that a stream of 60x104 latent frames gives with 2x2 patches: 1560 tokens a
frame, 21 frames for a clip of 81.  Inputs are synthetic, drawn from the seed
on the device.
"""
import math

import torch

own = False  # True: run() calls the framework's operators

DEVICE = "cuda"
BLOCK = 16      # tokens that share a scale
E4M3_MAX = 448.0
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


# ---------------------------------------------------------------- cases

def _norm(T, C, rows, dtype="bf16", post=True, **kw):
    return dict(kind="norm", T=T, C=C, rows=rows, dtype=dtype, post=post, **kw)


def _linear(M, K, N, dtype="bf16", pre=False, bias=True, **kw):
    return dict(kind="linear", M=M, K=K, N=N, dtype=dtype, pre=pre, bias=bias, **kw)


def _append(B, new_lo, new_hi, old_lo, old_hi, Hq, Hkv, D, page, rot, pairs="half", dtype="bf16", **kw):
    return dict(kind="append", B=B, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, Hq=Hq, Hkv=Hkv,
                D=D, page=page, rot=rot, pairs=pairs, dtype=dtype, **kw)


def _attend(B, new_lo, new_hi, old_lo, old_hi, Hq, Hkv, D, page, causal=True, window=0, dtype="bf16", **kw):
    return dict(kind="attend", B=B, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, Hq=Hq, Hkv=Hkv,
                D=D, page=page, causal=causal, window=window, dtype=dtype, **kw)


def listed():
    return [
        # one token of one stream: all latency
        _norm(1, 4096, 1, name="norm_token"),
        # a width that no vector load fits, full precision, a gate for each token
        _norm(777, 1531, 1, dtype="f32", name="norm_odd_f32"),
        # a whole clip of 21 frames, gates by frame: memory traffic alone
        _norm(32760, 5120, 1560, name="norm_clip"),
        # the query, key and value projection of one token: reads the weights once
        _linear(1, 4096, 6144, name="linear_token"),
        # sizes that fit no tile, half precision
        _linear(333, 1111, 777, dtype="f16", name="linear_odd_f16"),
        # a clip's projection, its activations already quantised by the norm
        _linear(32760, 5120, 5120, pre=True, name="linear_clip"),
        # one new token for each of 64 streams
        _append(64, 1, 1, 100, 2000, 32, 8, 128, 64, 128, name="append_token"),
        # a new frame of 1560 tokens for each of four streams, behind two frames
        _append(4, 1560, 1560, 3120, 3120, 12, 12, 128, 128, 128, pairs="next", name="append_frame"),
        # one stream's next token: few rows, a long axis
        _attend(1, 1, 1, 4096, 4096, 32, 8, 128, 64, name="attend_token"),
        # a batch of ragged streams, long ones among them: reads the cache once
        _attend(64, 1, 1, 1000, 32767, 32, 8, 128, 64, name="attend_batch"),
        # a frame that sees itself and a rolling context of five more
        _attend(2, 1560, 1560, 7800, 7900, 12, 12, 128, 128, causal=False, name="attend_frame"),
        # a long prompt, causal: matrix products and exponentials
        _attend(1, 8192, 8192, 0, 0, 32, 8, 128, 64, name="attend_prompt"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, multiple, odd=0.3):
    """A size between lo and hi, evenly over its logarithm: a multiple of
    ``multiple``, or (with probability ``odd``) any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < odd else max(multiple, n // multiple * multiple)


def _dtype(rng):
    return rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])


def draw(rng):
    kind = rng.choice(["norm", "linear", "append", "attend", "attend"])
    while True:
        if kind == "norm":
            c = _norm(_log_int(rng, 1, 32760), _size(rng, 64, 8192, 8), 1, _dtype(rng), rng.random() < 0.7)
            c["rows"] = rng.choice([1, c["T"], _log_int(rng, 1, 1560)])
            # outputs and inputs of the largest listed case in bytes
            if c["T"] * c["C"] * ESIZE[c["dtype"]] > 32760 * 5120 * 2:
                continue
        elif kind == "linear":
            c = _linear(_log_int(rng, 1, 32760), _size(rng, 64, 16384, 16), _size(rng, 64, 16384, 16), _dtype(rng),
                        rng.random() < 0.3, rng.random() < 0.5)
            if c["M"] * c["K"] * c["N"] > 32760 * 5120 * 5120 or c["M"] * max(c["K"], c["N"]) > 4e8:
                continue
        else:
            Hkv = rng.choice([1, 2, 4, 8, 12, 16])
            G = rng.choice([1, 1, 2, 4, 5, 8])
            D = rng.choice([64, 80, 96, 128, 128, 128, 256])
            page = rng.choice([16, 32, 64, 128])
            B = _log_int(rng, 1, 128)
            # single tokens, a few (drafted) tokens, or chunks
            new_hi = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 16, 8192)])
            new_lo = new_hi if new_hi == 1 else rng.randint(0, new_hi)
            old_hi = _log_int(rng, 1, 32768)
            old_lo = rng.randint(0, old_hi)
            if kind == "append":
                c = _append(B, new_lo, new_hi, old_lo, old_hi, G * Hkv, Hkv, D, page,
                            rng.choice([D, D, D // 2]), rng.choice(["half", "next"]), _dtype(rng))
                # the cache that comes back stays small next to what is read and written
                if B * (old_hi + new_hi + page) * Hkv * D > 2e8 or B * new_hi * G * Hkv * D > 1e8:
                    continue
            else:
                c = _attend(B, new_lo, new_hi, old_lo, old_hi, G * Hkv, Hkv, D, page, rng.random() < 0.7,
                            rng.choice([0, 0, _log_int(rng, 16, 8192)]), _dtype(rng))
                longest = old_hi + new_hi
                # the largest listed cases in cache, in products and in the plain form's scores
                if (B * longest * Hkv * D > 64 * 32768 * 8 * 128 or B * G * Hkv * new_hi * longest * D > 32 * 8192 * 8192 * 128
                        or B * G * Hkv * new_hi * longest > 32 * 8192 * 8192):
                    continue
        if 3072 not in c.values():
            return c


# ---------------------------------------------------------------- lengths

def _spread(lo, hi, B, k):
    """B lengths from lo to hi, both among them, in a mixed order."""
    if B == 1:
        return [hi]
    step = next(s for s in (k, k + 2, k + 4, k + 6, 1) if math.gcd(s, B) == 1)
    return [lo + (hi - lo) * ((b * step) % B) // (B - 1) for b in range(B)]


def _lengths(case):
    """New and earlier tokens of every sequence."""
    return (_spread(case["new_lo"], case["new_hi"], case["B"], 7), _spread(case["old_lo"], case["old_hi"], case["B"], 11))


def _seen(new, old, causal, window):
    """Pairs of query and key, and keys that any query sees."""
    pairs, first = 0, old + new
    if new and not window:
        pairs = new * old + (new * (new + 1) // 2 if causal else new * new)
        first = 0
    elif new:
        end = old + new
        first = max(0, old - window + 1)
        # query i sees from max(0, old + i - window + 1) to old + i (causal) or to the end
        for i in range(new):
            lo = max(0, old + i - window + 1)
            pairs += (old + i + 1 if causal else end) - lo
    return pairs, (old + new - first if new else 0)


def work(case):
    e = ESIZE[case["dtype"]]
    if case["kind"] == "norm":
        n = case["T"] * case["C"]
        gates = -(-case["T"] // case["rows"]) * case["C"]
        return dict(bytes=4 * n * e + gates * e + 4 * case["C"] * (2 if case["post"] else 1),
                    flops=n * (10 if case["post"] else 7))
    if case["kind"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        x = M * K + 4 * M if case["pre"] else M * K * e
        return dict(bytes=x + N * K + M * N * e + 4 * N * (2 if case["bias"] else 1), flops=2.0 * M * N * K)
    new, old = _lengths(case)
    T, Hq, Hkv, D = sum(new), case["Hq"], case["Hkv"], case["D"]
    if case["kind"] == "append":
        return dict(bytes=T * ((2 * Hq + 2 * Hkv) * D * e + 4 * case["rot"] + 2 * Hkv * D),
                    flops=T * ((Hq + Hkv) * case["rot"] * 3 + 2 * Hkv * D * 3) or 1)
    both = [_seen(n, o, case["causal"], case["window"]) for n, o in zip(new, old)]
    return dict(bytes=sum(k for _, k in both) * Hkv * (2 * D + 8.0 / BLOCK) + 2 * T * Hq * D * e + 4 * case["B"],
                flops=4.0 * D * Hq * sum(p for p, _ in both))


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) & ((1 << 62) - 1))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)


def _activations(g, rows, C):
    """Normal values whose channels have scales of their own, as a
    transformer's activations have."""
    return _randn(g, rows, C).mul_(torch.exp(0.5 * _randn(g, C)))


def _codes(x):
    """x [..., 16 tokens, D] in fp32 -> (codes, scale): e4m3 codes and the
    least power of two that brings the block's largest value to 448 or less."""
    scale = torch.exp2(_exponent(x.abs().amax((-2, -1))).float())
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn), scale


def _exponent(amax):
    """Least e >= -126 with amax <= 448 * 2^e (448 = 0.875 * 2^9)."""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.where(amax > 0, e, torch.full_like(e, -126)).clamp_(min=-126)


def _cache(g, case, new, old):
    """A cache whose pages hold every sequence's earlier tokens (for attention
    also the new ones), in a mixed order of pages; the pages' unused tokens
    hold other values."""
    B, Hkv, D, page = case["B"], case["Hkv"], case["D"], case["page"]
    cols = max(1, max(-(-(n + o) // page) for n, o in zip(new, old)))
    pages = sum(-(-(n + o) // page) for n, o in zip(new, old)) + 3
    nb = page // BLOCK
    k, ks = _codes(_randn(g, pages, Hkv, nb, BLOCK, D).mul_(torch.exp(0.5 * _randn(g, D))))
    v, vs = _codes(_randn(g, pages, Hkv, nb, BLOCK, D))
    order = torch.randperm(pages, generator=g, device=DEVICE).int()
    table = torch.zeros(B, cols, dtype=torch.int32, device=DEVICE)
    used = torch.tensor([-(-(n + o) // page) for n, o in zip(new, old)], device=DEVICE)
    here = torch.arange(cols, device=DEVICE)[None, :] < used[:, None]
    table[here] = order[:int(used.sum())]
    return dict(k=k.view(pages, Hkv, page, D), v=v.transpose(-1, -2).contiguous(), ks=ks, vs=vs, table=table)


def prepare(case, seed):
    g = _gen(seed)
    dt = DTYPES[case["dtype"]]
    s = dict(case=case)
    if case["kind"] == "norm":
        T, C = case["T"], case["C"]
        gates = -(-T // case["rows"])
        s.update(h=_activations(g, T, C).mul_(3.0).to(dt), y=_activations(g, T, C).to(dt),
                 gate=(0.3 * _randn(g, gates, C)).to(dt), alpha=0.9, pre=1 + 0.2 * _randn(g, C),
                 post=1 + 0.2 * _randn(g, C) if case["post"] else None)
        return s
    if case["kind"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        x = _activations(g, M, K)
        w = _randn(g, N, K).div_(math.sqrt(K))
        s["ws"] = w.abs().amax(1) / 127
        s["w"] = torch.round(w / s["ws"][:, None]).to(torch.int8)
        s["bias"] = 0.1 * _randn(g, N) if case["bias"] else None
        s["xs"] = x.abs().amax(1) / 127 if case["pre"] else None
        s["x"] = torch.round(x / s["xs"][:, None]).to(torch.int8) if case["pre"] else x.to(dt)
        return s
    new, old = _lengths(case)
    T, Hq, Hkv, D = sum(new), case["Hq"], case["Hkv"], case["D"]
    s.update(_cache(g, case, new, old))
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEVICE)
    s["len"] = torch.tensor([n + o for n, o in zip(new, old)], dtype=torch.int32, device=DEVICE)
    s["max_new"], s["max_len"] = max(new), max(n + o for n, o in zip(new, old))
    if case["kind"] == "append":
        # one projection's output: queries, keys and values side by side
        s["qkv"] = _activations(g, T, (Hq + 2 * Hkv) * D).to(dt)
        rows = s["max_len"] or 1
        freq = 10000.0 ** (-torch.arange(case["rot"] // 2, device=DEVICE, dtype=torch.float64) / (case["rot"] // 2))
        angle = torch.arange(rows, device=DEVICE, dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    else:
        s["q"] = _randn(g, T, Hq, D).to(dt)
    return s


# ---------------------------------------------------------------- plain forms

def _plain_norm(s):
    h, y = s["h"].float(), s["y"].float()
    if s["post"] is not None:
        y = y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS) * s["post"]
    group = torch.arange(h.shape[0], device=h.device) // s["case"]["rows"]
    h = s["alpha"] * h + s["gate"].float()[group] * y
    u = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["pre"]
    return dict(h=h.to(s["h"].dtype), u=u.to(s["h"].dtype))


def _plain_linear(s):
    x, xs = s["x"].float(), s["xs"]
    if xs is None:
        xs = x.abs().amax(1) / 127
        x = torch.where(xs[:, None] > 0, torch.round(x / xs[:, None]), 0.0)
    y = (x @ s["w"].float().t()) * xs[:, None] * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[s["case"]["dtype"]])


def _token_places(s, T):
    """Sequence and cache position of every new token."""
    t = torch.arange(T, device=DEVICE)
    b = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    return b, t - s["cu"].long()[b + 1] + s["len"].long()[b]


def _plain_rotate(x, cos, sin, rot, pairs):
    """x [T][H][D] fp32, cos and sin [T][rot / 2]."""
    c, sn = cos[:, None, :], sin[:, None, :]
    if pairs == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    return torch.cat([r, x[..., rot:]], -1)


def _plain_store(x, codes, scale, blocks, slot, first):
    """x [T][Hkv][D] fp32 into codes [blocks][Hkv][16][D] (a view); blocks and
    slot: the block and the place in it of every token; first [n blocks]: the
    first new place of every block (16: no new token)."""
    n, Hkv = scale.shape
    amax = torch.zeros(n, Hkv, device=x.device).scatter_reduce_(0, blocks[:, None].expand(-1, Hkv), x.abs().amax(-1), "amax")
    touched = first < BLOCK
    fresh = touched & (first == 0)
    e_old = torch.where(fresh[:, None], -126, torch.frexp(scale)[1] - 1)
    e = torch.maximum(_exponent(amax), e_old)
    new_scale = torch.where(touched[:, None], torch.exp2(e.float()), scale)
    part = torch.nonzero(touched & ~fresh)[:, 0]
    shrink = (scale[part] / new_scale[part])[..., None, None]
    kept = (codes[part].float() * shrink).to(codes.dtype)
    before = torch.arange(BLOCK, device=x.device) < first[part][:, None]
    codes[part] = torch.where(before[:, None, :, None], kept.float(), codes[part].float()).to(codes.dtype)
    scale.copy_(new_scale)
    codes[blocks, :, slot] = (x / new_scale[blocks][..., None]).to(codes.dtype)


def _plain_append(s):
    c = s["case"]
    Hq, Hkv, D, page, dt = c["Hq"], c["Hkv"], c["D"], c["page"], s["qkv"].dtype
    T, nb = s["qkv"].shape[0], page // BLOCK
    b, p = _token_places(s, T)
    q, k, v = s["qkv"].float().view(T, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
    cos, sin = s["cos"][p], s["sin"][p]
    q = _plain_rotate(q, cos, sin, c["rot"], c["pairs"])
    k = _plain_rotate(k, cos, sin, c["rot"], c["pairs"])
    blocks = s["table"][b, p // page].long() * nb + p % page // BLOCK
    slot = p % BLOCK
    n = s["k"].shape[0] * nb
    first = torch.full((n,), BLOCK, device=p.device).scatter_reduce_(0, blocks, slot, "amin")
    # copies with the blocks of every page first, [pages][nb][Hkv][16][D], written back where they came from
    kc = s["k"].clone().view(-1, Hkv, nb, BLOCK, D).transpose(1, 2).reshape(n, Hkv, BLOCK, D)
    vc = s["v"].clone().permute(0, 2, 1, 4, 3).reshape(n, Hkv, BLOCK, D)
    ks, vs = (t.clone().transpose(1, 2).reshape(n, Hkv) for t in (s["ks"], s["vs"]))
    _plain_store(k, kc, ks, blocks, slot, first)
    _plain_store(v, vc, vs, blocks, slot, first)
    s["k"].view(-1, Hkv, nb, BLOCK, D).copy_(kc.view(-1, nb, Hkv, BLOCK, D).transpose(1, 2))
    s["v"].copy_(vc.view(-1, nb, Hkv, BLOCK, D).permute(0, 2, 1, 4, 3))
    s["ks"].copy_(ks.view(-1, nb, Hkv).transpose(1, 2))
    s["vs"].copy_(vs.view(-1, nb, Hkv).transpose(1, 2))
    return dict(q=q.to(dt), k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])


def _plain_attend(s):
    c, q = s["case"], s["q"]
    B, Hq, Hkv, D, page = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    G, nb, L, n = Hq // Hkv, page // BLOCK, s["max_len"], s["max_new"]
    cols = -(-L // page)
    at = s["table"][:, :cols].long()
    k = s["k"].view(-1, Hkv, nb, BLOCK, D)[at].float() * s["ks"][at][..., None, None]  # [B][cols][Hkv][nb][16][D]
    k = k.transpose(1, 2).reshape(B, Hkv, cols * page, D)[:, :, :L]
    v = s["v"][at].float() * s["vs"][at][..., None, None]                              # [B][cols][Hkv][nb][D][16]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, Hkv, cols * page, D)[:, :, :L]
    length, cu = s["len"].long(), s["cu"].long()
    new = cu[1:] - cu[:-1]
    i, j = torch.arange(n, device=q.device), torch.arange(L, device=q.device)
    v = v * (j < length[:, None])[:, None, :, None]
    rows = (cu[:-1, None] + i).clamp(max=max(q.shape[0] - 1, 0))            # [B][n]
    x = q.float()[rows].view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    p = (length - new)[:, None] + i                                         # [B][n]
    see = (j < length[:, None])[:, None, :].expand(B, n, L)
    if c["causal"]:
        see = see & (j <= p[:, :, None])
    if c["window"]:
        see = see & (j > p[:, :, None] - c["window"])
    see = see[:, None, None]
    w = (x @ k.transpose(-1, -2)).mul_(D ** -0.5).view(B, Hkv, G, n, L)
    w.masked_fill_(~see, -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = w.sum(-1, keepdim=True)
    o = (w.view(B, Hkv, G * n, L) @ v).view(B, Hkv, G, n, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D)
    return o[i < new[:, None]].to(q.dtype)


# ---------------------------------------------------------------- the framework's operators

_kept = {}


def _framework(need):
    """The binding's modules and the one context of this program, whose
    workspace grows to what a call asks for."""
    from paper_2609_31938_amd import c3c, tokens
    if "ctx" not in _kept:
        _kept.update(ctx=c3c.Context(), bytes=0)
    n = need(tokens)
    if n > _kept["bytes"]:
        _kept["ctx"].set_workspace(torch.empty(n, dtype=torch.uint8, device=DEVICE))
        _kept["bytes"] = n
    return tokens, _kept["ctx"]


def _own_norm(s):
    tokens, ctx = _framework(lambda t: 0)
    h, u = tokens.norm_gate(ctx, s["h"], s["y"], s["gate"], post=s["post"], pre=s["pre"], alpha=s["alpha"], eps=EPS,
                            rows_per_gate=s["case"]["rows"])
    return dict(h=h, u=u)


def _own_linear(s):
    dt = s["case"]["dtype"]
    if "plan" not in s:
        c = s["case"]
        _framework(lambda t: t.linear_i8_workspace_bytes(c["M"], c["N"], c["K"], "i8" if c["pre"] else dt, dt))
        s["plan"] = True
    tokens, ctx = _framework(lambda t: 0)
    return tokens.linear_i8(ctx, s["x"], s["w"], s["ws"], bias=s["bias"], x_scale=s["xs"], out_dtype=dt)


def _paged(s):
    """The cache and the batch, as the program keeps them over a step."""
    if "plan" not in s:
        from paper_2609_31938_amd import tokens
        cache = tokens.KVCache(s["k"], s["v"], s["ks"], s["vs"])
        batch = tokens.Batch(s["table"], s["cu"], s["len"], max_new=s["max_new"], max_len=s["max_len"])
        if s["case"]["kind"] == "attend":
            _framework(lambda t: t.paged_attention_workspace_bytes(cache, s["q"], batch, causal=s["case"]["causal"],
                                                                   window=s["case"]["window"]))
        s["plan"] = (cache, batch)
    return s["plan"]


def _own_append(s):
    c = s["case"]
    cache, batch = _paged(s)
    tokens, ctx = _framework(lambda t: 0)
    q, k, v = s["qkv"].view(-1, c["Hq"] + 2 * c["Hkv"], c["D"]).split([c["Hq"], c["Hkv"], c["Hkv"]], 1)
    q = tokens.kv_append(ctx, cache, batch, k, v, q=q, cos=s["cos"], sin=s["sin"], pairs=c["pairs"])
    return dict(q=q, k=s["k"], v=s["v"], ks=s["ks"], vs=s["vs"])


def _own_attend(s):
    cache, batch = _paged(s)
    tokens, ctx = _framework(lambda t: 0)
    return tokens.paged_attention(ctx, cache, batch, s["q"], causal=s["case"]["causal"], window=s["case"]["window"])


_PLAIN = dict(norm=_plain_norm, linear=_plain_linear, append=_plain_append, attend=_plain_attend)
_OWN = dict(norm=_own_norm, linear=_own_linear, append=_own_append, attend=_own_attend)


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# ---------------------------------------------------------------- definitions in 64 bits

def _exact_norm(s):
    h, y = s["h"].double(), s["y"].double()
    if s["post"] is not None:
        y = y / ((y ** 2).mean(1) + EPS).sqrt()[:, None] * s["post"].double()
    gate = s["gate"].double().repeat_interleave(s["case"]["rows"], 0)[:h.shape[0]]
    h = h * s["alpha"] + y * gate
    return dict(h=h, u=h / ((h ** 2).mean(1) + EPS).sqrt()[:, None] * s["pre"].double())


def _exact_linear(s):
    x = s["x"].double()
    if s["xs"] is not None:
        xs = s["xs"].double()
    else:
        xs = x.abs().max(1).values / 127
        x = (x / xs[:, None]).nan_to_num(0.0).round()
    y = torch.mm(x, s["w"].double().t().contiguous()) * torch.outer(xs, s["ws"].double())
    return y if s["bias"] is None else y + s["bias"].double()


def _e4m3(x):
    """x (|x| <= 448) to the nearest e4m3 value, ties to even, in 64 bits."""
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-6).double() - 3)
    return (x / step).round() * step


def _exact_append(s):
    c = s["case"]
    Hq, Hkv, D, page, half = c["Hq"], c["Hkv"], c["D"], c["page"], c["rot"] // 2
    new, old = _lengths(c)
    x = s["qkv"].double().view(-1, Hq + 2 * Hkv, D).clone()
    p = torch.cat([torch.arange(o, o + n, device=DEVICE) for n, o in zip(new, old)])
    turn = torch.complex(s["cos"].double(), s["sin"].double())[p][:, None, :]
    first = torch.arange(half, device=DEVICE) * (1 if c["pairs"] == "half" else 2)
    second = first + (half if c["pairs"] == "half" else 1)
    r = torch.complex(x[:, :Hq + Hkv, first], x[:, :Hq + Hkv, second]) * turn
    x[:, :Hq + Hkv, first], x[:, :Hq + Hkv, second] = r.real, r.imag
    table = s["table"].tolist()
    out = dict(q=x[:, :Hq], k=s["k"].double(), v=s["v"].double(), ks=s["ks"].double(), vs=s["vs"].double())
    at = 0
    for b, (n, o) in enumerate(zip(new, old)):
        for lo in range(o // BLOCK * BLOCK, o + n if n else 0, BLOCK):
            f, t = max(lo, o), min(lo + BLOCK, o + n)     # new tokens of this block
            pg, blk = table[b][lo // page], lo % page // BLOCK
            for name, sc, h0 in (("k", "ks", Hq), ("v", "vs", Hq + Hkv)):
                block = out[name][pg, :, lo % page:lo % page + BLOCK] if name == "k" else out[name][pg, :, blk].transpose(1, 2)
                val = x[at + f - o:at + t - o, h0:h0 + Hkv].transpose(0, 1)
                top = val.abs().amax((1, 2))
                e = torch.where(top > 0, torch.ceil(torch.log2(top / E4M3_MAX)), -126.0).clamp(min=-126)
                if f > lo:
                    e = torch.maximum(e, torch.log2(out[sc][pg, :, blk]))
                    block[:, :f - lo] = _e4m3(block[:, :f - lo] * (out[sc][pg, :, blk] * torch.exp2(-e))[:, None, None])
                block[:, f - lo:t - lo] = _e4m3(val * torch.exp2(-e)[:, None, None])
                out[sc][pg, :, blk] = torch.exp2(e)
        at += n
    return out


def _exact_attend(s):
    c = s["case"]
    Hq, Hkv, D, page = c["Hq"], c["Hkv"], c["D"], c["page"]
    new, old = _lengths(c)
    q, out, at = s["q"].double(), torch.zeros_like(s["q"], dtype=torch.float64), 0
    for b, (n, o) in enumerate(zip(new, old)):
        L = n + o
        if not n or not L:
            at += n
            continue
        pages = s["table"][b, :-(-L // page)].long()
        k = s["k"][pages].double() * s["ks"][pages].double().repeat_interleave(BLOCK, 2)[..., None]
        v = s["v"][pages].double() * s["vs"][pages].double()[..., None, None]
        i, j = torch.arange(n, device=DEVICE)[:, None] + o, torch.arange(L, device=DEVICE)
        hidden = torch.zeros(n, L, dtype=torch.bool, device=DEVICE)
        if c["causal"]:
            hidden |= j > i
        if c["window"]:
            hidden |= j <= i - c["window"]
        for h in range(Hkv):
            kh = k[:, h].reshape(-1, D)[:L]
            vh = v[:, h].transpose(2, 3).reshape(-1, D)[:L]
            for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                w = torch.mm(q[at:at + n, g], kh.t().contiguous()) / math.sqrt(D)
                w = torch.softmax(w.masked_fill_(hidden, -math.inf), 1).nan_to_num_(0.0)
                out[at:at + n, g] = torch.mm(w, vh)
        at += n
    return out


def exact(case, seed):
    if case["kind"] == "append":
        new, _ = _lengths(case)
        if sum(-(-n // BLOCK) + 1 for n in new) > 4000:   # block by block: too long
            return None
    s = prepare(case, seed)
    return dict(norm=_exact_norm, linear=_exact_linear, append=_exact_append, attend=_exact_attend)[case["kind"]](s)
