"""Performance cases of a recurrent layer's operators: one call each, through the public binding.

They are the operators of a transformer layer whose memory of the stream is a
state of constant size, as the cached Conv3D's is, in place of a cache that
grows.  Every case carries a ``kind``:

  recur    linear attention with a decay for each head (``by`` "head": one for
           each head; "token": one for each token and head):
             S_t = exp(g_t) S_(t-1) + k_t v_t^T        o_t = scale q_t S_t
           with S (Dk x Dv) in fp32 for each head, updated in place
  linear   matrix product in 8-bit integers with an epilogue:
             y = alpha residual + gate act(x w^T + bias)
  gated    both projections of a gated feed-forward block, the activation and
           their product:
             y = act(x w_g^T + b_g) (x w_u^T + b_u)

Sequences are ragged: sequence b has ``new`` tokens in this call, behind
``old`` earlier ones; one without earlier tokens begins from a state of zeros.
Activations of the products come as floats (the call quantises them: a scale
for every token) or, with ``pre``, as 8-bit codes with their scales.  Sizes are
generic, or those that a stream of 60x104 latent frames gives with 2x2
patches: 1560 tokens a frame, 21 frames for a clip of 81.  Inputs are
synthetic, drawn from the seed on the device.
"""
import math

import torch

own = False  # True: run() calls the framework's operators

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f16": 2, "f32": 4}
CHUNK = 64  # tokens that the plain form takes together


# ---------------------------------------------------------------- cases

def _recur(B, new_lo, new_hi, old_lo, old_hi, H, Hk, Dk, Dv, by="head", dtype="bf16", **kw):
    return dict(kind="recur", B=B, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, H=H, Hk=Hk, Dk=Dk, Dv=Dv,
                by=by, dtype=dtype, **kw)


def _linear(M, K, N, act="none", residual=False, rows=0, bias=True, dtype="bf16", pre=False, **kw):
    # rows: tokens that share a row of gates (0: no gate)
    return dict(kind="linear", M=M, K=K, N=N, act=act, residual=residual, rows=rows, bias=bias, dtype=dtype, pre=pre, **kw)


def _gated(M, K, N, act="silu", bias=False, dtype="bf16", pre=False, **kw):
    return dict(kind="gated", M=M, K=K, N=N, act=act, bias=bias, dtype=dtype, pre=pre, **kw)


def listed():
    return [
        # one stream's next token: all latency
        _recur(1, 1, 1, 1000, 1000, 32, 32, 128, 128, name="recur_token"),
        # the next token of 64 streams: states in and out
        _recur(64, 1, 1, 0, 4000, 32, 8, 128, 128, by="token", name="recur_batch"),
        # a few drafted tokens for each of 16 streams, half precision
        _recur(16, 2, 8, 10, 900, 16, 16, 64, 128, by="token", dtype="f16", name="recur_draft_f16"),
        # odd ragged chunks in full precision, one of them empty, dims that fill no tile
        _recur(5, 0, 701, 0, 300, 6, 3, 80, 112, by="token", dtype="f32", name="recur_odd_f32"),
        # a new frame for each of two streams
        _recur(2, 1560, 1560, 3120, 7800, 12, 12, 128, 128, name="recur_frame"),
        # a whole clip of 21 frames as a prompt
        _recur(1, 32760, 32760, 0, 0, 32, 32, 128, 128, by="token", name="recur_clip"),
        # the up projection of one token with its activation
        _linear(1, 1536, 6144, act="gelu_tanh", name="linear_token"),
        # the down projection of 64 streams' tokens onto their residual stream, full precision, sizes that fit no tile
        _linear(61, 5003, 1531, residual=True, rows=1, dtype="f32", name="linear_odd_f32"),
        # a clip's output projection onto the residual stream, gates by frame, its activations already quantised
        _linear(32760, 5120, 5120, residual=True, rows=1560, pre=True, name="linear_clip"),
        # one token's gated block: reads the weights once
        _gated(1, 4096, 10240, name="gated_token"),
        # sizes that fit no tile, half precision
        _gated(333, 1111, 777, act="gelu", bias=True, dtype="f16", name="gated_odd_f16"),
        # a frame's gated block for each of four streams
        _gated(6240, 5120, 13312, name="gated_frame"),
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
    kind = rng.choice(["recur", "recur", "linear", "gated"])
    while True:
        if kind == "recur":
            H = rng.choice([1, 4, 6, 8, 12, 16, 24, 32])
            Hk = H // rng.choice([d for d in (1, 1, 2, 3, 4, 8) if H % d == 0])
            Dk, Dv = (rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256]) for _ in range(2))
            B = _log_int(rng, 1, 128)
            # single tokens, a few (drafted) tokens, or chunks
            new_hi = rng.choice([1, 1, rng.randint(2, 16), _log_int(rng, 16, 32760), _log_int(rng, 16, 8192)])
            new_lo = new_hi if new_hi == 1 else rng.randint(0, new_hi)
            old_hi = rng.choice([0, _log_int(rng, 1, 32768), _log_int(rng, 1, 32768)])
            c = _recur(B, new_lo, new_hi, rng.randint(0, old_hi), old_hi, H, Hk, Dk, Dv, rng.choice(["head", "token"]), _dtype(rng))
            # the largest listed case in products, in the plain form's memory and in the definition's steps
            if B * new_hi * H * Dk * Dv > 32760 * 32 * 128 * 128 or B * new_hi * H * max(Dk, Dv) > 32760 * 32 * 128:
                continue
        else:
            M, K, N = _log_int(rng, 1, 8192), _size(rng, 64, 16384, 16), _size(rng, 64, 16384, 16)
            act = rng.choice(["none", "silu", "gelu", "gelu_tanh"])
            rows = rng.choice([0, 1, M, _log_int(rng, 1, 1560)])
            if kind == "linear":
                c = _linear(M, K, N, act, rng.random() < 0.6, rows, rng.random() < 0.6, _dtype(rng), rng.random() < 0.4)
            else:
                c = _gated(M, K, N, act, rng.random() < 0.4, _dtype(rng), rng.random() < 0.4)
            if M * K * N * (2 if kind == "gated" else 1) > 6240 * 5120 * 13312 * 2:
                continue
            if kind == "linear" and act == "none" and not c["residual"] and not rows:
                continue  # no epilogue
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


def work(case):
    e = ESIZE[case["dtype"]]
    if case["kind"] == "recur":
        new, old = _lengths(case)
        T, H, Hk, Dk, Dv = sum(new), case["H"], case["Hk"], case["Dk"], case["Dv"]
        states = sum(1 + (o > 0) for n, o in zip(new, old) if n)
        return dict(bytes=T * (2 * Hk * Dk + 2 * H * Dv) * e + 4 * H * (T if case["by"] == "token" else 1) + states * H * Dk * Dv * 4,
                    flops=4.0 * T * H * Dk * Dv or 1)
    M, K, N, two = case["M"], case["K"], case["N"], 2 if case["kind"] == "gated" else 1
    x = M * K + 4 * M if case["pre"] else M * K * e
    more = M * N * e if case.get("residual") else 0
    if case.get("rows"):
        more += -(-M // case["rows"]) * N * e
    return dict(bytes=x + two * N * K + M * N * e + 4 * two * N * (2 if case["bias"] else 1) + more, flops=2.0 * two * M * N * K)


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


def _prepare_recur(case, g, dt):
    B, H, Hk, Dk, Dv = (case[n] for n in ("B", "H", "Hk", "Dk", "Dv"))
    new, old = _lengths(case)
    T = sum(new)
    # one projection's output: queries, keys and values side by side
    s = dict(qkv=_activations(g, T, 2 * Hk * Dk + H * Dv).to(dt))
    # a head forgets half within some 20 to 600 tokens, or as its tokens say
    rate = torch.exp2(-5 - 5 * torch.arange(H, device=DEVICE) / H)
    if case["by"] == "head":
        s["decay"] = torch.log1p(-rate)
    else:
        s["decay"] = -4 * rate * torch.nn.functional.softplus(_randn(g, T, H))
    s["state"] = _randn(g, B + 2, H, Dk, Dv)
    s["slot"] = torch.randperm(B + 2, generator=g, device=DEVICE)[:B].int()
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEVICE)
    s["len"] = torch.tensor([n + o for n, o in zip(new, old)], dtype=torch.int32, device=DEVICE)
    s["max_new"], s["max_len"] = max(new), max(n + o for n, o in zip(new, old))
    return s


def _prepare_product(case, g, dt):
    M, K, N = case["M"], case["K"], case["N"]
    rows = 2 * N if case["kind"] == "gated" else N
    x = _activations(g, M, K)
    w = _randn(g, rows, K).div_(math.sqrt(K))
    s = dict(ws=w.abs().amax(1) / 127)
    s["w"] = torch.round(w / s["ws"][:, None]).to(torch.int8)
    s["bias"] = 0.1 * _randn(g, rows) if case["bias"] else None
    s["xs"] = x.abs().amax(1) / 127 if case["pre"] else None
    s["x"] = torch.round(x / s["xs"][:, None]).to(torch.int8) if case["pre"] else x.to(dt)
    if case["kind"] == "linear":
        s["residual"] = _activations(g, M, N).mul_(3.0).to(dt) if case["residual"] else None
        s["gate"] = (0.3 * _randn(g, -(-M // case["rows"]), N)).to(dt) if case["rows"] else None
        s["alpha"] = 0.9
    return s


def prepare(case, seed):
    make = _prepare_recur if case["kind"] == "recur" else _prepare_product
    return dict(make(case, _gen(seed), DTYPES[case["dtype"]]), case=case)


# ---------------------------------------------------------------- plain forms

def _split(s):
    """Queries, keys and values (T, heads, dim) of the projection's output."""
    c = s["case"]
    Hk, Dk, H, Dv = c["Hk"], c["Dk"], c["H"], c["Dv"]
    q, k, v = s["qkv"].split([Hk * Dk, Hk * Dk, H * Dv], 1)
    return q.unflatten(1, (Hk, Dk)), k.unflatten(1, (Hk, Dk)), v.unflatten(1, (H, Dv))


def _plain_recur(s):
    """By chunks of tokens: products within a chunk, a state for each chunk, and
    a matrix of decays from chunk to chunk."""
    c, dt = s["case"], s["qkv"].dtype
    B, H, Hk, Dk, Dv = (c[n] for n in ("B", "H", "Hk", "Dk", "Dv"))
    C = max(1, min(CHUNK, s["max_new"]))
    N = max(1, -(-s["max_new"] // C))
    cu = s["cu"].long()
    i = torch.arange(N * C, device=DEVICE)
    here = i < (cu[1:] - cu[:-1])[:, None]                                   # [B][N C]
    rows = (cu[:-1, None] + i).clamp(max=max(s["qkv"].shape[0] - 1, 0))

    def padded(x):  # (T, heads, dim) -> [B][H][N][C][dim], zeros past a sequence's end
        x = x.float().repeat_interleave(H // x.shape[1], 1)[rows] * here[..., None, None]
        return x.view(B, N, C, H, -1).permute(0, 3, 1, 2, 4).contiguous()

    q, k, v = (padded(x) for x in _split(s))
    g = s["decay"].double()
    g = (g[rows] if c["by"] == "token" else g.expand(B, N * C, H)) * here[..., None]
    G = g.view(B, N, C, H).permute(0, 3, 1, 2).cumsum(-1)                    # [B][H][N][C]
    R = G[..., -1].cumsum(-1)                                                # [B][H][N], all chunks up to this one
    S0 = s["state"][s["slot"].long()]
    S0 = S0 * (s["len"].long() > cu[1:] - cu[:-1])[:, None, None, None]
    to_end = (G[..., -1:] - G).exp().float()
    U = (k * to_end[..., None]).transpose(-1, -2).contiguous() @ v           # a chunk's own part of the state
    before = (R - G[..., -1])[..., :, None] - R[..., None, :]                # from the end of chunk m to the start of n
    W = torch.where(torch.ones(N, N, device=DEVICE).tril(-1) > 0, before, -math.inf).exp().float()
    start = (W @ U.view(B, H, N, Dk * Dv)).view(B, H, N, Dk, Dv)
    start = start + (R - G[..., -1]).exp().float()[..., None, None] * S0[:, :, None]
    causal = torch.ones(C, C, device=DEVICE).tril() > 0
    P = (q @ k.transpose(-1, -2).contiguous()) * torch.where(causal, G[..., :, None] - G[..., None, :], -math.inf).exp().float()
    o = (P @ v + G.exp().float()[..., None] * (q @ start)) * Dk ** -0.5
    o = o.permute(0, 2, 3, 1, 4).reshape(B, N * C, H, Dv)[here].to(dt)
    end = G[..., -1, None, None].exp().float()[:, :, -1] * start[:, :, -1] + U[:, :, -1]
    some = cu[1:] > cu[:-1]
    s["state"][s["slot"].long()[some]] = end[some]
    return dict(o=o, state=s["state"])


def _act(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z


def _plain_product(s):
    x, xs = s["x"].float(), s["xs"]
    if xs is None:
        xs = x.abs().amax(1) / 127
        x = torch.where(xs[:, None] > 0, torch.round(x / xs[:, None]), 0.0)
    z = (x @ s["w"].float().t()) * xs[:, None] * s["ws"]
    return z if s["bias"] is None else z + s["bias"]


def _plain_linear(s):
    c = s["case"]
    y = _act(_plain_product(s), c["act"])
    if s["gate"] is not None:
        y = y * s["gate"].float()[torch.arange(c["M"], device=DEVICE) // c["rows"]]
    if s["residual"] is not None:
        y = y + s["alpha"] * s["residual"].float()
    return y.to(DTYPES[c["dtype"]])


def _plain_gated(s):
    z, N = _plain_product(s), s["case"]["N"]
    return (_act(z[:, :N], s["case"]["act"]) * z[:, N:]).to(DTYPES[s["case"]["dtype"]])


# ---------------------------------------------------------------- the framework's operators

_kept = {}


def _framework(need):
    """The binding and the one context of this program, whose workspace grows
    to what a call asks for."""
    from paper_2609_31938_amd import c3c, tokens
    if "ctx" not in _kept:
        _kept.update(ctx=c3c.Context(), bytes=0)
    n = need(tokens)
    if n > _kept["bytes"]:
        _kept["ctx"].set_workspace(torch.empty(n, dtype=torch.uint8, device=DEVICE))
        _kept["bytes"] = n
    return tokens, _kept["ctx"]


def _own_recur(s):
    c = s["case"]
    q, k, v = _split(s)
    if "plan" not in s:
        # the states and the batch, as the program keeps them over a step
        from paper_2609_31938_amd import tokens
        table = torch.empty(c["B"], 0, dtype=torch.int32, device=DEVICE)
        s["plan"] = (tokens.StateCache(s["state"]),
                     tokens.Batch(table, s["cu"], s["len"], max_new=s["max_new"], max_len=s["max_len"]))
        _framework(lambda t: t.linear_attention_workspace_bytes(*s["plan"], q))
    states, batch = s["plan"]
    tokens, ctx = _framework(lambda t: 0)
    o = tokens.linear_attention(ctx, states, batch, q, k, v, s["decay"], slots=s["slot"])
    return dict(o=o, state=s["state"])


def _own_linear(s):
    c = s["case"]
    if "plan" not in s:
        _framework(lambda t: t.linear_i8_workspace_bytes(c["M"], c["N"], c["K"], "i8" if c["pre"] else c["dtype"], c["dtype"]))
        s["plan"] = True
    tokens, ctx = _framework(lambda t: 0)
    return tokens.linear_i8(ctx, s["x"], s["w"], s["ws"], bias=s["bias"], x_scale=s["xs"], out_dtype=c["dtype"], act=c["act"],
                            residual=s["residual"], gate=s["gate"], alpha=s["alpha"], rows_per_gate=c["rows"] or 1)


def _own_gated(s):
    c = s["case"]
    if "plan" not in s:
        _framework(lambda t: t.gated_linear_i8_workspace_bytes(c["M"], c["N"], c["K"], "i8" if c["pre"] else c["dtype"], c["dtype"]))
        s["plan"] = True
    tokens, ctx = _framework(lambda t: 0)
    return tokens.gated_linear_i8(ctx, s["x"], s["w"], s["ws"], bias=s["bias"], x_scale=s["xs"], out_dtype=c["dtype"], act=c["act"])


_PLAIN = dict(recur=_plain_recur, linear=_plain_linear, gated=_plain_gated)
_OWN = dict(recur=_own_recur, linear=_own_linear, gated=_own_gated)


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# ---------------------------------------------------------------- definitions in 64 bits

def _exact_recur(s):
    """Token by token, all sequences and heads side by side."""
    c = s["case"]
    new, old = _lengths(c)
    H, Hk, Dk, Dv = (c[n] for n in ("H", "Hk", "Dk", "Dv"))
    q, k, v = s["qkv"].double().tensor_split([Hk * Dk, 2 * Hk * Dk], 1)
    q, k = (x.reshape(-1, Hk, Dk) for x in (q, k))
    v = v.reshape(-1, H, Dv)
    group = torch.arange(H, device=DEVICE) // (H // Hk)
    a = torch.exp(s["decay"].double())
    out, state = torch.zeros_like(v), s["state"].double()
    first, slot = s["cu"].tolist(), s["slot"].tolist()
    S = torch.stack([state[slot[b]] if old[b] else torch.zeros_like(state[0]) for b in range(c["B"])])
    for t in range(max(new)):
        live = [b for b in range(c["B"]) if t < new[b]]
        at = torch.tensor([first[b] + t for b in live], device=DEVICE)
        on = slice(None) if len(live) == c["B"] else torch.tensor(live, device=DEVICE)
        now = S[on]
        now = now * (a[at] if c["by"] == "token" else a.expand(len(live), H))[..., None, None]
        now += k[at][:, group].unsqueeze(-1) * v[at].unsqueeze(-2)
        out[at] = (q[at][:, group].unsqueeze(-1) * now).sum(-2) / math.sqrt(Dk)
        S[on] = now
    for b in range(c["B"]):
        if new[b]:
            state[slot[b]] = S[b]
    return dict(o=out, state=state)


def _exact_act(z, act):
    if act == "silu":
        return z * torch.special.expit(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.special.expit(math.sqrt(8 / math.pi) * (z + 0.044715 * z * z * z))
    return z


def _exact_product(s, first, last):
    """Output channels first to last of the product with its bias."""
    x = s["x"].double()
    if s["xs"] is not None:
        xs = s["xs"].double()
    else:
        xs = x.abs().max(1).values / 127
        x = (x / xs[:, None]).nan_to_num(0.0).round()
    y = torch.mm(x, s["w"][first:last].double().t().contiguous()) * torch.outer(xs, s["ws"][first:last].double())
    return y if s["bias"] is None else y + s["bias"][first:last].double()


def _exact_linear(s):
    c = s["case"]
    y = _exact_act(_exact_product(s, 0, c["N"]), c["act"])
    if s["gate"] is not None:
        y *= s["gate"].double().repeat_interleave(c["rows"], 0)[:c["M"]]
    return y if s["residual"] is None else torch.add(y, s["residual"].double(), alpha=s["alpha"])


def _exact_gated(s):
    N = s["case"]["N"]
    return _exact_act(_exact_product(s, 0, N), s["case"]["act"]) * _exact_product(s, N, 2 * N)


def exact(case, seed):
    if case["kind"] == "recur":
        # a step's launches, or four passes over the states in 64 bits at 3 TB/s
        step = max(2e-4, 4 * 16 * case["B"] * case["H"] * case["Dk"] * case["Dv"] / 3e12)
        if max(_lengths(case)[0]) * step > 15:
            return None
    return dict(recur=_exact_recur, linear=_exact_linear, gated=_exact_gated)[case["kind"]](prepare(case, seed))
