"""Plain forms of the token operators for the tests: numpy, 64 bits unless a
rule is stated in fp32 (scales and codes), sequence by sequence, written from
the definitions in include/c3c_tokens.h."""
import numpy as np
import torch

# unit roundoff of the output types, and the spacing of their subnormals
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 0.0, "f16": 2.0 ** -24, "f32": 0.0}
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS32 = 2.0 ** -24


def f64(t):
    return t.detach().cpu().double().numpy()


def randn(seed, *shape, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(device)


def assert_within(got, ref, tol, what=""):
    """Elementwise |got - ref| <= tol, with NaN and infinities where ref has them."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (what, "NaN differ")
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), (what, "infinities differ")
    fin = np.isfinite(ref)
    err, tol = np.abs(got - ref)[fin], np.broadcast_to(tol, ref.shape)[fin]
    if err.size:
        worst = np.argmax(err - tol)
        assert err[worst] <= tol[worst], (what, err[worst], tol[worst])


# ---------------------------------------------------------------- 8-bit rows

def quantize(x):
    """(codes int8, scale fp32) of x (rows, n) by the rule, in fp32."""
    x = f64(x).astype(np.float32)
    top = np.abs(x).max(1)
    ok = np.isfinite(x).all(1)
    with np.errstate(all="ignore"):
        s = np.where(ok, top / np.float32(127), np.float32(np.nan)).astype(np.float32)
        q = np.rint(x / s[:, None])
    q = np.where(s[:, None] > 0, np.clip(q, -127, 127), 0)
    return q.astype(np.int8), s


# ---------------------------------------------------------------- norms

def norm_gate(h, y, gate, post, pre, alpha, eps, rows):
    """(h', u, size of h's terms, size of u's terms) in 64 bits."""
    h = f64(h)
    size = np.abs(alpha * h)
    new = alpha * h
    if y is not None:
        y = f64(y)
        if post is not None:
            y = f64(post) * y / np.sqrt((y * y).mean(1, keepdims=True) + eps)
        if gate is not None:
            y = y * f64(gate)[np.arange(h.shape[0]) // rows]
        new, size = new + y, size + np.abs(y)
    if pre is None:
        return new, None, size, None
    r = f64(pre) / np.sqrt((new * new).mean(1, keepdims=True) + eps)
    # an error of h' reaches u directly and through the mean (relative size of the row's errors)
    with np.errstate(all="ignore"):
        through = np.sqrt((size * size).mean(1, keepdims=True) / ((new * new).mean(1, keepdims=True) + eps))
    return new, new * r, size, np.abs(r) * size + np.abs(new * r) * through


# ---------------------------------------------------------------- the cache

def e4m3_table():
    return f64(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float())


def to_e4m3(x):
    """Nearest e4m3 code (ties to even) of fp32 values of at most 448; NaN for
    what is not finite."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    code = t.to(torch.float8_e4m3fn).view(torch.uint8).numpy().copy()
    code[~np.isfinite(x)] = 0x7F
    return code


def exponent(top):
    e = -126
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def rotate(x, cos, sin, at, pairs):
    """x (heads, dim) fp32 by row ``at`` of the fp32 tables, rounded after
    every product and sum."""
    x = x.astype(np.float32).copy()
    half = cos.shape[1]
    if at < 0 or at >= cos.shape[0]:
        x[:] = np.nan
        return x
    i = np.arange(half)
    a, b = (i, i + half) if pairs == "half" else (2 * i, 2 * i + 1)
    c, s = cos[at], sin[at]
    u, v = x[:, a].copy(), x[:, b].copy()
    x[:, a], x[:, b] = u * c - v * s, v * c + u * s
    return x


class Pages:
    """Host copy of a cache, k and v both as (pages, heads, tokens, dim) codes."""

    def __init__(self, cache):
        self.page, self.heads, self.dim = cache.page, cache.heads, cache.dim
        self.k = cache.k.view(torch.uint8).cpu().numpy().copy()
        v = cache.v.view(torch.uint8).cpu().numpy()
        self.v = v.transpose(0, 1, 2, 4, 3).reshape(self.k.shape).copy()
        self.ks, self.vs = cache.k_scale.cpu().numpy().copy(), cache.v_scale.cpu().numpy().copy()

    def append(self, table, start, k, v):
        """Stores k, v (tokens, heads, dim) fp32 at the places from start on."""
        nb = self.page // 16
        n = len(k)
        for p0 in range(start // 16 * 16, start + n if n else 0, 16):
            lo, hi = max(p0, start), min(p0 + 16, start + n)
            col = p0 // self.page
            if p0 < 0 or col >= len(table) or not 0 <= table[col] < len(self.k):
                continue
            pg, at, blk = table[col], p0 % self.page, p0 % self.page // 16
            for codes, scale, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
                for h in range(self.heads):
                    new = x[lo - start:hi - start, h]
                    fin = np.where(np.isfinite(new), np.abs(new), 0)
                    e = exponent(float(fin.max()))
                    if lo > p0:
                        old = int(np.log2(scale[pg, h, blk]))
                        e = max(e, old)
                        was = e4m3_table()[codes[pg, h, at:at + lo - p0]].astype(np.float64) * 2.0 ** (old - e)
                        codes[pg, h, at:at + lo - p0] = to_e4m3(was)
                    scale[pg, h, blk] = 2.0 ** e
                    codes[pg, h, at + lo - p0:at + hi - p0] = to_e4m3(new.astype(np.float64) * 2.0 ** -e)

    def values(self, table, length):
        """(k, v, valid): 64-bit values (tokens, heads, dim) of a sequence, and
        which tokens have a page."""
        nb, t = self.page // 16, e4m3_table()
        length = max(0, min(length, len(table) * self.page))
        k = np.zeros((length, self.heads, self.dim))
        v = np.zeros_like(k)
        ok = np.zeros(length, bool)
        for p in range(length):
            pg, at = table[p // self.page], p % self.page
            if 0 <= pg < len(self.k):
                ok[p] = True
                k[p] = t[self.k[pg, :, at]] * self.ks[pg, :, at // 16, None]
                v[p] = t[self.v[pg, :, at]] * self.vs[pg, :, at // 16, None]
        return k, v, ok


def attend(q, k, v, ok, length, scale, causal, window):
    """One sequence in 64 bits: q (n, q_heads, dim) are its last n tokens.
    Returns out, lse, and the tolerance terms sum p |v| and the largest score
    with the size of its terms."""
    n, qh, dim = q.shape
    G = qh // k.shape[1]
    out, lse = np.zeros(q.shape), np.full((n, qh), -np.inf)
    mix, big, size = np.zeros(q.shape), np.zeros((n, qh, 1)), np.zeros((n, qh, 1))
    j = np.arange(len(k))
    for i in range(n):
        p = length - n + i
        see = ok.copy()
        if causal:
            see &= j <= p
        if window:
            see &= j > p - window
        if not see.any():
            continue
        for h in range(qh):
            kk, vv = k[see, h // G], v[see, h // G]
            s = kk @ q[i, h] * scale
            m = s.max()
            w = np.exp(s - (0 if np.isnan(m) else m))
            out[i, h] = w @ vv / w.sum()
            lse[i, h] = m + np.log(w.sum())
            mix[i, h] = (w / w.sum()) @ np.abs(vv)
            big[i, h] = np.abs(s).max()
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, lse, mix, big, size


def attend_tolerance(dtype, ref, mix, big, size, dim):
    """Output rounding; a probability's rounding to bf16 terms (1, 2 or 3 of
    them); errors of the fp32 score (its sum of dim products) and of the
    hardware exponential's argument, which are relative errors of p.  Both
    enter numerator and denominator, hence the factor 2."""
    terms = {"bf16": 2.0 ** -9, "f16": 2.0 ** -17, "f32": 2.0 ** -24}[dtype]
    score = EPS32 * (dim / 8 + 8) * size + 4 * EPS32 * (1.5 * big + 1)
    return UNIT[dtype] * np.abs(ref) + (terms + 2 * score + 32 * EPS32) * mix + TINY[dtype]
