"""Plain forms of a recurrent layer's operators for the tests: numpy, 64 bits,
token by token, written from the definitions in include/c3c_layers.h; and the
bounds that their kernels' roundings keep."""
import math

import numpy as np

from token_ref import EPS32, TINY, UNIT, f64


def linear_attention(q, k, v, g, S, scale):
    """One sequence: q, k (n, qk_heads, Dk), v (n, heads, Dv), g (n, heads), S
    (heads, Dk, Dv).  Returns out, S, and for each the sizes of its terms: their
    absolute sum, and that with every term times the sum of |g| that it has
    decayed by."""
    n, heads, _ = v.shape
    group = np.arange(heads) // (heads // q.shape[1])
    S, M = S.copy(), np.abs(S)
    G = np.zeros_like(M)
    out, om, og = (np.zeros(v.shape) for _ in range(3))
    with np.errstate(all="ignore"):
        for t in range(n):
            a = np.exp(g[t])[:, None, None]
            far = np.where(a > 0, np.abs(g[t])[:, None, None], 0)
            kv = k[t][group][:, :, None] * v[t][:, None, :]
            S, G, M = a * S + kv, a * (G + far * M), a * M + np.abs(kv)
            qt = q[t][group][:, :, None]
            out[t], om[t], og[t] = (scale * (x * y).sum(1) for x, y in ((qt, S), (np.abs(qt), M), (np.abs(qt), G)))
    return out, S, (np.abs(om), np.abs(og)), (M, G)


def attention_tolerance(dtype, ref, sizes, n, dim_k):
    """Rounding of the output; of the operands' bf16 terms: 2 terms hold 2^-18
    of a value, and the product of two second terms is left out (2^-18), at most
    four of these on a path (q k, P or S, its product with v or q), and 3 terms
    with the six largest products err by less than 2^-24 each; of the fp32 sums
    (any order of n terms errs by at most n roundings: dim_k products, n tokens, a
    decay and a sum for every chunk of 32); of the decays' exponentials, whose
    argument's rounding grows with it (log2(e) < 1.5, two roundings)."""
    terms = {"bf16": 2.0 ** -16, "f16": 2.0 ** -16, "f32": 4 * EPS32}[dtype]
    sums = EPS32 * (dim_k + n + 6 * (n / 32 + 1) + 16)
    return UNIT[dtype] * np.abs(ref) + (terms + sums) * sizes[0] + 4 * EPS32 * sizes[1] + TINY[dtype]


def state_tolerance(n, sizes):
    """3 terms hold all bits of a weighted value; its rounding, and the sums and
    decays as for the outputs."""
    return EPS32 * (n + 6 * (n / 32 + 1) + 16) * sizes[0] + 4 * EPS32 * sizes[1]


def quantize(x):
    """(codes, scale fp32) of x (rows, n): the integers nearest to 127 x / max|x|."""
    x = f64(x)
    top = np.abs(x).max(1)
    s = (top.astype(np.float32) / np.float32(127)).astype(np.float32)
    with np.errstate(all="ignore"):
        q = np.where(s[:, None] > 0, np.rint(x * 127 / top[:, None]), 0)
    return q.astype(np.int8), s


def act(z, name):
    """(act(z), bound on the relative error of its fp32 form without the
    argument's, bound on the absolute one)"""
    with np.errstate(all="ignore"):
        if name == "silu":
            return z / (1 + np.exp(-z)), (6 + 3 * np.abs(z)) * EPS32, 0
        if name == "gelu":
            return 0.5 * z * np.vectorize(math.erfc)(-z / math.sqrt(2)), 4 * EPS32, 4 * EPS32 * np.abs(z)
        if name == "gelu_tanh":
            u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
            return z / (1 + np.exp(-u)), (6 + 8 * np.abs(u)) * EPS32, 0
    return z, 0, 0


def product(q, s, w, ws, bias):
    """(z, bound on the error of its fp32 form): exact integer sums, their
    conversion, two products and a sum."""
    z = (q.astype(np.float64) @ f64(w).T) * s.astype(np.float64)[:, None] * f64(ws)
    size = np.abs(z)
    if bias is not None:
        z, size = z + f64(bias), size + np.abs(f64(bias))
    return z, 4 * EPS32 * size


def epilogue(z, err, name, gate, residual, alpha, dtype):
    """(y, tolerance).  No act's slope exceeds 1.13."""
    a, rel, off = act(z, name)
    err = 1.2 * err + np.abs(a) * rel + off if name != "none" else err
    y = a
    if gate is not None:
        y, err = y * gate, np.abs(gate) * (err + EPS32 * np.abs(a))
    if residual is not None:
        y = y + alpha * residual
        err = err + 2 * EPS32 * (np.abs(alpha * residual) + np.abs(y))
    return y, UNIT[dtype] * np.abs(y) + err + TINY[dtype]
