"""Plain 64-bit implementations of the block operators, written from their formulas, and error bounds for them
(derived from the formulas and the types' roundoff, element by element).  No code of the package is used."""
import math

import numpy as np

U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}      # half a unit in the last place
SMALLEST = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


def philox(seed, counter):
    """Philox 4x32-10: four words from a 64-bit key and a 64-bit counter (Salmon et al., 2011)."""
    return philox_words([counter & 0xFFFFFFFF, counter >> 32, 0, 0], [seed & 0xFFFFFFFF, seed >> 32])


def philox_words(c, k):
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_factors(rows, cols, p, seed, offset=0):
    """dropout factor of every element, float64 [rows][cols]"""
    cut = int(p * 65536 + 0.5)
    e = np.arange(offset, offset + rows * cols, dtype=object)
    words = {}
    out = np.empty(rows * cols)
    for i, v in enumerate(e):
        b = v // 8
        if b not in words:
            words = {b: philox(seed, b)} if len(words) > 4 else {**words, b: philox(seed, b)}
        w = words[b][(v % 8) // 2]
        bits = (w >> 16) if v % 2 else (w & 0xFFFF)
        out[i] = 0.0 if bits < cut else 65536.0 / (65536 - cut)
    return out.reshape(rows, cols)


def unit(v, kind, eps):
    v = v - v.mean(1, keepdims=True) if kind == "layer" else v
    return v / np.sqrt((v * v).mean(1, keepdims=True) + eps)


def norm_forward(x, y, w_post, w_pre, gate, per, alpha, keep, kind, eps):
    out = alpha * x
    if y is not None:
        n = y if w_post is None else unit(y, kind, eps) * w_post
        g = 1.0 if gate is None else gate[np.arange(len(x)) // per]
        out = out + np.where(keep > 0, g * n * keep, 0.0)
    return out, None if w_pre is None else unit(out, kind, eps) * w_pre


def act(name, h):
    """act, act', a bound of |act''|"""
    if name == "silu":
        s = 1 / (1 + np.exp(-h))
        return h * s, s * (1 + h * (1 - s)), 0.5
    if name == "gelu":
        c = 0.5 * (1 + np.vectorize(math.erf)(h / math.sqrt(2))) if h.size else h
        return h * c, c + h * np.exp(-h * h / 2) / math.sqrt(2 * math.pi), 0.8
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = np.tanh(k * (h + 0.044715 * h ** 3))
        return 0.5 * h * (1 + t), 0.5 * (1 + t) + 0.5 * h * (1 - t * t) * k * (1 + 3 * 0.044715 * h * h), 0.9
    return np.maximum(h, 0), (h > 0) * 1.0, 0.0


def ffn(x, wg, wu, wd, name, dy, dtype, grad_dtype=None):
    """{name: (value, error bound)} of the block and its gradients in 64 bits.

    Bounds: a sum of K products in binary32, in any order, is within (K + 8) 2^-23 of the sum of the absolute
    products (2^-23: products may be added with truncation); a binary32 block's operands may carry 2^-22 of
    relative error (a product of operands split into three 16-bit terms); h, u, a, dh and du are rounded to the
    tensors' type; act, act' and the elementwise products add a few units of 2^-22."""
    u, g = U[dtype], U[grad_dtype or dtype]
    tiny = SMALLEST[dtype]
    split = 2.0 ** -21 if dtype == "float32" else 0.0

    def product(a, da, b, db):
        """a b^T with elementwise errors da, db of its operands"""
        aa, ab = np.abs(a), np.abs(b)
        k = a.shape[1]
        return a @ b.T, da @ ab.T + aa @ db.T + da @ db.T + ((k + 8) * 2.0 ** -23 + split) * (aa @ ab.T)

    def rounded(v, dv, by, least=tiny):
        return dv + by * (np.abs(v) + dv) + least

    z = np.zeros_like
    h, eh = product(x, z(x), wg, z(wg))
    t, et = product(x, z(x), wu, z(wu))
    f, df, d2 = act(name, h)
    few = 2.0 ** -19
    ef = np.abs(df) * eh + 0.5 * d2 * eh * eh + few * (np.abs(f) + 0.2 * (np.abs(f) > 0))
    a = f * t
    ea = rounded(a, ef * np.abs(t) + (np.abs(f) + ef) * et, u)
    y, ey = product(a, ea, wd, z(wd))
    r = {"y": (y, rounded(y, ey, u))}
    if dy is None:
        return r
    hs, ts = rounded(h, eh, u), rounded(t, et, u)               # h and u as they are kept
    da, eda = product(dy, z(dy), wd.T.copy(), z(wd.T))
    edf = d2 * hs + few
    if name == "relu":
        edf = np.where(np.abs(h) <= eh + tiny, 1.0, 0.0)        # the step may fall on either side
    edf = np.minimum(edf, 1.3)
    ef = np.minimum(np.abs(df) * hs + 0.5 * d2 * hs * hs, 1.2 * hs) + few * (1 + np.abs(f))

    def scaled(v, ev, s, es):
        return v * s, ev * np.abs(s) + np.abs(v) * es + ev * es

    dh, edh = scaled(*scaled(da, eda, t, ts), df, edf)
    du, edu = scaled(da, eda, f, ef)
    edh, edu = rounded(dh, edh, u), rounded(du, edu, u)
    dx1, e1 = product(dh, edh, wg.T.copy(), z(wg.T))
    dx2, e2 = product(du, edu, wu.T.copy(), z(wu.T))
    # one accumulator may run over both sums
    e = e1 + e2 + (dh.shape[1] + 8) * 2.0 ** -23 * (np.abs(dh) @ np.abs(wg) + np.abs(du) @ np.abs(wu))
    r["dx"] = (dx1 + dx2, rounded(dx1 + dx2, e, u))
    for k, (p, ep, q, eq) in {"dw_gate": (dh, edh, x, z(x)), "dw_up": (du, edu, x, z(x)), "dw_down": (dy, z(dy), a, ea)}.items():
        v, ev = product(p.T.copy(), ep.T.copy(), q.T.copy(), eq.T.copy())
        r[k] = (v, rounded(v, ev, g, SMALLEST[grad_dtype or dtype]))
    return r
