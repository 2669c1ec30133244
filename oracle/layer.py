"""Oracle of the operators around the matmuls: paged KV cache, attention over it,
gated residual norms.  Plain NumPy in float64, from the definitions.

Parity unpinned: the paper has no values for these operators; closed forms and
special cases in the CPU tests pin this file.
"""

from __future__ import annotations

import numpy as np

LEVELS = {"int8": 255, "int4": 15}


def bf16_ceil(x):
    """The smallest bf16 not below x > 0 (float64 in, float64 out)."""
    m, e = np.frexp(np.asarray(x, np.float64))
    e = np.maximum(e, -125)                     # bf16 subnormals share the exponent of 2^-126
    return np.ldexp(np.ceil(np.ldexp(x, 8 - e)), e - 8)


def quantise_rows(x, kind):
    """Rows x [..., D] (values of bf16 numbers) -> codes, scale, zero-point."""
    x = np.asarray(x, np.float64)
    top = LEVELS[kind]
    with np.errstate(invalid="ignore", over="ignore"):
        hi = np.maximum(x.max(-1, keepdims=True), 0.0)
        lo = np.minimum(x.min(-1, keepdims=True), 0.0)
        span = (hi - lo).astype(np.float32).astype(np.float64)
    bad = ~np.isfinite(span) | ~np.isfinite(x).all(-1, keepdims=True)
    safe = np.where(bad | (span == 0), 1.0, span)
    s = np.where(span == 0, 1.0, bf16_ceil(safe / top))
    with np.errstate(invalid="ignore"):
        z = np.clip(np.rint(-np.where(bad, 0.0, lo) / s), 0, top)
        c = np.clip(np.rint(np.where(bad, 0.0, x) / s) + z, 0, top)
    return c, np.where(bad, np.nan, s), z


def held_rows(x, kind):
    """What a cache of this kind holds of rows x."""
    x = np.asarray(x, np.float64)
    if kind == "bf16":
        return x
    c, s, z = quantise_rows(x, kind)
    return s * (c - z)


def visible(p, n_keys, window, sinks):
    """Which of keys 0 .. n_keys - 1 a token at position p sees."""
    j = np.arange(n_keys)
    see = j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def attention_row(q, k, v, see, scale):
    """One row: q [D], k, v [S][D], see [S] -> (o [D], lse, sum w |v| [D], max score
    magnitude sum |q||k| scale).  Keys that are not seen take no part at all."""
    k, v = k[see], v[see]
    if k.shape[0] == 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), 0.0
    with np.errstate(all="ignore"):
        t = scale * (k @ q)
        top = t.max()
        if top == -np.inf:
            return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), 0.0
        w = np.exp(t - top)
        lse = top + np.log(w.sum())
        w = w / w.sum()
        o = np.where(w[:, None] == 0, 0.0, w[:, None] * v).sum(0) if np.isfinite(v).all() else \
            (w[:, None] * v).sum(0)
        return o, lse, w @ np.abs(v), float((np.abs(k) @ np.abs(q)).max() * abs(scale))


def gated_residual_norm(x, residual, pre, post, gate, alpha, eps):
    """(r, h, |alpha residual| + |gate u|)."""
    u = np.asarray(x, np.float64)
    if post is not None:
        u = u / np.sqrt((u * u).mean(-1, keepdims=True) + eps) * post
    if gate is not None:
        u = gate * u
    res = np.zeros_like(u) if residual is None else alpha * np.asarray(residual, np.float64)
    r = res + u
    h = None if pre is None else r / np.sqrt((r * r).mean(-1, keepdims=True) + eps) * pre
    return r, h, np.abs(res) + np.abs(u)
