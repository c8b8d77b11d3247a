"""The 4-bit KV cache in plain numpy: its quantiser, and attention over what it holds, in 64 bits.

Definition (include/rollpack.h): blocks of 32 dimensions, a scale s that is the least power of two
with amax <= 7 s (2^-125 <= s <= 2^125), values s times 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign: the
nearest, ties to the even mantissa.  A block with an infinity or a NaN holds NaN.
"""
from __future__ import annotations

import numpy as np

from oracle import model as om

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _nearest(a: np.ndarray) -> np.ndarray:
    """Magnitudes to the nearest grid value; ties to the even index (an even mantissa), beyond 6 to 6."""
    hi = np.clip(np.searchsorted(GRID, a, side="left"), 0, 7)
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0))
    return np.where(a >= 6.0, 6.0, np.where(take_hi, GRID[hi], GRID[lo]))


def held(x) -> np.ndarray:
    """What the cache holds of x [..., hd] (float64)."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, BLOCK)
    finite = np.isfinite(b).all(-1, keepdims=True)
    amax = np.abs(np.where(finite, b, 0.0)).max(-1, keepdims=True)
    e = np.clip(np.frexp(amax)[1] - 4, -125, 125)  # amax >= 2^(e + 3): too small, or at a limit
    for _ in range(4):
        e = np.where((amax > 7.0 * np.ldexp(1.0, e)) & (e < 125), e + 1, e)
    s = np.ldexp(1.0, e)
    with np.errstate(invalid="ignore"):
        v = _nearest(np.abs(b) / s) * s
    return np.where(finite, np.where(np.signbit(b), -v, v), np.nan).reshape(x.shape)


def attend(q, k, v, pos, scale):
    """q [n, n_q, hd] at positions pos [n] over keys k, v [ctx, n_kv, hd] (values, float64).
    Returns (out, weighted |v|, largest |q|.|k| scale over visible keys); rows that see no key give zeros."""
    n, n_q, hd = q.shape
    n_kv = k.shape[1]
    g = n_q // n_kv
    out = np.zeros((n, n_q, v.shape[2]))
    mag = np.zeros_like(out)
    top = np.zeros((n, n_q))
    see = np.arange(k.shape[0])[None, :] <= np.asarray(pos)[:, None]  # [n, ctx]
    some = see.any(1)
    if not some.any():
        return out, mag, top
    for h in range(n_q):
        kk, vv = k[:, h // g], v[:, h // g]
        with np.errstate(invalid="ignore"):
            s = np.where(see, q[:, h] @ kk.T * scale, -np.inf)[some]
            p = np.exp(s - s.max(1, keepdims=True))  # a NaN among a row's scores makes all of it NaN
            p = p / p.sum(1, keepdims=True)
            # a key that a row does not see counts nothing, whatever its value
            out[some, h] = _weigh(p, vv, see[some])
            mag[some, h] = _weigh(p, np.abs(vv), see[some])
            top[some, h] = np.where(see, np.abs(q[:, h]) @ np.abs(kk).T * scale, 0.0)[some].max(1)
    return out, mag, top


def _weigh(p, v, see):
    if np.isfinite(v).all():
        return p @ v
    return np.stack([p[i, see[i]] @ v[see[i]] for i in range(len(p))])


def forward_over_cache(w, shape, tokens, cache):
    """The model's forward over a whole sequence whose attention reads cache[layer] = (K, V) [n, n_kv, hd] (what a
    4-bit cache holds) in the place of its own.  Returns the logits [n, V] and its own (K, V) of every layer."""
    tokens = np.asarray(tokens)
    n = len(tokens)
    pos = np.arange(n)
    cos, sin = om.rope_cos_sin(pos, shape.head_dim, shape.theta)
    x = w["embed"][tokens].astype(np.float64)
    mine = []
    for layer, (ck, cv) in zip(w["layers"], cache):
        h = om.rmsnorm(x, layer["attn_norm"], shape.eps)
        q, k, v = om._qkv(layer, h, shape)
        q, k = om.apply_rope(q, cos, sin), om.apply_rope(k, cos, sin)
        mine.append((k, v))
        x = x + om.attention(q, ck, cv, pos, pos).reshape(n, -1) @ layer["wo"].T
        x = x + om._mlp(layer, x, shape)
    return om.lm_head(w, x, shape), mine
