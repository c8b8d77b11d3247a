"""Attention over the 4-bit cache where the softmax is hard: weights far below a row's largest, and maxima that move.

Every key has its first block of 32 dimensions aimed at the queries' first block, so that a count 0 .. 32 sets its score;
the other dimensions are random.  The bar is test_gpu_kvq's, from the roundings: scores and sums in fp32, a weight
rounded once to 11 bits (bf16 queries; fp32: 24), the output's own rounding; all but the last relative to sum p|v|,
whatever the size of p.  What may be dropped besides are weights below 2^-50 of a row's largest: vmax 2^-50 a key.
"""
import numpy as np
import pytest

from oracle import kvq as okvq
from tests.test_gpu_kvq import DEV, Setup, _f64, _room

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _bar(ref, mag, top, ctx, hd, dtype, vmax):
    u = 2.0 ** -24
    e_p = (hd + 6) * u * top[..., None] + 2.0 ** -21
    p, out = (2.0 ** -11, 2.0 ** -8) if dtype == "bf16" else (u, u)
    return out * np.abs(ref) * (1 + 2.0 ** -7) + mag * (2 * e_p + 2 * (ctx + 64) * u + p) * 1.01 + ctx * vmax * 2.0 ** -50 + 1e-37


def _check(s, out):
    out, q, held, at = _f64(out), _f64(s.q), s.held(), 0
    for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
        if n:
            k, v = held[b]
            ref, mag, top = okvq.attend(q[at:at + n], k, v, np.arange(c - n, c), s.hd ** -0.5)
            err, bar = np.abs(out[at:at + n] - ref), _bar(ref, mag, top, c, s.hd, s.dtype, np.abs(v).max(initial=0))
            assert (err <= bar).all(), (b, c, n, float((err / bar).max()), np.argwhere(~(err <= bar))[:4].tolist())
        at += n


def _aim(s, counts, nats):
    """Scores of counts[b][t] / 32 * nats for token t of sequence b, besides the random part."""
    n = torch.from_numpy(np.concatenate(counts)).to(DEV)
    s.k[:, :, :32] = 4.0 * (torch.arange(32, device=DEV) < n[:, None])[:, None, :].to(s.dt)
    s.q[:, :, :32] = nats * s.hd ** 0.5 / 128
    return s


# n_q, n_kv, hd, contexts, rows, bounds: the kernel for few columns with 4 waves, 1 and 8, its pages in one item and in
# several; the one for many, whole tiles, split ones, and of 8 waves
FORMS = {
    "four": (7, 1, 128, [1024, 700, 130, 64, 1], [1, 9, 2, 1, 1], ""),
    "four-64": (6, 2, 64, [1000, 640, 65, 30], [1, 3, 1, 7], ""),
    "one": (64, 64, 64, [512, 130] + [1] * 62, None, ""),
    "eight-waves": (12, 4, 128, [1300, 1100] + [3] * 62, None, ""),
    "joined": (7, 1, 128, [5000], [1], ""),
    "joined-64": (14, 2, 64, [4300, 900], [2, 1], ""),
    "prompt-tiles": (28, 4, 128, [900, 130, 40], [60, 40, 1], "tiles"),
    "prompt-tiles-64": (14, 2, 64, [900, 130, 40], [60, 130, 1], "tiles"),
    "prompt-split": (28, 4, 128, [1300, 130], [40, 90], "split"),
    "prompt-split-64": (14, 2, 64, [1300, 130], [40, 90], "split"),
    "prompt-eight": (28, 4, 128, [1300, 130], [60, 40], "eight"),
}


def _setup(form, dtype, seed):
    n_q, n_kv, hd, ctx, rows, kind = FORMS[form]
    return Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=seed, room=_room(kind, n_q, hd))


def _types(form):
    return ("bf16",) if form.startswith("prompt") else ("bf16", "f32")


@pytest.mark.parametrize("form", FORMS)
def test_weights_far_below_the_largest(form):
    """One key carries the weight and its value is zero: the output is made of weights of any size."""
    for dtype in _types(form):
        for nats in (10.0, 13.0, 16.0, 27.0):
            s = _setup(form, dtype, 41)
            off, counts = np.concatenate([[0], np.cumsum(s.ctx)]), []
            for b, c in enumerate(s.ctx):
                at = 0 if b % 2 == 0 else c // 2  # the first key, or one with smaller ones before it
                counts.append(np.where(np.arange(c) == at, 32, 0))
                s.v[off[b] + at] = 0
            _aim(s, counts, nats).fill()
            _check(s, s.cache.attend(s.batch(), s.q))


@pytest.mark.parametrize("form", ["four", "four-64", "prompt-tiles", "prompt-split-64", "prompt-eight"])
def test_strong_keys_everywhere(form):
    """Strong keys with a value of zero in all pages: the weights beside them are off by 2^-11 of what the keys around them weigh
    together at most (include/rollpack.h), times the largest of their values."""
    for nats in (12.0, 18.0, 27.0):
        s = _setup(form, "bf16", 47)
        pos = np.concatenate([np.arange(c) for c in s.ctx])
        s.v[torch.from_numpy(pos % 11 == 3).to(DEV)] = 0
        _aim(s, [np.where(np.arange(c) % 11 == 3, 32, 0) for c in s.ctx], nats).fill()
        out, q, at, g = _f64(s.cache.attend(s.batch(), s.q)), _f64(s.q), 0, s.n_q // s.n_kv
        for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
            k, v = s.held()[b]
            ref, mag, top = okvq.attend(q[at:at + n], k, v, np.arange(c - n, c), s.hd ** -0.5)
            bar = _bar(ref, mag, top, c, s.hd, "bf16", np.abs(v).max())
            for h in range(s.n_q):
                z = np.where(np.arange(c)[None] <= np.arange(c - n, c)[:, None], q[at:at + n, h] @ k[:, h // g].T * s.hd ** -0.5, -np.inf)
                p = np.exp(z - z.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                pad = -(-c // 64) * 64 - c
                around = np.pad(p, ((0, 0), (0, pad))).reshape(n, -1, 64).sum(-1)                         # of a page
                most = np.pad(np.abs(v[:, h // g]), ((0, pad), (0, 0))).reshape(-1, 64, s.hd).max(1)
                bar[:, h] += 2.0 ** -11 * around @ most
            assert (np.abs(out[at:at + n] - ref) <= bar).all(), (b, c, n, nats)
            at += n


def test_many_keys_beside_a_dominant_one():
    """A tenth of a percent of the weight in 40,000 keys of a wave, each about 2^-25 of the first, whose value is zero."""
    s = Setup(2, 1, 64, [40000] + [1] * 257, seed=42)
    s.v[:, 0] = 1.0 + s.v[:, 0].abs()
    s.v[0] = 0
    _aim(s, [np.where(np.arange(40000) == 0, 32, 0)] + [np.zeros(1)] * 257, 18.0).fill()
    _check(s, s.cache.attend(s.batch(), s.q))


STEPS = {
    "steep": lambda page: np.minimum(32, 5 * page),   # ~14 bits a page
    "slow": lambda page: np.minimum(32, page),        # ~3
    "down": lambda page: np.maximum(0, 32 - 5 * page),
    "spikes": lambda page: np.where(page % 3 == 2, 32, 0),
    "mixed": lambda page: (page * 2654435761 >> 7) % 33,
}


@pytest.mark.parametrize("form", FORMS)
def test_maxima_that_move(form):
    """Scores that rise, fall or jump by many bits from page to page: what was summed before is rescaled, once."""
    for dtype in _types(form):
        for step in STEPS.values():
            s = _setup(form, dtype, 43)
            _aim(s, [step(np.arange(c) // 64) for c in s.ctx], 64.0).fill()
            _check(s, s.cache.attend(s.batch(), s.q))


@pytest.mark.parametrize("form", [f for f in FORMS if f not in ("one", "eight-waves")])
def test_values_beyond_half_precision_after_a_move(form):
    """Values that fp16 does not hold from the middle of each sequence on, after the reference has moved and with small
    weights on both sides."""
    for step in ("slow", "mixed"):
        s = _setup(form, "bf16", 44)
        off = np.concatenate([[0], np.cumsum(s.ctx)])
        _aim(s, [STEPS[step](np.arange(c) // 64) for c in s.ctx], 64.0)
        for b, c in enumerate(s.ctx):
            s.v[off[b] + c // 2:off[b + 1]:7] *= 2.0 ** 30
            s.v[off[b] + c // 2 + 3:off[b + 1]:11] *= 2.0 ** -40
        s.fill()
        _check(s, s.cache.attend(s.batch(), s.q))


@pytest.mark.parametrize("kind", ["", "tiles", "split", "eight"])
def test_large_scores_have_the_right_values(kind):
    """Scores in the thousands: one key takes nearly all of the weight, and which one changes all the time."""
    for dtype in ("bf16", "f32"):
        s = Setup(7, 1, 128, [700, 65, 1], rows=[30 if kind else 3, 65, 1], dtype=dtype, seed=45, gain=6.0, room=_room(kind, 7, 128)).fill()
        s.q *= 4
        _check(s, s.cache.attend(s.batch(), s.q))


@pytest.mark.parametrize("form", ["four", "joined-64", "prompt-tiles", "prompt-eight"])
def test_values_near_the_end_of_the_range(form):
    """Sums stay finite while the largest value times the context is below 2^119 (include/rollpack.h)."""
    for dtype in _types(form):
        s = _setup(form, dtype, 46)
        s.v *= 2.0 ** (118 - 13 - 3)  # contexts below 2^13, values below 2^3
        s.q *= 0.25
        s.fill()
        _check(s, s.cache.attend(s.batch(), s.q))
