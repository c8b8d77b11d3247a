"""Attention over picked pages of the 4-bit cache where the softmax is hard: weights far below a row's largest, maxima that move from
page to page, values beyond fp16.  Every page is listed, ascending or in an order of its own, so that the sum is attention's over the
whole context, with its bar (tests/test_gpu_kvq_softmax.py).
"""
import numpy as np
import pytest

from oracle import kvq as okvq
from tests.test_gpu_kvq import DEV, Setup, _f64
from tests.test_gpu_kvq_softmax import STEPS, _aim, _bar, _check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# n_q, n_kv, hd, contexts, rows: up to eight heads and more, blocks of 4 waves, 8 and 2, lists whole and split
FORMS = {
    "four": (7, 1, 128, [1024, 700, 130, 64, 1], [1, 9, 2, 1, 1]),
    "four-64": (6, 2, 64, [1000, 640, 65, 30], [1, 3, 1, 7]),
    "wide": (32, 2, 128, [900, 130, 64, 1], [1, 9, 2, 1]),
    "wide-64": (9, 1, 64, [1000, 640, 65], [1, 3, 1]),
    "eight": (10, 2, 64, [1400, 1100] + [3] * 78, [1] * 80),
    "eight-128": (8, 1, 128, [1400, 130] + [3] * 148, [1] * 150),
    "two": (28, 4, 128, [700, 130], [100, 60]),
    "two-64": (14, 2, 64, [700, 130], [200, 100]),
    "split": (7, 1, 128, [5000], [1]),
    "split-64": (14, 2, 64, [4300, 900], [2, 1]),
}


def _attend(s, seed=None):
    width = s.table.shape[1]
    order = np.arange(width) if seed is None else np.random.default_rng(seed).permutation(width)
    picks = torch.from_numpy(order.astype(np.int32)).to(DEV).expand(sum(s.rows), s.n_kv, width).contiguous()
    return s.cache.attend_picked(s.batch(), s.q, picks)


def _setup(form, dtype, seed):
    n_q, n_kv, hd, ctx, rows = FORMS[form]
    return Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=seed)


@pytest.mark.parametrize("form", FORMS)
def test_weights_far_below_the_largest(form):
    """One key carries the weight and its value is zero: the output is made of weights of any size."""
    for dtype in ("bf16", "f32"):
        for nats in (10.0, 16.0, 27.0):
            s = _setup(form, dtype, 41)
            off, counts = np.concatenate([[0], np.cumsum(s.ctx)]), []
            for b, c in enumerate(s.ctx):
                at = 0 if b % 2 == 0 else c // 2  # the first key, or one with smaller ones before it
                counts.append(np.where(np.arange(c) == at, 32, 0))
                s.v[off[b] + at] = 0
            _aim(s, counts, nats).fill()
            _check(s, _attend(s))
            _check(s, _attend(s, 3))


@pytest.mark.parametrize("form", FORMS)
def test_maxima_that_move(form):
    """Scores that rise, fall or jump by many bits from page to page: what was summed before is rescaled, once."""
    for dtype in ("bf16", "f32"):
        for step in STEPS.values():
            s = _setup(form, dtype, 43)
            _aim(s, [step(np.arange(c) // 64) for c in s.ctx], 64.0).fill()
            _check(s, _attend(s))


@pytest.mark.parametrize("form", FORMS)
def test_values_beyond_half_precision_after_a_move(form):
    """Values that fp16 does not hold from the middle of each sequence on, after the reference has moved and with small weights on
    both sides."""
    for step in ("slow", "mixed"):
        s = _setup(form, "bf16", 44)
        off = np.concatenate([[0], np.cumsum(s.ctx)])
        _aim(s, [STEPS[step](np.arange(c) // 64) for c in s.ctx], 64.0)
        for b, c in enumerate(s.ctx):
            s.v[off[b] + c // 2:off[b + 1]:7] *= 2.0 ** 30
            s.v[off[b] + c // 2 + 3:off[b + 1]:11] *= 2.0 ** -40
        s.fill()
        _check(s, _attend(s))
        _check(s, _attend(s, 5))


@pytest.mark.parametrize("form", ["four", "four-64", "wide", "two"])
def test_strong_keys_everywhere(form):
    """Strong keys with a value of zero in all pages: the weights beside them are off by 2^-11 of what the keys around them weigh
    together at most (include/rollpack.h), times the largest of their values."""
    for nats in (12.0, 18.0, 27.0):
        s = _setup(form, "bf16", 47)
        pos = np.concatenate([np.arange(c) for c in s.ctx])
        s.v[torch.from_numpy(pos % 11 == 3).to(DEV)] = 0
        _aim(s, [np.where(np.arange(c) % 11 == 3, 32, 0) for c in s.ctx], nats).fill()
        out, q, at, g = _f64(_attend(s)), _f64(s.q), 0, s.n_q // s.n_kv
        held = s.held()
        for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
            k, v = held[b]
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
    """A tenth of a percent of the weight in 40,000 keys, each about 2^-25 of the first, whose value is zero."""
    s = Setup(2, 1, 64, [40000] + [1] * 150, seed=42)
    s.v[:, 0] = 1.0 + s.v[:, 0].abs()
    s.v[0] = 0
    _aim(s, [np.where(np.arange(40000) == 0, 32, 0)] + [np.zeros(1)] * 150, 18.0).fill()
    _check(s, _attend(s))


@pytest.mark.parametrize("form", ["four", "four-64", "wide", "two"])
def test_large_scores_and_values_near_the_end_of_the_range(form):
    """Scores in the thousands, where one key takes nearly all of the weight; sums stay finite while the largest value times the
    context is below 2^119 (include/rollpack.h)."""
    for dtype in ("bf16", "f32"):
        n_q, n_kv, hd, ctx, rows = FORMS[form]
        s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=45, gain=6.0).fill()
        s.q *= 4
        _check(s, _attend(s))
        s = _setup(form, dtype, 46)
        s.v *= 2.0 ** (118 - 13 - 3)  # contexts below 2^13, values below 2^3
        s.q *= 0.25
        s.fill()
        _check(s, _attend(s))
