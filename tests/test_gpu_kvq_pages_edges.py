"""The 4-bit cache's page calls on the GPU where their bounds end, and every form of the scores of pages and of
attention over picked ones (oracle/kvq_pages.py).  Tolerances are those of tests/test_gpu_kvq_pages.py and tests/test_gpu_kvq_softmax.py.
"""
import numpy as np
import pytest

from oracle import kvq as okvq
from oracle import kvq_pages as op
from tests import test_gpu_kvq_picked_softmax as softmax
from tests.gpu_helpers import rp
from tests.kvq_page_forms import CALLS, HARD, SCORES
from tests.test_gpu_kvq_pages import DEV, Decode, Pools, Setup, _check_picked, _check_scores, _f64, _ints, _lists, _score_bar

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


# ---- bounds of the batch that fit makes ----------------------------------------------

class Bounded(Pools):
    def fit(self, lengths, n_rows, **bounds):
        """Both pools, with the same bounds; the GPU's is looked at as a whole."""
        table = self.gpu.page_table.clone()
        batch, positions, slots = self.gpu.fit(_ints(np.asarray(lengths)), n_rows, **bounds)
        error, off, pos, slot = self.plain.fit(lengths, n_rows, **bounds)
        st = self.check_state()
        assert (st["error"], st["missing_pages"], st["rows"]) == (error, self.plain.missing, off[-1])
        assert st["message"] == rp().KVQ_FIT_ERRORS[error]
        assert np.array_equal(batch.row_offsets.cpu().numpy(), off)
        assert np.array_equal(positions.cpu().numpy(), pos) and np.array_equal(slots.cpu().numpy(), slot)
        assert not error or torch.equal(self.gpu.page_table, table)
        assert (batch.struct.max_rows, batch.struct.max_context) == (bounds.get("max_rows", n_rows), bounds.get("max_context", self.gpu.max_context))
        return error


def test_a_sequence_with_more_rows_than_max_rows_changes_nothing():
    p = Bounded(9, 3, 640, 4)
    assert p.fit([10, 5, 0], 16) == 0
    assert p.fit([11, 7, 0], 16, max_rows=1) == 5
    assert p.fit([11, 6, 64], 100, max_rows=1) == 5     # a prompt in a step of single tokens
    assert p.fit([11, 6, 1], 100, max_rows=0) == 5
    assert p.fit([11, 6, 1], 100, max_rows=1) == 0
    assert p.fit([0, 70, 1], 100, max_rows=64) == 0
    assert p.fit([0, 135, 66], 200, max_rows=64) == 5
    assert p.fit([0, 135, 66], 200, max_rows=65) == 0
    assert p.fit([0, 130, 0], 5, max_rows=0) == 0       # taking back needs none


def test_a_length_above_the_calls_max_context_changes_nothing():
    p = Bounded(12, 3, 640, 4)
    assert p.fit([10, 5, 0], 16, max_context=10) == 0
    assert p.fit([11, 5, 0], 16, max_context=10) == 2
    assert p.fit([10, 5, 0], 16, max_context=9) == 2    # one that has no new token
    assert p.fit([9, 5, 3], 16, max_context=9) == 0     # a longer one that shrinks is within
    assert p.fit([0, 0, 1], 16, max_context=0) == 2
    assert p.fit([0, 0, 0], 16, max_context=0) == 0
    assert p.fit([640, 0, 0], 640, max_context=640) == 0


def test_which_error_is_told():
    """A length out of range, too few pages, too many rows, too many of a sequence: the first of these."""
    p = Bounded(4, 2, 640, 1)
    assert p.fit([3, 3], 6) == 0
    assert p.fit([301, 9], 4, max_rows=1, max_context=300) == 2
    assert p.fit([300, 9], 4, max_rows=1, max_context=300) == 1
    assert p.fit([100, 9], 4, max_rows=1, max_context=300) == 3
    assert p.fit([100, 9], 103, max_rows=96, max_context=300) == 5
    assert p.fit([100, 9], 103, max_rows=97, max_context=300) == 0


@pytest.mark.parametrize("n", [64, 65, 1024, 1025, 3000])
def test_bounds_of_any_one_sequence(n):
    """The first, one in the middle and the last; up to 1,024 sequences and more, one block and many."""
    p = Bounded(2 * n, n, 128, 2)
    now = np.random.default_rng(n).integers(0, 64, n)
    assert p.fit(now.tolist(), 64 * n) == 0
    for b in (0, n // 2, n - 1):
        for room in (3 * n, 70_000):
            to = now + 1
            to[b] += 1
            assert p.fit(to.tolist(), room, max_rows=1) == 5
            to[b] = 101
            assert p.fit(to.tolist(), room, max_rows=101, max_context=100) == 2
    assert p.fit((now + 1).tolist(), n, max_rows=1, max_context=64) == 0


def test_rows_past_the_bounds_reach_no_cache():
    """A prompt in a step of single tokens: nothing of the pool, the cache or the ranges changes, and the same lengths under bounds that
    hold attend to what was appended."""
    d = Decode(11)
    q, k, v = d.tensors(94)
    d.step(_ints([30, 0, 0, 64, 0]), 94, q, k, v)
    kept = [t.clone() for t in (d.cache.blocks, d.ranges, d.pages.contexts, d.pages.page_table, d.pages.free_pages)]
    lengths = [31, 0, 2, 65, 0]
    q, k, v = d.tensors(6)
    batch, positions, slots = d.pages.fit(_ints(lengths), 6, max_rows=1)
    assert d.pages.status()["error"] == 5 and (positions == -1).all() and (slots == -1).all()
    d.cache.append(batch, k, v)
    d.cache.update_ranges(batch, d.ranges)
    for a, b in zip((d.cache.blocks, d.ranges, d.pages.contexts, d.pages.page_table, d.pages.free_pages), kept):
        assert torch.equal(a, b)
    out, picks, scores, positions, slots = d.step(_ints(lengths), 6, q, k, v)
    assert torch.isfinite(out[:4]).all() and positions.tolist() == [30, 0, 1, 64, -1, -1]


def test_bounds_in_a_graph():
    """Replays read the lengths that are there: those past the bounds change nothing, those within are served."""
    p, lengths = Bounded(40, 8, 300, 3), _ints(np.zeros(8))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        p.gpu.fit(lengths, 8, max_rows=1, max_context=200)
    torch.cuda.current_stream().wait_stream(stream)
    with torch.cuda.graph(graph):
        batch, positions, slots = p.gpu.fit(lengths, 8, max_rows=1, max_context=200)
    assert p.fit([70, 1, 199, 0, 5, 6, 200, 8], 500) == 0
    now = np.array(p.plain.contexts)
    for grow, error in (([1, 1, 1, 1, 1, 1, 0, 1], 0), ([0, 0, 1, 0, 0, 0, 0, 0], 2), ([2, 0, 0, 0, 0, 0, 0, 0], 5), ([1, 0, 0, 2, 1, 0, -3, 0], 5),
                        ([1, 0, 0, 1, 1, 0, -3, 0], 0)):
        to = (now + np.array(grow)).tolist()
        lengths.copy_(_ints(to))
        graph.replay()
        want, off, pos, slot = p.plain.fit(to, 8, 1, 200)
        assert p.check_state()["error"] == want == error
        assert np.array_equal(batch.row_offsets.cpu().numpy(), off)
        assert np.array_equal(positions.cpu().numpy(), pos) and np.array_equal(slots.cpu().numpy(), slot)
        now = np.array(p.plain.contexts)


# ---- a batch in parts ------------------------------------------------------------------

@pytest.mark.parametrize("cuts", [[0, 2, 5], [0, 1, 3, 4, 5]])
def test_a_batch_cut_between_sequences(cuts):
    """Prompts of a pool, whose scores, picks and attention take more rows than a call may have: parts of the batch give what it gives."""
    d = Decode(13)
    before = [30, 0, 64, 129, 0]
    d.step(_ints(before), 223, *(first := d.tensors(223)))
    d.k, d.v = ([x[a:b] for a, b in ((0, 30), (30, 30), (30, 94), (94, 223), (223, 223))] for x in (okvq.held(_f64(t)) for t in first[1:]))
    lengths = [31, 700, 64, 300, 5]
    rows = np.maximum(np.array(lengths) - np.array(before), 0)
    q, k, v = d.tensors(int(rows.sum()))
    batch, _, _ = d.pages.fit(_ints(lengths), len(q))
    d.cache.append(batch, k, v)
    d.cache.update_ranges(batch, d.ranges)
    scores = d.cache.page_scores(batch, q, d.ranges)
    picks = d.cache.pick_pages(batch, scores, 4)
    at, out = np.concatenate([[0], np.cumsum(rows)]), torch.full_like(q, 9.0)
    for a, b in zip(cuts, cuts[1:]):
        part = slice(int(at[a]), int(at[b]))
        offsets = batch.row_offsets[a:b + 1] - batch.row_offsets[a]
        n = part.stop - part.start
        cut = d.cache.batch(d.pages.contexts[a:b], d.pages.page_table[a:b], row_offsets=offsets, n_rows=n, max_rows=int(rows[a:b].max()))
        assert torch.equal(d.cache.page_scores(cut, q[part], d.ranges), scores[part])
        assert torch.equal(d.cache.pick_pages(cut, scores[part], 4), picks[part])
        d.cache.attend_picked(cut, q[part], picks[part], out=out[part])
    d.check(before, lengths, q, k, v, out, picks, scores)


# ---- scores as a bound -----------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd", [(28, 4, 128), (14, 2, 64), (17, 1, 128), (2, 2, 64)])
def test_scores_bound_keys_up_to_their_rounding(n_q, n_kv, hd, dtype):
    """No key's q . k exceeds its page's score by more than the error of the score's sum; a page of one token has that token's."""
    for rows in ([9, 2, 1, 3], [1, 1, 1, 1]):
        s = Setup(n_q, n_kv, hd, [500, 65, 1, 129 + 2], rows, dtype, seed=8 + rows[0]).fill()
        ranges = s.cache.update_ranges(s.batch(s.ctx), s.cache.new_ranges())
        got, q, at, alone = _f64(s.cache.page_scores(s.batch(), s.q, ranges)), _f64(s.q), 0, 0
        for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
            k = s.held()[b][0]
            _, mag = op.page_scores(q[at:at + n], op.key_ranges(k), np.arange(c - n, c), got.shape[2])
            bar = _score_bar(None, mag, hd, dtype)
            dot = np.einsum("nhgd,thd->nhgt", q[at:at + n].reshape(n, n_kv, -1, hd), k).max(2)
            for i in range(n):
                for p in range((c - n + i) // 64 + 1):
                    top = dot[i, :, p * 64:min(c, (p + 1) * 64)].max(-1)  # of all of the page's keys, those behind the row among them
                    assert (got[at + i, :, p] >= top - bar[i, :, p]).all()
                    if min(c, (p + 1) * 64) - p * 64 == 1:
                        assert (np.abs(got[at + i, :, p] - top) <= bar[i, :, p]).all()
                        alone += 1
            at += n
        assert alone >= 2


# ---- every form of scores, and of attention over picked pages --------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("call", SCORES)
def test_every_form_of_page_scores(call, dtype):
    n_q, n_kv, hd, ctx, rows, room, columns = SCORES[call]
    s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=hd + columns).fill()
    ranges, n = s.cache.update_ranges(s.batch(s.ctx), s.cache.new_ranges()), sum(s.rows)
    q = torch.full((room, n_q, hd), float("nan"), device=DEV, dtype=s.dt)
    q[:n] = s.q
    out = torch.full((room, n_kv, columns), 7.0, device=DEV)
    s.cache.page_scores(s.batch(n_rows=room, max_rows=1 if rows is None else room), q, ranges, out=out)
    _check_scores(out[:n], s, s.held(), _f64(s.q))
    assert (out[n:] == 7.0).all()
    table = s.dev_table.clone()
    s.dev_table[torch.arange(s.table.shape[1], device=DEV) >= torch.tensor([-(-c // 64) for c in ctx], device=DEV)[:, None]] = 2 ** 31 - 1
    again = torch.full_like(out, 7.0)  # what the table has behind a context does not count
    s.cache.page_scores(s.batch(n_rows=room, max_rows=1 if rows is None else room), q, ranges, out=again)
    s.dev_table.copy_(table)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("call", CALLS)
def test_every_form_of_attend_picked(call, dtype):
    n_q, n_kv, hd, ctx, rows, n = CALLS[call]
    s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=n + hd).fill()
    rng = np.random.default_rng(n)
    for style in ("picks", "any"):
        picks = _lists(s, n, rng, style)
        out = torch.full_like(s.q, 9.0)
        assert s.cache.attend_picked(s.batch(), s.q, torch.from_numpy(picks).to(DEV), out=out) is out
        _check_picked(s, out, picks)


@pytest.mark.parametrize("form", HARD)
def test_eight_waves_where_the_softmax_is_hard(form, monkeypatch):
    monkeypatch.setitem(softmax.FORMS, form, HARD[form])
    softmax.test_weights_far_below_the_largest(form)
    softmax.test_maxima_that_move(form)
    softmax.test_values_beyond_half_precision_after_a_move(form)
    softmax.test_strong_keys_everywhere(form)
    softmax.test_large_scores_and_values_near_the_end_of_the_range(form)


@pytest.mark.parametrize("form", ["four", "four-64", "wide", "wide-64", "two", "eight-128", "eight-wide-128", "eight-wide-64-rows"])
def test_small_weights_beside_the_keys_of_their_lane(form, monkeypatch):
    """Strong keys with a value of zero in all pages, as softmax.test_strong_keys_everywhere has them, but only where they share no lane's
    sum with what the output is made of: 4 of each 16 tokens of a page are a lane's, with up to eight query heads of half a page.  A weight
    below 2^-14 of fp16's is off by 2^-25 where its lane's N <= 16 keys sum to 2^-9 at least, by N 2^-25 <= 2^-21 < 2^-11 2^-9 of
    them together; where they do not, each is off by 2^-11 of itself alone.  The sum of a row's weights has the same errors (another
    2^-11 of the output)."""
    if form in HARD:
        monkeypatch.setitem(softmax.FORMS, form, HARD[form])
    for nats in (12.0, 18.0, 27.0):
        s = softmax._setup(form, "bf16", 48)
        narrow = s.n_q // s.n_kv <= 8
        lane = lambda t: (t % 16) // 4 + 4 * ((t % 64) // 32 if narrow else 0) + 8 * (t // 64)  # noqa: E731
        strong = lambda t: (t % 16) // 4 == 1  # noqa: E731
        pos = np.concatenate([np.arange(c) for c in s.ctx])
        s.v[torch.from_numpy(strong(pos)).to(DEV)] = 0
        softmax._aim(s, [np.where(strong(np.arange(c)), 32, 0) for c in s.ctx], nats).fill()
        out, q, at, g = _f64(softmax._attend(s)), _f64(s.q), 0, s.n_q // s.n_kv
        held = s.held()
        for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
            k, v = held[b]
            ref, mag, top = okvq.attend(q[at:at + n], k, v, np.arange(c - n, c), s.hd ** -0.5)
            bar = softmax._bar(ref, mag, top, c, s.hd, "bf16", np.abs(v).max()) + 2.0 ** -11 * mag
            mine = lane(np.arange(c))[:, None] == np.arange(8 * (-(-c // 64)))
            for h in range(s.n_q):
                z = np.where(np.arange(c)[None] <= np.arange(c - n, c)[:, None], q[at:at + n, h] @ k[:, h // g].T * s.hd ** -0.5, -np.inf)
                p = np.exp(z - z.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                most = np.where(mine[:, :, None], np.abs(v[:, None, h // g]), 0.0).max(0)  # of a lane's keys
                bar[:, h] += 2.0 ** -11 * (p @ mine) @ most
            assert (np.abs(out[at:at + n] - ref) <= bar).all(), (b, c, n, nats)
            at += n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("call", ["eight-wide-128", "eight-wide-64-rows", "eight-17-heads", "eight-narrow-128-rows"])
def test_eight_waves_of_bad_pages_and_empty_lists(call, dtype):
    """Ids outside the cache and NaN keys make their row and KV head NaN where they are listed; lists without a page that the row sees give
    zeros, rows of no sequence are left as they are."""
    n_q, n_kv, hd, ctx, rows, n = CALLS[call]
    s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=3)
    s.k[ctx[0] + 70, 0, 5] = float("nan")                # of the second sequence, page 1
    s.fill()
    picks = _lists(s, n, np.random.default_rng(5))
    first = np.concatenate([[0], np.cumsum(s.rows)])[:-1]
    picks[first[0], 0] = [0, 3, 5] + [-1] * (n - 3)      # page 3 is lost
    picks[first[1], 0] = [0, 1, 2] + [-1] * (n - 3)
    picks[first[3], 0] = [-1] * (n - 2) + [11, 2 ** 31 - 1]  # of 700 tokens: pages 0 .. 10
    s.dev_table[0, 3] = s.cache.n_pages
    room = sum(s.rows) + 3
    q = torch.cat([s.q, s.q[:3]])
    out = torch.full_like(q, 5.0)
    all_picks = torch.from_numpy(np.concatenate([picks, picks[:3]])).to(DEV)
    s.cache.attend_picked(s.batch(n_rows=room), q, all_picks, out=out)
    assert torch.isnan(out[first[0]]).all() and torch.isnan(out[first[1]]).all() and (out[first[3]] == 0).all()
    assert (out[sum(s.rows):] == 5.0).all()
    _check_picked(s, out, picks, seqs=[2, 4, 5])
