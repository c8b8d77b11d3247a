"""The 4-bit cache's pages on the GPU against their plain forms (oracle/kvq_pages.py): handed out, ranges of keys, scores, picks,
attention over picked pages.

Pages, offsets, slots, ranges and picks have one right result and are compared exactly.

Scores: 2 hd products in fp32, those with one sign of q being zeros: products of bf16 are exact; fp32 queries go in three pieces
of bf16, whose sum has an error of 2^-24 of each query and whose products are 6 hd.  Every addition is off by at most one
step, 2^-23 of a partial sum (half of it where it rounds to nearest): (2 hd, or 6 hd, + 2) 2^-23 sum |q| |range| in all; the
largest of several such sums is off by no more than the worst of them.
Attention over a list has the bar of attention over a sequence of the list's tokens (tests/test_gpu_kvq.py).
"""
import numpy as np
import pytest

from oracle import kvq as okvq
from oracle import kvq_pages as op
from tests.gpu_helpers import rp
from tests.test_gpu_kvq import DEV, TYPES, Setup, _bound, _f64, _ints

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


# ---- pages handed out ----------------------------------------------------------------

class Pools:
    """A pool on the GPU beside the plain one."""

    def __init__(self, n_pages, n_seqs, max_context, seed=0):
        free = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
        self.gpu = rp().KvqPages(n_pages, n_seqs, max_context, device=DEV)
        self.gpu.free_pages.copy_(torch.from_numpy(free))
        self.plain = op.Pool(free.tolist(), n_seqs, max_context)

    def check_state(self, rows=None):
        st, pl = self.gpu.status(), self.plain
        n = len(pl.free)
        assert st["free_pages"] == n
        assert self.gpu.free_pages[:n].tolist() == pl.free
        assert self.gpu.contexts.tolist() == pl.contexts
        table = self.gpu.page_table.cpu().numpy()
        for b, held in enumerate(pl.table):
            assert table[b, :len(held)].tolist() == held, b
        return st

    def fit(self, lengths, n_rows, **kw):
        batch, positions, slots = self.gpu.fit(_ints(np.asarray(lengths)), n_rows, **kw)
        error, off, pos, slot = self.plain.fit(lengths, n_rows)
        st = self.check_state()
        assert (st["error"], st["missing_pages"], st["rows"]) == (error, self.plain.missing, off[-1])
        assert np.array_equal(batch.row_offsets.cpu().numpy(), off)
        assert np.array_equal(positions.cpu().numpy(), pos) and np.array_equal(slots.cpu().numpy(), slot)
        return batch


@pytest.mark.parametrize("n_seqs,max_context,steps,seed", [
    (1, 1, 4, 0), (1, 64, 5, 1), (3, 65, 8, 2), (64, 700, 8, 3), (65, 130, 6, 4), (1023, 200, 4, 5), (1024, 100, 4, 6),
    (1025, 129, 4, 7), (2500, 90, 4, 8), (7, 33000, 5, 9),
])
def test_pool_follows_lengths(n_seqs, max_context, steps, seed):
    """Sequences come, grow, shrink, stay and go, in any mix; up to 1,024 rows are one block's, and those of more than 1,024
    sequences a launch of their own."""
    rng = np.random.default_rng(seed)
    p = Pools(n_seqs * op.pages(max_context), n_seqs, max_context, seed)
    now = np.zeros(n_seqs, np.int64)
    for _ in range(steps):
        to = rng.integers(0, max_context + 1, n_seqs)
        kind = rng.integers(0, 5, n_seqs)
        now = np.select([kind == 0, kind == 1, kind == 2, kind == 3], [np.minimum(now + 1, max_context), now, np.maximum(now - 3, 0), 0], to)
        rows = int(np.maximum(now - np.array(p.plain.contexts), 0).sum())
        p.fit(now.tolist(), rows + int(rng.integers(0, 70)))
        assert p.plain.contexts == now.tolist()
    p.fit([0] * n_seqs, 0)
    assert p.gpu.status()["free_pages"] == p.gpu.n_pages


def test_pool_of_very_many_sequences():
    """Sums over tiles of 1,024 sequences and over many of them to a thread."""
    n = 70001
    p = Pools(2 * n, n, 70, 1)
    rng = np.random.default_rng(4)
    for most in (3, 70, 66):
        to = rng.integers(0, most + 1, n)
        p.fit(to.tolist(), int(np.maximum(to - np.array(p.plain.contexts), 0).sum()))
    p.fit([70] * n, n)  # more rows than room for them
    assert p.gpu.status()["error"] == 3
    p.fit([0] * n, 0)


@pytest.mark.parametrize("n_seqs,max_context", [(1, 500_000), (3, 150_000), (300, 1500), (1000, 400), (1024, 300)])
def test_rows_of_many_blocks(n_seqs, max_context):
    """Up to 256 blocks, of 1,024 rows and more, share a call; pages that it takes back serve it; and a call of padded rows, one that
    fails and one that changes nothing leave the blocks' counts ready for the next."""
    rng = np.random.default_rng(n_seqs)
    p = Pools(n_seqs * op.pages(max_context) * 2 // 3 + 1, n_seqs, max_context, 5)
    half = rng.permutation(n_seqs) < (n_seqs + 1) // 2
    a = np.where(half, rng.integers(max_context // 2, max_context + 1, n_seqs), 1) if n_seqs > 1 else np.array([max_context // 2])
    b = np.where(half, 30, a[::-1] // 2 + 65) if n_seqs > 1 else np.array([max_context * 3 // 5])
    for to in (a, b, a):
        p.fit(to.tolist(), int(np.maximum(to - np.array(p.plain.contexts), 0).sum()) + 1500)
        assert p.gpu.status()["error"] == 0
    p.fit(a.tolist(), 5000)                    # nothing to do
    p.fit(np.full(n_seqs, max_context).tolist(), 300_000)   # too few pages
    assert p.gpu.status()["error"] == 1
    p.fit((a - 1).tolist(), 70_000)
    p.fit(np.zeros(n_seqs, int).tolist(), 2000)
    p.fit(b.tolist(), 400_000)
    assert p.gpu.status()["error"] == 0


def test_rows_of_many_blocks_in_a_graph():
    """Replays with other lengths, the pool used eagerly in between."""
    p, lengths = Pools(900, 40, 2000, 6), _ints(np.zeros(40))
    rng = np.random.default_rng(8)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        p.gpu.fit(lengths, 30_000)
    torch.cuda.current_stream().wait_stream(stream)
    with torch.cuda.graph(graph):
        batch, positions, slots = p.gpu.fit(lengths, 30_000)
    for i in range(6):
        to = rng.integers(0, 1100, 40)
        lengths.copy_(_ints(to))
        graph.replay()
        error, off, pos, slot = p.plain.fit(to.tolist(), 30_000)
        assert p.check_state()["error"] == error == 0
        assert np.array_equal(batch.row_offsets.cpu().numpy(), off)
        assert np.array_equal(positions.cpu().numpy(), pos) and np.array_equal(slots.cpu().numpy(), slot)
        if i % 2:
            p.fit((to + 1).tolist(), [40, 3000][i // 2 % 2])


def test_a_call_and_its_taking_back_leave_the_pool_as_it_was():
    rng = np.random.default_rng(3)
    p = Pools(300, 40, 600, 1)
    a, b = rng.integers(0, 400, 40).tolist(), rng.integers(0, 400, 40).tolist()
    p.fit(a, 40 * 400)
    before = [t.clone() for t in (p.gpu.free_pages, p.gpu.state)]
    p.fit(b, 40 * 400)
    p.fit(a, 40 * 400)
    n = int(before[1][0])
    assert torch.equal(p.gpu.free_pages[:n], before[0][:n]) and int(p.gpu.state[0]) == n


def test_pages_given_back_serve_the_same_call():
    p = Pools(4, 3, 256, 2)
    p.fit([256, 0, 0], 256)
    p.fit([0, 100, 128], 300)  # all of the first one's
    p.fit([0, 100, 128], 0)    # nothing to do


@pytest.mark.parametrize("lengths,n_rows,error", [
    ([64 * 5, 10, 64 * 4], 4096, 1), ([-1, 0, 0], 10, 2), ([0, 641, 0], 700, 2), ([2 ** 31 - 1, 2 ** 31 - 1, 5], 10, 2),
    ([20, 7, 31], 32, 3), ([20, 7, 31], 0, 3), ([640, 640, 640], 1920, 1), ([640, 640, 640], 5, 1),
])
def test_what_does_not_fit_changes_nothing(lengths, n_rows, error):
    """And has no rows, so that the calls that take the batch do nothing; the next call that fits is served."""
    p = Pools(9, 3, 640, 4)
    p.fit([10, 5, 10], 30)
    batch = p.fit(lengths, n_rows)
    assert p.gpu.status()["error"] == error and p.gpu.status()["message"] == rp().KVQ_FIT_ERRORS[error]
    cache = rp().KvqCache(9, 2, 64, device=DEV)
    before = cache.blocks.clone()
    x = torch.ones((n_rows, 2, 64), device=DEV)
    cache.append(batch, x, x)
    assert torch.equal(cache.blocks, before)
    p.fit([11, 0, 90], 200)


@pytest.mark.parametrize("n_rows", [33, 37])
def test_what_just_fits(n_rows):
    """(20 - 10) + (7 - 5) + (31 - 10) = 33 new tokens."""
    p = Pools(9, 3, 640, 4)
    p.fit([10, 5, 10], 30)
    p.fit([20, 7, 31], n_rows)
    assert p.gpu.status()["error"] == 0 and p.gpu.status()["rows"] == 33


@pytest.mark.parametrize("spoil", ["free", "free_low", "context", "context_low"])
def test_a_state_that_no_calls_have_made_is_refused(spoil):
    p = Pools(9, 3, 640, 4)
    p.fit([10, 70, 10], 100)
    t, i, v = {"free": (p.gpu.state, 0, 6), "free_low": (p.gpu.state, 0, -1), "context": (p.gpu.contexts, 1, 641),
               "context_low": (p.gpu.contexts, 1, -64)}[spoil]
    keep, t[i] = int(t[i]), v
    table, free = p.gpu.page_table.clone(), p.gpu.free_pages.clone()
    batch, positions, slots = p.gpu.fit(_ints([0, 0, 0]), 4)
    assert p.gpu.status()["error"] == 4 and batch.row_offsets.tolist() == [0] * 4 and positions.tolist() == [-1] * 4
    assert torch.equal(table, p.gpu.page_table) and torch.equal(free, p.gpu.free_pages)
    t[i] = keep
    p.fit([0, 71, 200], 500)


def test_no_sequences():
    p = rp().KvqPages(3, 0, 64, device=DEV)
    batch, positions, slots = p.fit(_ints([]), 5)
    assert batch.row_offsets.tolist() == [0] and positions.tolist() == slots.tolist() == [-1] * 5
    assert p.status()["error"] == 0 and p.status()["free_pages"] == 3
    for n_rows in (0, 70_000, 2000):
        batch, positions, slots = p.fit(_ints([]), n_rows)
        assert batch.row_offsets.tolist() == [0] and bool((positions == -1).all()) and bool((slots == -1).all())
        assert p.status() == {"free_pages": 3, "error": 0, "message": rp().KVQ_FIT_ERRORS[0], "rows": 0, "missing_pages": 0}


# ---- ranges --------------------------------------------------------------------------

def _plain_ranges(s, held, ranges, rows):
    """What update_ranges leaves of `ranges` (numpy) after the last `rows` tokens of each sequence were appended."""
    for b, (c, n) in enumerate(zip(s.ctx, rows)):
        if not n or not c:
            continue
        r = op.key_ranges(held[b][0])
        for p in range(max(0, c - n) // 64, op.pages(c)):
            ranges[s.table[b, p]] = r[p]
    return ranges


@pytest.mark.parametrize("n_kv,hd,dtype,ctx,rows", [
    (4, 128, "bf16", [1, 63, 64, 65, 130, 7], None),
    (2, 64, "f32", [1, 63, 64, 65, 130, 7], None),
    (3, 64, "bf16", [5, 200, 1, 400], [5, 3, 1, 330]),
    (1, 128, "f32", [70, 64, 3, 129] * 20, [9, 64, 1, 2] * 20),
    (2, 64, "bf16", [3, 1, 0, 70, 2, 0, 0] * 40, [2, 1, 0, 70, 2, 0, 0] * 40),
    (8, 128, "bf16", [4000, 700], [4000, 65]),
    (2, 128, "bf16", [40, 3], [50, 7]),   # more rows than tokens
])
def test_ranges_are_the_keys(n_kv, hd, dtype, ctx, rows):
    s = Setup(n_kv, n_kv, hd, ctx, rows, dtype, seed=len(ctx) + hd).fill()
    start = torch.randn((s.cache.n_pages, n_kv, 2, hd), device=DEV).to(torch.bfloat16)
    got = s.cache.update_ranges(s.batch(), start.clone())
    assert np.array_equal(_f64(got), _plain_ranges(s, s.held(), _f64(start), s.rows))
    if rows is None:  # the form without offsets
        b = s.cache.batch(_ints(ctx), s.dev_table)
        assert torch.equal(s.cache.update_ranges(b, start.clone()), got)


@pytest.mark.parametrize("hd", [64, 128])
def test_ranges_of_odd_keys(hd):
    """NaN and infinity make NaN of their block's dimensions; zeros, one sign only, huge and tiny values; the sign of zero."""
    s = Setup(2, 2, hd, [100, 64, 30, 64], [100, 64, 30, 64], "f32", seed=5)
    k = s.k
    k[3, 0, 5], k[70, 1, hd - 1], k[99, 0, 40] = float("nan"), float("inf"), float("-inf")
    k[100:164, 0] = k[100:164, 0].abs()
    k[100:164, 1] = -k[100:164, 1].abs()
    k[164:180] *= 1e-38
    k[180:194] *= 1e37
    k[194:, 0] = 0.0
    k[194:, 1] = -0.0
    s.fill()
    got = _f64(s.cache.update_ranges(s.batch(), s.cache.new_ranges()))
    ref = _plain_ranges(s, s.held(), np.zeros(got.shape), s.rows)
    assert np.isnan(ref).any() and np.array_equal(got, ref, equal_nan=True)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv", [1, 3, 8])
def test_ranges_of_whole_pages_of_every_magnitude(n_kv, hd):
    """Whole pages whose scales lie within fp16's exact range, at its ends and past them, and pages with a NaN, an infinity."""
    s = Setup(n_kv, n_kv, hd, [64 * 24, 64 * 3 + 5], [64 * 24, 64 * 3 + 5], "f32", seed=n_kv + hd)
    for p, e in enumerate([-30, -25, -24, -23, -22, -21, -20, -10, -3, 0, 3, 6, 7, 8, 9, 10, 11, 12, 20, 100]):
        x = s.k[64 * p:64 * p + 64]
        x.clamp_(-3.0, 3.0).mul_(2.0 ** e)
    s.k[64 * 20 + 11, 0, 7], s.k[64 * 21, n_kv - 1, hd - 1], s.k[64 * 22 + 63, 0, 40] = float("nan"), float("inf"), float("-inf")
    s.k[64 * 23:64 * 24] = 0.0
    s.fill()
    got = _f64(s.cache.update_ranges(s.batch(), s.cache.new_ranges()))
    assert np.array_equal(got, _plain_ranges(s, s.held(), np.zeros(got.shape), s.rows), equal_nan=True)


def test_ranges_of_many_rows():
    """Waves with one row and with 64; sequences of every length side by side, some without rows, many such in a row, so that 64 rows
    are of more than 64 sequences."""
    rng = np.random.default_rng(2)
    ctx = rng.integers(0, 300, 250)
    rows = np.where(rng.random(250) < 0.3, 0, np.minimum(ctx, rng.integers(0, 400, 250)))
    rows[60:200:2] = 0
    rows[61:200:2] = np.minimum(ctx[61:200:2], 1)
    for n_kv, hd in ((4, 64), (2, 128)):
        s = Setup(n_kv, n_kv, hd, ctx.tolist(), rows.tolist(), "bf16", seed=n_kv).fill()
        start = torch.randn((s.cache.n_pages, n_kv, 2, hd), device=DEV).to(torch.bfloat16)
        want = _plain_ranges(s, s.held(), _f64(start), s.rows)
        assert np.array_equal(_f64(s.cache.update_ranges(s.batch(), start.clone())), want)
        many = s.batch(n_rows=70000, max_rows=400)  # with the rows behind the last sequence
        assert np.array_equal(_f64(s.cache.update_ranges(many, start.clone())), want)


def test_ranges_of_bad_batches_are_left_alone():
    s = Setup(2, 2, 64, [70, 70, 70, 70], None, seed=6).fill()
    start = torch.randn((s.cache.n_pages, 2, 2, 64), device=DEV).to(torch.bfloat16)
    table = s.dev_table.clone()
    table[1, 1], table[2, 1] = -5, s.cache.n_pages
    b = s.cache.batch(_ints([-3, 70, 70, 200]), table, n_rows=6, row_offsets=_ints([0, 1, 2, 3, 5]), max_rows=1)
    assert torch.equal(s.cache.update_ranges(b, start.clone()), start)


# ---- scores --------------------------------------------------------------------------

def _score_bar(ref, mag, hd, dtype):
    return mag * ((2 if dtype == "bf16" else 6) * hd + 2) * 2.0 ** -23 + 1e-37


def _check_scores(got, s, held, q):
    got, at = _f64(got), 0
    for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
        if n:
            pos = np.arange(c - n, c)
            ref, mag = op.page_scores(q[at:at + n], op.key_ranges(held[b][0]), pos, got.shape[2])
            part = got[at:at + n]
            assert np.array_equal(np.isfinite(part), np.isfinite(ref)), b
            inf = ~np.isfinite(ref)
            assert np.array_equal(part[inf], ref[inf], equal_nan=True), b
            assert (np.abs(part[~inf] - ref[~inf]) <= _score_bar(ref, mag, s.hd, s.dtype)[~inf]).all(), b
        at += n


SHAPES = [(4, 2, 64), (14, 2, 64), (28, 4, 128), (40, 8, 128), (2, 2, 128), (16, 1, 64), (17, 1, 128), (40, 1, 64), (9, 3, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd", SHAPES)
def test_scores(n_q, n_kv, hd, dtype):
    """One row each, and several of each, of contexts that end inside, at and behind a page and a tile of 16 pages."""
    for ctx, rows in (([1, 64, 65, 1024, 1025, 700], None), ([5, 130, 1030, 0, 3], [5, 7, 66, 0, 0]), ([2, 900], [4, 40])):
        s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=n_q + len(ctx)).fill()
        every = s.batch(s.ctx)
        ranges = s.cache.update_ranges(every, s.cache.new_ranges())
        got = s.cache.page_scores(s.batch(), s.q, ranges)
        assert got.shape == (sum(s.rows), n_kv, s.table.shape[1])
        _check_scores(got, s, s.held(), _f64(s.q))
        if rows is None:
            b = s.cache.batch(_ints(ctx), s.dev_table)
            assert torch.equal(s.cache.page_scores(b, s.q, ranges), got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("room", [10, 1000])
@pytest.mark.parametrize("n_q,n_kv,hd", [(2, 2, 64), (28, 4, 128), (17, 1, 128), (40, 1, 64), (16, 1, 128)])
def test_scores_of_long_sequences(n_q, n_kv, hd, room, dtype):
    """One row each, of contexts that end inside, at and behind 16, 64 and 256 pages; columns past all of them, and rows of no sequence
    (so many that a wave has 64 pages); a page id outside the cache makes its own score NaN."""
    s = Setup(n_q, n_kv, hd, [4096, 4097, 1024, 1025, 6200, 16385, 1, 3000], None, dtype, seed=n_q).fill()
    ranges = s.cache.update_ranges(s.batch(s.ctx), s.cache.new_ranges())
    out = torch.full((room, n_kv, 300), 7.0, device=DEV)
    q = torch.full((room, n_q, hd), float("nan"), device=DEV, dtype=s.dt)
    q[:8] = s.q
    b = s.cache.batch(_ints(s.ctx), s.dev_table, row_offsets=_ints(range(9)), n_rows=room, max_rows=1)
    s.cache.page_scores(b, q, ranges, out=out)
    _check_scores(out[:8], s, s.held(), _f64(s.q))
    assert (out[8:] == 7.0).all()
    want = out.clone()
    s.dev_table[4, 70], want[4, :, 70] = s.cache.n_pages, float("nan")
    s.dev_table[5, 3], want[5, :, 3] = -1, float("nan")
    s.cache.page_scores(b, q, ranges, out=out)
    assert torch.equal(out.nan_to_num(nan=9e30), want.nan_to_num(nan=9e30))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd,room,columns", [(14, 2, 64, 1700, 15), (28, 4, 128, 3000, 100), (28, 4, 128, 3000, 1024), (40, 1, 64, 5000, 200)])
def test_scores_of_many_rows(n_q, n_kv, hd, room, columns, dtype):
    """Bounds under which a wave has several rows and 32 or 64 pages, whatever the sequences: short ones and long ones side by side,
    some without rows, rows of no sequence behind them."""
    s = Setup(n_q, n_kv, hd, [900, 40, 0, 3, 64, 700, 1], [130, 40, 0, 3, 1, 65, 0], dtype, seed=hd + columns).fill()
    ranges = s.cache.update_ranges(s.batch(s.ctx), s.cache.new_ranges())
    q = torch.full((room, n_q, hd), float("nan"), device=DEV, dtype=s.dt)
    q[:len(s.q)] = s.q
    out = torch.full((room, n_kv, columns), 7.0, device=DEV)
    s.cache.page_scores(s.batch(n_rows=room, max_rows=room), q, ranges, out=out)
    _check_scores(out[:len(s.q)], s, s.held(), _f64(s.q))
    assert (out[len(s.q):] == 7.0).all()


@pytest.mark.parametrize("n_q,n_kv,hd", [(28, 4, 128), (14, 2, 64)])
def test_scores_bound_every_key(n_q, n_kv, hd):
    s = Setup(n_q, n_kv, hd, [500, 77], [9, 2], "bf16", seed=8).fill()
    ranges = s.cache.update_ranges(s.batch(s.ctx), s.cache.new_ranges())
    got, q, at = _f64(s.cache.page_scores(s.batch(), s.q, ranges)), _f64(s.q), 0
    for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
        k = s.held()[b][0]
        dot = np.einsum("nhgd,thd->nhgt", q[at:at + n].reshape(n, n_kv, -1, hd), k).max(2)
        for p in range((c - n) // 64 + 1):  # pages that every row sees
            top = dot[..., p * 64:min(c - n, (p + 1) * 64 - 1) + 1].max(-1)
            assert (got[at:at + n, :, p] >= top - 1e-3).all()
        at += n


def test_scores_of_odd_inputs():
    """NaN queries of one head, NaN keys, page ids outside the cache, contexts outside the bounds, rows before the first token,
    rows of no sequence, more columns than pages."""
    s = Setup(8, 2, 128, [200, 200, 200, 30, 200], [3, 3, 1, 40, 1], "bf16", seed=9)
    s.k[70, 1, 3] = float("nan")
    s.fill()
    ranges = s.cache.update_ranges(s.batch(s.ctx), s.cache.new_ranges())
    q = s.q.clone()
    q[1, 2, 7] = float("nan")    # row 1, KV head 0
    table = s.dev_table.clone()
    table[1, 1], table[1, 2] = -1, 1 << 24
    ctx = _ints([200, 200, 300, 30, -1])
    b = s.cache.batch(ctx, table, row_offsets=_ints([0, 3, 6, 7, 47, 48]), n_rows=50, max_rows=40, max_context=256)
    out = torch.full((50, 2, 9), 7.0, device=DEV)
    q = torch.cat([q, q[:2]])
    s.cache.page_scores(b, q, ranges, out=out)
    got = _f64(out)
    assert np.isnan(got[0, 1, 1]) and np.isfinite(got[0, 0, :4]).all() and np.isfinite(got[0, 1, [0, 2, 3]]).all()
    assert np.isnan(got[1, 0, :4]).all() and np.isfinite(got[1, 1, [0, 2, 3]]).all()
    assert (got[:3, :, 4:] == -np.inf).all()
    assert np.isnan(got[3:6, :, 1:3]).all() and np.isfinite(got[3:6][:, :, [0, 3]]).all()
    assert np.isnan(got[6]).all() and np.isnan(got[47]).all()      # out of bounds
    assert (got[7:17] == -np.inf).all()                            # positions -10 .. -1
    assert np.isfinite(got[17:47, :, 0]).all() and (got[17:47, :, 1:] == -np.inf).all()
    assert (got[48:] == 7.0).all()                                 # of no sequence


def test_scores_take_strided_queries():
    s = Setup(6, 2, 64, [300, 90], [4, 1], "bf16", seed=10).fill()
    ranges = s.cache.update_ranges(s.batch(s.ctx), s.cache.new_ranges())
    want = s.cache.page_scores(s.batch(), s.q, ranges)
    wide = torch.full((5, 9, 65), float("nan"), device=DEV, dtype=torch.bfloat16)
    wide[:, 2:8, 1:] = s.q
    assert torch.equal(s.cache.page_scores(s.batch(), wide[:, 2:8, 1:], ranges), want)
    assert torch.equal(s.cache.page_scores(s.batch(), s.q.transpose(0, 1).contiguous().transpose(0, 1), ranges), want)


# ---- picks ---------------------------------------------------------------------------

def _pick_case(ctx, rows, n_kv, n, first, last, seed, make=None, columns=None):
    width = columns or max(op.pages(max(ctx)), 1)
    table = torch.zeros((len(ctx), max(1, op.pages(max(ctx)))), dtype=torch.int32, device=DEV)  # not read
    rng = np.random.default_rng(seed)
    scores = rng.standard_normal((sum(rows), n_kv, width)).astype(np.float32)
    if make is not None:
        scores = make(scores, rng)
    cache = rp().KvqCache(1, n_kv, 64, device=DEV)
    b = cache.batch(_ints(ctx), table, row_offsets=_ints(np.concatenate([[0], np.cumsum(rows)])), n_rows=sum(rows), max_rows=max(rows))
    guard = torch.full((sum(rows) * n_kv * n + 64,), -77, dtype=torch.int32, device=DEV)
    out = guard[32:-32].view(sum(rows), n_kv, n)
    cache.pick_pages(b, torch.from_numpy(scores).to(DEV), n, first=first, last=last, out=out)
    got, r = out.cpu().numpy(), 0
    for c, k in zip(ctx, rows):
        for i in range(k):
            seen = max(0, op.pages(c - k + i + 1)) if c - k + i >= 0 else 0
            for h in range(n_kv):
                ref = op.pick(scores[r, h], seen, first, last, n)
                assert np.array_equal(got[r, h], ref), (c, i, h, got[r, h], ref)
            r += 1
    assert (guard[:32] == -77).all() and (guard[-32:] == -77).all()


def _ties(scores, rng):
    return np.round(scores)


def _same(scores, rng):
    return np.zeros_like(scores)


def _odd(scores, rng):
    return rng.choice(np.array([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3e38, -3e38, 1.0], np.float32), scores.shape)


@pytest.mark.parametrize("make", [None, _ties, _same, _odd])
@pytest.mark.parametrize("pages_", [1, 2, 63, 64, 65, 128, 200, 300, 600, 1024, 1500, 2048, 2049, 5000])
def test_picks(pages_, make):
    """Lists of every length that has a kernel of its own, at budgets around their ends."""
    ctx = [pages_ * 64, max(1, pages_ * 64 - 64), max(1, pages_ * 32 + 1)]
    for n, first, last in ((1, 0, 0), (2, 1, 1), (5, 0, 2), (16, 1, 2), (max(1, pages_ - 1), 0, 0), (pages_, 0, 1), (pages_ + 3, 2, 1), (40, 20, 20)):
        if first + last <= n:
            _pick_case(ctx, [1, 1, 1], 2, n, first, last, pages_ + n, make)


def test_picks_of_many_rows():
    _pick_case([500, 64, 1000, 0, 30], [400, 3, 130, 0, 35], 3, 6, 1, 2, 1, _ties)
    _pick_case([900] * 70, [3] * 70, 1, 4, 0, 1, 2, _ties, columns=33)


def test_picks_of_bad_batches():
    """A sequence out of bounds has -1 alone; rows of no sequence are left as they are."""
    cache = rp().KvqCache(1, 2, 64, device=DEV)
    b = cache.batch(_ints([640, 700, -1]), _ints(np.zeros((3, 10))), row_offsets=_ints([0, 1, 2, 5]), n_rows=7, max_rows=2, max_context=640)
    out = torch.full((7, 2, 4), 9, dtype=torch.int32, device=DEV)
    cache.pick_pages(b, torch.zeros((7, 2, 10), device=DEV), 4, out=out)
    assert out[0].tolist() == [[0, 1, 2, 9]] * 2 and (out[1:4] == -1).all() and (out[4:] == 9).all()


# ---- attention over picked pages -----------------------------------------------------

def _lists(s, n, rng, style="picks"):
    """Random lists of the rows: ascending, then -1 (as pick_pages); or in any order with -1 among them."""
    out = np.full((sum(s.rows), s.n_kv, n), -1, np.int32)
    r = 0
    for c, k in zip(s.ctx, s.rows):
        for i in range(k):
            seen = op.pages(c - k + i + 1) if c - k + i >= 0 else 0
            for h in range(s.n_kv):
                m = min(seen, n) if style == "picks" else int(rng.integers(0, min(seen, n) + 1))
                got = np.sort(rng.permutation(seen)[:m]) if style == "picks" else rng.permutation(seen)[:m]
                at = np.arange(m) if style == "picks" else np.sort(rng.permutation(n)[:m])
                out[r, h, at] = got
            r += 1
    return out


def _check_picked(s, out, picks, held=None, q=None, seqs=None):
    out, q = _f64(out), _f64(s.q if q is None else q)
    held = s.held() if held is None else held
    g, r = s.n_q // s.n_kv, 0
    for b, (c, k) in enumerate(zip(s.ctx, s.rows)):
        for i in range(k):
            for h in range(s.n_kv if seqs is None or b in seqs else 0):
                t = op.listed_tokens(picks[r, h], c - k + i)
                kk, vv = held[b][0][t, h:h + 1], held[b][1][t, h:h + 1]
                heads = slice(h * g, (h + 1) * g)
                ref, mag, top = okvq.attend(q[r:r + 1, heads], kk, vv, np.array([len(t) - 1]), s.hd ** -0.5)
                bar = _bound(ref, mag, top, len(t), s.hd, s.dtype, np.nanmax(np.abs(vv), initial=0))
                err = np.abs(out[r:r + 1, heads] - ref)
                assert (err <= bar).all(), (b, i, h, float((err / bar).max()))
            r += 1


@pytest.mark.parametrize("style", ["picks", "any"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd", SHAPES)
def test_attend_picked(n_q, n_kv, hd, dtype, style):
    rng = np.random.default_rng(n_q + hd)
    for ctx, rows, n in (([1, 64, 65, 700, 130], None, 3), ([1500, 63], None, 40), ([5, 200, 300, 0], [5, 6, 3, 0], 4), ([40, 70], [45, 2], 1)):
        s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=n).fill()
        picks = _lists(s, n, rng, style)
        out = s.cache.attend_picked(s.batch(), s.q, torch.from_numpy(picks).to(DEV))
        _check_picked(s, out, picks)
        if rows is None:
            b = s.cache.batch(_ints(ctx), s.dev_table)
            assert torch.equal(s.cache.attend_picked(b, s.q, torch.from_numpy(picks).to(DEV)), out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd,ctx,rows,n", [
    (28, 4, 128, [20000], None, 313),        # one row: split as far as it goes
    (4, 2, 64, [9000, 100], None, 90),
    (28, 4, 128, [3000] * 3, [70] * 3, 9),   # many blocks: no split
    (2, 1, 128, [6000], None, 200),
    (6, 3, 64, [700, 64, 1] * 26 + [300, 5], None, 20),      # eight waves
    (6, 3, 64, [700, 2] * 40, [2, 0] * 40, 20),              # and rows that share pages
    (7, 1, 128, [2500, 130, 60] * 5, [4, 4, 4] * 5, 40),     # split, rows that share pages
    (40, 2, 64, [900] * 3, [70] * 3, 9),     # two waves, more than 16 heads
    (9, 1, 128, [900, 5] * 3, [250, 5] * 3, 4),
])
def test_attend_picked_split_and_whole(n_q, n_kv, hd, ctx, rows, n, dtype):
    s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=n).fill()
    picks = _lists(s, n, np.random.default_rng(n))
    _check_picked(s, s.cache.attend_picked(s.batch(), s.q, torch.from_numpy(picks).to(DEV)), picks)


def test_all_pages_listed_is_attention():
    s = Setup(28, 4, 128, [700, 64, 3], [20, 1, 3], "bf16", seed=11).fill()
    picks = torch.arange(-1, 12, device=DEV, dtype=torch.int32).expand(24, 4, 13).contiguous()
    s.check(s.cache.attend_picked(s.batch(), s.q, picks))


def test_entries_that_name_no_seen_page_count_nothing():
    s = Setup(4, 2, 64, [200, 130], [2, 1], "bf16", seed=12).fill()
    rows = [[1, 7, -1, 4, 2 ** 31 - 1, -2 ** 31, 0, 3], [3, -9, 64, 4, 5, 1000, 2, -1], [0, 3, 3, 3, 2, -1, -1, 1]]
    picks = np.array(rows, np.int32)[:, None].repeat(2, 1)
    _check_picked(s, s.cache.attend_picked(s.batch(), s.q, torch.from_numpy(picks).to(DEV)), picks)


@pytest.mark.parametrize("n", [3, 70, 600])
def test_lists_that_leave_nothing_give_zeros(n):
    s = Setup(4, 2, 64, [200, 130, 10], [1, 1, 12], "bf16", seed=13).fill()
    picks = torch.full((14, 2, n), -1, dtype=torch.int32, device=DEV)
    picks[1, 1, n // 2] = 1
    out = s.cache.attend_picked(s.batch(), s.q, picks)
    _check_picked(s, out, picks.cpu().numpy())
    assert (out[0] == 0).all() and (out[1, :2] == 0).all() and (out[1, 2:] != 0).any() and (out[2:] == 0).all()


@pytest.mark.parametrize("n", [6, 300])
def test_a_page_listed_twice_counts_twice(n):
    s = Setup(4, 2, 64, [300], [1], "bf16", seed=14).fill()
    picks = np.full((1, 2, n), -1, np.int32)
    picks[0, :, :5] = [2, 0, 2, 4, 2]
    _check_picked(s, s.cache.attend_picked(s.batch(), s.q, torch.from_numpy(picks).to(DEV)), picks)


@pytest.mark.parametrize("n", [4, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_picked_bad_batches(dtype, n):
    """Bad page ids and contexts give NaN where they are listed; NaN keys and values behind the position or on pages that are not
    listed change nothing; rows of no sequence are left as they are."""
    s = Setup(4, 2, 64, [200, 200, 200, 200], [1, 1, 1, 1], dtype, seed=15)
    s.v[130, 0, 3], s.k[70, 1, 5] = float("nan"), float("inf")  # of the first sequence: pages 2 and 1
    s.fill()
    table = s.dev_table.clone()
    table[1, 1], table[2, 0] = s.cache.n_pages, -1
    picks = np.full((6, 2, n), -1, np.int32)
    picks[:, :, :3] = [0, 1, 3]
    picks[2, 1, 0] = -1
    b = s.cache.batch(_ints([200, 200, 200, 257]), table, row_offsets=_ints([0, 1, 2, 3, 4]), n_rows=6, max_rows=1, max_context=256)
    q = torch.cat([s.q, s.q[:2]])
    out = torch.full((6, 4, 64), 5.0, device=DEV, dtype=TYPES[dtype])
    s.cache.attend_picked(b, q, torch.from_numpy(picks).to(DEV), out=out)
    assert torch.isfinite(out[0, :2]).all() and torch.isnan(out[0, 2:]).all()
    assert torch.isnan(out[1]).all()
    assert torch.isnan(out[2, :2]).all() and torch.isfinite(out[2, 2:]).all()
    assert torch.isnan(out[3]).all() and (out[4:] == 5.0).all()
    held = s.held()
    t = op.listed_tokens(picks[0, 0], 199)
    ref, mag, top = okvq.attend(_f64(s.q[:1, :2]), held[0][0][t, :1], held[0][1][t, :1], np.array([len(t) - 1]), 0.125)
    assert (np.abs(_f64(out[:1, :2]) - ref) <= _bound(ref, mag, top, len(t), 64, dtype, 6.0)).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_nan_values_and_values_beyond_fp16(hd):
    """A NaN value block makes its 32 dimensions NaN for rows that attend to it; values that fp16 does not hold, on some pages of
    the list, go in bf16."""
    s = Setup(4, 2, hd, [640, 640], [1, 1], "bf16", seed=16)
    s.v[100, 0, 1] = float("nan")                    # page 1
    s.v[640 + 200:640 + 210] *= 2.0 ** 40            # page 3
    s.v[640 + 330:640 + 340] *= 2.0 ** -60
    s.fill()
    picks = np.array([[[0, 1, 5, 9]] * 2, [[0, 3, 5, 9]] * 2], np.int32)
    out = _f64(s.cache.attend_picked(s.batch(), s.q, torch.from_numpy(picks).to(DEV)))
    assert np.isnan(out[0, :2, :32]).all() and np.isfinite(out[0, :2, 32:]).all() and np.isfinite(out[0, 2:]).all()
    _check_picked(s, out if isinstance(out, torch.Tensor) else torch.from_numpy(out), picks, seqs=[1])


def test_attend_picked_strong_and_weak_pages():
    """Pages whose weights lie many orders apart, in the order of the list and against it."""
    s = Setup(14, 2, 64, [640], [1], "bf16", seed=17)
    for p in range(10):
        s.k[64 * p:64 * p + 64] *= 0.2
        s.k[64 * p:64 * p + 64] += s.q[0, ::7].float().sign().to(s.dt) * 0.35 * p
    s.fill()
    for order in (list(range(10)), list(range(9, -1, -1)), [9, 0, 5, 1]):
        picks = np.array([[order] * 2], np.int32)
        _check_picked(s, s.cache.attend_picked(s.batch(), s.q, torch.from_numpy(picks).to(DEV)), picks)


def test_attend_picked_strides_and_reuse_of_a_workspace():
    s = Setup(6, 2, 64, [3000], None, "bf16", seed=18).fill()
    picks = torch.from_numpy(_lists(s, 40, np.random.default_rng(1))).to(DEV)
    want = s.cache.attend_picked(s.batch(), s.q, picks)
    ws = s.cache.attend_picked_workspace(s.batch(), 6, 40)
    assert ws.numel() > 0
    ws.fill_(255)
    wide = torch.zeros((1, 8, 65), device=DEV, dtype=torch.bfloat16)
    wide[:, 1:7, 1:] = s.q
    out = torch.full((1, 9, 66), 3.0, device=DEV, dtype=torch.bfloat16)
    s.cache.attend_picked(s.batch(), wide[:, 1:7, 1:], picks, out=out[:, 2:8, 1:65], workspace=ws)
    assert torch.equal(out[:, 2:8, 1:65], want)
    assert (out[:, :2] == 3).all() and (out[:, 8:] == 3).all() and (out[:, :, 0] == 3).all() and (out[:, :, 65] == 3).all()


# ---- together ------------------------------------------------------------------------

class Decode:
    """A layer's decode loop over a pool that the GPU keeps: `n` sequences, prompts, then a token at a time."""

    def __init__(self, seed=0, n=5, n_q=14, n_kv=2, hd=64, max_context=900):
        self.n, self.n_q, self.n_kv, self.hd = n, n_q, n_kv, hd
        self.pages = rp().KvqPages(n * op.pages(max_context), n, max_context, device=DEV)
        self.pages.free_pages.copy_(torch.randperm(self.pages.n_pages).to(torch.int32))
        self.cache = rp().KvqCache(self.pages.n_pages, n_kv, hd, device=DEV)
        self.ranges = self.cache.new_ranges()
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(seed)
        self.k = [np.zeros((0, n_kv, hd)) for _ in range(n)]
        self.v = [np.zeros((0, n_kv, hd)) for _ in range(n)]

    def tensors(self, rows):
        rnd = lambda h: torch.randn((rows, h, self.hd), generator=self.gen, device=DEV).to(torch.bfloat16)  # noqa: E731
        return rnd(self.n_q), rnd(self.n_kv), rnd(self.n_kv)

    def step(self, lengths, n_rows, q, k, v, n_picks=4):
        batch, positions, slots = self.pages.fit(lengths, n_rows)
        self.cache.append(batch, k, v)
        self.cache.update_ranges(batch, self.ranges)
        scores = self.cache.page_scores(batch, q, self.ranges)
        picks = self.cache.pick_pages(batch, scores, n_picks, first=1, last=1)
        return self.cache.attend_picked(batch, q, picks), picks, scores, positions, slots

    def check(self, before, lengths, q, k, v, out, picks, scores, n_picks=4):
        """Against the plain forms; picks against those of the GPU's own scores."""
        r = 0
        for b, (c0, c1) in enumerate(zip(before, lengths)):
            self.k[b], self.v[b] = self.k[b][:c1], self.v[b][:c1]
            if c1 > c0:
                self.k[b] = np.concatenate([self.k[b], okvq.held(_f64(k[r:r + c1 - c0]))])
                self.v[b] = np.concatenate([self.v[b], okvq.held(_f64(v[r:r + c1 - c0]))])
            for i in range(max(0, c1 - c0)):
                pos = c0 + i
                ref, mag = op.page_scores(_f64(q[r:r + 1]), op.key_ranges(self.k[b]), [pos], scores.shape[2])
                got = _f64(scores[r:r + 1])
                fin = np.isfinite(ref)
                assert np.array_equal(fin, np.isfinite(got)) and (np.abs(got[fin] - ref[fin]) <= _score_bar(ref, mag, self.hd, "bf16")[fin]).all()
                g = self.n_q // self.n_kv
                for h in range(self.n_kv):
                    mine = picks[r, h].cpu().numpy()
                    assert np.array_equal(mine, op.pick(scores[r, h].cpu().numpy(), op.pages(pos + 1), 1, 1, n_picks))
                    t = op.listed_tokens(mine, pos)
                    heads = slice(h * g, (h + 1) * g)
                    want, m, top = okvq.attend(_f64(q[r:r + 1, heads]), self.k[b][t, h:h + 1], self.v[b][t, h:h + 1], np.array([len(t) - 1]), self.hd ** -0.5)
                    err = np.abs(_f64(out[r:r + 1, heads]) - want)
                    assert (err <= _bound(want, m, top, len(t), self.hd, "bf16", 6.0)).all()
                r += 1


def test_a_decode_loop():
    """Prompts, tokens, a sequence that ends and one that takes its place, a few tokens taken back."""
    d = Decode(1)
    steps = [[30, 700, 0, 64, 129], [31, 701, 0, 65, 130], [32, 702, 200, 66, 0], [33, 0, 201, 60, 150], [34, 800, 202, 61, 151],
             [35, 801, 198, 62, 152]]
    before = [0] * 5
    for lengths in steps:
        rows = sum(max(0, a - b) for a, b in zip(lengths, before))
        q, k, v = d.tensors(rows + 2)
        out, picks, scores, positions, slots = d.step(_ints(lengths), rows + 2, q, k, v)
        d.check(before, lengths, q, k, v, out, picks, scores)
        assert positions[rows:].tolist() == [-1, -1]
        before = lengths


def test_a_decode_loop_in_a_graph():
    """A captured step whose lengths grow between replays follows them; eager steps between the replays, on a pool of their own,
    give the same."""
    d, e = Decode(2, n=4), Decode(2, n=4)
    e.pages.free_pages.copy_(d.pages.free_pages)
    lengths = _ints([63, 127, 500, 1])
    for x in (d, e):
        q, k, v = x.tensors(691)
        x.step(lengths, 691, q, k, v)
    grown = lengths.clone()
    q, k, v = d.tensors(4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        warm = Decode(3, n=4)
        warm.step(_ints([1, 2, 3, 0]), 6, *warm.tensors(6))
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, picks, scores, positions, slots = d.step(grown, 4, q, k, v)
    for i in range(5):
        grown += 1
        for a, b in zip((q, k, v), d.tensors(4)):
            a.copy_(b)
        graph.replay()
        want = e.step(grown, 4, q.clone(), k.clone(), v.clone())
        torch.cuda.synchronize()
        for a, b in zip((out, picks, scores, positions, slots), want):
            assert torch.equal(a, b), i
        assert torch.equal(d.pages.page_table, e.pages.page_table) and torch.equal(d.pages.state, e.pages.state)
        assert torch.equal(d.ranges, e.ranges) and torch.equal(d.cache.blocks, e.cache.blocks)


def test_calls_on_a_stream_of_their_own():
    d, e = Decode(4), Decode(4)
    e.pages.free_pages.copy_(d.pages.free_pages)
    lengths = _ints([300, 64, 65, 0, 700])
    q, k, v = d.tensors(1129)
    want = d.step(lengths, 1129, q, k, v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = e.step(lengths, 1129, q, k, v)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_results_do_not_vary():
    d = Decode(5)
    q, k, v = d.tensors(2000)
    lengths = _ints([400, 400, 400, 400, 400])
    first = [t.clone() for t in d.step(lengths, 2000, q, k, v)]
    for _ in range(3):
        d.pages.fit(_ints([0] * 5), 0)
        for a, b in zip(d.step(lengths, 2000, q, k, v), first):
            assert torch.equal(a, b)


def test_refusals_on_the_device():
    R = rp()
    s = Setup(4, 2, 64, [100], None, "bf16").fill()
    b, c = s.batch(), s.cache
    ranges, scores, picks = c.new_ranges(), torch.zeros((1, 2, 2), device=DEV), torch.zeros((1, 2, 2), dtype=torch.int32, device=DEV)
    bad = [lambda: c.update_ranges(b, ranges.float()), lambda: c.update_ranges(b, ranges[:1]), lambda: c.update_ranges(b, ranges.cpu()),
           lambda: c.page_scores(b, s.q, ranges.transpose(0, 1)), lambda: c.page_scores(b, s.q[0], ranges),
           lambda: c.page_scores(b, s.q.half(), ranges), lambda: c.page_scores(b, s.q, ranges, out=scores[:, :1]),
           lambda: c.pick_pages(b, scores.double(), 2), lambda: c.pick_pages(b, scores, 2 ** 32 + 2), lambda: c.pick_pages(b, scores, 2, first=-1),
           lambda: c.pick_pages(b, scores, 2, out=picks[..., :1].contiguous()), lambda: c.attend_picked(b, s.q, picks.long()),
           lambda: c.attend_picked(b, s.q, picks[:, :1]), lambda: c.attend_picked(b, s.q[0], picks),
           lambda: c.attend_picked(b, s.q, picks, workspace=torch.empty(4096, dtype=torch.uint8))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: c.pick_pages(b, scores, 2, first=2, last=1), lambda: c.pick_pages(b, scores, 0, first=0, last=0),
                 lambda: c.page_scores(b, s.q, ranges, out=scores[..., :1].contiguous()), lambda: c.attend_picked(b, s.q, picks[..., :0].contiguous()),
                 lambda: c.attend_picked(b, s.q, picks, out=s.q), lambda: c.attend_picked(b, s.q, picks, scale=0.0)):
        with pytest.raises(R.RollpackError):
            call()
    p = R.KvqPages(4, 2, 100, device=DEV)
    for args in ((_ints([1]), 1), (_ints([1, 1]).long(), 2), (_ints([1, 1]).cpu(), 2), (_ints([1, 1]), -1), (_ints([1, 1]), 2 ** 24 + 1)):
        with pytest.raises(ValueError):
            p.fit(*args)


def test_tensors_that_need_a_gradient_are_refused():
    s = Setup(4, 2, 64, [100], None, "bf16").fill()
    b, c = s.batch(), s.cache
    ranges, picks, q = c.new_ranges(), torch.zeros((1, 2, 2), dtype=torch.int32, device=DEV), s.q.clone().requires_grad_()
    scores = torch.zeros((1, 2, 2), device=DEV)
    for call in (lambda: c.update_ranges(b, ranges.clone().requires_grad_()), lambda: c.page_scores(b, q, ranges), lambda: c.attend_picked(b, q, picks),
                 lambda: c.page_scores(b, s.q, ranges.clone().requires_grad_()), lambda: c.pick_pages(b, scores.clone().requires_grad_(), 2)):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()


def test_ranges_of_a_page_whose_last_tokens_were_taken_back():
    """Bounds of what is left; exact again with the next token."""
    d = Decode(7, n=1)
    q, k, v = d.tensors(100)
    d.step(_ints([100]), 100, q, k, v)
    d.pages.fit(_ints([70]), 0)
    held = okvq.held(_f64(k))[:70]
    table = d.pages.page_table[0, :2].cpu().numpy()
    lo, hi = (_f64(d.ranges)[table][:, :, i] for i in (0, 1))                   # [pages, n_kv, hd]
    for p, t in ((0, slice(0, 64)), (1, slice(64, 70))):
        assert (lo[p] <= held[t].min(0)).all() and (hi[p] >= held[t].max(0)).all()
    q2, k2, v2 = d.tensors(1)
    d.step(_ints([71]), 1, q2, k2, v2)
    held = np.concatenate([held, okvq.held(_f64(k2))])[64:]
    got = _f64(d.ranges)[table[1]]
    assert np.array_equal(got[:, 0], held.min(0)) and np.array_equal(got[:, 1], held.max(0))


def test_a_workspace_that_another_pool_used():
    """Of more than 1,024 sequences it keeps sums, of fewer what counts blocks, each in its own part."""
    a, b = Pools(3000, 1500, 128, 1), Pools(900, 100, 700, 2)
    b.gpu.struct.workspace = a.gpu.struct.workspace
    rng = np.random.default_rng(3)
    for _ in range(3):
        a.fit(rng.integers(0, 129, 1500).tolist(), 200_000)
        b.fit(rng.integers(0, 500, 100).tolist(), 60_000)
