"""The 4-bit KV cache on the GPU against its plain form in 64 bits (oracle/kvq.py).

What the cache holds is compared exactly: a power-of-two scale and a rounding have one right result.

Attention's bar comes from its roundings.  With u = 2^-24 and ctx keys, hd dimensions:
  scores   sums of hd products in fp32, in any order: (hd + 2) u sum|q||k| scale at most; the scaling to
           base 2 and the exponent's argument add two roundings of |s| (with the maximum's), the
           exponential 2^-21.  A probability is then off by the factor 1 + e_p, e_p = (hd + 6) u T + 2^-21,
           T the largest sum |q||k| scale; numerator and denominator both have it.
  sums     over keys, ctx additions and their products in fp32: (ctx + 64) u, twice.
  P        bf16 queries: rounded to fp16, 2^-11 of it, and where fp16 is subnormal 2^-25 for every key, the
           probabilities being at least 1 in sum (of pages with values beyond fp16: two pieces of bf16,
           2^-16).  fp32: three pieces of bf16, 2^-24.
  output   half a step: 2^-8 of the value in bf16, 2^-24 in fp32.
All but the last are relative to sum p|v|.
"""
import numpy as np
import pytest

from oracle import kvq as okvq
from tests.gpu_helpers import rp

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DEV = torch.device("cuda:0")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
P_BITS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -11}


def _bound(ref, mag, top, ctx, hd, dtype, vmax=0.0):
    u = 2.0 ** -24
    e_p = (hd + 6) * u * top[..., None] + 2.0 ** -21
    out = 2.0 ** -8 if dtype == "bf16" else u
    return out * np.abs(ref) * (1 + 2.0 ** -7) + mag * (2 * e_p + 2 * (ctx + 64) * u + P_BITS[dtype]) * 1.01 \
        + (ctx * vmax * 2.0 ** -25 if dtype == "bf16" else 0.0) + 1e-37


def _f64(t):
    return t.detach().to("cpu").double().numpy()


def _ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _room(kind, n_q, hd):
    """Bounds of a call (rows, context) under which sequences of many rows go to each form of the kernel for them,
    however few rows they have: many tiles; fewer of more pages, split over the keys; blocks of eight waves."""
    return {"": None, "tiles": (-(-8192 * 16 // n_q), 0), "split": (-(-512 * 16 // n_q), 64 * 8192 // hd),
            "eight": (-(-81920 // n_q), 4096)}[kind]


class Setup:
    """Sequences with random K and V in a cache whose pages are shuffled; numpy copies of what it holds.
    room: rows and context of the calls' bounds, if more than the sequences'; the rows behind the last one are NaN."""

    def __init__(self, n_q, n_kv, hd, ctx, rows=None, dtype="bf16", seed=0, spare=2, gain=1.0, room=None):
        self.n_q, self.n_kv, self.hd, self.ctx = n_q, n_kv, hd, list(ctx)
        self.rows = [1] * len(ctx) if rows is None else list(rows)
        self.dtype, self.dt = dtype, TYPES[dtype]
        rng = np.random.default_rng(seed)
        need = [-(-c // 64) for c in ctx]
        self.cache = rp().KvqCache(sum(need) + spare, n_kv, hd, device=DEV)
        perm = rng.permutation(sum(need) + spare).astype(np.int32)
        self.room = room = room and (max(room[0], sum(self.rows)), room[1])
        self.table = np.full((len(ctx), max(need + [1, room[1] // 64 if room else 0])), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.dev_table = torch.from_numpy(self.table).to(DEV)
        tot = sum(ctx)
        chan = np.where(rng.random((n_kv, hd)) < 0.05, 6.0, 1.0) * gain
        self.k = torch.from_numpy((rng.standard_normal((tot, n_kv, hd)) * chan).astype(np.float32)).to(DEV).to(self.dt)
        self.v = torch.from_numpy(rng.standard_normal((tot, n_kv, hd)).astype(np.float32)).to(DEV).to(self.dt)
        q = rng.standard_normal((sum(self.rows), n_q, hd)).astype(np.float32)
        if room:
            q = np.concatenate([q, np.full((room[0] - len(q), n_q, hd), np.nan, np.float32)])
        self.q = torch.from_numpy(q).to(DEV).to(self.dt)

    def batch(self, rows=None, ctx=None, **kw):
        if rows is None and self.room:
            kw = {**dict(n_rows=self.room[0], max_rows=self.room[0]), **kw}
        rows = self.rows if rows is None else rows
        ctx = self.ctx if ctx is None else ctx
        off = _ints(np.concatenate([[0], np.cumsum(rows)]))
        return self.cache.batch(_ints(ctx), self.dev_table, row_offsets=off,
                                **{**dict(n_rows=int(sum(rows)), max_rows=int(max(rows))), **kw})

    def fill(self):
        self.cache.append(self.batch(self.ctx), self.k, self.v)
        return self

    def held(self):
        off = np.concatenate([[0], np.cumsum(self.ctx)])
        k, v = okvq.held(_f64(self.k)), okvq.held(_f64(self.v))
        return [(k[off[b]:off[b + 1]], v[off[b]:off[b + 1]]) for b in range(len(self.ctx))]

    def check(self, out, q=None, held=None, seqs=None):
        q = _f64(self.q if q is None else q)
        out = _f64(out)
        held = self.held() if held is None else held
        at = 0
        worst = 0.0
        for b, (c, n) in enumerate(zip(self.ctx, self.rows)):
            if n and (seqs is None or b in seqs):
                pos = np.arange(c - n, c)
                ref, mag, top = okvq.attend(q[at:at + n], *held[b], pos, self.hd ** -0.5)
                err, bar = np.abs(out[at:at + n] - ref), _bound(ref, mag, top, c, self.hd, self.dtype, np.nanmax(np.abs(held[b][1]), initial=0))
                assert (err <= bar).all(), (b, c, n, float((err / bar).max()), np.argwhere(~(err <= bar))[:4].tolist())
                worst = max(worst, float((err / bar).max()))
            at += n
        return worst


# ---- append and read -----------------------------------------------------------------

@pytest.mark.parametrize("n_kv,hd,dtype,ctx,rows", [
    (4, 128, "bf16", [1, 63, 64, 65, 130, 7], None),
    (2, 64, "f32", [1, 63, 64, 65, 130, 7], None),
    (3, 64, "bf16", [5, 200, 1], [5, 3, 1]),
    (1, 128, "f32", [70, 64, 3, 129] * 20, [9, 64, 1, 2] * 20),     # 80 sequences: offsets past one wave's 64
    (5, 64, "bf16", [3] * 131, [1] * 131),
    (2, 64, "bf16", [3, 1, 0, 70, 2, 0, 0] * 40, [2, 1, 0, 70, 2, 0, 0] * 40),
    (2, 128, "f32", [2] * 65, [2] * 65),
    (2, 64, "f32", [1, 2] * 64 + [9], [1, 2] * 64 + [0]),
])
def test_append_then_read_holds_the_oracles_values(n_kv, hd, dtype, ctx, rows):
    s = Setup(n_kv, n_kv, hd, ctx, rows, dtype, seed=len(ctx)).fill()
    ref = s.held()
    for out_type in (torch.float32, torch.bfloat16):
        k, v = s.cache.read(s.batch(), dtype=out_type)
        at = 0
        for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
            assert np.array_equal(_f64(k[at:at + n]), ref[b][0][c - n:]), (b, out_type)
            assert np.array_equal(_f64(v[at:at + n]), ref[b][1][c - n:]), (b, out_type)
            at += n


@pytest.mark.parametrize("hd", [64, 128])
def test_append_row_by_row_equals_whole(hd):
    """A token's bytes are its own: appended one at a time, in any order, the cache ends the same."""
    s = Setup(2, 2, hd, [131, 1, 64], seed=1).fill()
    whole = s.cache.blocks.clone()
    s.cache.blocks.zero_()
    off = np.concatenate([[0], np.cumsum(s.ctx)])
    order = [(b, t) for b, c in enumerate(s.ctx) for t in range(c)]
    np.random.default_rng(0).shuffle(order)
    for b, t in order:
        one = s.cache.batch(_ints([t + 1]), s.dev_table[b:b + 1])
        s.cache.append(one, s.k[off[b] + t:off[b] + t + 1], s.v[off[b] + t:off[b] + t + 1])
    assert torch.equal(s.cache.blocks, whole)


def test_quantiser_ties_extremes_and_nan():
    """Ties, the border of the scales, tiny and huge blocks, infinities and NaN, in both types."""
    rng = np.random.default_rng(9)
    rows = [np.r_[[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], -np.r_[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], np.zeros(16)]]
    for e in (-149, -133, -127, -126, -125, -124, -30, 0, 40, 124, 125, 126, 127):
        for m in (1.0, 1.5, 1.75, 1.7578125, 1.9921875):
            x = rng.uniform(-1, 1, 32)
            with np.errstate(over="ignore"):
                x = np.ldexp(x * m, e)
            x[rng.integers(32)] = np.ldexp(m, e)
            rows.append(x)
    for bad in (np.inf, -np.inf, np.nan):
        x = rng.uniform(-1, 1, 32)
        x[rng.integers(32)] = bad
        rows.append(x)
    rows.append(np.zeros(32))
    while len(rows) % 4:
        rows.append(rng.uniform(-1, 1, 32))
    x = np.concatenate(rows).reshape(-1, 1, 128)
    n = len(x)
    for name, dt in TYPES.items():
        t = torch.from_numpy(x.astype(np.float32)).to(DEV).to(dt)
        cache = rp().KvqCache(-(-n // 64), 1, 128, device=DEV)
        b = cache.batch(_ints([n]), _ints([list(range(-(-n // 64)))]), row_offsets=_ints([0, n]), n_rows=n)
        cache.append(b, t, -t)
        ref = okvq.held(_f64(t))
        for out in TYPES.values():
            k, v = cache.read(b, dtype=out)
            assert np.array_equal(_f64(k), ref, equal_nan=True), name
            assert np.array_equal(_f64(v), -ref, equal_nan=True), name


def test_strided_and_misaligned_tensors():
    """Rows inside wider tensors, heads outermost, odd offsets: element accesses where 16 bytes do not fit."""
    for dtype in ("bf16", "f32"):
        s = Setup(6, 2, 64, [100, 33], rows=[9, 33], dtype=dtype, seed=4).fill()
        base = s.cache.blocks.clone()
        tot = sum(s.ctx)
        wide = torch.zeros((tot, 5 * 64 + 3), dtype=s.dt, device=DEV)
        heads = torch.zeros((2, tot, 64), dtype=s.dt, device=DEV)
        k = wide[:, 3:3 + 128].view(tot, 2, 64)
        k.copy_(s.k)
        v = heads.permute(1, 0, 2)
        v.copy_(s.v)
        s.cache.blocks.zero_()
        s.cache.append(s.batch(s.ctx), k, v)
        assert torch.equal(s.cache.blocks, base)
        n = sum(s.rows)
        kw = torch.full((n, 5 * 64 + 3), 7.0, dtype=s.dt, device=DEV)
        vw = torch.full((2, n, 64), 7.0, dtype=s.dt, device=DEV)
        s.cache.read(s.batch(), out=(kw[:, 3:3 + 128].view(n, 2, 64), vw.permute(1, 0, 2)))
        rk, rv = s.cache.read(s.batch(), dtype=s.dt)
        assert torch.equal(kw[:, 3:3 + 128].reshape(n, 2, 64), rk) and torch.equal(vw.permute(1, 0, 2), rv)
        assert (kw[:, :3] == 7).all() and (kw[:, 131:] == 7).all()
        qw = torch.zeros((n, 6 * 64 + 5), dtype=s.dt, device=DEV)
        q = qw[:, 1:1 + 6 * 64].view(n, 6, 64)
        q.copy_(s.q)
        ow = torch.full((6, n, 64 + 1), 7.0, dtype=s.dt, device=DEV)
        s.cache.attend(s.batch(), q, out=ow[:, :, :64].permute(1, 0, 2))
        assert torch.equal(ow[:, :, :64].permute(1, 0, 2), s.cache.attend(s.batch(), s.q)) and (ow[:, :, 64] == 7).all()
        one = s.q[:, :1].expand(n, 6, 64)  # one query for every head: a stride of zero
        assert torch.equal(s.cache.attend(s.batch(), one), s.cache.attend(s.batch(), one.contiguous()))


# ---- attention -----------------------------------------------------------------------

EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 191, 192, 255, 256, 257, 320, 513]
HEADS = [(28, 4, 128), (14, 2, 64), (7, 1, 128), (4, 4, 64), (16, 1, 64), (20, 1, 128), (40, 2, 64), (5, 5, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd", HEADS)
def test_attend_single_tokens(n_q, n_kv, hd, dtype):
    s = Setup(n_q, n_kv, hd, EDGES, dtype=dtype, seed=n_q).fill()
    out = s.cache.attend(s.batch(), s.q)
    s.check(out)
    # without row offsets: the same rows, the same result
    plain = s.cache.batch(_ints(s.ctx), s.dev_table)
    assert torch.equal(s.cache.attend(plain, s.q), out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd", [(28, 4, 128), (14, 2, 64), (5, 1, 128), (3, 3, 64)])
def test_attend_several_rows(n_q, n_kv, hd, dtype):
    """Prompts (every row of the context), later pieces of a context, and single tokens in one batch."""
    ctx = [1, 2, 16, 17, 63, 64, 65, 100, 128, 129, 200, 40, 300, 65, 192]
    rows = [1, 2, 16, 17, 63, 64, 65, 30, 128, 5, 1, 39, 3, 64, 2]
    s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=n_q + 1).fill()
    s.check(s.cache.attend(s.batch(), s.q))


@pytest.mark.parametrize("n_q,n_kv,hd,kind", [
    (28, 4, 128, "tiles"), (28, 4, 128, "split"), (28, 4, 128, "eight"), (14, 2, 64, "tiles"), (14, 2, 64, "split"),
    (40, 2, 128, "split"), (40, 2, 128, "eight"), (3, 3, 64, "tiles"), (3, 1, 128, "eight"), (6, 1, 64, "split"),
])
def test_attend_prompts_and_long_pieces(n_q, n_kv, hd, kind):
    """Sequences below, at and above 64 columns, tiles of 128 and 256 columns that end anywhere, contexts of several
    items, and rows behind the last sequence, which stay as they were."""
    group = n_q // n_kv
    edge = [max(1, c // group) for c in (63, 64, 65, 127, 128, 129, 255, 256, 257)]
    rows = [1, 2] + edge + [e + 1 for e in edge] + [100, 1, 30, 0, 17]
    ctx = [1, 9] + edge + [e + 64 for e in edge] + [700, 1100, 1200, 50, 513]
    s = Setup(n_q, n_kv, hd, ctx, rows, seed=n_q + 2, room=_room(kind, n_q, hd)).fill()
    out = torch.full_like(s.q, 5.0)
    s.cache.attend(s.batch(), s.q, out=out)
    s.check(out)
    assert (out[sum(rows):] == 5).all()


@pytest.mark.parametrize("n_q,n_kv,hd,kind", [(28, 4, 128, "tiles"), (28, 4, 128, "eight"), (28, 4, 128, "split"), (14, 2, 64, "split")])
def test_attend_one_sequence_of_many_rows(n_q, n_kv, hd, kind):
    """All sequences have as many rows as the bound: nothing is left for the other kernel."""
    n, c = _room(kind, n_q, hd)
    n = min(n, 300)
    s = Setup(n_q, n_kv, hd, [900], [n], seed=31)
    wide = torch.full((1, max(15, -(-c // 64))), -1, dtype=torch.int32, device=DEV)
    wide[:, :15] = s.dev_table
    s.fill()
    rows = _room(kind, n_q, hd)[0]
    q = torch.zeros((rows, n_q, hd), dtype=s.dt, device=DEV)
    q[:n] = s.q
    b = s.cache.batch(_ints([900]), wide, row_offsets=_ints([0, n]), n_rows=rows, max_rows=rows)
    out = s.cache.attend(b, q)
    s.check(out)


@pytest.mark.parametrize("dtype,ctx,rows", [
    ("bf16", [5000], [1]),                              # one row, split over the GPU and joined
    ("f32", [4100], [2]),
    ("bf16", [3000, 1, 700, 4097, 64, 0], [1, 1, 1, 1, 1, 1]),   # ragged: some rows of one item, some of many
    ("bf16", [2500, 900], [3, 20]),
    ("bf16", [1500, 64, 1], [200, 64, 1]),
])
def test_attend_long_contexts(dtype, ctx, rows):
    s = Setup(7, 1, 128, ctx, rows, dtype, seed=3).fill()
    s.check(s.cache.attend(s.batch(), s.q))
    s = Setup(6, 2, 64, ctx, rows, dtype, seed=4).fill()
    s.check(s.cache.attend(s.batch(), s.q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
def test_attend_as_many_blocks_as_compute_units(hd, dtype):
    """256 blocks with long contexts among them: blocks of eight waves."""
    rng = np.random.default_rng(37)
    ctx = [1300, 1100, 0] + rng.integers(1, 90, 61).tolist()
    s = Setup(12, 4, hd, ctx, [1, 1, 0] + [1] * 61, dtype=dtype, seed=38).fill()
    s.check(s.cache.attend(s.batch(), s.q))


def test_attend_many_sequences():
    """More sequences than a wave has lanes, empty ones among them, and none at all in the last places."""
    rng = np.random.default_rng(8)
    ctx = rng.integers(1, 150, 300).tolist()
    rows = [int(min(c, rng.integers(0, 4))) for c in ctx]
    s = Setup(14, 2, 64, ctx, rows, seed=5).fill()
    s.check(s.cache.attend(s.batch(), s.q))
    out = s.cache.attend(s.cache.batch(_ints(ctx), s.dev_table), s.q[:1].expand(300, 14, 64))
    s.rows = [1] * 300
    s.check(out, q=s.q[:1].expand(300, 14, 64))


@pytest.mark.parametrize("kind", ["tiles", "eight"])
def test_prompts_of_more_sequences_than_lanes(kind):
    rng = np.random.default_rng(34)
    ctx = rng.integers(1, 200, 150).tolist()
    rows = [int(min(c, rng.integers(0, 25))) for c in ctx]
    s = Setup(28, 4, 128, ctx, rows, seed=35, room=_room(kind, 28, 128)).fill()
    out = torch.full_like(s.q, 5.0)
    s.cache.attend(s.batch(), s.q, out=out)
    s.check(out)
    assert (out[sum(rows):] == 5).all()


@pytest.mark.parametrize("kind", ["", "tiles", "split", "eight"])
def test_more_rows_than_tokens(kind):
    """Rows before a sequence's first token are zero, in the middle of a tile and a page too; the others are right."""
    ctx, rows = [70, 1, 40, 300, 0], [100, 90, 40, 310, 20]
    s = Setup(14, 2, 64, ctx, rows, seed=36, room=_room(kind if kind != "eight" else "", 14, 64)) if kind != "eight" else \
        Setup(28, 4, 128, ctx, rows, seed=36, room=_room(kind, 28, 128))
    s.fill()
    out = _f64(s.cache.attend(s.batch(), s.q))
    q, at = _f64(s.q), 0
    for b, (c, n) in enumerate(zip(ctx, rows)):
        assert (out[at:at + n - c] == 0).all()
        if c:
            k, v = s.held()[b]
            ref, mag, top = okvq.attend(q[at + n - c:at + n], k, v, np.arange(c), s.hd ** -0.5)
            bar = _bound(ref, mag, top, c, s.hd, "bf16", np.abs(v).max())
            assert (np.abs(out[at + n - c:at + n] - ref) <= bar).all(), b
        at += n


def test_rows_without_keys_are_zero():
    """Empty contexts and rows before their sequence's first token."""
    s = Setup(14, 2, 64, [0, 3, 0, 70], rows=[2, 5, 1, 1], seed=6)
    k = torch.zeros((sum(s.rows), 2, 64), device=DEV, dtype=s.dt)
    b = s.batch()
    s.cache.append(b, k + 1, k + 2)  # rows 0 and 1 of sequence 1 have no position, those of 0 and 2 neither
    out = s.cache.attend(b, s.q)
    assert (out[:4] == 0).all() and (out[7] == 0).all()
    assert (out[4:7] == 2).all()
    rk, rv = s.cache.read(b)
    assert (rk[:4] == 0).all() and (rv[:4] == 0).all() and (rk[7] == 0).all() and (rv[4:7] == 2).all()


@pytest.mark.parametrize("n_q,n_kv,hd", [(28, 4, 128), (14, 2, 64)])
def test_what_lies_behind_the_context_does_not_matter(n_q, n_kv, hd):
    """Bytes of places that no sequence holds, table entries past a context and padding rows may be anything."""
    ctx = [1, 37, 64, 70, 129, 300]
    s = Setup(n_q, n_kv, hd, ctx, seed=7)
    s.cache.blocks.fill_(255)  # every scale a NaN
    s.fill()
    s.check(s.cache.attend(s.batch(), s.q))
    s.rows = [1, 20, 64, 3, 128, 40]
    q = torch.randn((sum(s.rows) + 9, n_q, hd), device=DEV, dtype=torch.float32).to(s.dt)
    q[-9:] = float("nan")
    out = torch.full_like(q, 5.0)
    s.cache.attend(s.batch(n_rows=sum(s.rows) + 9), q, out=out)
    s.check(out, q=q)
    assert (out[-9:] == 5).all()
    k = torch.full((sum(s.rows) + 9, n_kv, hd), 3.0, device=DEV, dtype=s.dt)
    v = k.clone()
    s.cache.read(s.batch(n_rows=sum(s.rows) + 9), out=(k, v))
    assert (k[-9:] == 3).all() and (v[-9:] == 3).all()
    before = s.cache.blocks.clone()
    s.cache.append(s.batch(n_rows=sum(s.rows) + 9), k, v)  # what was read, again; the padding nowhere
    assert torch.equal(s.cache.blocks, before)


@pytest.mark.parametrize("hd,rows,kind", [
    (64, [1, 1, 1], ""), (128, [1, 1, 1], ""), (64, [90, 130, 20], ""), (128, [90, 130, 20], ""),
    (64, [90, 130, 30], "tiles"), (128, [90, 130, 30], "tiles"), (64, [90, 130, 30], "split"), (128, [90, 130, 30], "split"),
    (128, [90, 130, 30], "eight"),
])
def test_nan_and_infinities_reach_only_rows_that_see_them(hd, rows, kind):
    """A NaN key makes its readers' rows NaN, a NaN value block its 32 dimensions of them; earlier rows are untouched."""
    n_q, n_kv = 6, 2
    ctx = [100, 130, 1200]
    s = Setup(n_q, n_kv, hd, ctx, rows, seed=8, room=_room(kind, n_q, hd))
    s.k[40, 0, 5] = float("nan")       # sequence 0, position 40, head 0
    s.v[100 + 60, 1, 40] = float("inf")  # sequence 1, position 60, head 1, dimensions 32..63
    s.v[230 + 1195, 0, hd - 1] = float("nan")
    s.fill()
    out = _f64(s.cache.attend(s.batch(), s.q))
    held = s.held()
    clean = [(np.nan_to_num(k), np.nan_to_num(v)) for k, v in held]
    at = 0
    for b, (c, n) in enumerate(zip(ctx, rows)):
        pos = np.arange(c - n, c)
        ref, mag, top = okvq.attend(_f64(s.q[at:at + n]), *clean[b], pos, hd ** -0.5)
        want = np.zeros(ref.shape, bool)
        if b == 0:
            want[pos >= 40, :3] = True
        elif b == 1:
            want[pos >= 60, 3:, 32:64] = True
        else:
            want[pos >= 1195, :3, hd - 32:] = True
        got = out[at:at + n]
        assert np.array_equal(np.isnan(got), want), b
        bar = _bound(ref, mag, top, c, hd, "bf16", np.abs(clean[b][1]).max())
        assert (np.abs(got - ref)[~want] <= bar[~want]).all(), b
        at += n
    q = s.q.clone()
    q[0, 1] = float("nan")
    q[0, 2] = float("inf")
    out = s.cache.attend(s.batch(), q)
    assert torch.isnan(out[0, 1:3]).all() and (rows[0] == 1 or not torch.isnan(out[0, 3:]).any())


@pytest.mark.parametrize("kind", ["", "tiles", "split", "eight"])
def test_large_scores_do_not_overflow(kind):
    """Scores in the thousands, and equal ones: the running maximum keeps every exponent in range."""
    for dtype in ("bf16", "f32"):
        s = Setup(7, 1, 128, [700, 65, 1], rows=[30 if kind else 3, 65, 1], dtype=dtype, seed=10, gain=30.0, room=_room(kind, 7, 128)).fill()
        s.q *= 20
        out = _f64(s.cache.attend(s.batch(), s.q))[:sum(s.rows)]
        assert np.isfinite(out).all()
        s.q *= 0  # every key alike: the mean of the values
        s.check(s.cache.attend(s.batch(), s.q))


@pytest.mark.parametrize("hd,kind", [(64, ""), (128, ""), (64, "tiles"), (128, "tiles"), (64, "split"), (128, "split"), (128, "eight")])
def test_values_beyond_half_precision(hd, kind):
    """Value blocks that fp16 does not hold, tiny and huge, among ordinary ones; keys likewise."""
    for dtype in ("bf16", "f32"):
        s = Setup(7, 1, hd, [700, 130, 64, 200], rows=[12 if kind else 1, 130, 3, 1], dtype=dtype, seed=21, room=_room(kind, 7, hd))
        s.v[5::64] *= 2.0 ** 20
        s.v[9::32, :, :32] *= 2.0 ** -40
        s.v[700:830] *= 2.0 ** -30
        s.v[830:894] *= 2.0 ** 90
        s.k[3::16] *= 2.0 ** -20
        s.fill()
        s.check(s.cache.attend(s.batch(), s.q))


def test_device_values_out_of_bounds_are_not_followed():
    """Page ids outside the cache, contexts past the bound, too many rows: NaN for those rows alone, and no append."""
    ctx = [70, 70, 70, 70, 70, 130]
    s = Setup(14, 2, 64, ctx, seed=11).fill()
    good = s.cache.attend(s.batch(), s.q)
    t = s.dev_table.clone()
    t[1, 1] = s.cache.n_pages          # the page of its last token
    t[2, 0] = -7
    t[5, 2] = 2 ** 31 - 1
    c = _ints([70, 70, 70, 129 + 64, -3, 130])
    b = s.cache.batch(c, t, max_context=192)
    out = s.cache.attend(b, s.q)
    assert torch.equal(out[0], good[0])
    for i in (1, 2, 3, 4, 5):
        assert torch.isnan(out[i]).all(), i
    before = s.cache.blocks.clone()
    k = torch.full((6, 2, 64), 9.0, device=DEV, dtype=s.dt)
    t[0, 1] = -1
    t[2, 1] = 2 ** 31 - 1
    s.cache.append(s.cache.batch(c, t, max_context=192), k, k)
    assert torch.equal(s.cache.blocks, before)
    rk, rv = s.cache.read(s.cache.batch(c, t, max_context=192))
    assert torch.isnan(rk).all() and torch.isnan(rv).all()
    # more rows than max_rows: those up to it NaN, the others left; descending offsets touch nothing outside the rows
    s.rows = [1, 4, 1, 1, 1, 1]
    q = torch.randn((9, 14, 64), device=DEV).to(s.dt)
    out = torch.full_like(q, 5.0)
    s.cache.attend(s.batch(max_rows=2), q, out=out)
    assert torch.isnan(out[1:3]).all() and (out[3:5] == 5).all() and not torch.isnan(out[5:]).any()
    wild = s.cache.batch(_ints(ctx), s.dev_table, row_offsets=_ints([0, 2 ** 31 - 1, -5, 3, 9, 2, 4]), n_rows=9)
    s.cache.attend(wild, q)
    s.cache.read(wild)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["tiles", "split", "eight"])
def test_bad_pages_and_contexts_of_prompts(kind):
    """As above where sequences have many rows: a bad page's readers are NaN, bad contexts' rows too, the rest right."""
    ctx, rows = [600, 300, 300, 128, 70], [100, 80, 60, 128, 1]
    s = Setup(28, 4, 128, ctx, rows, seed=32, room=_room(kind, 28, 128)).fill()
    t = s.dev_table.clone()
    t[0, 8] = s.cache.n_pages  # of tokens 512 to 575
    t[3, 1] = -1
    b = s.cache.batch(_ints([600, 2 ** 31 - 1, -5, 128, 70]), t, row_offsets=_ints(np.concatenate([[0], np.cumsum(rows)])),
                      n_rows=s.room[0], max_rows=s.room[0])
    out = torch.full_like(s.q, 5.0)
    s.cache.attend(b, s.q, out=out)
    nan = torch.isnan(out).flatten(1)
    want = np.zeros(s.room[0], bool)
    want[12:100] = True          # positions 512 on
    want[100:240] = True
    want[240 + 64:368] = True
    assert np.array_equal(nan.all(1).cpu().numpy(), want) and np.array_equal(nan.any(1).cpu().numpy(), want)
    assert (out[369:] == 5).all()
    good = s.cache.attend(s.batch(), s.q)
    keep = torch.from_numpy(~want[:369]).to(DEV)
    assert torch.equal(out[:369][keep], good[:369][keep])
    # too many rows for the bound
    out = torch.full_like(s.q, 5.0)
    s.cache.attend(s.batch(max_rows=90), s.q, out=out)
    assert torch.isnan(out[:90]).all() and (out[90:100] == 5).all() and torch.isnan(out[240:330]).all() and (out[330:368] == 5).all()
    assert torch.equal(out[100:240], s.cache.attend(s.batch(max_rows=90), s.q)[100:240]) and torch.isfinite(out[100:240]).all()
    # offsets that descend or run away stay inside the tensors
    s.cache.attend(s.cache.batch(_ints(ctx), s.dev_table, row_offsets=_ints([0, 2 ** 31 - 1, -5, 300, 90, 400]),
                                 n_rows=s.room[0], max_rows=s.room[0]), s.q)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["tiles", "split", "eight"])
def test_prompts_captured_and_replayed(kind):
    """One graph for steps whose rows and contexts change on the device, sequences moving between the two kernels."""
    s = Setup(28, 4, 128, [700, 900, 64, 513], [100, 1, 64, 9], seed=33, room=_room(kind, 28, 128)).fill()
    n = s.room[0]
    ctx, off = _ints(s.ctx), _ints([0, 0, 0, 0, 0])
    q = torch.zeros((n, 28, 128), dtype=s.dt, device=DEV)
    b = s.cache.batch(ctx, s.dev_table, row_offsets=off, n_rows=n, max_rows=n)
    ws = s.cache.attend_workspace(b, 28)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.cache.attend(b, q, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    out = torch.zeros_like(q)
    with torch.cuda.graph(graph):
        s.cache.attend(b, q, out=out, workspace=ws)
    held = s.held()
    for i, (c, rows) in enumerate([([700, 900, 64, 513], [100, 1, 64, 9]), ([700, 900, 64, 513], [0, 90, 1, 100]),
                                   ([1, 899, 0, 200], [1, 10, 0, 200])]):
        ctx.copy_(_ints(c))
        off.copy_(_ints(np.concatenate([[0], np.cumsum(rows)])))
        q.copy_(torch.randn(q.shape, device=DEV, generator=torch.Generator(DEV).manual_seed(i)))
        ws.fill_(float("nan")) if ws.is_floating_point() else ws.fill_(255)
        out.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        now = Setup(28, 4, 128, c, rows, seed=0)
        now.check(out, q=q, held=[(k[:x], v[:x]) for (k, v), x in zip(held, c)])
        assert (out[sum(rows):] == 5).all()
        assert torch.equal(out, s.cache.attend(b, q, out=torch.full_like(q, 5.0)))


def test_offsets_that_claim_far_more_rows_than_there_are():
    """Every second sequence claims all rows: 2^31 tiles between them, of which as many are taken as fit the bound."""
    n_rows, n_seqs = 1 << 15, 1 << 15
    cache = rp().KvqCache(2, 1, 64, device=DEV)
    off = torch.zeros(n_seqs + 1, dtype=torch.int32, device=DEV)
    off[1::2] = n_rows
    b = cache.batch(torch.ones(n_seqs, dtype=torch.int32, device=DEV), torch.zeros((n_seqs, 1), dtype=torch.int32, device=DEV),
                    row_offsets=off, n_rows=n_rows, max_rows=n_rows)
    q = torch.zeros((n_rows, 64, 64), dtype=torch.bfloat16, device=DEV)
    out = cache.attend(b, q)
    k, v = cache.read(b)
    torch.cuda.synchronize()
    assert out.shape == q.shape and k.shape == (n_rows, 1, 64)


def test_shared_pages_and_strided_tables():
    """Sequences that share a prefix's pages, a table that is a slice of a wider one."""
    s = Setup(14, 2, 64, [200, 200], seed=12).fill()
    wide = torch.full((2, 11), -1, dtype=torch.int32, device=DEV)
    wide[0, :4] = s.dev_table[0, :4]
    wide[1, :2] = s.dev_table[0, :2]
    wide[1, 2:4] = s.dev_table[1, 2:4]
    b = s.cache.batch(_ints(s.ctx), wide[:, :4])
    assert b.struct.table_stride == 11
    held = s.held()
    mixed = [held[0], tuple(np.concatenate([held[0][i][:128], held[1][i][128:]]) for i in range(2))]
    s.check(s.cache.attend(b, s.q), held=mixed)


def test_cache_beyond_four_gib():
    """Offsets past 32 bits: the pages at the end of a 4.6 GB cache."""
    n_pages, n_kv = 132000, 4
    cache = rp().KvqCache(n_pages, n_kv, 128, device=DEV)
    assert cache.blocks.numel() > 2 ** 32
    s = Setup(28, n_kv, 128, [130, 64], seed=13)
    s.cache, s.dev_table = cache, _ints([[n_pages - 1, 7, n_pages - 2], [n_pages - 3, 0, 0]])
    s.fill()
    s.check(s.cache.attend(s.batch(), s.q))
    k, v = s.cache.read(s.batch())
    assert np.array_equal(_f64(k[0]), s.held()[0][0][-1])


# ---- streams, graphs, and the operators together ----------------------------------------

def test_other_streams():
    """Work on torch's current stream: behind what was queued there, with results ready there."""
    s = Setup(28, 4, 128, [300, 2000, 65], seed=14).fill()
    ref = s.cache.attend(s.batch(), s.q)
    b = s.batch()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q = torch.zeros_like(s.q)
        big = torch.randn(4096, 4096, device=DEV)
        for _ in range(10):
            big = big @ big * 1e-3
        q.copy_(s.q)
        out = s.cache.attend(b, q)
    side.synchronize()
    assert torch.equal(out, ref)


def test_two_calls_at_once():
    """Two streams with a workspace each; results equal those of one after the other."""
    a = Setup(28, 4, 128, [3000], seed=15).fill()
    b = Setup(28, 4, 128, [2900, 100], seed=16).fill()
    ra, rb = a.cache.attend(a.batch(), a.q), b.cache.attend(b.batch(), b.q)
    ba, bb = a.batch(), b.batch()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(20):
        with torch.cuda.stream(s1):
            x = a.cache.attend(ba, a.q)
        with torch.cuda.stream(s2):
            y = b.cache.attend(bb, b.q)
        outs.append((x, y))
    torch.cuda.synchronize()
    assert all(torch.equal(x, ra) and torch.equal(y, rb) for x, y in outs)


@pytest.mark.parametrize("n_q,n_kv,hd", [(28, 4, 128), (14, 2, 64)])
def test_decode_loop_captured_and_replayed(n_q, n_kv, hd):
    """Prompts enter the cache and are attended; then every step appends a token per sequence and attends, as one
    graph whose replays follow the contexts on the device.  Each step equals the eager calls and the oracle."""
    ctx0, steps = [61, 127, 1, 1000], 5
    full = [c + steps for c in ctx0]
    s = Setup(n_q, n_kv, hd, full, seed=17)
    off = np.concatenate([[0], np.cumsum(full)])
    pick = torch.cat([torch.arange(off[i], off[i] + c, device=DEV) for i, c in enumerate(ctx0)])
    prompt = s.batch(ctx0, ctx0)
    s.cache.append(prompt, s.k[pick], s.v[pick])
    ps = Setup(n_q, n_kv, hd, ctx0, ctx0, seed=18)
    held = s.held()
    ps.check(s.cache.attend(prompt, ps.q), held=[(k[:c], v[:c]) for (k, v), c in zip(held, ctx0)], seqs=[0, 1, 2])

    ctx = _ints(ctx0)
    k, v = torch.zeros((4, n_kv, hd), dtype=s.dt, device=DEV), torch.zeros((4, n_kv, hd), dtype=s.dt, device=DEV)
    q = torch.zeros((4, n_q, hd), dtype=s.dt, device=DEV)
    b = s.cache.batch(ctx, s.dev_table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # once before the capture
        s.cache.attend(b, q)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.cache.append(b, k, v)
        out = s.cache.attend(b, q)
        kr, vr = s.cache.read(b)
    for step in range(steps):
        rows = torch.tensor([off[i] + c + step for i, c in enumerate(ctx0)], device=DEV)
        k.copy_(s.k[rows])
        v.copy_(s.v[rows])
        q.copy_(torch.randn((4, n_q, hd), device=DEV, generator=torch.Generator(DEV).manual_seed(step)))
        ctx.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        eager = s.cache.attend(b, q)
        assert torch.equal(out, eager)
        now = Setup(n_q, n_kv, hd, [c + step + 1 for c in ctx0], seed=0, spare=0)
        now.check(out, q=q, held=[(a[:c + step + 1], d[:c + step + 1]) for (a, d), c in zip(held, ctx0)])
        for i, c in enumerate(ctx0):
            assert np.array_equal(_f64(kr[i]), held[i][0][c + step]) and np.array_equal(_f64(vr[i]), held[i][1][c + step])


def test_runs_repeat_bit_for_bit():
    s = Setup(28, 4, 128, [5000, 300, 1200], rows=[1, 40, 2], seed=19).fill()
    first = s.cache.attend(s.batch(), s.q)
    for _ in range(5):
        assert torch.equal(s.cache.attend(s.batch(), s.q), first)


def test_python_refusals():
    s = Setup(6, 2, 64, [70, 70], seed=20)
    R = rp()
    with pytest.raises(ValueError):
        s.cache.batch(torch.tensor([1, 2], device=DEV), s.dev_table)                 # int64
    with pytest.raises(ValueError):
        s.cache.batch(torch.tensor([1, 2], dtype=torch.int32), s.dev_table)          # host memory
    with pytest.raises(ValueError):
        s.cache.batch(_ints([1, 2, 3]), s.dev_table)
    with pytest.raises(ValueError):
        s.cache.batch(_ints([1, 2]), s.dev_table, row_offsets=_ints([0, 1, 2]))      # without n_rows
    with pytest.raises(ValueError):
        s.cache.batch(_ints([1, 2]), s.dev_table, max_context=129)
    b = s.cache.batch(_ints([1, 2]), s.dev_table)
    for bad in (s.q[:1], s.q.half(), s.q.cpu(), s.q[..., :32], s.q[0], torch.zeros((2, 6, 128), device=DEV, dtype=s.dt)[..., ::2]):
        with pytest.raises(ValueError):
            s.cache.attend(b, bad)
    with pytest.raises(R.RollpackError):
        s.cache.attend(b, s.q[:, :5])
    with pytest.raises(R.RollpackError):
        s.cache.attend(b, s.q, scale=0.0)
    with pytest.raises(R.RollpackError):
        s.cache.attend(b, s.q, out=s.q)
    for dt in (torch.float16, torch.int32):
        with pytest.raises(ValueError):
            s.cache.read(b, dtype=dt)
    with pytest.raises(ValueError):
        R.KvqCache(4, 2, 64, device="cpu")
