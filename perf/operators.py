"""Measured cases of the 4-bit KV cache: its quantising append, its read-back and the attention over it.

The cache keeps K and V of a token and KV head in blocks of 32 dimensions: one scale, a power of
two, and 32 codes of four bits (sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6).  It is paged in pages
of 64 tokens; a page table gives each sequence's pages.  Every call takes the batch that a step of
the rollout engine has: how many rows (tokens) each sequence brings, its context with those rows,
and the page table.

Kinds of case:
  attend   attention of the rows over their sequences' cached keys, causal: `rows` query rows per
           sequence (0: the whole context, a prompt), the last of its context of lo..hi tokens.
  write    the rows' K and V are quantised into the cache, and what the cache now holds of them
           is read back.
  read     the last `rows` positions of each sequence (0: all of them) are read back.

Heads are those of the repository's models: 4/2 heads of 64 (the small fp32 decoder), 14/2 of 64
(0.5B), 28/4 of 128 (7B), 40/8 of 128 (32B).
"""
from __future__ import annotations

import random
import types

import torch

own = False

_PAGE, _BLOCK = 64, 32
_HEADS = {"tiny": (4, 2, 64), "0.5b": (14, 2, 64), "7b": (28, 4, 128), "32b": (40, 8, 128)}
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # The smallest serving call: a handful of rows of the 0.5B model decode one token; latency counts.
        dict(name="attend-0.5b-4", kind="attend", heads="0.5b", dtype="bf16", seqs=4, lo=65, hi=500, rows=1),
        # The end of a long round: the longest response decodes alone.
        dict(name="attend-7b-1", kind="attend", heads="7b", dtype="bf16", seqs=1, lo=12001, hi=12001, rows=1),
        # The full long round: 64 rows at ragged contexts.
        dict(name="attend-7b-64", kind="attend", heads="7b", dtype="bf16", seqs=64, lo=600, hi=4500, rows=1),
        # A short round at its full width.
        dict(name="attend-7b-330", kind="attend", heads="7b", dtype="bf16", seqs=330, lo=200, hi=1700, rows=1),
        # A 32B round at long contexts: the largest decode step.
        dict(name="attend-32b-96", kind="attend", heads="32b", dtype="bf16", seqs=96, lo=900, hi=8300, rows=1),
        # The fp32 decoder's types, several rows per sequence (given tokens are scored).
        dict(name="attend-tiny-f32", kind="attend", heads="tiny", dtype="f32", seqs=8, lo=40, hi=330, rows=9),
        # Admission of a round's prompts, U[128, 1024].
        dict(name="attend-7b-prompts", kind="attend", heads="7b", dtype="bf16", seqs=20, lo=128, hi=1024, rows=0),
        # A preempted long response resumes: its whole history is prefilled again.
        dict(name="attend-7b-resume", kind="attend", heads="7b", dtype="bf16", seqs=1, lo=14500, hi=14500, rows=0),
        # A decode step's new tokens enter the cache.
        dict(name="write-7b-64", kind="write", heads="7b", dtype="bf16", seqs=64, lo=600, hi=4500, rows=1),
        # A chunk of prompts enters the cache.
        dict(name="write-7b-prompts", kind="write", heads="7b", dtype="bf16", seqs=20, lo=128, hi=1024, rows=0),
        # A few short sequences are taken out of the cache, in fp32.
        dict(name="read-0.5b-f32", kind="read", heads="0.5b", dtype="f32", seqs=5, lo=33, hi=700, rows=0),
        # A round's sequences are taken out of the cache: they move to another replica.
        dict(name="read-7b-64", kind="read", heads="7b", dtype="bf16", seqs=64, lo=600, hi=4500, rows=0),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    heads = rng.choice(["tiny", "0.5b", "7b", "7b", "32b"])
    kind = rng.choice(["decode", "decode", "decode", "extend", "prompt", "prompt", "write", "read"])
    dtype = "f32" if heads == "tiny" or rng.random() < 0.15 else "bf16"
    kv = _HEADS[heads][1] * _HEADS[heads][2]
    seqs = _log(rng, 1, {"decode": 330, "extend": 48, "prompt": 24, "write": 256, "read": 64}[kind])
    # cached elements of a head side in all: the largest decode case's for one token, fewer for prompts
    most = {"decode": 4.5e8, "extend": 1.0e8, "prompt": 7.0e6, "write": 3.0e7, "read": 8.0e7}[kind]
    if dtype == "f32" and kind in ("extend", "prompt"):
        most /= 4
    hi = _log(rng, 1, max(2, int(min(14500, most / (kv * seqs)))))
    lo = max(1, hi // rng.choice([1, 2, 8]))
    rows = {"decode": 1, "extend": rng.randint(2, 40), "prompt": 0, "write": rng.choice([0, 1, 5]), "read": 0}[kind]
    return dict(kind=kind if kind in ("write", "read") else "attend", heads=heads, dtype=dtype, seqs=seqs, lo=lo, hi=hi,
                rows=rows)


def _sizes(case):
    """Contexts, spread evenly over [lo, hi] in an order of the case's own (the same for every seed), and rows."""
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    ctx = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(n * 1000003 + hi).shuffle(ctx)
    return ctx, [c if case["rows"] == 0 else min(case["rows"], c) for c in ctx]


def _inputs(case, seed):
    """Keys with a few strong channels per head, as rotated keys with a bias have; plain values; queries."""
    n_q, n_kv, hd = _HEADS[case["heads"]]
    dt = _TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 9176 + 11)
    ctx, rows = _sizes(case)
    tokens = sum(ctx)

    def normal(*dims):
        return torch.randn(dims, generator=gen, device="cuda", dtype=torch.float32)

    gain = 1.0 + 5.0 * (torch.rand((n_kv, hd), generator=gen, device="cuda") < 0.04)
    s = types.SimpleNamespace(case=case, ctx=ctx, rows=rows, dt=dt, n_q=n_q, n_kv=n_kv, hd=hd)
    s.k = (normal(tokens, n_kv, hd) * gain).to(dt)
    s.v = normal(tokens, n_kv, hd).to(dt)
    s.q = normal(sum(rows), n_q, hd).to(dt) if case["kind"] == "attend" else None
    # the pages of a pool that sequences of other lengths have come and gone from: any order, some of others between
    need = [-(-c // _PAGE) for c in ctx]
    s.n_pages = sum(need) + 3
    perm = torch.randperm(s.n_pages, generator=gen, device="cuda").to(torch.int32)
    s.table = torch.zeros((len(ctx), max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        s.table[b, :n] = perm[at:at + n]
        at += n
    return s


def _last_rows(s, x):
    """The rows of the call out of all tokens: each sequence's last ones."""
    keep = []
    at = 0
    for c, r in zip(s.ctx, s.rows):
        keep.append(torch.arange(at + c - r, at + c, device="cuda"))
        at += c
    return x[torch.cat(keep)]


def _batch(cache, s, rows):
    """The batch descriptor of a step: one row per sequence, or `rows` of each."""
    ctx = torch.tensor(s.ctx, dtype=torch.int32, device="cuda")
    if all(r == 1 for r in rows):
        return cache.batch(ctx, s.table, max_context=max(s.ctx))
    off = torch.tensor([0] + rows, device="cuda").cumsum(0).to(torch.int32)
    return cache.batch(ctx, s.table, row_offsets=off, n_rows=sum(rows), max_rows=max(rows), max_context=max(s.ctx))


def prepare(case, seed):
    """The cache with the sequences' tokens in it (a `write` case: without the call's rows), and the call's tensors."""
    s = _inputs(case, seed)
    k, v = s.k, s.v
    s.k, s.v = (_last_rows(s, k), _last_rows(s, v)) if case["kind"] == "write" else (None, None)
    if own:
        from paper_2509_21009_amd import rollpack
        s.cache = rollpack.KvqCache(s.n_pages, s.n_kv, s.hd, device="cuda")
        if case["kind"] != "write":
            s.cache.append(_batch(s.cache, s, s.ctx), k, v)
        s.batch = _batch(s.cache, s, s.rows)
        if case["kind"] == "attend":
            s.workspace = s.cache.attend_workspace(s.batch, s.n_q)
        return s
    s.codes = torch.zeros((2, s.n_pages, _PAGE, s.n_kv, s.hd // 2), dtype=torch.uint8, device="cuda")
    s.scales = torch.zeros((2, s.n_pages, _PAGE, s.n_kv, s.hd // _BLOCK), dtype=torch.uint8, device="cuda")
    s.slots = []  # of every token: page * 64 + place
    for b, c in enumerate(s.ctx):
        t = torch.arange(c, device="cuda")
        s.slots.append(s.table[b].long()[t // _PAGE] * _PAGE + t % _PAGE)
    if case["kind"] != "write":
        _plain_write(s, torch.cat(s.slots), k, v)
    return s


# ---- the plain forms -----------------------------------------------------------------

def _plain_write(s, slots, k, v):
    for i, x in enumerate((k, v)):
        b = x.float().unflatten(-1, (-1, _BLOCK))
        amax = b.abs().amax(-1, keepdim=True)
        mant, expo = torch.frexp(amax)  # amax = mant * 2^expo, 0.5 <= mant < 1
        e = (expo - 3 + (mant > 0.875).int()).clamp(-125, 125)
        a = torch.ldexp(b.abs(), -e)
        code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int()
                + (a >= 3.5).int() + (a > 5.0).int() + 8 * (b < 0).int())
        code = code.flatten(-2).to(torch.uint8)
        flat = s.codes[i].view(-1, s.n_kv, s.hd // 2)
        flat[slots] = code[..., 0::2] | (code[..., 1::2] << 4)
        s.scales[i].view(-1, s.n_kv, s.hd // _BLOCK)[slots] = (e.squeeze(-1) + 127).to(torch.uint8)


def _plain_read(s, i, slots):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    grid = torch.cat([grid, -grid])
    byte = s.codes[i].view(-1, s.n_kv, s.hd // 2)[slots].int()
    x = torch.stack([grid[byte & 15], grid[byte >> 4]], -1).flatten(-2)
    e = s.scales[i].view(-1, s.n_kv, s.hd // _BLOCK)[slots].int() - 127
    return torch.ldexp(x.unflatten(-1, (-1, _BLOCK)), e.unsqueeze(-1)).flatten(-2)


def _plain_attend(s):
    out = torch.empty_like(s.q)
    g = s.n_q // s.n_kv
    at = 0
    for c, n, slots in zip(s.ctx, s.rows, s.slots):
        k = _plain_read(s, 0, slots).permute(1, 2, 0).contiguous()  # [n_kv, hd, c]
        v = _plain_read(s, 1, slots).permute(1, 0, 2).contiguous()
        step = max(1, (1 << 28) // (c * s.n_q))
        for o in range(0, n, step):
            m = min(n, o + step)
            q = s.q[at + o:at + m].float().view(m - o, s.n_kv, g, s.hd).permute(1, 2, 0, 3).reshape(s.n_kv, -1, s.hd)
            end = c - n + m  # no row of the piece sees a key past it
            sc = torch.bmm(q, k[:, :, :end].contiguous()) * s.hd ** -0.5
            if m - o > 1:
                t = torch.arange(end, device="cuda")
                pos = torch.arange(c - n + o, c - n + m, device="cuda")
                sc = sc.view(s.n_kv, g, m - o, end).masked_fill(t > pos[:, None], -float("inf")).view(sc.shape)
            sc = torch.exp(sc - sc.amax(-1, keepdim=True))
            y = torch.bmm(sc, v[:, :end].contiguous()) / sc.sum(-1, keepdim=True)
            out[at + o:at + m] = y.view(s.n_kv, g, m - o, s.hd).permute(2, 0, 1, 3).reshape(m - o, s.n_q, s.hd).to(s.dt)
        at += n
    return out


def run(s):
    kind = s.case["kind"]
    if own:
        if kind == "attend":
            return s.cache.attend(s.batch, s.q, workspace=s.workspace)
        if kind == "write":
            s.cache.append(s.batch, s.k, s.v)
        return s.cache.read(s.batch, dtype=s.dt)
    if kind == "attend":
        return _plain_attend(s)
    slots = torch.cat([x[len(x) - n:] for x, n in zip(s.slots, s.rows)])
    if kind == "write":
        _plain_write(s, slots, s.k, s.v)
    return _plain_read(s, 0, slots).to(s.dt), _plain_read(s, 1, slots).to(s.dt)


def work(case):
    n_q, n_kv, hd = _HEADS[case["heads"]]
    ctx, rows = _sizes(case)
    esz = 4 if case["dtype"] == "f32" else 2
    held = 2 * n_kv * (hd // 2 + hd // _BLOCK)  # bytes of a token in the cache
    dense = 2 * n_kv * hd * esz                 # and of its K and V rows
    if case["kind"] == "attend":
        seen = sum(r * (c - r) + r * (r + 1) // 2 for c, r in zip(ctx, rows))
        return {"bytes": sum(ctx) * held + 2 * sum(rows) * n_q * hd * esz, "flops": 4 * n_q * hd * seen}
    if case["kind"] == "write":  # rows in, the cache written, rows out; a maximum, a scaling and a rounding each
        return {"bytes": sum(rows) * (2 * dense + held), "flops": sum(rows) * 2 * n_kv * hd * 4}
    return {"bytes": sum(rows) * (dense + held), "flops": sum(rows) * 2 * n_kv * hd}


# ---- the same in 64 bits -------------------------------------------------------------

def _held(x):
    """What the cache holds of x: the nearest of its values, in 64 bits."""
    b = x.double().reshape(*x.shape[:-1], -1, _BLOCK)
    top = b.abs().max(-1, keepdim=True).values
    s = 2.0 ** torch.ceil(torch.log2(torch.clamp(top / 7.0, min=2.0 ** -125)))
    a = b.abs() / s
    r = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2)))
    return (torch.sign(b) * torch.clamp(r, max=6.0) * s).reshape(x.shape)


def exact(case, seed):
    s = _inputs(case, seed)
    k, v = _held(s.k), _held(s.v)
    if case["kind"] != "attend":
        return _last_rows(s, k), _last_rows(s, v)
    out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    grp = s.n_q // s.n_kv
    qa = ka = 0
    for c, n in zip(s.ctx, s.rows):
        for h in range(s.n_q):
            kk, vv = k[ka:ka + c, h // grp].t().contiguous(), v[ka:ka + c, h // grp].contiguous()
            for o in range(0, n, 4096):
                m = min(n, o + 4096)
                z = s.q[qa + o:qa + m, h].double() @ kk / float(s.hd) ** 0.5
                late = torch.ones((m - o, c), dtype=torch.bool, device="cuda").triu(c - n + o + 1)
                out[qa + o:qa + m, h] = torch.softmax(z.masked_fill(late, -float("inf")), -1) @ vv
        qa += n
        ka += c
    return out
