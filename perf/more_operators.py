"""Measured cases of the 4-bit KV cache's page operators: its pages handed out on the GPU, and attention over
the pages that a cheap score picks for each query.

The cache keeps K and V of a token and KV head in blocks of 32 dimensions (a scale, a power of two, and codes of four
bits), in pages of 64 tokens that a page table names.  A step of a rollout with long responses is: the pages and slots of
the new tokens (`fit`), the smallest and largest key of every dimension in the pages that they went to (`ranges`), a
bound of each page's scores by these (`scores`), the pages to attend to (`pick`), and attention over those (`picked`).

Kinds of case:
  fit      lengths in, pages out: sequences that got longer take pages from the free list, in order, shorter ones give
           theirs back; row offsets, positions and slots of the new tokens.  One pass is a step and its taking back.
  ranges   after the rows (`rows` of each sequence, 0: all of its tokens) were appended: their pages' ranges.
  scores   for each row, KV head and page that the row sees: the largest, over the query heads of the KV head, of
           sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d.
  pick     from such scores: the first page, the last two, and the best of the others, `n` in all; ascending, then -1.
  picked   causal attention of each row over the tokens of its picked pages.

Heads are those of the repository's models: 4/2 heads of 64 (the small fp32 decoder), 14/2 of 64 (0.5B), 28/4 of 128
(7B), 40/8 of 128 (32B).
"""
from __future__ import annotations

import random
import types

import torch

own = False

_PAGE, _BLOCK = 64, 32
_FIRST, _LAST = 1, 2  # pages that are always picked
_HEADS = {"tiny": (4, 2, 64), "0.5b": (14, 2, 64), "7b": (28, 4, 128), "32b": (40, 8, 128)}
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # A decode step of the long round: every sequence gets a token; latency counts.
        dict(name="fit-64", kind="fit", seqs=64, lo=600, hi=4500, step="decode"),
        # A full short round turns over: a third of the sequences finish, a third are admitted, the others decode.
        dict(name="fit-512-turn", kind="fit", seqs=512, lo=200, hi=1700, step="turn"),
        # All prompts of a large RL step are admitted at once.
        dict(name="fit-1024-prompts", kind="fit", seqs=1024, lo=128, hi=1024, step="admit"),
        # A decode step's new tokens change their pages' ranges.
        dict(name="ranges-7b-64", kind="ranges", heads="7b", dtype="bf16", seqs=64, lo=600, hi=4500, rows=1),
        # Long prompts have entered the cache.
        dict(name="ranges-32b-prompts", kind="ranges", heads="32b", dtype="bf16", seqs=20, lo=256, hi=8192, rows=0),
        # The fp32 decoder's types, several rows per sequence.
        dict(name="scores-tiny-f32", kind="scores", heads="tiny", dtype="f32", seqs=8, lo=40, hi=330, rows=9),
        # A 32B round whose responses are up to 32k tokens long: one token each.
        dict(name="scores-32b-64", kind="scores", heads="32b", dtype="bf16", seqs=64, lo=6000, hi=33000, rows=1),
        # Decoding at a context of several thousand tokens: short lists; latency counts.
        dict(name="pick-7b-64", kind="pick", heads="7b", seqs=64, lo=600, hi=4500, rows=1, n=16),
        # A piece of a long prompt: every row has its lists.
        dict(name="pick-7b-512rows", kind="pick", heads="7b", seqs=1, lo=14000, hi=14000, rows=512, n=32),
        # The smallest attention call.
        dict(name="picked-tiny-f32", kind="picked", heads="tiny", dtype="f32", seqs=8, lo=40, hi=330, rows=9, n=4),
        # The 32B round with responses up to 32k tokens: 48 of up to 516 pages each.
        dict(name="picked-32b-64", kind="picked", heads="32b", dtype="bf16", seqs=64, lo=6000, hi=33000, rows=1, n=48),
        # The last piece of a long prompt, 2,048 of its 14,000 keys for each row.
        dict(name="picked-7b-512rows", kind="picked", heads="7b", dtype="bf16", seqs=1, lo=14000, hi=14000, rows=512, n=32),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["fit", "ranges", "scores", "pick", "picked", "picked", "picked"])
    if kind == "fit":
        seqs = _log(rng, 1, 4096)
        hi = _log(rng, 1, max(2, min(33000, 580000 // seqs)))
        return dict(kind="fit", seqs=seqs, lo=max(1, hi // rng.choice([1, 2, 8])), hi=hi,
                    step=rng.choice(["decode", "turn", "admit", "rewind"]))
    heads = rng.choice(["tiny", "0.5b", "7b", "32b"])
    n_q, n_kv, hd = _HEADS[heads]
    # one token of each sequence, a few, or many (a prompt's piece)
    shape = rng.choice(["one", "one", "few", "many"])
    seqs = _log(rng, 1, {"one": 192, "few": 40, "many": 8}[shape])
    rows = {"one": 1, "few": rng.randint(2, 24), "many": _log(rng, 32, 2000)}[shape]
    # elements of a side of the cache in all, and of the lists' pages
    hi = _log(rng, 1, max(2, min(33000, 1.2e9 // (n_kv * hd * seqs))))
    if kind == "pick":  # lists that leave a choice
        hi = max(hi, 2048)
    if kind == "ranges":
        hi = min(hi, max(2, int(8e7 // (n_kv * hd * seqs))))
        rows = rng.choice([0, rows])
    if kind in ("scores", "pick"):
        rows = min(rows, max(1, int((4e7 / n_q if kind == "scores" else 4e6 / n_kv) // (seqs * -(-hi // _PAGE)))))
    rows = min(rows, hi)
    case = dict(kind=kind, heads=heads, seqs=seqs, lo=max(1, hi // rng.choice([1, 2, 8])), hi=hi, rows=rows)
    if kind != "pick":
        case["dtype"] = "f32" if heads == "tiny" or rng.random() < 0.2 else "bf16"
    if kind in ("pick", "picked"):
        most = -(-hi // _PAGE)
        least = _FIRST + _LAST + (kind == "pick")
        case["n"] = rng.randint(least, max(least, min(96, most + (2 if kind == "picked" else -2))))
        if kind == "picked":
            case["rows"] = max(1, min(rows, int(4e8 // (seqs * n_kv * hd * _PAGE * case["n"]))))
    return case


def _sizes(case):
    """Contexts, spread evenly over [lo, hi] in an order of the case's own (the same for every seed), and rows."""
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    ctx = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    random.Random(n * 1000003 + hi).shuffle(ctx)
    rows = case.get("rows", 1)
    return ctx, [c if rows == 0 else min(rows, c) for c in ctx]


def _lengths(case):
    """Of a fit case: the sequences' lengths before and after the step."""
    ctx, _ = _sizes(case)
    step = case["step"]
    if step == "decode":
        return ctx, [c + 1 for c in ctx]
    if step == "admit":
        return [0] * len(ctx), ctx
    if step == "rewind":  # tokens that were only guessed are taken back
        return ctx, [max(0, c - 1 - b % 9) for b, c in enumerate(ctx)]
    return ([c if b % 3 != 1 else 0 for b, c in enumerate(ctx)],
            [0 if b % 3 == 0 else c if b % 3 == 1 else c + 1 for b, c in enumerate(ctx)])


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 5)
    return gen


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    """The sequences' places in a shuffled pool, and the kind's tensors: keys with a few strong channels per head, as
    rotated keys with a bias have; values, queries; ranges as wide as 64 such keys'; scores with a few that tie."""
    n_q, n_kv, hd = _HEADS[case["heads"]]
    kind, gen = case["kind"], _generator(seed)
    ctx, rows = _sizes(case)

    def normal(*dims):
        return torch.randn(dims, generator=gen, device="cuda", dtype=torch.float32)

    s = types.SimpleNamespace(case=case, ctx=ctx, rows=rows, n_q=n_q, n_kv=n_kv, hd=hd, dt=_TYPES[case.get("dtype", "bf16")])
    need = [-(-c // _PAGE) for c in ctx]
    s.n_pages, s.width = sum(need) + 3, max(need)
    perm = torch.randperm(s.n_pages, generator=gen, device="cuda").to(torch.int32)
    s.table = torch.zeros((len(ctx), s.width), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        s.table[b, :n] = perm[at:at + n]
        at += n
    gain = 1.0 + 5.0 * (torch.rand((n_kv, hd), generator=gen, device="cuda") < 0.04)
    if kind in ("ranges", "picked"):
        s.k = normal(sum(ctx), n_kv, hd).mul_(gain).to(s.dt)
        s.v = normal(sum(ctx), n_kv, hd).to(s.dt)
    if kind == "scores":
        mid, wide = normal(s.n_pages, n_kv, hd).mul_(0.3), normal(s.n_pages, n_kv, hd).mul_(0.4).add_(2.4).abs_()
        s.ranges = torch.stack([(mid - wide) * gain, (mid + wide) * gain], 2).to(torch.bfloat16)
    if kind in ("scores", "picked"):
        s.q = normal(sum(rows), n_q, hd).to(s.dt)
    if kind in ("pick", "picked"):
        s.scores = normal(sum(rows), n_kv, s.width).mul_(30.0).to(torch.bfloat16).float()
    return s


def prepare(case, seed):
    """The pool as the sequences' lengths before the step left it; or the cache with the sequences' tokens, and the call's tensors."""
    if case["kind"] == "fit":
        return _prepare_fit(case, seed)
    s = _inputs(case, seed)
    kind = case["kind"]
    k, v = (s.k, s.v) if kind in ("ranges", "picked") else (None, None)
    s.k = s.v = None
    s.ctx_t, s.rows_t = _ints(s.ctx), _ints(s.rows)
    s.off = torch.cat([_ints([0]), s.rows_t.cumsum(0).to(torch.int32)])
    if kind == "ranges":
        s.ranges = torch.zeros((s.n_pages, s.n_kv, 2, s.hd), dtype=torch.bfloat16, device="cuda")
    if kind == "picked":
        s.picks = _plain_pick(s)
        s.scores = None
    if own:
        from paper_2509_21009_amd import rollpack
        s.cache = rollpack.KvqCache(s.n_pages, s.n_kv, s.hd, device="cuda")
        if k is not None:
            all_rows = torch.cat([_ints([0]), s.ctx_t.cumsum(0).to(torch.int32)])
            s.cache.append(s.cache.batch(s.ctx_t, s.table, row_offsets=all_rows, n_rows=sum(s.ctx), max_rows=max(s.ctx)), k, v)
        if max(s.rows) == min(s.rows) == 1:
            s.batch = s.cache.batch(s.ctx_t, s.table, max_context=max(s.ctx))
        else:
            s.batch = s.cache.batch(s.ctx_t, s.table, row_offsets=s.off, n_rows=sum(s.rows), max_rows=max(s.rows),
                                    max_context=max(s.ctx))
        if kind == "picked":
            s.workspace = s.cache.attend_picked_workspace(s.batch, s.n_q, case["n"])
    elif k is not None:
        s.codes = torch.zeros((2, s.n_pages, s.n_kv, _PAGE, s.hd // 2), dtype=torch.uint8, device="cuda")
        s.scales = torch.zeros((2, s.n_pages, s.n_kv, _PAGE, s.hd // _BLOCK), dtype=torch.uint8, device="cuda")
        at = 0
        for b, c in enumerate(s.ctx):
            _plain_write(s, b, k[at:at + c], v[at:at + c])
            at += c
    return s


def _prepare_fit(case, seed):
    before, after = _lengths(case)
    s = types.SimpleNamespace(case=case, n=len(before))
    s.most = max(max(before), max(after), 1)
    s.width = -(-s.most // _PAGE)
    s.n_pages = sum(max(-(-a // _PAGE), -(-b // _PAGE)) for a, b in zip(before, after)) + 5
    order = torch.randperm(s.n_pages, generator=_generator(seed), device="cuda").to(torch.int32)
    s.before, s.after = _ints(before), _ints(after)
    s.n_rows = sum(max(0, b - a) for a, b in zip(before, after))
    s.n_back = sum(max(0, a - b) for a, b in zip(before, after))
    if own:
        from paper_2509_21009_amd import rollpack
        s.pages = rollpack.KvqPages(s.n_pages, s.n, s.width * _PAGE, device="cuda")
        s.pages.free_pages.copy_(order)
        s.pages.fit(s.before, sum(before))
        return s
    s.free, s.n_free = order, torch.tensor(s.n_pages, device="cuda")
    s.table = torch.zeros((s.n, s.width), dtype=torch.int32, device="cuda")
    s.contexts = torch.zeros(s.n, dtype=torch.int32, device="cuda")
    _plain_fit(s, s.before, sum(before))
    return s


# ---- the plain forms -----------------------------------------------------------------

def _plain_fit(s, lengths, n_rows):
    """Row offsets, positions and slots of the new tokens; pages are taken from and given back to the end of the free list."""
    old, new = s.contexts.long(), lengths.long()
    page = torch.arange(s.width, device="cuda")
    have, want = -(-old // _PAGE), -(-new // _PAGE)
    gone = (page >= want[:, None]) & (page < have[:, None])    # in the order of sequences, then pages
    fresh = (page >= have[:, None]) & (page < want[:, None])
    back, need = gone.flatten().cumsum(0) - 1, fresh.flatten().cumsum(0) - 1
    n_back, n_need = back[-1] + 1, need[-1] + 1
    end = s.n_pages  # entries of no page are written behind the list
    free = torch.cat([s.free, s.free[:1]])
    free[torch.where(gone.flatten(), s.n_free + n_back - 1 - back, end)] = s.table.flatten()
    s.free = free[:end].contiguous()
    s.n_free = s.n_free + n_back
    taken = s.free[torch.where(fresh.flatten(), s.n_free - 1 - need, 0)].view(s.n, s.width)
    s.table = torch.where(fresh, taken, s.table)
    s.n_free = s.n_free - n_need
    rows = (new - old).clamp(min=0)
    off = torch.cat([rows.new_zeros(1), rows.cumsum(0)])
    seq = torch.repeat_interleave(torch.arange(s.n, device="cuda"), rows, output_size=n_rows)
    pos = old[seq] + torch.arange(n_rows, device="cuda") - off[seq]
    slots = s.table[seq, pos // _PAGE] * _PAGE + pos % _PAGE
    s.contexts = lengths.clone()
    return off.to(torch.int32), pos.to(torch.int32), slots.to(torch.int32)


def _plain_write(s, b, k, v):
    t = torch.arange(len(k), device="cuda")
    page = s.table[b].long()[t // _PAGE]
    x = torch.stack([k, v]).float().unflatten(-1, (-1, _BLOCK))
    amax = x.abs().amax(-1, keepdim=True)
    mant, expo = torch.frexp(amax)  # amax = mant * 2^expo, 0.5 <= mant < 1
    e = (expo - 3 + (mant > 0.875).int()).clamp(-125, 125)
    a = torch.ldexp(x.abs(), -e)
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int()
            + (a >= 3.5).int() + (a > 5.0).int() + 8 * (x < 0).int())
    code = code.flatten(-2).to(torch.uint8)
    s.codes[:, page, :, t % _PAGE] = (code[..., 0::2] | (code[..., 1::2] << 4)).transpose(0, 1).contiguous()
    s.scales[:, page, :, t % _PAGE] = (e.squeeze(-1) + 127).to(torch.uint8).transpose(0, 1).contiguous()


def _values(byte, scale):
    """What codes and scales of whole head dimensions stand for."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    grid = torch.cat([grid, -grid])
    x = torch.stack([grid[(byte & 15).int()], grid[(byte >> 4).int()]], -1).flatten(-2)
    return torch.ldexp(x.unflatten(-1, (-1, _BLOCK)), (scale.int() - 127).unsqueeze(-1)).flatten(-2)


def _plain_ranges(s):
    first, last = (s.ctx_t - s.rows_t).long() // _PAGE, (s.ctx_t.long() - 1) // _PAGE
    most = max((c - 1) // _PAGE - (c - n) // _PAGE + 1 for c, n in zip(s.ctx, s.rows))
    p = first[:, None] + torch.arange(most, device="cuda")                     # [seqs, pages of the call's rows]
    there = p <= last[:, None]
    b, i = there.nonzero(as_tuple=True)
    p = p[b, i]
    page = s.table[b, p].long()
    k = _values(s.codes[0, page], s.scales[0, page])                           # [pages, n_kv, 64, hd]
    out = p[:, None] * _PAGE + torch.arange(_PAGE, device="cuda") >= s.ctx_t[b][:, None]
    out = out[:, None, :, None]
    lo, hi = k.masked_fill(out, float("inf")).amin(2), k.masked_fill(out, -float("inf")).amax(2)
    s.ranges[page] = torch.stack([lo, hi], 2).to(torch.bfloat16)
    return s.ranges


def _row_places(s):
    """Of each row: its sequence, and its position."""
    seq = torch.repeat_interleave(torch.arange(len(s.ctx), device="cuda"), s.rows_t, output_size=sum(s.rows))
    return seq, (s.ctx_t - s.rows_t)[seq] + torch.arange(sum(s.rows), device="cuda") - s.off[seq]


def _plain_scores(s):
    seq, pos = _row_places(s)
    i = torch.arange(sum(s.rows), device="cuda") - s.off[seq]                  # of its sequence's rows
    n, g = len(s.ctx), s.n_q // s.n_kv
    q = s.q.new_zeros((n, max(s.rows), s.n_q, s.hd), dtype=torch.float32)
    q[seq, i] = s.q.float()
    q = q.view(n, -1, s.n_kv, g, s.hd).permute(0, 2, 1, 3, 4).reshape(n * s.n_kv, -1, s.hd)
    r = s.ranges[s.table.long()].float().permute(3, 0, 2, 4, 1).reshape(2, n * s.n_kv, s.hd, s.width)
    x = torch.bmm(q.clamp(min=0), r[1].contiguous()) + torch.bmm(q.clamp(max=0), r[0].contiguous())
    x = x.view(n, s.n_kv, -1, g, s.width).amax(3)[seq, :, i]                   # [rows, n_kv, pages]
    return x.masked_fill((torch.arange(s.width, device="cuda") * _PAGE > pos[:, None])[:, None], -float("inf"))


def _plain_pick(s):
    _, pos = _row_places(s)
    n = s.case["n"]
    seen = (pos // _PAGE + 1)[:, None, None]                                   # pages
    page = torch.arange(s.width, device="cuda")
    bits = (s.scores + 0.0).view(torch.int32).long()                           # in the order of the values, -0 being 0
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF) - 1)
    key = torch.where(torch.isnan(s.scores), 1 << 31, key)                     # above every number
    key = torch.where((page < _FIRST) | (page >= seen - _LAST), 1 << 32, key)
    key = torch.where(page < seen, key, -(1 << 40))
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :n]  # ties: the lower page
    best = torch.where(best < seen, best, 1 << 30).sort(-1).values
    best = torch.where(best < 1 << 30, best, -1).to(torch.int32)
    return torch.cat([best, best.new_full((*best.shape[:2], n - best.shape[2]), -1)], -1)


def _plain_picked(s):
    seq, pos = _row_places(s)
    g = s.n_q // s.n_kv
    p = s.picks.clamp(min=0).long()                                            # [rows, n_kv, n]
    page = s.table[seq[:, None, None], p].long()
    head = torch.arange(s.n_kv, device="cuda")[:, None]
    t = (p[..., None] * _PAGE + torch.arange(_PAGE, device="cuda"))
    out = ((s.picks < 0)[..., None] | (t > pos[:, None, None, None])).flatten(-2).flatten(0, 1)  # [rows n_kv, n 64]
    k = _values(s.codes[0][page, head], s.scales[0][page, head]).view(len(out), -1, s.hd)
    sc = torch.bmm(s.q.float().view(len(out), g, s.hd), k.transpose(1, 2).contiguous()) * s.hd ** -0.5
    del k
    sc = sc.masked_fill(out[:, None], -float("inf"))
    sc = torch.exp(sc - sc.amax(-1, keepdim=True))
    v = _values(s.codes[1][page, head], s.scales[1][page, head]).view(len(out), -1, s.hd)
    return (torch.bmm(sc, v) / sc.sum(-1, keepdim=True)).view(-1, s.n_q, s.hd).to(s.dt)


def run(s):
    kind = s.case["kind"]
    if kind == "fit":
        if own:
            batch, positions, slots = s.pages.fit(s.after, s.n_rows)
            back, back_positions, back_slots = s.pages.fit(s.before, s.n_back)
            return (batch.row_offsets, positions, slots, back.row_offsets, back_positions, back_slots,
                    s.pages.contexts, s.pages.page_table, s.pages.free_pages)
        return (*_plain_fit(s, s.after, s.n_rows), *_plain_fit(s, s.before, s.n_back), s.contexts, s.table, s.free)
    if kind == "ranges":
        return s.cache.update_ranges(s.batch, s.ranges) if own else _plain_ranges(s)
    if kind == "scores":
        return s.cache.page_scores(s.batch, s.q, s.ranges) if own else _plain_scores(s)
    if kind == "pick":
        return s.cache.pick_pages(s.batch, s.scores, s.case["n"], first=_FIRST, last=_LAST) if own else _plain_pick(s)
    return s.cache.attend_picked(s.batch, s.q, s.picks, workspace=s.workspace) if own else _plain_picked(s)


def work(case):
    if case["kind"] == "fit":  # two calls
        before, after = _lengths(case)
        moved = sum(abs(-(-a // _PAGE) + -b // _PAGE) for a, b in zip(before, after))
        rows = sum(abs(a - b) for a, b in zip(before, after))
        # lengths in, contexts in and out, offsets out; a page id in and out, twice; a position and a slot out
        return {"bytes": 2 * len(before) * 16 + 2 * moved * 8 + rows * 8, "flops": 2 * len(before) * 8 + rows * 4}
    n_q, n_kv, hd = _HEADS[case["heads"]]
    ctx, rows = _sizes(case)
    esz = 4 if case.get("dtype") == "f32" else 2
    side = n_kv * (hd // 2 + hd // _BLOCK)  # bytes of a token's K, or V, in the cache
    held = n_kv * 2 * hd * 2                # of a page's ranges
    pages = [-(-c // _PAGE) for c in ctx]
    seen = [[(c - n + i) // _PAGE + 1 for i in range(n)] for c, n in zip(ctx, rows)]  # pages of each row
    if case["kind"] == "ranges":
        first = [(c - n) // _PAGE for c, n in zip(ctx, rows)]
        tokens = sum(c - f * _PAGE for c, f in zip(ctx, first))
        return {"bytes": tokens * side + sum(p - f for p, f in zip(pages, first)) * held, "flops": tokens * n_kv * hd * 2}
    lists = sum(sum(x) for x in seen) * n_kv
    if case["kind"] == "scores":
        return {"bytes": sum(pages) * held + sum(rows) * (n_q * hd * esz + n_kv * max(pages) * 4), "flops": lists * n_q // n_kv * hd * 4}
    if case["kind"] == "pick":
        return {"bytes": lists * 4 + sum(rows) * n_kv * case["n"] * 4, "flops": lists}
    n = case["n"]
    taken = sum(min(n, p) for x in seen for p in x)
    # a sequence's rows share what they pick: at most all its pages, at least one row's
    read = sum(min(p * 1.0, sum(min(n, y) for y in x)) for p, x in zip(pages, seen))
    return {"bytes": read * _PAGE * 2 * side + sum(rows) * (2 * n_q * hd * esz + n_kv * n * 4),
            "flops": taken * _PAGE * n_q * hd * 4}


# ---- the same in 64 bits -------------------------------------------------------------

def _held(x):
    """What the cache holds of x: the nearest of its values, in 64 bits."""
    b = x.double().reshape(*x.shape[:-1], -1, _BLOCK)
    top = b.abs().max(-1, keepdim=True).values
    s = 2.0 ** torch.ceil(torch.log2(torch.clamp(top / 7.0, min=2.0 ** -125)))
    a = b.abs() / s
    r = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2)))
    return (torch.sign(b) * torch.clamp(r, max=6.0) * s).reshape(x.shape)


def _exact_fit(case, seed):
    before, after = _lengths(case)
    pages = lambda n: (n + _PAGE - 1) // _PAGE  # noqa: E731
    width = max(pages(max(before + after)), 1)
    n_pages = sum(max(pages(a), pages(b)) for a, b in zip(before, after)) + 5
    free = torch.randperm(n_pages, generator=_generator(seed), device="cuda").tolist()
    top = n_pages
    table = [[0] * width for _ in before]
    now = [0] * len(before)
    out = []
    for step in (before, after, before):
        back = [table[b][p] for b in range(len(now)) for p in range(pages(step[b]), pages(now[b]))]
        top += len(back)
        for j, page in enumerate(back):
            free[top - 1 - j] = page
        off, positions, slots = [0], [], []
        for b, n in enumerate(step):
            for p in range(pages(now[b]), pages(n)):
                top -= 1
                table[b][p] = free[top]
            off.append(off[-1] + max(0, n - now[b]))
            positions.extend(range(now[b], n))
            slots.extend(table[b][t // _PAGE] * _PAGE + t % _PAGE for t in range(now[b], n))
        now = list(step)
        out.append((_ints(off), _ints(positions), _ints(slots)))
    return (*out[1], *out[2], _ints(now), _ints(table), _ints(free))


def exact(case, seed):
    if case["kind"] == "fit":
        return _exact_fit(case, seed)
    s = _inputs(case, seed)
    g = s.n_q // s.n_kv
    page_ends = [sum(-(-c // _PAGE) for c in s.ctx[:b]) for b in range(len(s.ctx) + 1)]
    if case["kind"] == "ranges":
        out = torch.zeros((s.n_pages, s.n_kv, 2, s.hd), dtype=torch.float64, device="cuda")
        at = 0
        for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
            f = (c - n) // _PAGE
            k = _held(s.k[at + f * _PAGE:at + c])
            fill = -len(k) % _PAGE  # the last key again
            k = torch.cat([k, k[-1:].expand(fill, -1, -1)]).unflatten(0, (-1, _PAGE))
            out[s.table[b, f:page_ends[b + 1] - page_ends[b]].long()] = torch.stack([k.min(1).values, k.max(1).values], 2)
            at += c
        return out
    if case["kind"] == "scores":
        out = torch.full((sum(s.rows), s.n_kv, s.width), -float("inf"), dtype=torch.float64, device="cuda")
        at = 0
        for b, (c, n) in enumerate(zip(s.ctx, s.rows)):
            r = s.ranges[s.table[b, :-(-c // _PAGE)].long()].double()          # [pages, n_kv, 2, hd]
            for h in range(s.n_kv):
                q = s.q[at:at + n, h * g:(h + 1) * g].double()
                x = torch.stack([q[:, i].clamp(min=0) @ r[:, h, 1].t().contiguous() + q[:, i].clamp(max=0) @ r[:, h, 0].t().contiguous()
                                 for i in range(g)]).max(0).values
                late = torch.arange(len(r), device="cuda") * _PAGE > torch.arange(c - n, c, device="cuda")[:, None]
                out[at:at + n, h, :len(r)] = x.masked_fill(late, -float("inf"))
            at += n
        return out
    seen = [(c - n + i) // _PAGE + 1 for c, n in zip(s.ctx, s.rows) for i in range(n)]
    if len(seen) * s.n_kv > (20000 if case["kind"] == "pick" else 5000):
        return None
    picks = torch.full((len(seen), s.n_kv, case["n"]), -1, dtype=torch.int32)
    lists = s.scores.double().cpu().numpy()
    for r, m in enumerate(seen):
        for h in range(s.n_kv):
            x = lists[r, h, :m].tolist()
            always = [p for p in range(m) if p < _FIRST or p >= m - _LAST]
            rest = sorted((p for p in range(m) if _FIRST <= p < m - _LAST), key=lambda p: (-x[p], p))
            got = sorted(always + rest[:max(0, case["n"] - len(always))])
            picks[r, h, :len(got)] = torch.tensor(got, dtype=torch.int32)
    if case["kind"] == "pick":
        return picks.to("cuda")
    out = torch.empty(s.q.shape, dtype=torch.float64, device="cuda")
    starts = [sum(s.ctx[:b]) for b in range(len(s.ctx))]
    owner = [b for b, n in enumerate(s.rows) for _ in range(n)]
    place = [c - n + i for c, n in zip(s.ctx, s.rows) for i in range(n)]
    picks = picks.tolist()
    for r, (b, pos) in enumerate(zip(owner, place)):
        for h in range(s.n_kv):
            t = torch.tensor([starts[b] + u for p in picks[r][h] if p >= 0 for u in range(p * _PAGE, min((p + 1) * _PAGE, pos + 1))],
                             device="cuda")
            k, v = _held(s.k[t, h]), _held(s.v[t, h])
            w = torch.softmax(s.q[r, h * g:(h + 1) * g].double() @ k.t().contiguous() / float(s.hd) ** 0.5, -1)
            out[r, h * g:(h + 1) * g] = w @ v
    return out
