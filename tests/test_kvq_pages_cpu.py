"""The 4-bit cache's page calls without a GPU: their refusals, what needs no launch, and their plain forms."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import kvq_pages as op
from paper_2509_21009_amd import build
from paper_2509_21009_amd import rollpack as rp
from tests.test_kvq_cpu import BAD_BATCHES, BAD_CACHES, BAD_TENSORS, OVERLAPS, PTR, _batch, _cache, _host_cache, _refused, _tensor

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PLAN = os.path.join(ROOT, "tests", "cpp", "kvq_pages_plan.cpp")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return rp.load_library()


def _pool(**kw):
    return rp.RpKvqPool(**{**dict(page_table=PTR, table_stride=4, contexts=PTR, free_pages=PTR, state=PTR, workspace=PTR, n_seqs=3,
                                  max_context=256, n_pages=8), **kw})


def test_fit_refuses_bad_arguments(lib):
    ok = dict(pool=_pool(), lengths=PTR, n_rows=6, off=PTR, positions=PTR, slots=PTR)

    def call(**kw):
        a = {**ok, **kw}
        rp.rp_kvq_fit_pages(a["pool"], a["lengths"], a["n_rows"], a["off"], a["positions"], a["slots"], 0)

    bad = [dict(page_table=0), dict(page_table=PTR + 2), dict(table_stride=0), dict(table_stride=-4), dict(table_stride=1 << 33), dict(contexts=0),
           dict(free_pages=0), dict(state=0), dict(state=PTR + 1), dict(workspace=0), dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1), dict(max_context=-1),
           dict(max_context=257), dict(max_context=(1 << 30) + 1, table_stride=1 << 30), dict(n_pages=0), dict(n_pages=(1 << 24) + 1)]
    for kw in bad:
        _refused(lambda: call(pool=_pool(**kw)))
    for kw in (dict(pool=None), dict(lengths=0), dict(lengths=PTR + 2), dict(n_rows=-1), dict(n_rows=(1 << 24) + 1), dict(off=0), dict(positions=0),
               dict(slots=0), dict(slots=PTR + 1)):
        _refused(lambda: call(**kw))


def test_ranges_refuse_bad_arguments(lib):
    for bad in BAD_CACHES:
        _refused(rp.rp_kvq_key_ranges, _cache(**bad), _batch(), 4 * PTR, 0)
    for bad in BAD_BATCHES:
        _refused(rp.rp_kvq_key_ranges, _cache(), _batch(**bad), 4 * PTR, 0)
    for args in ((None, _batch(), 4 * PTR), (_cache(), None, 4 * PTR), (_cache(), _batch(), 0), (_cache(), _batch(), 4 * PTR + 8)):
        _refused(rp.rp_kvq_key_ranges, *args, 0)
    _refused(rp.rp_kvq_key_ranges, _cache(n_kv_heads=1024), _batch(n_rows=(1 << 16) + 1), 4 * PTR, 0)


def test_scores_refuse_bad_arguments(lib):
    ok = dict(cache=_cache(), batch=_batch(), n_q=6, q=_tensor(6), ranges=4 * PTR, scores=PTR, n=4)

    def call(**kw):
        a = {**ok, **kw}
        rp.rp_kvq_page_scores(a["cache"], a["batch"], a["n_q"], a["q"], a["ranges"], a["scores"], a["n"], 0)

    cases = [dict(cache=_cache(**b)) for b in BAD_CACHES if "blocks" not in b] + [dict(batch=_batch(**b)) for b in BAD_BATCHES]
    cases += [dict(q=_tensor(6, **b)) for b in BAD_TENSORS] + [dict(n_q=n) for n in (0, -2, 7, 65538)]
    cases += [dict(n=n) for n in (0, -1, 3, (1 << 21) + 1)] + [dict(ranges=0), dict(ranges=PTR + 4), dict(scores=0), dict(scores=PTR + 2)]
    cases += [dict(cache=None), dict(batch=None), dict(q=None)]
    cases += [dict(cache=_cache(n_kv_heads=1024), batch=_batch(n_rows=1 << 12), n_q=1024, q=_tensor(1024))]  # more lists than a launch can have
    for kw in cases:
        _refused(lambda: call(**kw))


def test_picks_refuse_bad_arguments(lib):
    ok = dict(batch=_batch(), n_kv=2, scores=PTR, columns=4, first=1, last=1, n=4, picks=2 * PTR)

    def call(**kw):
        a = {**ok, **kw}
        rp.rp_kvq_pick_pages(a["batch"], a["n_kv"], a["scores"], a["columns"], a["first"], a["last"], a["n"], a["picks"], 0)

    cases = [dict(batch=_batch(**b)) for b in BAD_BATCHES] + [dict(n_kv=n) for n in (0, -1, 1025)] + [dict(columns=n) for n in (0, 3, (1 << 21) + 1)]
    cases += [dict(first=-1), dict(last=-1), dict(first=5), dict(first=2, last=3), dict(first=2 ** 31 - 1, last=2 ** 31 - 1), dict(n=0, first=0, last=0),
              dict(n=-1), dict(n=(1 << 24) + 1), dict(scores=0), dict(scores=PTR + 1), dict(picks=0), dict(picks=PTR + 3), dict(batch=None),
              dict(n_kv=1024, batch=_batch(n_rows=1 << 12))]
    for kw in cases:
        _refused(lambda: call(**kw))


def test_attend_picked_refuses_bad_arguments(lib):
    big = 1 << 40
    ok = dict(cache=_cache(), batch=_batch(max_context=1 << 13, table_stride=1 << 7), n_q=6, scale=0.1, q=_tensor(6), picks=PTR, n=40,
              out=_tensor(6, data=2 * PTR), ws=4 * PTR, size=big)

    def call(**kw):
        a = {**ok, **kw}
        rp.rp_kvq_attend_picked(a["cache"], a["batch"], a["n_q"], a["scale"], a["q"], a["picks"], a["n"], a["out"], a["ws"], a["size"], 0)

    cases = [dict(cache=_cache(**b)) for b in BAD_CACHES] + [dict(batch=_batch(**b)) for b in BAD_BATCHES]
    cases += [dict(q=_tensor(6, **b)) for b in BAD_TENSORS]
    cases += [dict(out=_tensor(6, **{**dict(data=2 * PTR), **b})) for b in BAD_TENSORS + OVERLAPS]
    cases += [dict(n_q=n) for n in (0, -2, 7, 65538)] + [dict(scale=s) for s in (0.0, -0.1, float("nan"), float("inf"))]
    need = rp.rp_kvq_attend_picked_workspace(_cache(), ok["batch"], 6, 40)
    assert need > 0
    cases += [dict(out=_tensor(6)), dict(out=_tensor(6, data=2 * PTR, dtype=0)), dict(ws=0), dict(ws=4 * PTR + 16), dict(size=need - 1), dict(picks=0),
              dict(picks=PTR + 2), dict(n=0), dict(n=-1), dict(n=(1 << 24) + 1), dict(cache=None), dict(batch=None), dict(q=None), dict(out=None)]
    for kw in cases:
        _refused(lambda: call(**kw))
    for kw in (dict(batch=_batch(max_rows=-1)), dict(n_q=7), dict(cache=_cache(head_dim=80)), dict(n=0),
               dict(cache=_cache(n_kv_heads=1024), batch=_batch(n_rows=1 << 12), n_q=1024)):
        a = {**ok, **kw}
        _refused(rp.rp_kvq_attend_picked_workspace, a["cache"], a["batch"], a["n_q"], a["n"])


def test_empty_batches_do_nothing(lib):
    """No sequences, no rows, or none that a sequence may have: RP_OK before any array or tensor is looked at."""
    for kw in (dict(n_seqs=0, n_rows=0, max_rows=0), dict(n_seqs=0, contexts=0, page_table=0), dict(n_seqs=3, n_rows=0, max_rows=0), dict(max_rows=0)):
        b = _batch(**kw)
        rp.rp_kvq_key_ranges(_cache(), b, 4 * PTR, 0)
        rp.rp_kvq_page_scores(_cache(), b, 6, _tensor(6), 4 * PTR, PTR, 4, 0)
        rp.rp_kvq_pick_pages(b, 2, PTR, 4, 1, 1, 4, PTR, 0)
        rp.rp_kvq_attend_picked(_cache(), b, 6, 0.1, _tensor(6), PTR, 4, _tensor(6, data=2 * PTR), 4 * PTR, 1 << 40, 0)


def test_workspace_is_bounded(lib):
    """Long lists do not grow it without end; short ones, and many rows, need none."""
    c = _cache(n_kv_heads=4)
    one = _batch(n_seqs=1, n_rows=1, row_offsets=0, max_context=1 << 20, table_stride=1 << 14)
    assert 0 < rp.rp_kvq_attend_picked_workspace(c, one, 28, 1 << 14) <= 64 * 4 * 16 * 130 * 4
    assert rp.rp_kvq_attend_picked_workspace(c, one, 28, 4) == 0
    many = _batch(n_seqs=1, n_rows=4096, max_rows=4096, max_context=1 << 20, table_stride=1 << 14)
    assert rp.rp_kvq_attend_picked_workspace(c, many, 28, 512) == 0


def test_tensors_that_need_gradients_are_refused(lib):
    torch = pytest.importorskip("torch")
    c = _host_cache(torch)
    b = c.batch(torch.ones(3, dtype=torch.int32), torch.zeros((3, 1), dtype=torch.int32))
    q = torch.zeros(3, 4, 64).requires_grad_()
    picks = torch.zeros((3, 2, 1), dtype=torch.int32)
    scores = torch.zeros(3, 2, 1).requires_grad_()
    for call in (lambda: c.page_scores(b, q, c.new_ranges()), lambda: c.attend_picked(b, q, picks), lambda: c.attend_picked(b, q.detach(), picks, out=q),
                 lambda: c.page_scores(b, q.detach(), c.new_ranges(), out=scores), lambda: c.pick_pages(b, scores, 1, first=0)):
        with pytest.raises(ValueError, match="gradient"):
            call()


def test_tensors_of_other_shapes_and_types_are_refused(lib):
    torch = pytest.importorskip("torch")
    c = _host_cache(torch)
    b = c.batch(torch.ones(3, dtype=torch.int32), torch.zeros((3, 1), dtype=torch.int32))
    q, ranges, scores = torch.zeros(3, 4, 64), c.new_ranges(), torch.zeros(3, 2, 1)
    picks = torch.zeros((3, 2, 1), dtype=torch.int32)
    for call in (lambda: c.update_ranges(b, ranges.float()), lambda: c.update_ranges(b, ranges[1:]), lambda: c.update_ranges(b, ranges.to("meta")),
                 lambda: c.page_scores(b, q, ranges[:, :, :1]), lambda: c.page_scores(b, q[:2], ranges), lambda: c.page_scores(b, q[..., :32], ranges),
                 lambda: c.page_scores(b, q, ranges, out=scores[:2]), lambda: c.pick_pages(b, scores[:, :1], 1), lambda: c.pick_pages(b, scores.half(), 1),
                 lambda: c.pick_pages(b, scores, 1 << 32), lambda: c.pick_pages(b, scores, 1, first=-1), lambda: c.pick_pages(b, scores, 2, out=picks),
                 lambda: c.attend_picked(b, q, picks.short()), lambda: c.attend_picked(b, q, picks[1:]), lambda: c.attend_picked(b, q, picks[0])):
        with pytest.raises(ValueError):
            call()


def test_pools_live_in_gpu_memory_and_within_their_limits(lib):
    pytest.importorskip("torch")
    for args in ((4, 2, 64), (0, 2, 64), ((1 << 24) + 1, 2, 64), (4, -1, 64), (4, (1 << 20) + 1, 64), (4, 2, -1), (4, 2, (1 << 30) + 1), (2 ** 32 + 4, 2, 64)):
        with pytest.raises(ValueError):
            rp.KvqPages(*args, device="cpu")


# ---- which kernel takes a call -------------------------------------------------------

def test_plan_under_sanitizers(tmp_path):
    exe = tmp_path / "kvq_pages_plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", f"-I{build.CSRC}", PLAN,
                    "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "plan tests passed" in r.stdout, r.stderr


def test_gpu_tests_reach_every_kernel(tmp_path):
    """The calls of tests/test_gpu_kvq_pages.py that are there for a form of a kernel are of that form."""
    so = tmp_path / "plan.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}", PLAN, "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))

    def plan(n_q, n_kv, hd, bf16, n_rows, max_rows, columns, n):
        out = (ctypes.c_int * 6)()
        lib.kvq_pages_plan_of(n_q, n_kv, hd, bf16, n_rows, max_rows, columns, n, out)
        return tuple(out)

    for bf16 in (1, 0):  # test_attend_picked_split_and_whole: items, waves, shared
        assert plan(28, 4, 128, bf16, 1, 1, 313, 313)[3:] == (64, 4, 0) and plan(4, 2, 64, bf16, 2, 1, 141, 90)[3:] == (23, 4, 0)
        assert plan(28, 4, 128, bf16, 210, 70, 47, 9)[3:] == (1, 2, 1) and plan(6, 3, 64, bf16, 80, 1, 12, 20)[3:] == (1, 8, 0)
        assert plan(6, 3, 64, bf16, 80, 2, 12, 20)[3:] == (1, 8, 1) and plan(7, 1, 128, bf16, 60, 4, 40, 40)[3:] == (8, 4, 1)
        assert plan(40, 2, 64, bf16, 210, 70, 47, 9)[3:] == (1, 2, 1)
        # tests/test_gpu_kvq_picked_softmax.py's forms
        for (n_q, n_kv, hd), n_rows, most, pages, want in (
                ((7, 1, 128), 14, 9, 16, (1, 4, 1)), ((32, 2, 128), 13, 9, 15, (1, 4, 1)), ((10, 2, 64), 80, 1, 22, (1, 8, 0)),
                ((8, 1, 128), 150, 1, 22, (1, 8, 0)), ((28, 4, 128), 160, 100, 11, (1, 2, 1)), ((14, 2, 64), 300, 200, 11, (1, 2, 1)),
                ((7, 1, 128), 1, 1, 79, (20, 4, 0)), ((14, 2, 64), 3, 2, 68, (17, 4, 1))):
            assert plan(n_q, n_kv, hd, bf16, n_rows, most, pages, pages)[3:] == want
        # test_scores_of_many_rows: rows, tiles, shared
        assert plan(14, 2, 64, bf16, 1700, 1700, 15, 1)[:3] == (2, 2, 1) and plan(28, 4, 128, bf16, 3000, 3000, 100, 1)[:3] == (16, 2, 1)
        assert plan(28, 4, 128, bf16, 3000, 3000, 1024, 1)[:3] == (32, 4 if bf16 else 2, 1)
        assert plan(28, 4, 128, bf16, 6, 1, 17, 1)[:3] == (1, 1, 0)
        # test_scores_of_long_sequences
        for n_q, n_kv, hd in ((2, 2, 64), (28, 4, 128), (16, 1, 128)):
            assert plan(n_q, n_kv, hd, bf16, 10, 1, 300, 1)[:3] == (1, 1, 0) and plan(n_q, n_kv, hd, bf16, 1000, 1, 300, 1)[:3] == (1, 4, 0)


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")
@pytest.mark.parametrize("source,least,limits", [
    ("k_kvq_picked.hip", 16, (("attend_pickedILi128ELb0ELi4ELb0ELb1E", 128), ("attend_pickedILi128ELb0ELi2ELb1ELb1E", 128), ("attend_pickedILi128ELb0ELi4ELb0ELb0E", 168),
                              ("attend_pickedILi64ELb0ELi4E", 128), ("attend_pickedILi128ELb1ELi8E", 256))),
    ("k_kvq_pages.hip", 18, (("scores_walkILi128ELb0E", 168), ("scores_walkILi128ELb1E", 256), ("k_kvq_scoresILi128ELb0ELi4E", 256), ("k_kvq_scoresILi128ELb1ELi2E", 256),
                             ("k_kvq_rangesILi128E", 128)))])
def test_registers_and_scratch(source, least, limits):
    """No kernel spills, and the waves of a SIMD are those that the launch bounds and plans count with."""
    asm = subprocess.run([build.HIPCC, *build.COMMON, *build.DEVICE, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", "-"],
                         check=True, capture_output=True, text=True, timeout=300).stdout
    info = {m.group(1): (int(m.group(2)), int(m.group(3))) for m in
            re.finditer(r"^(_Z\w+):.*?; TotalNumVgprs: (\d+).*?; ScratchSize: (\d+)", asm, flags=re.S | re.M)}
    assert len(info) >= least and not [k for k, (_, scratch) in info.items() if scratch]
    for name, most in limits:
        found = [v for k, (v, _) in info.items() if name in k]
        assert found and max(found) <= most, (name, found)


# ---- the plain forms -----------------------------------------------------------------

def test_plain_pool():
    """No page has two owners, none is lost, and slots are the table's."""
    rng = np.random.default_rng(0)
    p = op.Pool(range(60), 6, 640)
    for _ in range(50):
        to = np.where(rng.random(6) < 0.3, rng.integers(0, 641, 6), np.minimum(np.array(p.contexts) + 1, 640))
        old = list(p.contexts)
        error, off, pos, slots = p.fit(to, 4000)
        assert error == 0
        owned = sum(p.table, []) + p.free
        assert sorted(owned) == list(range(60))
        for b in range(6):
            assert pos[off[b]:off[b + 1]].tolist() == list(range(old[b], to[b]))
            assert all(p.table[b][t // 64] == s // 64 and t % 64 == s % 64 for t, s in zip(pos[off[b]:off[b + 1]], slots[off[b]:off[b + 1]]))


def test_plain_scores_are_a_bound():
    rng = np.random.default_rng(1)
    k, q = rng.standard_normal((130, 2, 64)), rng.standard_normal((3, 6, 64))
    r = op.key_ranges(k)
    s, _ = op.page_scores(q, r, [129, 64, 10], 4)
    dot = np.einsum("nhgd,thd->nhgt", q.reshape(3, 2, 3, 64), k).max(2)
    assert (s[0, :, 0] >= dot[0, :, :64].max(-1)).all() and (s[0, :, 2] >= dot[0, :, 128:].max(-1)).all()
    assert (s[:, :, 3] == -np.inf).all() and (s[1, :, 2] == -np.inf).all() and (s[2, :, 1:] == -np.inf).all()


def test_plain_picks():
    s = np.array([0.0, 5.0, np.nan, 5.0, -np.inf, 7.0, 1.0, 2.0], np.float32)
    assert op.pick(s, 8, 1, 1, 4).tolist() == [0, 2, 5, 7] and op.pick(s, 8, 0, 0, 3).tolist() == [1, 2, 5]
    assert op.pick(s, 3, 1, 1, 4).tolist() == [0, 1, 2, -1] and op.pick(s, 8, 2, 2, 4).tolist() == [0, 1, 6, 7]
    assert op.pick(s, 0, 1, 1, 3).tolist() == [-1] * 3
    assert op.listed_tokens([0, -1, 2, 5], 130).tolist() == list(range(64)) + [128, 129, 130]
