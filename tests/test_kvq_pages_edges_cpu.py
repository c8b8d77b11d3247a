"""The 4-bit cache's page calls without a GPU: the bounds of a batch that a pool hands out, what is read of a page table, and
which kernel takes a call."""
import ctypes
import os
import re
import subprocess

import pytest

from oracle import kvq_pages as op
from paper_2509_21009_amd import build
from paper_2509_21009_amd import rollpack as rp
from tests.kvq_page_forms import CALLS, HARD, SCORES
from tests.test_kvq_cpu import PTR, _host_cache, _refused
from tests.test_kvq_pages_cpu import _pool

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return rp.load_library()


def test_fit_refuses_bad_bounds(lib):
    """Of a sequence: more rows than the batch has, more tokens than the pool's sequences may have."""
    def call(max_rows=6, max_context=256, **kw):
        rp.rp_kvq_fit_pages_within(kw.get("pool", _pool()), PTR, 6, max_rows, max_context, PTR, PTR, PTR, 0)

    for kw in (dict(max_rows=-1), dict(max_rows=7), dict(max_context=-1), dict(max_context=257), dict(pool=None),
               dict(pool=_pool(max_context=100), max_context=101), dict(pool=_pool(n_pages=0))):
        _refused(lambda: call(**kw))


def test_plain_pool_bounds():
    """A sequence past them changes nothing, whatever it shares the call with."""
    p = op.Pool(range(20), 3, 640)
    assert p.fit([10, 70, 0], 80, max_rows=70, max_context=70)[0] == 0
    for lengths, n_rows, max_rows, max_context, error in (
            ([12, 71, 0], 80, 1, 640, 5), ([11, 71, 1], 80, 1, 640, 0), ([11, 72, 1], 80, 0, 640, 5), ([0, 73, 1], 80, 2, 72, 2),
            ([0, 71, 3], 80, 2, 640, 0), ([0, 71, 3], 2, 2, 640, 0), ([0, 71, 3], 80, 2, 70, 2), ([0, 71, 3], 80, 2, 71, 0),
            ([0, 71, 3], 0, 0, 71, 0), ([0, 71, 6], 2, 2, 640, 3), ([0, 71, 6], 80, 2, 640, 5)):
        before = list(p.contexts)
        got = p.fit(lengths, n_rows, max_rows, max_context)
        assert got[0] == error and p.contexts == (before if error else lengths) and (not error or got[1].tolist() == [0] * 4)


def test_a_batch_keeps_the_arrays_that_it_is_given(lib):
    """All three, as its makers give them, or those that a structure made elsewhere points to."""
    torch = pytest.importorskip("torch")
    c = _host_cache(torch)
    ctx, table, off = torch.ones(3, dtype=torch.int32), torch.zeros((3, 1), dtype=torch.int32), torch.arange(4, dtype=torch.int32)
    b = c.batch(ctx, table, row_offsets=off, n_rows=3)
    assert b.contexts is ctx and b.page_table is table and b.row_offsets is off
    assert c.batch(ctx, table).row_offsets is None
    for kept in ((ctx,), (ctx, table)):
        again = rp.KvqBatch(b.struct, kept)
        assert again.tensors is kept and again.device == ctx.device and again.contexts is ctx


# ---- the page table ------------------------------------------------------------------

def test_scores_read_no_entry_past_a_context(tmp_path):
    exe = tmp_path / "kvq_pages_table"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", f"-I{build.CSRC}",
                    os.path.join(ROOT, "tests", "cpp", "kvq_pages_table.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "table tests passed" in r.stdout, r.stderr
    # and the kernels take their entries from there alone
    text = open(os.path.join(build.CSRC, "k_kvq_pages.hip")).read()
    text = text[text.index("// ---- scores"):text.index("// ---- picks")]
    assert text.count("kvq_seen_entry(") == 2 and re.findall(r"(?:\bpt|table_of\(bt, b\))\[(.*?)\]", text) == ["entry", "entry"]


# ---- which kernel takes a call -------------------------------------------------------

@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    so = tmp_path_factory.mktemp("forms") / "forms.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}", os.path.join(ROOT, "tests", "cpp", "kvq_page_forms.cpp"),
                    "-o", str(so)], check=True)
    return ctypes.CDLL(str(so))


def test_gpu_tests_reach_every_form_of_attention(forms):
    """Every form that some call has is one of tests/kvq_page_forms.py's, for both head dimensions (and both types, which
    do not count here); each of these has the form that its name says."""
    reached = {64: set(), 128: set()}
    for name, (n_q, n_kv, hd, ctx, rows, n) in {**CALLS, **{"hard " + k: (*v, -(-max(v[3]) // 64)) for k, v in HARD.items()}}.items():
        f = forms.kvq_picked_form_of(n_q, n_kv, hd, sum(rows or [1] * len(ctx)), max(rows or [1]), n)
        said = name.split()[-1].split("-")
        assert f >> 3 == {"eight": 8, "four": 4, "two": 2, "split": 4}[said[0]] and bool(f & 4) == (said[0] == "split"), name
        assert bool(f & 2) == (n_q // n_kv > 8) and bool(f & 1) == (rows is not None and max(rows) > 1), name
        reached[hd].add(f)
    for hd in (64, 128):
        seen = (ctypes.c_ubyte * 128)()
        forms.kvq_picked_forms(hd, seen)
        assert {i for i in range(128) if seen[i]} <= reached[hd]
        assert len(reached[hd]) == 14


def test_gpu_tests_reach_every_form_of_scores(forms):
    """The same; here the type counts."""
    for hd in (64, 128):
        for bf16 in (0, 1):
            reached = set()
            for name, (n_q, n_kv, hd_, ctx, rows, room, columns) in SCORES.items():
                if hd_ == hd:
                    f = forms.kvq_score_form_of(n_q, n_kv, hd, bf16, room, 1 if rows is None else room, columns)
                    said = name.split("-")
                    assert f & 3 == (1 if said[0] == "rows" else 2 if said[1] == "heads" else 0), name
                    assert f >> 2 == (1 if said[1] == "heads" else int(said[1]) // 16 if said[0] == "walk" or bf16 else 2), name
                    reached.add(f)
            seen = (ctypes.c_ubyte * 64)()
            forms.kvq_score_forms(hd, bf16, seen)
            assert {i for i in range(64) if seen[i]} <= reached and len(reached) == 4 + bf16
