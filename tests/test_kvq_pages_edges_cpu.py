"""The 4-bit cache's page calls without a GPU: the bounds of a batch that a pool hands out, what is read of a page table."""
import os
import re
import subprocess

import pytest

from oracle import kvq_pages as op
from paper_2509_21009_amd import build
from paper_2509_21009_amd import rollpack as rp
from tests.test_kvq_cpu import PTR, _refused
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
