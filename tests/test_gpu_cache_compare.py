"""paper_2509_21009_amd/cache_compare.py runs and writes its two tables."""
import sys

import pytest

from tests.gpu_helpers import rp

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def test_tables(monkeypatch, tmp_path, capsys):
    rp()
    from paper_2509_21009_amd import cache_compare
    out = tmp_path / "t.md"
    monkeypatch.setattr(sys, "argv", ["cache_compare", "--workload", "0.5b", "--sets", "3:20:90", "--new", "6", "--layers", "1", "--out", str(out)])
    cache_compare.main()
    text = out.read_text()
    assert text in capsys.readouterr().out
    rows = [line.split(" | ") for line in text.splitlines() if line.startswith("| 3, 20")]
    assert len(rows) == 2 and rows[0][1] == "bf16" and rows[1][1] == "4 bits"
    pools = [float(r[7].split()[0]) for r in rows]
    assert pools[1] < pools[0]
    assert text.splitlines()[-1].startswith("| 1 | ")
