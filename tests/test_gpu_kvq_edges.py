"""Attention over the 4-bit cache at the edges of what its arrays may say."""
import numpy as np
import pytest

from tests.test_gpu_kvq import DEV, Setup, _ints, _room

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("byte", [253, 254, 255])
@pytest.mark.parametrize("n_q,n_kv,hd,kind", [
    (28, 4, 128, ""), (14, 2, 64, ""), (28, 4, 128, "tiles"), (28, 4, 128, "split"), (14, 2, 64, "split"), (28, 4, 128, "eight")])
def test_a_bad_page_beside_rows_that_do_not_see_it(n_q, n_kv, hd, kind, byte):
    """A page id outside the cache is not followed, and no other page's bytes are in its place: the rows of its tile that
    end before it are as they are without it, whatever the first page of a cache that nobody cleared holds."""
    for dtype in ("bf16",) if kind else ("bf16", "f32"):
        ctx, rows = [70, 300, 130], [12, 60, 1]
        s = Setup(n_q, n_kv, hd, ctx, rows, dtype, seed=51, room=_room(kind, n_q, hd), spare=3)
        used = set(s.table[s.table >= 0].tolist())
        spare = next(i for i in range(1, s.cache.n_pages) if i not in used)
        s.table[s.table == 0] = spare  # the first page is nobody's
        s.dev_table = torch.from_numpy(s.table).to(DEV)
        s.cache.blocks.fill_(byte)
        s.fill()
        good = s.cache.attend(s.batch(), s.q)
        s.check(good)
        t = s.dev_table.clone()
        t[0, 1] = s.cache.n_pages  # positions 64 on, rows 6 on
        t[1, 4] = -1               # positions 256 on
        b = s.cache.batch(_ints(ctx), t, row_offsets=_ints(np.concatenate([[0], np.cumsum(rows)])),
                          n_rows=s.q.shape[0], max_rows=s.q.shape[0] if kind else max(rows))
        out = torch.full_like(s.q, 5.0)
        s.cache.attend(b, s.q, out=out)
        n = sum(rows)
        want = torch.zeros(n, dtype=torch.bool, device=DEV)
        want[6:12] = True
        want[12 + 16:72] = True
        assert torch.isnan(out[:n][want]).all()
        assert torch.equal(out[:n][~want], good[:n][~want])
        assert (out[n:] == 5).all()
