"""rp_read_kv: which sequences hold a cache, and which outputs it writes."""
import numpy as np
import pytest

from tests.gpu_helpers import rp
from workloads import ModelShape, make_weights

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DEV = torch.device("cuda:0")
SMALL = ModelShape("small", 2, 384, 6, 2, 64, 640, 1152, False, "bf16")


def _engine(plens, n_new, kv_pages, policy=None):
    R = rp()
    wd = R.weights_for_engine(make_weights(SMALL, seed=3, device=DEV))
    eng = R.Engine(SMALL, wd, max_seqs=len(plens), max_prefill_tokens=256, max_context=max(plens) + n_new, kv_pages=kv_pages, kv4=True)
    if policy is not None:
        eng.set_kv_policy(policy)
    toks = np.random.default_rng(2).integers(0, SMALL.vocab, sum(plens)).astype(np.int32)
    eng.prefill(np.arange(len(plens)) + 5, toks, np.concatenate([[0], np.cumsum(plens)]), np.full(len(plens), n_new, np.int32))
    return R, eng


def test_a_preempted_sequence_holds_no_cache():
    R, eng = _engine([60, 61], 20, 3, rp().KV_ON_DEMAND)
    assert torch.isfinite(torch.stack(eng.read_kv(6, 1, 0, 61))).all()
    for _ in range(12):  # until a step leaves sequences waiting, the latest arrival among them
        eng.decode_step()
        if eng.kv_status()["waiting"]:
            break
    assert eng.kv_status()["waiting"] >= 1
    with pytest.raises(R.RollpackError) as e:
        eng.read_kv(6, 0, 0, 1)
    assert e.value.status == 5 and "preempted" in str(e.value)
    with pytest.raises(R.RollpackError) as e:
        eng.read_kv(7, 0, 0, 1)
    assert e.value.status == 4
    eng.close()


def test_overlapping_outputs_are_refused():
    """Each element would hold either's value."""
    R, eng = _engine([60], 4, 1)
    row = 2 * 64 * 2  # bytes of a position
    buf = torch.full((40 * row // 2,), 7.0, dtype=torch.bfloat16, device=DEV)
    at = buf.data_ptr()
    for k, v in ((at, at), (at, at + 19 * row), (at + 19 * row, at), (at, at + 2)):
        with pytest.raises(R.RollpackError) as e:
            R.rp_read_kv(eng.handle, 5, 0, 0, 20, k, v)
        assert e.value.status == 1
    assert (buf == 7).all()
    R.rp_read_kv(eng.handle, 5, 0, 0, 20, at + 20 * row, at)  # side by side
    k, v = eng.read_kv(5, 0, 0, 20)
    assert torch.equal(buf.view(2, 20, 2, 64)[1], k) and torch.equal(buf.view(2, 20, 2, 64)[0], v)
    eng.close()
