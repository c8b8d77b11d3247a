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
