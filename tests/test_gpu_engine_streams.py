"""An engine on a stream of its own: its outputs on the caller's stream, its inputs from there."""
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


def _busy():
    """Some milliseconds of work on the current stream."""
    x = torch.randn(4096, 4096, device=DEV)
    for _ in range(12):
        x = x @ x * 1e-3
    return x


@pytest.mark.parametrize("kv4", [True, False])
def test_outputs_are_ready_on_the_callers_stream(kv4):
    R = rp()
    wd = R.weights_for_engine(make_weights(SMALL, seed=3, device=DEV))
    rng = np.random.default_rng(1)
    toks, offs = rng.integers(0, SMALL.vocab, 130).astype(np.int32), np.array([0, 50, 130])
    ids, mn = np.array([5, 9]), np.full(2, 6, np.int32)

    def run(stream, busy):
        eng = R.Engine(SMALL, wd, max_seqs=2, max_prefill_tokens=256, max_context=128, kv_pages=4, stream=stream, kv4=kv4)
        outs = []
        for step in range(4):
            if busy:
                with torch.cuda.stream(stream):
                    _busy()  # the engine's call queues behind it, and its output comes late
            out = eng.prefill(ids, toks, offs, mn, 7, 0.0, logits=True)[0] if step == 0 else eng.decode_step(logits=True)[2]
            outs.append(out.clone())  # on the current stream
            del out
        if kv4:
            if busy:
                with torch.cuda.stream(stream):
                    _busy()
            outs += [t.clone() for t in eng.read_kv(9, 1, 0, 80)]
        torch.cuda.synchronize()
        eng.close()
        return outs

    want = run(None, False)
    got = run(torch.cuda.Stream(), True)
    assert len(want) == len(got) and all(torch.equal(a, b) for a, b in zip(want, got))


def test_weights_may_still_be_on_their_way():
    """Weights written by work that is queued on the caller's stream when the engine is made."""
    R = rp()
    w = make_weights(SMALL, seed=3, device=DEV)
    rng = np.random.default_rng(1)
    toks, offs, ids, mn = rng.integers(0, SMALL.vocab, 130).astype(np.int32), np.array([0, 50, 130]), np.array([5, 9]), np.full(2, 6, np.int32)
    lim = R.RpEngineLimits(2, 256, 128, 64, 4)
    want = R.generate(SMALL, R.weights_for_engine(w), ids, toks, offs, mn, 7, 0.0, limits=lim)[0]
    late = {k: torch.zeros_like(v) if torch.is_tensor(v) else v for k, v in w.items() if k != "layers"}
    late["layers"] = [{k: torch.zeros_like(v) for k, v in layer.items()} for layer in w["layers"]]
    for one_shot in (True, False):
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        _busy()
        for k, v in late.items():
            if torch.is_tensor(v):
                v.copy_(w[k])
        for a, b in zip(late["layers"], w["layers"]):
            for k in a:
                a[k].copy_(b[k])
        if one_shot:
            got = R.generate(SMALL, R.weights_for_engine(late), ids, toks, offs, mn, 7, 0.0, limits=lim, stream=side)[0]
        else:
            eng = R.Engine(SMALL, R.weights_for_engine(late), max_seqs=2, max_prefill_tokens=256, max_context=128, kv_pages=4, stream=side)
            got = eng.rollout(ids, toks, offs, mn, 7, 0.0)[0]
            eng.close()
        assert np.array_equal(got, want)
        for v in [v for v in late.values() if torch.is_tensor(v)] + [v for layer in late["layers"] for v in layer.values()]:
            v.zero_()
