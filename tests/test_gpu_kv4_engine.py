"""The rollout engine with its KV cache in 4 bits (RP_DTYPE_BF16_KV4), against the fp64 oracle.

What the cache holds is read back and given to the oracle, whose logits over it are compared: the bar is the
other bf16 parity tests' (2e-2 of the largest logit of a position).  The held K and V themselves are within the
quantiser's error of the oracle's own: at most one scale step (include/rollpack.h), for a block whose largest
element may be off by the bf16 forward's error, 2e-2 of the row's largest.
"""
import numpy as np
import pytest

from oracle import kvq as okvq
from tests.gpu_helpers import rp
from workloads import SHAPES, ModelShape, make_weights, weights_to_numpy
from workloads.gen import truncated

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DEV = torch.device("cuda:0")
SMALL = ModelShape("small", 2, 384, 6, 2, 64, 640, 1152, False, "bf16")


def _engine(shape, wd, plens, n_new, max_prefill=4096, kv_pages=None, **kw):
    R = rp()
    pages = sum((p + n_new + 63) // 64 for p in plens) if kv_pages is None else kv_pages
    return R.Engine(shape, R.weights_for_engine(wd), max_seqs=len(plens), max_prefill_tokens=max_prefill,
                    max_context=max(plens) + n_new, kv_pages=pages, kv4=True, **kw)


def _prompts(shape, plens, seed):
    rng = np.random.default_rng(seed)
    prompts = [rng.integers(0, shape.vocab, size=p).astype(np.int32) for p in plens]
    offs = np.concatenate([[0], np.cumsum(plens)]).astype(np.int64)
    return prompts, np.concatenate(prompts), offs, rng


def _parity(shape, plens, n_new, max_prefill=4096, check=None, tol=2e-2):
    wd = make_weights(shape, seed=3, device=DEV)
    w64 = weights_to_numpy(wd)
    prompts, toks, offs, rng = _prompts(shape, plens, sum(plens))
    n = len(plens)
    ids = np.arange(700, 700 + n, dtype=np.int64)
    eng = _engine(shape, wd, plens, n_new, max_prefill)
    forced = rng.integers(0, shape.vocab, size=(n, n_new)).astype(np.int32)
    out, _ = eng.prefill(ids, toks, offs, np.full(n, n_new, np.int32), 11, 1.0, logits=True)
    logits = [out.cpu().numpy().astype(np.float64)]
    for j in range(1, n_new):
        b, rows, lg = eng.decode_step(forced_tokens=forced[:, j - 1], logits=True)
        assert b == n and np.array_equal(rows, ids)
        logits.append(lg.cpu().numpy().astype(np.float64))
    worst = 0.0
    for i in range(n) if check is None else check:
        seq = np.concatenate([prompts[i], forced[i, :n_new - 1]])
        cache = [tuple(t.double().cpu().numpy() for t in eng.read_kv(int(ids[i]), li, 0, len(seq))) for li in range(shape.layers)]
        ref, mine = okvq.forward_over_cache(w64, shape, seq, cache)
        ref = ref[len(prompts[i]) - 1:]
        got = np.stack([lg[i] for lg in logits])
        err = (np.abs(got - ref).max(-1) / np.abs(ref).max(-1)).max()
        worst = max(worst, err)
        for own, held in zip(mine[0], cache[0]):  # layer 0: its inputs are the embeddings
            noise = 2e-2 * np.abs(own).max(axis=(1, 2), keepdims=True)
            top = np.abs(own.reshape(*own.shape[:2], -1, 32)).max(-1) + noise
            step = 2.0 ** np.ceil(np.log2(np.maximum(top / 7, 2.0 ** -125)))
            assert (np.abs(own - held) <= np.repeat(step, 32, -1) + noise).all(), i
    assert worst <= tol, worst
    assert sorted(eng.free_finished().tolist()) == ids.tolist()
    assert eng.kv_status()["free_pages"] == sum((p + n_new + 63) // 64 for p in plens)
    eng.close()


def test_small_model_edges():
    """Two layers; prompts around pages and tiles, decoded side by side."""
    _parity(SMALL, [1, 2, 63, 64, 65, 127, 128, 129, 200, 33], 6)


def test_prompts_in_pieces():
    """Prompts longer than a prefill chunk: later pieces attend to what earlier ones appended."""
    _parity(SMALL, [300, 40, 129, 1], 3, max_prefill=96)


@pytest.mark.parametrize("n_q,n_kv,hd", [(7, 1, 128), (16, 1, 64), (3, 3, 128), (8, 2, 128)])
def test_head_layouts(n_q, n_kv, hd):
    shape = ModelShape("heads", 1, 384, n_q, n_kv, hd, 384, 640, False, "bf16")
    if (n_q + 2 * n_kv) * hd % 128 or n_q * hd % 128:
        pytest.skip("not a bf16 shape")
    _parity(shape, [70, 1, 64, 200], 3)


@pytest.mark.parametrize("name,plens,check", [
    ("qwen2.5-0.5b", [65, 400, 130], None),
    ("qwen2.5-7b", [200, 1000, 64], [0, 1]),
    ("qwen2.5-7b", [60 + i for i in range(80)], [0, 41, 79]),     # more rows than the decode GEMMs' 64
])
def test_real_layer_shapes(name, plens, check):
    _parity(truncated(SHAPES[name], 1, 2048), plens, 3, check=check)


def test_long_context():
    """Contexts that decode splits over the GPU, and a long prompt's columns in many tiles."""
    _parity(truncated(SHAPES["qwen2.5-0.5b"], 1, 1024), [5000, 30], 3, max_prefill=2048)


def test_rollout_under_pressure_and_one_shot():
    """Rounds, pages on demand with preemption, and the one-shot form: lengths, finite log-probabilities, and the one-shot
    form's tokens equal to the engine's."""
    R = rp()
    wd = make_weights(SMALL, seed=3, device=DEV)
    plens = [50, 60, 70, 64, 30, 90, 20, 55]
    n_new = 80
    prompts, toks, offs, rng = _prompts(SMALL, plens, 5)
    ids = np.arange(len(plens), dtype=np.int64)
    mn = np.full(len(plens), n_new, np.int32)
    eng = _engine(SMALL, wd, plens, n_new)
    resp, logp, lens, stats = eng.rollout(ids, toks, offs, mn, 7, 1.0, details=True)
    assert (lens == n_new).all() and np.isfinite(logp).all() and (logp <= 0).all() and (resp >= 0).all() and (resp < SMALL.vocab).all()
    eng.close()
    lim = R.RpEngineLimits(len(plens), 4096, max(plens) + n_new, 64, sum((p + n_new + 63) // 64 for p in plens))
    one = R.generate(SMALL, R.weights_for_engine(wd), ids, toks, offs, mn, 7, 1.0, limits=lim, kv4=True)
    assert np.array_equal(one[0], resp) and np.array_equal(one[1], logp)
    eng = _engine(SMALL, wd, plens, n_new, kv_pages=9)
    eng.set_kv_policy(R.KV_ON_DEMAND)
    resp2, logp2, lens2, _ = eng.rollout(ids, toks, offs, mn, 7, 1.0, details=True)
    st = eng.kv_status()
    assert st["preemptions"] > 0 and st["free_pages"] == 9
    assert (lens2 == n_new).all() and np.isfinite(logp2).all()
    first = np.arange(len(plens)) * n_new
    assert np.array_equal(resp2[first], resp[first])  # sampled from the same prefill rows
    eng.close()


def test_static_workspace():
    R = rp()
    wd = make_weights(SMALL, seed=3, device=DEV)
    plens, n_new = [50, 30], 12
    prompts, toks, offs, rng = _prompts(SMALL, plens, 5)
    ids = np.arange(2, dtype=np.int64)
    mn = np.full(2, n_new, np.int32)
    lim = R.RpEngineLimits(2, 128, 64, 64, 4)
    w = R.weights_for_engine(wd)
    a = R.generate(SMALL, w, ids, toks, offs, mn, 7, 1.0, limits=lim, kv4=True)
    st, layers = R.weights_struct(SMALL, w)
    b = R.rp_generate_static(R.model_config(SMALL, kv4=True), st, lim, torch.cuda.current_stream().cuda_stream, ids, toks, offs,
                             mn, 7, 1.0)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_read_kv_refusals():
    R = rp()
    wd = make_weights(SMALL, seed=3, device=DEV)
    prompts, toks, offs, _ = _prompts(SMALL, [50], 5)
    buf = torch.zeros(50 * 2 * 64 * 2, dtype=torch.bfloat16, device=DEV)
    k, v = buf.data_ptr(), buf.data_ptr() + 50 * 2 * 64 * 2
    eng = _engine(SMALL, wd, [50], 4)
    eng.prefill(np.array([5]), toks, offs, np.array([4], np.int32))
    for args, status in (((6, 0, 0, 1, k, v), 4), ((5, 2, 0, 1, k, v), 1), ((5, -1, 0, 1, k, v), 1), ((5, 0, -1, 1, k, v), 1),
                         ((5, 0, 0, 51, k, v), 1), ((5, 0, 50, 1, k, v), 1), ((5, 0, 0, 1, 0, v), 1), ((5, 0, 0, 1, k, k), 1),
                         ((5, 0, 0, 1, k + 1, v), 1)):
        with pytest.raises(R.RollpackError) as e:
            R.rp_read_kv(eng.handle, *args)
        assert e.value.status == status, args
    part = eng.read_kv(5, 1, 20, 30)
    whole = eng.read_kv(5, 1, 0, 50)
    assert all(torch.equal(a, b[20:]) for a, b in zip(part, whole))
    eng.close()
    eng = R.Engine(SMALL, R.weights_for_engine(wd), max_seqs=1, max_prefill_tokens=64, max_context=64, kv_pages=1)
    eng.prefill(np.array([5]), toks, offs, np.array([4], np.int32))
    with pytest.raises(R.RollpackError) as e:
        R.rp_read_kv(eng.handle, 5, 0, 0, 1, k, v)
    assert e.value.status == 5
    eng.close()


def test_every_layer_holds_its_own_keys_and_values():
    """What each layer's cache holds is the oracle's own K and V of that layer, over the same held cache: within the quantiser's
    step for a block whose largest element, and each element, may be off by the bf16 forward's error.  Another layer's is not."""
    shape = ModelShape("three", 3, 384, 6, 2, 64, 640, 1152, False, "bf16")
    wd = make_weights(shape, seed=4, device=DEV)
    w64 = weights_to_numpy(wd)
    plens, n_new = [70, 129, 5], 4
    prompts, toks, offs, rng = _prompts(shape, plens, 9)
    ids = np.arange(3, dtype=np.int64)
    eng = _engine(shape, wd, plens, n_new, max_prefill=96)  # the second prompt in two pieces
    forced = rng.integers(0, shape.vocab, size=(3, n_new)).astype(np.int32)
    eng.prefill(ids, toks, offs, np.full(3, n_new, np.int32), 11, 1.0)
    for j in range(n_new - 1):
        eng.decode_step(forced_tokens=forced[:, j])

    def within(own, held):
        noise = 2e-2 * np.abs(own).max(axis=(1, 2), keepdims=True)
        top = np.abs(own.reshape(*own.shape[:2], -1, 32)).max(-1) + noise
        step = 2.0 ** np.ceil(np.log2(np.maximum(top / 7, 2.0 ** -125)))
        return np.abs(own - held) <= np.repeat(step, 32, -1) + noise

    for i in range(3):
        seq = np.concatenate([prompts[i], forced[i, :n_new - 1]])
        cache = [tuple(t.double().cpu().numpy() for t in eng.read_kv(i, li, 0, len(seq))) for li in range(3)]
        _, mine = okvq.forward_over_cache(w64, shape, seq, cache)
        for a in range(3):
            for b in range(3):
                for own, held in zip(mine[a], cache[b]):
                    ok = within(own, held)
                    assert ok.all() if a == b else ok.mean() < 0.9, (i, a, b, float(ok.mean()))
    eng.close()
