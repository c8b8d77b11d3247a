"""The 4-bit KV cache without a GPU: its format and plan under the sanitizers, its refusals, its oracle."""
import os
import subprocess

import numpy as np
import pytest

from oracle import kvq as okvq
from paper_2509_21009_amd import rollpack as rp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 1 << 20  # stands for device memory: every call here is refused, or has nothing to do, before it is used


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rp.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return rp.load_library()


def test_format_and_plan_under_sanitizers(tmp_path):
    exe = tmp_path / "kvq_host"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    f"-I{os.path.join(ROOT, 'paper_2509_21009_amd', 'csrc')}",
                    os.path.join(ROOT, "tests", "cpp", "kvq_host.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "host tests passed" in r.stdout, r.stderr


def test_cache_bytes(lib):
    """4.25 bits per element: 17/64 of the bf16 pages."""
    assert rp.rp_kvq_cache_bytes(10, 4, 128) == 10 * 4 * 64 * 128 * 2 * 2 * 17 // 64
    assert rp.rp_kvq_cache_bytes(1, 2, 64) == 2 * 64 * 64 * 2 * 2 * 17 // 64
    for args in ((0, 4, 128), (1 << 25, 4, 128), (1, 0, 128), (1, 2000, 128), (1, 1, 96), (-1, 1, 64)):
        with pytest.raises(rp.RollpackError) as e:
            rp.rp_kvq_cache_bytes(*args)
        assert e.value.status == 1


def _cache(**kw):
    return rp.RpKvqCache(**{**dict(blocks=PTR, n_pages=8, n_kv_heads=2, head_dim=128), **kw})


def _batch(**kw):
    return rp.RpKvqBatch(**{**dict(n_seqs=3, n_rows=6, max_rows=4, max_context=256, row_offsets=PTR, contexts=PTR,
                                   page_table=PTR, table_stride=4), **kw})


def _tensor(heads=2, **kw):
    return rp.RpKvqTensor(**{**dict(data=PTR, row_stride=heads * 128, head_stride=128, dtype=1), **kw})


BAD_CACHES = [dict(blocks=0), dict(blocks=PTR + 128), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(n_kv_heads=0),
              dict(n_kv_heads=1025), dict(head_dim=32), dict(head_dim=0)]
BAD_BATCHES = [dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1), dict(n_rows=-1), dict(n_rows=(1 << 24) + 1),
               dict(max_rows=-1), dict(max_rows=7), dict(max_context=-1), dict(max_context=(1 << 30) + 1, table_stride=1 << 30),
               dict(max_context=257), dict(contexts=0), dict(page_table=0), dict(table_stride=0), dict(table_stride=-4),
               dict(row_offsets=0, n_rows=2)]
BAD_TENSORS = [dict(data=0), dict(data=PTR + 1), dict(dtype=2), dict(dtype=-1), dict(row_stride=-1), dict(head_stride=-128),
               dict(row_stride=1 << 39)]
OVERLAPS = [dict(row_stride=128), dict(row_stride=0), dict(head_stride=64), dict(head_stride=0), dict(row_stride=255)]


def _refused(f, *args):
    with pytest.raises(rp.RollpackError) as e:
        f(*args)
    assert e.value.status == 1 and rp.rp_last_error()


@pytest.mark.parametrize("f", [rp.rp_kvq_append, rp.rp_kvq_read])
def test_append_and_read_refuse_bad_arguments(lib, f):
    for bad in BAD_CACHES:
        _refused(f, _cache(**bad), _batch(), _tensor(), _tensor(data=2 * PTR), 0)
    for bad in BAD_BATCHES:
        _refused(f, _cache(), _batch(**bad), _tensor(), _tensor(data=2 * PTR), 0)
    for bad in BAD_TENSORS:
        _refused(f, _cache(), _batch(), _tensor(**bad), _tensor(data=2 * PTR), 0)
        _refused(f, _cache(), _batch(), _tensor(), _tensor(**{**dict(data=2 * PTR), **bad}), 0)
    _refused(f, _cache(), _batch(), _tensor(dtype=0), _tensor(data=2 * PTR), 0)  # two types
    _refused(f, None, _batch(), _tensor(), _tensor(data=2 * PTR), 0)
    _refused(f, _cache(), None, _tensor(), _tensor(data=2 * PTR), 0)
    _refused(f, _cache(), _batch(), None, _tensor(), 0)


def test_read_refuses_overlapping_outputs(lib):
    for bad in OVERLAPS:
        _refused(rp.rp_kvq_read, _cache(), _batch(), _tensor(**bad), _tensor(data=2 * PTR), 0)
    _refused(rp.rp_kvq_read, _cache(), _batch(), _tensor(), _tensor(), 0)  # both into one tensor


def test_attend_refuses_bad_arguments(lib):
    big = 1 << 40
    ok = dict(cache=_cache(), batch=_batch(max_context=1 << 13, table_stride=1 << 7), n_q=6, scale=0.1, q=_tensor(6), out=_tensor(6, data=2 * PTR), ws=4 * PTR, n=big)

    def call(**kw):
        a = {**ok, **kw}
        rp.rp_kvq_attend(a["cache"], a["batch"], a["n_q"], a["scale"], a["q"], a["out"], a["ws"], a["n"], 0)

    cases = [dict(cache=_cache(**b)) for b in BAD_CACHES] + [dict(batch=_batch(**b)) for b in BAD_BATCHES]
    cases += [dict(q=_tensor(6, **b)) for b in BAD_TENSORS]
    cases += [dict(out=_tensor(6, **{**dict(data=2 * PTR), **b})) for b in BAD_TENSORS + OVERLAPS]
    cases += [dict(n_q=n) for n in (0, -2, 7, 65538)] + [dict(scale=s) for s in (0.0, -0.1, float("nan"), float("inf"))]
    need = rp.rp_kvq_attend_workspace(_cache(), ok["batch"], 6)
    assert need > 0
    cases += [dict(out=_tensor(6)), dict(out=_tensor(6, data=2 * PTR, dtype=0)), dict(ws=0), dict(ws=4 * PTR + 16), dict(n=need - 1),
              dict(cache=None), dict(batch=None), dict(q=None), dict(out=None)]
    for kw in cases:
        _refused(lambda: call(**kw))
    for kw in (dict(batch=_batch(max_rows=-1)), dict(n_q=7), dict(cache=_cache(head_dim=80))):
        a = {**ok, **kw}
        _refused(rp.rp_kvq_attend_workspace, a["cache"], a["batch"], a["n_q"])
    # more blocks than a launch can have
    _refused(rp.rp_kvq_append, _cache(n_kv_heads=1024), _batch(n_rows=(1 << 16) + 1), _tensor(1024), _tensor(1024, data=2 * PTR), 0)
    _refused(rp.rp_kvq_attend_workspace, _cache(n_kv_heads=1024), _batch(n_rows=1 << 24, n_seqs=1 << 20, max_rows=1 << 24, max_context=256), 1 << 16)


def test_empty_batches_do_nothing(lib):
    """No sequences or no rows: RP_OK before any array or tensor is looked at."""
    for kw in (dict(n_seqs=0, n_rows=0, max_rows=0), dict(n_seqs=0, contexts=0, page_table=0), dict(n_seqs=3, n_rows=0, max_rows=0)):
        rp.rp_kvq_append(_cache(), _batch(**kw), _tensor(), _tensor(), 0)
        rp.rp_kvq_read(_cache(), _batch(**kw), _tensor(), _tensor(), 0)
        rp.rp_kvq_attend(_cache(), _batch(**kw), 6, 0.1, _tensor(6), _tensor(6), 4 * PTR, 1 << 40, 0)


def test_batches_whose_sequences_have_no_row_do_nothing(lib):
    """max_rows = 0: the tensors' rows are all behind the last sequence, however many there are; also where a long context
    splits attention into items and a second kernel joins them (its grid has as many blocks as a tile has columns)."""
    for kw in (dict(max_rows=0), dict(max_rows=0, n_seqs=1, max_context=8192, table_stride=128)):
        b = _batch(**kw)
        rp.rp_kvq_append(_cache(), b, _tensor(), _tensor(data=2 * PTR), 0)
        rp.rp_kvq_read(_cache(), b, _tensor(), _tensor(data=2 * PTR), 0)
        rp.rp_kvq_attend(_cache(), b, 6, 0.1, _tensor(6), _tensor(6, data=2 * PTR), 4 * PTR, 1 << 40, 0)


def test_workspace_is_bounded(lib):
    """Long contexts do not grow it without end, and a context of a page needs none."""
    c = _cache(n_kv_heads=4)
    one = rp.rp_kvq_attend_workspace(c, _batch(n_seqs=1, n_rows=1, row_offsets=0, max_context=1 << 20, table_stride=1 << 14), 28)
    assert 0 < one <= 64 * 4 * (16 * 128 + 32) * 4
    assert rp.rp_kvq_attend_workspace(c, _batch(n_seqs=64, n_rows=64, row_offsets=0, max_context=64), 28) == 0


def test_oracle_quantiser():
    """Its values are the nearest of the grid: never further than half a step, or s beyond 6 s."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((40, 64)) * np.exp(rng.normal(0, 3, (40, 1)))
    y = okvq.held(x)
    b, r = x.reshape(40, 2, 32), y.reshape(40, 2, 32)
    amax = np.abs(b).max(-1)
    s = 2.0 ** np.ceil(np.log2(amax / 7))
    a = np.abs(b) / s[..., None]
    step = np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0))
    assert (np.abs(b - r) <= step * s[..., None] * (1 + 1e-12)).all()
    assert np.array_equal(okvq.held(y), y)  # what is held is held again
    assert np.isnan(okvq.held(np.r_[np.inf, np.zeros(31), np.ones(32)])[:32]).all()
    ties = np.r_[[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], np.zeros(24)]
    assert okvq.held(ties)[:8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]


def test_engine_sizes_with_the_cache_in_four_bits(lib):
    """A token takes 17/64 of its bf16 bytes, the pool with it; packed weights stay; fp32 models are refused."""
    import dataclasses
    from workloads import SHAPES
    s = SHAPES["qwen2.5-7b"]
    cfg, bf16 = rp.model_config(s, kv4=True), rp.model_config(s)
    assert rp.rp_kv_bytes_per_token(cfg) == 57344 * 17 // 64
    lim = rp.RpEngineLimits(64, 4096, 17408, 64, 1000)
    assert rp.rp_workspace_size(cfg, lim)[0] == 1000 * 64 * 57344 * 17 // 64
    assert rp.rp_packed_weights_bytes(cfg) == rp.rp_packed_weights_bytes(bf16) > 0
    with pytest.raises(ValueError):
        rp.model_config(SHAPES["tiny"], kv4=True)
    bad = rp.model_config(dataclasses.replace(s, n_q=20, n_kv=1), kv4=True)
    with pytest.raises(rp.RollpackError):
        rp.rp_workspace_size(bad, lim)
    cfg.dtype = 3
    with pytest.raises(rp.RollpackError):
        rp.rp_workspace_size(cfg, lim)
    with pytest.raises(rp.RollpackError) as e:
        rp.rp_read_kv(None, 1, 0, 0, 1, PTR, 2 * PTR)
    assert e.value.status == 1


def _host_cache(torch):
    """A KvqCache over host memory, for calls that are refused before the library is called."""
    c = object.__new__(rp.KvqCache)
    c.torch, c.n_pages, c.n_kv_heads, c.head_dim = torch, 4, 2, 64
    c.blocks = torch.zeros(rp.rp_kvq_cache_bytes(4, 2, 64), dtype=torch.uint8)
    c.device, c.struct = c.blocks.device, rp.RpKvqCache(c.blocks.data_ptr(), 4, 2, 64)
    c._types = {torch.float32: rp.RP_DTYPE_F32, torch.bfloat16: rp.RP_DTYPE_BF16}
    c._call = lambda *a: pytest.fail("called")
    return c


def test_tensors_that_need_gradients_are_refused(lib):
    """The calls have no backward: a gradient would end at them without a word."""
    torch = pytest.importorskip("torch")
    c = _host_cache(torch)
    b = c.batch(torch.ones(3, dtype=torch.int32), torch.zeros((3, 1), dtype=torch.int32))
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    grad = lambda t: t.clone().requires_grad_()
    for call in (lambda: c.attend(b, grad(q)), lambda: c.attend(b, q, out=grad(q)), lambda: c.append(b, grad(k), k),
                 lambda: c.append(b, k, grad(k)), lambda: c.read(b, out=(k, grad(k)))):
        with pytest.raises(ValueError, match="gradient"):
            call()
    c._call = lambda *a: None
    with torch.no_grad():
        c.attend(b, grad(q))
        c.append(b, grad(k), k)


def test_a_batch_on_another_device_is_refused(lib):
    """A batch's arrays are read by kernels on the cache's device."""
    torch = pytest.importorskip("torch")
    c = _host_cache(torch)
    far = _host_cache(torch)
    far.device = torch.device("meta")
    b = far.batch(torch.ones(3, dtype=torch.int32, device="meta"), torch.zeros((3, 1), dtype=torch.int32, device="meta"))
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    c._call = lambda *a: rp.KvqCache._call(c, *a)
    for call in (lambda: c.attend(b, q), lambda: c.append(b, k, k), lambda: c.read(b), lambda: c.read(b, out=(k, k.clone()))):
        with pytest.raises(ValueError, match="batch"):
            call()


def test_bounds_that_do_not_fit_an_int_are_refused(lib):
    """The C structure has 32-bit fields, which would hold a larger number's lower half."""
    torch = pytest.importorskip("torch")
    c = _host_cache(torch)
    ctx, table, off = torch.ones(3, dtype=torch.int32), torch.zeros((3, 1), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for kw in (dict(n_rows=2 ** 32 + 6), dict(max_rows=2 ** 32 + 1), dict(max_rows=2 ** 31), dict(max_context=-2 ** 32 + 5), dict(n_rows=-1),
               dict(max_rows=-1)):
        with pytest.raises(ValueError, match="between"):
            c.batch(ctx, table, row_offsets=off, **{**dict(n_rows=6), **kw})
    b = c.batch(ctx, table, row_offsets=off, n_rows=6, max_rows=4, max_context=64)
    assert (b.struct.n_rows, b.struct.max_rows, b.struct.max_context) == (6, 4, 64)
    for args in ((4, 2 ** 32 + 2, 64), (4, 2, 2 ** 32 + 64), (2 ** 64 + 4, 2, 64)):
        with pytest.raises((ValueError, rp.RollpackError)):
            rp.KvqCache(*args, device="cpu")
        with pytest.raises((ValueError, rp.RollpackError)):
            rp.rp_kvq_cache_bytes(*args)
