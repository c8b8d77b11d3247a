"""Device outputs of an engine whose stream is not the caller's, on a recording stand-in for torch."""
import contextlib
import types

import numpy as np
import pytest

from paper_2509_21009_amd import rollpack as rp


class _Stream:
    def __init__(self, name, log):
        self.name, self.log, self.cuda_stream = name, log, 1

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


class _Out:
    def __init__(self, log, on):
        self.log, self.on = log, on

    def data_ptr(self):
        return 4096

    def record_stream(self, s):
        self.log.append(("output of", self.on.name, "used on", s.name))

    def __getitem__(self, _):
        return self


def _engine(log, engine_stream, caller_stream):
    now = [caller_stream]

    @contextlib.contextmanager
    def stream(s):
        now.append(s)
        yield
        now.pop()

    torch = types.SimpleNamespace(float32="f32", bfloat16="bf16", empty=lambda *a, **k: log.append(("empty", now[-1].name)) or _Out(log, now[-1]),
                                  cuda=types.SimpleNamespace(stream=stream, current_stream=lambda dev=None: now[-1]))
    e = object.__new__(rp.Engine)
    e.torch, e.stream, e.handle, e.max_seqs = torch, engine_stream, None, 2
    e.kv = types.SimpleNamespace(device="dev")
    e.shape = types.SimpleNamespace(vocab=8, n_kv=2, head_dim=64)
    return e


@pytest.mark.parametrize("call", ["prefill", "decode_step", "read_kv"])
def test_outputs_cross_streams_in_order(monkeypatch, call):
    """Memory of the engine's stream, which writes it; the caller's stream waits for the engine's, and the allocator knows it."""
    for same in (False, True):
        log = []
        mine = _Stream("engine's", log)
        e = _engine(log, mine, mine if same else _Stream("caller's", log))
        for name in ("rp_prefill", "rp_decode_step", "rp_read_kv"):
            monkeypatch.setattr(rp, name, lambda *a: log.append("call") or (2, np.zeros(2)))
        {"prefill": lambda: e.prefill([1], [0], [0, 1], [4], logits=True), "decode_step": lambda: e.decode_step(logits=True),
         "read_kv": lambda: e.read_kv(1, 0, 0, 4)}[call]()
        outs = 2 if call == "read_kv" else 1
        want = [("empty", "engine's")] * outs + ["call"]
        if not same:
            want += [("caller's", "waits for", "engine's")] + [("output of", "engine's", "used on", "caller's")] * outs
        assert log == want
