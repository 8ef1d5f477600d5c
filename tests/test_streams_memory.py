"""Memory that a call allocates itself comes from the memory of the stream it runs on, on the
host: the calls are made with the library and torch's streams replaced."""
import contextlib
import types

import pytest
import torch

from paper_2606_29629_amd import _lib as T

CFG = T.LayerConfig(hidden=64, n_q_heads=1, n_kv_heads=1, head_dim=64, ffn_dim=64, rms_eps=1e-6,
                    rope_base=1e6)
HANDLE = 1234


@pytest.fixture
def made(monkeypatch):
    """(bytes, whether within the call's stream) of each torch.empty and torch.empty_like."""
    state, log = {"on": None}, []

    @contextlib.contextmanager
    def on(stream):
        state["on"] = stream
        yield
        state["on"] = None

    def recorded(make):
        def call(*args, **kw):
            t = make(*args, **kw)
            log.append((t.nbytes, state["on"] == HANDLE))
            return t
        return call

    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda s, device=None: s)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", recorded(torch.empty))
    monkeypatch.setattr(torch, "empty_like", recorded(torch.empty_like))
    monkeypatch.setattr(T, "_on_gpu", lambda what, stream, *tensors: stream)
    monkeypatch.setattr(T, "workspace_size", lambda *a: 4096)
    monkeypatch.setattr(T, "linear_workspace_size", lambda *a: 4096)
    monkeypatch.setattr(T, "lib", lambda: types.SimpleNamespace(**{n: lambda *a: 0 for n in T._FUNCS}))
    return log


def caches():
    kv = torch.zeros(1, 1, 64, 64, dtype=torch.bfloat16)
    return {"bf16": (kv, kv.clone()), "8-bit": T.KV8Cache.empty(CFG, 1, 64, device="cpu")}


@pytest.mark.parametrize("call", [T.layer_prefill, T.layer_decode])
@pytest.mark.parametrize("kind", ["bf16", "8-bit"])
def test_layer_calls(made, kind, call):
    cache, x = caches()[kind], torch.zeros(1, 64, dtype=torch.bfloat16)
    batch = T.DeviceBatch([0], [3], [1], device="cpu")
    made.clear()
    out, ws = call(CFG, {}, cache, batch, x, stream=HANDLE)
    assert made == [(out.nbytes, True), (ws.nbytes, True)] and ws.nbytes == 4096


def test_linear_and_the_step_without_a_workspace(made):
    x = torch.zeros(1, 64, dtype=torch.bfloat16)
    made.clear()
    out = T.linear(x, torch.zeros(32, 64, dtype=torch.bfloat16), stream=HANDLE)
    assert made == [(out.nbytes, True), (4096, True)]
    cache, batch = caches()["bf16"], T.DeviceBatch([0], [3], [1], device="cpu")
    made.clear()
    out = T.layer_decode_noalloc(CFG, {}, cache, batch, x, stream=HANDLE)
    assert made == [(out.nbytes, True)]


def test_a_stream_of_another_gpu_is_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    tensor = types.SimpleNamespace(get_device=lambda: 0, device="cuda:0")
    stream = types.SimpleNamespace(cuda_stream=HANDLE, device_index=0)
    assert T._on_gpu("call", stream, tensor, None, tensor) == T._on_gpu("call", HANDLE, tensor) == HANDLE
    stream.device_index = 1
    with pytest.raises(ValueError, match="stream of GPU 1"):
        T._on_gpu("call", stream, tensor, tensor)
