"""Layer calls on a stream of their own whose workspace the caller drops: what the current
stream allocates right after does not reach into it."""
import pytest

from paper_2606_29629_amd import _lib as T
from paper_2606_29629_amd.workload import DeviceLayer, to_device_bf16
from synth import LayerConfig, make_weights, make_x
from test_gpu_kv8 import make_cache

pytestmark = pytest.mark.gpu

CFG = LayerConfig(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=1024)


@pytest.mark.parametrize("kind", ["bf16", "8-bit"])
@pytest.mark.parametrize("name", ["decode", "prefill"])
def test_dropped_workspace_of_a_layer_call(name, kind):
    import torch
    dl = DeviceLayer(CFG, make_weights(CFG, 3))
    if kind == "8-bit":
        cache = make_cache(dl.cfg, 3, 4096, "int8", 64, seed=7)
    else:
        cache = tuple(torch.randn(3, 2, 4096, 64, device="cuda").bfloat16() for _ in range(2))
    q = [1, 1, 1] if name == "decode" else [200, 33, 1]
    db = T.DeviceBatch([1, 0, 2], [3000, 31, 2000], q)
    x = to_device_bf16(make_x(CFG, db.n_tokens, 3))
    call = T.layer_decode if name == "decode" else T.layer_prefill
    want, ws = call(dl.cfg, dl.w, cache, db, x)
    size = ws.nbytes
    del ws
    stream = torch.cuda.Stream()
    for given in (stream, stream.cuda_stream):
        torch.cuda.synchronize()
        got = call(dl.cfg, dl.w, cache, db, x, stream=given)[0]
        junk = [torch.full((size,), 77, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(got, want), junk[0][0]
