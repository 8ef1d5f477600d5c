"""The decoder layer over an 8-bit cache, stage by stage: the rows it appends are those of
the layer on a bf16 cache put through the append's definition (bit for bit), its attention
keeps the bounds of tests/kv8_ref.py on the cache as it stands, and what follows is the
layer's own (x1 within float32 sums and half a bf16 step, the dense output within the
strict end-to-end bound of the small shapes)."""
import numpy as np
import pytest

import kv8_ref
import oracle.layer as ol
from paper_2606_29629_amd import _lib as T
from paper_2606_29629_amd.workload import DeviceLayer, to_device_bf16, to_host_f64
from synth import LayerConfig, bf16_to_f32, layer_talker, make_weights, make_x
from test_gpu_kv8 import make_cache, same_cache

pytestmark = pytest.mark.gpu

TINY = LayerConfig(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=1024)
WIDE = LayerConfig(hidden=512, n_q_heads=7, n_kv_heads=1, head_dim=128, ffn_dim=256, qkv_bias=True)
NORMED = LayerConfig(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=512, qk_norm=True,
                     mrope_section=(8, 12, 12))
MOE = LayerConfig(hidden=256, n_q_heads=4, n_kv_heads=1, head_dim=128, n_experts=8, top_k=2,
                  expert_ffn_dim=128)
BATCHES = {
    "decode": ([1, 0, 2], [300, 31, 0], [1, 1, 1]),
    "prefill": ([0, 2], [0, 40], [200, 33]),
    "mixed": ([2, 0, 1], [250, 0, 64], [1, 150, 1]),
}


def run_layer(cfg, name, fmt, page):
    import torch
    slot, ctx, q = BATCHES[name]
    wb = make_weights(cfg, 3)
    dl = DeviceLayer(cfg, wb)
    cache = make_cache(dl.cfg, 3, 512, fmt, 64 if page else 32, page, seed=7)
    pos = None
    if cfg.mrope_section:
        pos = np.stack([np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, q)])] * 3)
        pos[1] //= 2
    db = T.DeviceBatch(slot, ctx, q, pos=pos)
    x = to_device_bf16(make_x(cfg, db.n_tokens, 3))
    step = T.layer_decode if name == "decode" else T.layer_prefill
    # the new rows, from the layer on a bf16 cache
    shape = 3, cfg.n_kv_heads, 512, cfg.head_dim
    twin = [torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    step(dl.cfg, dl.w, tuple(twin), db, x)
    new = [np.concatenate([to_host_f64(t)[s, :, c:c + n].transpose(1, 0, 2)
                           for s, c, n in zip(slot, ctx, q)]) for t in twin]
    ref = kv8_ref.Cache(cache)
    ref.append(db.host, new[0], new[1], db.pos.cpu().numpy()[:db.n_tokens])
    out, ws = step(dl.cfg, dl.w, cache, db, x)
    torch.cuda.synchronize()
    m, n = T.workspace_layout(dl.cfg, db), db.n_tokens
    heads = cfg.n_q_heads * cfg.head_dim

    def at(offset, cols):
        return to_host_f64(ws[offset:offset + n * cols * 2].view(torch.bfloat16).view(n, cols))

    queries, attn, x1 = at(m.q, heads), at(m.attn, heads), at(m.x1, cfg.hidden)
    want, tol, mass, mtol = ref.attention(db.host, queries.reshape(n, cfg.n_q_heads, cfg.head_dim))
    assert (np.abs(attn.reshape(want.shape) - want) <= tol).all()
    ref.mass = mass
    same_cache(cache, ref, mtol)
    w = {k: bf16_to_f32(v).astype(np.float64) for k, v in wb.items()}
    x64 = to_host_f64(x)
    w1 = x64 + attn @ w["w_o"].T
    sums = (heads + 8) * 2.0 ** -24 * (np.abs(x64) + np.abs(attn) @ np.abs(w["w_o"]).T)
    assert (np.abs(x1 - w1) <= 2.0 ** -8 * np.abs(w1) + sums).all()
    got = to_host_f64(out)
    assert np.isfinite(got).all()
    if not cfg.moe:
        h2 = ol.round_bf16(ol.rmsnorm(x1, w["mlp_norm"], cfg.rms_eps))
        gu = h2 @ w["w_gate_up"].T
        act = ol.round_bf16(ol.silu(gu[:, :cfg.ffn_dim]) * gu[:, cfg.ffn_dim:])
        r = x1 + act @ w["w_down"].T
        assert (np.abs(got - r) <= np.maximum(2e-2, 1e-2 * np.abs(r))).all()
    return cache, db, x, out, dl


@pytest.mark.parametrize("name", sorted(BATCHES))
@pytest.mark.parametrize("page", [0, 128])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_layer(fmt, page, name):
    run_layer(TINY, name, fmt, page)


@pytest.mark.parametrize("name", sorted(BATCHES))
@pytest.mark.parametrize("cfg", [WIDE, NORMED, MOE, layer_talker()], ids=["bias", "normed", "moe", "talker"])
def test_layer_variants(cfg, name):
    run_layer(cfg, name, "int8", 0)


def test_layer_step_in_a_graph():
    """A decode step captured and replayed between eager work: the same output each time (the
    step rewrites its own rows), with the weights' sums put back before each."""
    import torch
    cache, db, x, _, dl = run_layer(TINY, "decode", "e4m3", 0)
    ws = torch.empty(T.workspace_size(dl.cfg, db, cache), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    st = torch.cuda.Stream()
    call = lambda: T.layer_decode(dl.cfg, dl.w, cache, db, x, out=out, workspace=ws, stream=st)
    start = cache.mass.clone()
    torch.cuda.synchronize()
    call()
    st.synchronize()
    ref, mass = out.clone(), cache.mass.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        call()
    for i in range(3):
        cache.mass.copy_(start)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(cache.mass, mass), i
        junk = torch.randn(1 << 20, device="cuda") * 3.0
        del junk
        torch.cuda.synchronize()


def test_generation_under_a_budget():
    """Prompt, steps and evictions through the layer: the cache never holds more than the
    budget between steps, and every step keeps its stages' bounds."""
    import torch
    cfg, budget = TINY, 128
    dl = DeviceLayer(cfg, make_weights(cfg, 5))
    cache = T.KV8Cache.empty(dl.cfg, 2, 384, "int8", mass=True, stamp=True)
    ctx, seen = [0, 0], [0, 0]
    for i, q in enumerate([[180, 60], [1, 1], [1, 90], [1, 1]]):
        pos = np.concatenate([np.arange(s, s + n) for s, n in zip(seen, q)])
        db = T.DeviceBatch([1, 0], ctx, q, pos=pos)
        x = to_device_bf16(make_x(cfg, db.n_tokens, 5, step=i))
        before = kv8_ref.Cache(cache)
        out, ws = T.layer_prefill(dl.cfg, dl.w, cache, db, x)
        m, n = T.workspace_layout(dl.cfg, db), db.n_tokens
        rows = lambda o: to_host_f64(ws[o:o + n * 512].view(torch.bfloat16).view(n, 4, 64))
        ref = kv8_ref.Cache(cache)
        want, tol, mass, mtol = ref.attention(db.host, rows(m.q))
        assert (np.abs(rows(m.attn) - want) <= tol).all()
        # (the sums of before: new rows begin at 0)
        for s, c, k in zip([1, 0], ctx, q):
            add = mass[s] - ref.mass[s]
            before.mass[s, :, c:c + k] = 0
            assert (np.abs(ref.mass[s, :, :c + k] - before.mass[s, :, :c + k] - add[:, :c + k])
                    <= mtol[s, :, :c + k] + 1e-6).all()
        assert torch.isfinite(out).all()
        plan, new_len = T.kv8_select(dl.cfg, cache, db, budget, 4, 32)
        T.kv8_move(dl.cfg, cache, db, plan)
        ctx, seen = new_len.tolist(), [s + k for s, k in zip(seen, q)]
        assert ctx == [min(budget, c) for c in ctx] and max(seen) > budget
