"""The long-context operators' refusals and the host side of their references, no GPU:
every call below fails validation before any launch (fake device addresses)."""
import ctypes
import math
import os
import subprocess
import tempfile

import numpy as np
import pytest

import kv8_ref
from paper_2606_29629_amd import _lib as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000  # 256-byte aligned fake device address, never dereferenced


@pytest.fixture(scope="module")
def lib():
    import torch
    if torch.cuda.is_available():
        pytest.skip("fake-address validation tests run only where no GPU is visible")
    if not os.path.exists(T.LIB_PATH):
        pytest.skip("libtri.so not built (run python -m paper_2606_29629_amd.build)")
    return T.lib()


STRUCTS = {"tri_kv8_cache": T.KV8CacheStruct, "tri_rope_config": T.RopeConfig,
           "tri_rope_table": T.RopeTable}


def test_struct_layout_matches_header():
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "tri.h"', "int main(void){"]
    for name, cls in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "probe.c"), os.path.join(d, "probe")
        open(c, "w").write("\n".join(lines + ["return 0;}"]))
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe],
                       check=True)
        got = iter(subprocess.run([exe], capture_output=True, text=True).stdout.split())
    for cls in STRUCTS.values():
        assert int(next(got)) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(next(got)) == getattr(cls, f).offset, f


def cfg(**kw):
    base = dict(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=1024, n_experts=0,
                top_k=0, expert_ffn_dim=0, rms_eps=1e-6, rope_base=1e6, dtype=T.TRI_BF16, flags=0)
    base.update(kw)
    return T.LayerConfig(**base)


def cache(**kw):
    base = dict(k=FAKE, v=FAKE + (1 << 20), k_scale=FAKE + (2 << 20), v_scale=FAKE + (3 << 20),
                mass=FAKE + (4 << 20), stamp=FAKE + (5 << 20), n_slots=2, max_seq=256,
                block_table=None, block_size=0, n_blocks=0, format=0, scale_rows=32)
    base.update(kw)
    return T.KV8CacheStruct(**base)


def paged(**kw):
    base = dict(block_table=FAKE + (6 << 20), block_size=128, n_blocks=4)
    base.update(kw)
    return cache(**base)


def batch(n_seqs=2, n_tokens=5, max_q=4, max_ctx=100, **kw):
    b = T.BatchStruct(n_seqs, n_tokens, max_q, max_ctx, FAKE + (7 << 20), FAKE + (7 << 20) + 64,
                      FAKE + (7 << 20) + 128, FAKE + (7 << 20) + 192)
    for name, v in kw.items():
        setattr(b, name, v)
    return b


def append(lib, c=None, kv=None, b=None, k=FAKE + (8 << 20), v=FAKE + (9 << 20), stride=128):
    return lib.tri_kv8_append(ctypes.byref(c or cfg()), ctypes.byref(kv or cache()),
                              ctypes.byref(b or batch()), k, v, stride, None)


def attend(lib, c=None, kv=None, b=None, q=FAKE + (8 << 20), stride=256, out=FAKE + (9 << 20),
           ws=FAKE + (10 << 20), ws_bytes=1 << 30):
    return lib.tri_kv8_attention(ctypes.byref(c or cfg()), ctypes.byref(kv or cache()),
                                 ctypes.byref(b or batch()), q, stride, out, ws, ws_bytes, None)


def select(lib, c=None, kv=None, b=None, budget=64, first=4, recent=16, plan=FAKE + (8 << 20),
           new_len=FAKE + (9 << 20), ws=FAKE + (10 << 20), ws_bytes=1 << 30):
    return lib.tri_kv8_select(ctypes.byref(c or cfg()), ctypes.byref(kv or cache()),
                              ctypes.byref(b or batch()), budget, first, recent, plan, new_len, ws,
                              ws_bytes, None)


def move(lib, c=None, kv=None, b=None, plan=FAKE + (8 << 20), budget=64):
    return lib.tri_kv8_move(ctypes.byref(c or cfg()), ctypes.byref(kv or cache()),
                            ctypes.byref(b or batch()), plan, budget, None)


def test_every_call_checks_config_cache_and_batch(lib):
    for call in (append, attend, select, move):
        assert call(lib, c=cfg(dtype=T.TRI_F32)) == T.TRI_ERR_UNSUPPORTED
        assert call(lib, c=cfg(head_dim=96)) == T.TRI_ERR_UNSUPPORTED
        assert call(lib, c=cfg(n_kv_heads=0)) == T.TRI_ERR_SHAPE
        assert call(lib, c=cfg(n_kv_heads=70000, n_q_heads=70000)) == T.TRI_ERR_RANGE
        for name in ("k", "v", "k_scale", "v_scale"):
            assert call(lib, kv=cache(**{name: None})) == T.TRI_ERR_NULL, name
        assert call(lib, kv=cache(format=2)) == T.TRI_ERR_UNSUPPORTED
        assert call(lib, kv=cache(scale_rows=48)) == T.TRI_ERR_UNSUPPORTED
        assert call(lib, kv=cache(n_slots=0)) == T.TRI_ERR_SHAPE
        assert call(lib, kv=cache(max_seq=(1 << 23) + 1)) == T.TRI_ERR_RANGE
        assert call(lib, kv=cache(k=FAKE + 8)) == T.TRI_ERR_ALIGN
        assert call(lib, kv=cache(v_scale=FAKE + 2)) == T.TRI_ERR_ALIGN
        assert call(lib, kv=cache(mass=FAKE + 1)) == T.TRI_ERR_ALIGN
        assert call(lib, kv=paged(block_size=96)) == T.TRI_ERR_UNSUPPORTED
        assert call(lib, kv=paged(block_size=192)) == T.TRI_ERR_SHAPE        # does not divide 256
        assert call(lib, kv=paged(block_size=64, scale_rows=128)) == T.TRI_ERR_SHAPE
        assert call(lib, kv=paged(n_blocks=0)) == T.TRI_ERR_SHAPE
        assert call(lib, b=batch(max_ctx=256)) == T.TRI_ERR_RANGE            # no row left
        assert call(lib, b=batch(n_seqs=1, n_tokens=257, max_q=257)) == T.TRI_ERR_RANGE
        assert call(lib, b=batch(n_seqs=65536, n_tokens=65536, max_q=4)) == T.TRI_ERR_RANGE
        assert call(lib, b=batch(n_seqs=-1)) == T.TRI_ERR_SHAPE
        assert call(lib, b=batch(slot=None)) == T.TRI_ERR_NULL
        # a batch without sequences is done before anything else is looked at
        assert call(lib, kv=cache(k=None), b=batch(n_seqs=0, n_tokens=0, max_q=0)) == T.TRI_OK
    for call in (append, attend):  # without tokens likewise
        assert call(lib, b=batch(n_tokens=0, max_q=0, cu_q=None)) == T.TRI_OK


def test_append_refusals(lib):
    assert append(lib, k=None) == T.TRI_ERR_NULL
    assert append(lib, v=FAKE + 8) == T.TRI_ERR_ALIGN
    assert append(lib, stride=120) == T.TRI_ERR_SHAPE
    assert append(lib, stride=132) == T.TRI_ERR_ALIGN
    assert append(lib, b=batch(pos=None)) == T.TRI_ERR_NULL                  # stamps need positions


def test_attention_refusals(lib):
    assert attend(lib, c=cfg(n_q_heads=5)) == T.TRI_ERR_SHAPE
    assert attend(lib, c=cfg(n_q_heads=66)) == T.TRI_ERR_UNSUPPORTED         # group of 33
    assert attend(lib, q=None) == T.TRI_ERR_NULL
    assert attend(lib, q=FAKE + 2) == T.TRI_ERR_ALIGN
    assert attend(lib, stride=252) == T.TRI_ERR_SHAPE
    assert attend(lib, stride=260) == T.TRI_ERR_ALIGN
    assert attend(lib, out=FAKE + (8 << 20) + 512) == T.TRI_ERR_ALIAS
    assert attend(lib, ws=FAKE + (8 << 20)) == T.TRI_ERR_ALIAS
    assert attend(lib, ws=None) == T.TRI_ERR_WORKSPACE
    assert attend(lib, ws_bytes=8) == T.TRI_ERR_WORKSPACE
    assert attend(lib, ws=FAKE + 16) == T.TRI_ERR_ALIGN


def test_layer_refusals(lib):
    w = T.LayerWeights(*[FAKE + (20 << 20) + 4096 * i for i in range(10)])

    def layer(name="prefill", c=None, kv=None, b=None, x=FAKE + (8 << 20), out=FAKE + (9 << 20),
              ws=FAKE + (10 << 20), ws_bytes=1 << 30):
        c = c or cfg(dtype=T.TRI_BF16)
        return getattr(lib, f"tri_layer_{name}_kv8")(
            ctypes.byref(c), ctypes.byref(w), None if kv == 0 else ctypes.byref(kv or cache()),
            ctypes.byref(b or batch()), x, out, None, None, ws, ws_bytes, None)

    one = batch(n_seqs=2, n_tokens=2, max_q=1)
    for name, b in (("prefill", None), ("decode", one)):
        assert layer(name, b=b, kv=0) == T.TRI_ERR_NULL
        assert layer(name, b=b, c=cfg(dtype=T.TRI_F32)) == T.TRI_ERR_UNSUPPORTED
        assert layer(name, b=b, kv=cache(scale_rows=16)) == T.TRI_ERR_UNSUPPORTED
        assert layer(name, b=b, kv=cache(v=FAKE + 4)) == T.TRI_ERR_ALIGN
        assert layer(name, b=b, x=None) == T.TRI_ERR_NULL
        assert layer(name, b=b, ws_bytes=4096) == T.TRI_ERR_WORKSPACE
        assert layer(name, b=b, out=FAKE + (8 << 20)) == T.TRI_ERR_ALIAS
    assert layer(b=batch(max_ctx=256)) == T.TRI_ERR_RANGE
    assert layer("decode", b=batch()) == T.TRI_ERR_SHAPE                     # a chunk
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    size = lib.tri_workspace_size_kv8
    assert size(ctypes.byref(cfg()), ctypes.byref(cache()), ctypes.byref(batch()), None) == T.TRI_ERR_NULL
    assert size(ctypes.byref(cfg()), None, ctypes.byref(batch()), ctypes.byref(n)) == T.TRI_ERR_NULL
    last = 0
    for tokens in (5, 40, 200, 1000):                                       # never shrinks
        b = batch(n_tokens=tokens, max_q=min(tokens, 256) // 2 + 1 if tokens < 500 else 256, n_seqs=8)
        assert size(ctypes.byref(cfg()), ctypes.byref(cache()), ctypes.byref(b), ctypes.byref(n)) == T.TRI_OK
        assert lib.tri_workspace_size(ctypes.byref(cfg()), ctypes.byref(b), ctypes.byref(m)) == T.TRI_OK
        assert n.value > m.value and n.value >= last
        last = n.value


@pytest.mark.parametrize("mass", [False, True])
def test_attention_workspace_never_shrinks(lib, mass):
    """As tokens or the longest prefix grow, other scalars the same."""
    kv = cache(max_seq=1 << 20, **({} if mass else {"mass": None}))
    n = ctypes.c_size_t()

    def size(b):
        assert lib.tri_kv8_attention_workspace_size(ctypes.byref(cfg(n_q_heads=28, n_kv_heads=4, head_dim=128)),
                                                    ctypes.byref(kv), ctypes.byref(b),
                                                    ctypes.byref(n)) == T.TRI_OK
        return n.value

    for seqs, max_q in ((1, 1), (8, 1), (8, 300), (100, 7)):
        tokens = sorted({min(seqs * max_q, max(seqs, max_q) + k) for k in range(0, 2500, 37)})
        sizes = [size(batch(n_seqs=seqs, n_tokens=t, max_q=max_q, max_ctx=5000)) for t in tokens]
        assert sizes == sorted(sizes)
        sizes = [size(batch(n_seqs=seqs, n_tokens=tokens[0], max_q=max_q, max_ctx=c))
                 for c in range(0, 100000, 777)]
        assert sizes == sorted(sizes)


def test_attention_rows_of_heads_within_32_bits(lib):
    c, b = cfg(n_q_heads=64, n_kv_heads=2), batch(n_seqs=60000, n_tokens=60000 * 2000, max_q=2000)
    kv = cache(max_seq=4096)
    assert attend(lib, c=c, kv=kv, b=b) == T.TRI_ERR_RANGE


def test_eviction_refusals(lib):
    assert select(lib, kv=cache(mass=None)) == T.TRI_ERR_NULL
    assert select(lib, plan=None) == T.TRI_ERR_NULL
    for budget in (0, -32, 48):
        assert select(lib, budget=budget) == T.TRI_ERR_SHAPE
        assert move(lib, budget=budget) == T.TRI_ERR_SHAPE
    assert select(lib, budget=288) == T.TRI_ERR_RANGE
    assert move(lib, budget=288) == T.TRI_ERR_RANGE
    assert select(lib, first=-1) == T.TRI_ERR_SHAPE
    assert select(lib, first=40, recent=40) == T.TRI_ERR_SHAPE
    assert select(lib, plan=FAKE + 2) == T.TRI_ERR_ALIGN
    assert move(lib, plan=None) == T.TRI_ERR_NULL
    long = dict(kv=cache(max_seq=1 << 17), b=batch(max_ctx=100000))       # a workspace is needed
    assert select(lib, ws=None, **long) == T.TRI_ERR_WORKSPACE
    assert select(lib, ws_bytes=4096, **long) == T.TRI_ERR_WORKSPACE
    assert select(lib, ws=FAKE + 16, **long) == T.TRI_ERR_ALIGN
    assert select(lib, ws=FAKE + (8 << 20), **long) == T.TRI_ERR_ALIAS    # the plan's own memory
    n = ctypes.c_size_t(1)
    for rows, some in ((16380, False), (16381, True)):                    # and max_q_len 4
        b = batch(max_ctx=rows)
        kv = cache(max_seq=1 << 17)
        assert lib.tri_kv8_select_workspace_size(ctypes.byref(cfg()), ctypes.byref(kv),
                                                 ctypes.byref(b), 64, ctypes.byref(n)) == T.TRI_OK
        assert (n.value > 0) == some


def rope(lib, c=None, x=FAKE, xs=512, y=FAKE + (1 << 20), ys=512, pos=FAKE + (2 << 20), tokens=4,
         heads=4, dtype=0):
    return lib.tri_rope(ctypes.byref(c or T.make_rope(128)), x, xs, y, ys, pos, tokens, heads,
                        dtype, None)


def rope_status(*args, **kw):
    with pytest.raises(T.TriError) as e:
        T.make_rope(*args, **kw)
    return e.value.status


def test_rope_table_refusals(lib):
    assert rope_status(258) == T.TRI_ERR_UNSUPPORTED
    assert rope_status(127) == T.TRI_ERR_UNSUPPORTED
    for r in (0, 1, 63, 130):
        assert rope_status(128, rotary_dim=r) == T.TRI_ERR_SHAPE
    table = T.RopeTable()
    for name, status in (("layout", T.TRI_ERR_UNSUPPORTED), ("scaling", T.TRI_ERR_UNSUPPORTED)):
        c = T.RopeConfig(128, 128, 0, 0, 0, 1e6, 1.0, 1.0, 32.0, 1.0)
        setattr(c, name, 5)
        assert lib.tri_rope_table_make(ctypes.byref(c), ctypes.byref(table)) == status
    assert lib.tri_rope_table_make(None, ctypes.byref(table)) == T.TRI_ERR_NULL
    assert lib.tri_rope_table_make(ctypes.byref(c), None) == T.TRI_ERR_NULL
    assert rope_status(128, base=0.0) == T.TRI_ERR_RANGE
    assert rope_status(128, magnitude=math.inf) == T.TRI_ERR_RANGE
    assert rope_status(128, scaling="linear", factor=0.0) == T.TRI_ERR_RANGE
    for kw in (dict(original_len=0), dict(original_len=4096, low=0.0),
               dict(original_len=4096, low=2.0, high=2.0)):
        for scaling in ("turns", "index"):
            assert rope_status(128, scaling=scaling, **kw) == T.TRI_ERR_RANGE
    assert rope_status(128, scaling="index", base=1.0, original_len=9) == T.TRI_ERR_RANGE
    with pytest.raises(ValueError):
        T.make_rope(128, scaling="cubic")


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=3.0),
                                dict(scaling="base", factor=8.0),
                                dict(scaling="turns", factor=8.0, original_len=8192, high=4.0),
                                dict(scaling="index", factor=40.0, original_len=4096)])
@pytest.mark.parametrize("rotary", [128, 20, 2])
def test_rope_table_is_the_formulas(lib, kw, rotary):
    table = T.make_rope(128, rotary, base=1e4, **kw)
    want = kv8_ref.rope_freqs(rotary, 1e4, **kw) / (2 * math.pi)
    assert np.allclose(table.turns[:rotary // 2], want, rtol=1e-12, atol=0)


def test_rope_refusals(lib):
    assert lib.tri_rope(None, FAKE, 512, FAKE, 512, FAKE, 1, 1, 0, None) == T.TRI_ERR_NULL
    for name, v, status in (("head_dim", 300, T.TRI_ERR_UNSUPPORTED), ("rotary_dim", 0, T.TRI_ERR_SHAPE),
                            ("layout", 2, T.TRI_ERR_UNSUPPORTED), ("magnitude", math.nan, T.TRI_ERR_RANGE)):
        c = T.make_rope(128)
        setattr(c, name, v)
        assert rope(lib, c=c) == status
    assert rope(lib, dtype=2) == T.TRI_ERR_UNSUPPORTED
    assert rope(lib, xs=511) == T.TRI_ERR_SHAPE
    assert rope(lib, tokens=-1) == T.TRI_ERR_SHAPE
    assert rope(lib, x=None) == T.TRI_ERR_NULL
    assert rope(lib, pos=None) == T.TRI_ERR_NULL
    assert rope(lib, x=FAKE + 1) == T.TRI_ERR_ALIGN
    assert rope(lib, y=FAKE + 256) == T.TRI_ERR_ALIAS
    assert rope(lib, y=FAKE, ys=520) == T.TRI_ERR_ALIAS                      # itself, another stride
    assert rope(lib, tokens=0, x=None) == T.TRI_OK


def test_binding_refuses_before_the_call():
    import torch
    c = cfg(n_kv_heads=2, head_dim=64)
    kv = T.KV8Cache.empty(c, 2, 64, device="cpu", mass=True)
    b = T.DeviceBatch([0, 1], [3, 0], [1, 2], device="cpu")
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current GPU"):                     # host tensors
        T.kv8_append(c, kv, b, x, x)
    with pytest.raises(ValueError, match="current GPU"):
        T.layer_prefill(c, {}, kv, b, torch.zeros(3, 256, dtype=torch.bfloat16))
    with pytest.raises(ValueError):                                          # a token too few
        T.kv8_append(c, kv, b, x[:2], x[:2])
    with pytest.raises(ValueError):
        T.kv8_append(c, kv, b, x.float(), x.float())
    with pytest.raises(ValueError):
        T.kv8_append(cfg(n_kv_heads=1), kv, b, x[:, :1], x[:, :1])
    with pytest.raises(ValueError):
        T.kv8_attention(c, kv, b, x)                                         # 2 of 4 query heads
    with pytest.raises(ValueError):
        T.kv8_move(c, kv, b, torch.zeros(1, 2, 32, dtype=torch.int32))
    with pytest.raises(ValueError):
        T.KV8Cache(kv.k, kv.v, kv.k_scale, kv.v_scale[:, :, :1], 32)
    with pytest.raises(ValueError):
        T.KV8Cache(kv.k.float(), kv.v.float(), kv.k_scale, kv.v_scale, 32)
    with pytest.raises(ValueError):
        T.rope(T.make_rope(64), x.half(), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        T.rope(T.make_rope(64), x, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        T.rope(T.make_rope(32), x, torch.zeros(3, dtype=torch.int32))


# ------------------------------------------------- the references themselves --

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_reference_scale_and_numbers(fmt):
    import torch
    top = kv8_ref.TOP[fmt]
    for amax in (top, np.nextafter(top, 1e9), top / 2, 1.0, 3e38, 1e-30, 0.0):
        s = kv8_ref.scale_of(amax, fmt)
        assert amax <= top * s and (s == 2.0 ** -100 or amax > top * s / 2)
    assert math.isnan(kv8_ref.scale_of(math.inf, fmt))
    x = np.concatenate([np.linspace(-top, top, 20001), np.random.default_rng(0).normal(0, 1e-2, 4000)])
    dt = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    t = torch.from_numpy(x)
    want = t.round().to(dt).double() if fmt == "int8" else t.float().to(dt).double()
    assert np.array_equal(kv8_ref.number(x.astype(np.float32).astype(np.float64), fmt), want.numpy())


def test_reference_rope_properties():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(5, 3, 32))
    pos = np.array([0, 1, 77, 100000, -3])
    for inter in (False, True):
        f = kv8_ref.rope_freqs(16, 1e4)
        y = kv8_ref.rope(x, pos, f, inter)
        assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 16:], x[..., 16:])
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        back = kv8_ref.rope(y, -pos, f, inter)
        assert np.allclose(back, x)
    # one layout is the other with its values in another order
    order = np.concatenate([np.arange(0, 32, 2), np.arange(1, 32, 2)])
    f = kv8_ref.rope_freqs(32, 1e4)
    assert np.allclose(kv8_ref.rope(x, pos, f, True)[..., order], kv8_ref.rope(x[..., order], pos, f))
    # the ends of the scaled kinds: fast pairs as they were, slow ones interpolated
    w = kv8_ref.rope_freqs(128, 1e6)
    for kind in ("turns", "index"):
        f = kv8_ref.rope_freqs(128, 1e6, kind, 4.0, original_len=32768)
        assert f[0] == w[0] and np.isclose(f[-1], w[-1] / 4) and (np.diff(f) < 0).all()
