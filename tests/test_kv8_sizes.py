"""Workspaces of the calls over an 8-bit cache, and of the layer's: one sized for the largest batch serves every
smaller one.  Host only: no call here reads a device address."""
import ctypes

import pytest

from paper_2606_29629_amd import _lib as T
from test_kv8_abi import batch, cache, cfg, lib  # noqa: F401  (lib: the fixture)

LAYERS = [dict(n_q_heads=28, n_kv_heads=4, head_dim=128), dict(n_q_heads=32, n_kv_heads=1, head_dim=128),
          dict(n_q_heads=14, n_kv_heads=2, head_dim=64), dict(n_q_heads=3, n_kv_heads=3, head_dim=64),
          dict(n_q_heads=512, n_kv_heads=512, head_dim=64)]


def attention_size(lib, c, kv, b):
    n = ctypes.c_size_t()
    assert lib.tri_kv8_attention_workspace_size(ctypes.byref(c), ctypes.byref(kv), ctypes.byref(b),
                                                ctypes.byref(n)) == T.TRI_OK
    return n.value


def layer_size(lib, c, kv, b):
    n = ctypes.c_size_t()
    assert lib.tri_workspace_size_kv8(ctypes.byref(c), ctypes.byref(kv), ctypes.byref(b),
                                      ctypes.byref(n)) == T.TRI_OK
    return n.value


def bf16_layer_size(lib, c, kv, b):
    n = ctypes.c_size_t()
    assert lib.tri_workspace_size(ctypes.byref(c), ctypes.byref(b), ctypes.byref(n)) == T.TRI_OK
    return n.value


def select_size(lib, c, kv, b):
    n = ctypes.c_size_t()
    assert lib.tri_kv8_select_workspace_size(ctypes.byref(c), ctypes.byref(kv), ctypes.byref(b), 4096,
                                             ctypes.byref(n)) == T.TRI_OK
    return n.value


@pytest.mark.parametrize("size", [attention_size, layer_size, bf16_layer_size, select_size])
@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("layer", LAYERS, ids=lambda kw: "%d-%d-%d" % tuple(kw.values()))
def test_never_shrinks(lib, layer, mass, size):  # noqa: F811
    """As sequences are added: steps of one token each, chunks beside them, idle ones."""
    c, kv = cfg(**layer), cache(max_seq=1 << 20, **({} if mass else {"mass": None}))
    for ctx in (0, 127, 1000, 4095, 70000):
        for b in (lambda n: batch(n, n, 1, ctx), lambda n: batch(n, n + 299, 300, ctx),
                  lambda n: batch(n, 77, 77, ctx), lambda n: batch(n, 4 * n, 4, ctx)):
            sizes = [size(lib, c, kv, b(n)) for n in range(1, 600)]
            assert sizes == sorted(sizes)
    for n in (1, 13, 300):  # and as the longest chunk does
        sizes = [size(lib, c, kv, batch(n, 900, q, 3000)) for q in range(900 // n + 1, 901, 7)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("layer", LAYERS, ids=lambda kw: "%d-%d-%d" % tuple(kw.values()))
def test_layer_never_shrinks_as_tokens_are_added(lib, layer):  # noqa: F811
    c, kv = cfg(**layer), cache(max_seq=1 << 20)
    for n_seqs, q in ((1, 2000), (8, 500), (100, 40), (300, 300)):
        for ctx in (0, 4095, 70000):
            for size in (layer_size, bf16_layer_size):
                sizes = [size(lib, c, kv, batch(n_seqs, t, q, ctx))
                         for t in range(max(n_seqs, q), min(n_seqs * q, 3000))]
                assert sizes == sorted(sizes)


def test_layer_checks_the_batch_as_its_attention_does(lib):  # noqa: F811
    """Host scalars that the attention refuses are refused by the layer's size and calls."""
    n = ctypes.c_size_t(77)
    w = T.LayerWeights(*[0x7F0000000000 + (20 << 20) + 4096 * i for i in range(10)])
    one, many = cfg(), cfg(n_q_heads=64, n_kv_heads=2)
    for c, kv, b in ((one, cache(), batch(max_ctx=256)), (one, cache(), batch(max_ctx=1 << 30)),
                     (one, cache(), batch(max_ctx=(1 << 31) - 1)),
                     (one, cache(), batch(n_seqs=1, n_tokens=257, max_q=257)),
                     (one, cache(), batch(n_seqs=65536, n_tokens=65536, max_q=4)),
                     (cfg(n_q_heads=65540, n_kv_heads=65540, head_dim=64), cache(), batch()),
                     (many, cache(max_seq=4096), batch(n_seqs=60000, n_tokens=60000 * 2000, max_q=2000)),
                     (cfg(n_q_heads=1, n_kv_heads=1), cache(max_seq=1 << 23),
                      batch(n_seqs=256, n_tokens=(1 << 31) - 1, max_q=1 << 23))):
        args = [ctypes.byref(a) for a in (c, kv, b)]
        assert lib.tri_workspace_size_kv8(*args, ctypes.byref(n)) == T.TRI_ERR_RANGE and n.value == 77
        assert lib.tri_kv8_attention_workspace_size(*args, ctypes.byref(n)) == T.TRI_ERR_RANGE
        x = [0x7F0000000000 + (k << 40) for k in (1, 2, 3)]
        assert lib.tri_layer_prefill_kv8(args[0], ctypes.byref(w), *args[1:], x[0], x[1], None, None, x[2],
                                         (1 << 64) - 1, None) == T.TRI_ERR_RANGE
    b = batch(n_tokens=0, max_q=0, max_ctx=256)         # a full cache, nothing new
    assert lib.tri_workspace_size_kv8(*[ctypes.byref(a) for a in (one, cache(), b)], ctypes.byref(n)) == T.TRI_OK
