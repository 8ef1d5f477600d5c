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
