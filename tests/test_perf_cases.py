"""The cases of perf/operators.py, listed and drawn, are calls that the entry points accept:
their host checks on each case's sizes (fake device addresses, nothing is launched)."""
import ctypes
import random

import perf.operators as po
from paper_2606_29629_amd import _lib as T
from test_kv8_abi import FAKE, lib  # noqa: F401  (lib: the fixture)


def check(lib, c):  # noqa: F811
    L = po.LAYERS[c["layer"]]
    if c["op"] == "rope":
        T.make_rope(L["d"], rotary_dim=c["rotary"], base=po.BASE, interleaved=c["interleaved"],
                    scaling=c["scaling"], factor=c["factor"], low=1.0, high=32.0,
                    original_len=c["original"])
        return
    seqs = po._seqs(c)
    n, max_seq = len(seqs), po._max_seq(c, seqs)
    cfg = T.LayerConfig(hidden=64, n_q_heads=L["hq"], n_kv_heads=L["hkv"], head_dim=L["d"])
    kv = T.KV8CacheStruct(*[FAKE + (k << 30) for k in range(6)], n, max_seq, FAKE if c["paged"] else None,
                          po.BLOCK, n * max_seq // po.BLOCK + 3, 0, c["scale_rows"])
    batch = T.BatchStruct(n, sum(q for q, _ in seqs), max(q for q, _ in seqs), max(k for _, k in seqs),
                          *[FAKE + (k << 20) for k in range(4)])
    size, args = ctypes.c_size_t(), [ctypes.byref(a) for a in (cfg, kv, batch)]
    assert lib.tri_kv8_attention_workspace_size(*args, ctypes.byref(size)) == T.TRI_OK, c
    if c["op"] == "evict":
        assert lib.tri_kv8_select_workspace_size(*args, c["budget"], ctypes.byref(size)) == T.TRI_OK, c
        assert c["first"] + c["recent"] <= c["budget"], c


def test_listed_and_drawn_cases_are_accepted(lib):  # noqa: F811
    for c in po.listed() + [po.draw(random.Random(seed)) for seed in range(3000)]:
        check(lib, c)
