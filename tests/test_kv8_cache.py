"""The KV8Cache object on the host: the calls see the tensors that it names now."""
import copy

import pytest
import torch

from paper_2606_29629_amd import _lib as T

TENSORS = ("k", "v", "k_scale", "v_scale", "mass", "stamp")


class Shape:
    n_kv_heads, head_dim = 2, 64


def make(paged=False, **kw):
    kw = dict(dict(mass=True, stamp=True), **kw)
    if paged:
        table = torch.arange(4, dtype=torch.int32).view(2, 2)
        return T.KV8Cache.empty(Shape, 2, 256, block_table=table, block_size=128, n_blocks=5, device="cpu", **kw)
    return T.KV8Cache.empty(Shape, 2, 64, device="cpu", **kw)


def addresses(cache):
    s = cache.struct()
    return {n: getattr(s, n) for n in TENSORS + ("block_table",)}


def named(cache):
    return {n: None if getattr(cache, n) is None else getattr(cache, n).data_ptr()
            for n in TENSORS + ("block_table",)}


@pytest.mark.parametrize("paged", [False, True])
def test_a_replaced_tensor_is_the_one_the_calls_get(paged):
    cache = make(paged)
    assert addresses(cache) == named(cache)
    for name in TENSORS + (("block_table",) if paged else ()):
        before = getattr(cache, name)
        setattr(cache, name, before.clone())
        assert getattr(cache, name).data_ptr() != before.data_ptr()
        assert addresses(cache) == named(cache), name
    cache.mass = cache.mass * 0.5
    assert addresses(cache) == named(cache)
    cache.mass = None                                   # as shared pages require
    cache.stamp = None
    assert cache.struct().mass is None and cache.struct().stamp is None
    cache.mass = torch.zeros(cache.k.shape[:3])
    assert addresses(cache) == named(cache)


def test_what_may_not_replace_a_tensor():
    cache = make()
    before, kept = addresses(cache), {n: getattr(cache, n) for n in TENSORS}
    for name, t in (("mass", cache.mass.double()), ("mass", cache.mass[:1]), ("stamp", cache.mass),
                    ("mass", torch.zeros(2, 64, 2).transpose(1, 2)), ("k", None), ("v_scale", None),
                    ("k", cache.k.view(torch.uint8)), ("v", cache.v[..., :32]),
                    ("k_scale", torch.ones(2, 2, 3)), ("mass", cache.mass.to("meta")),
                    ("block_table", torch.zeros(2, 1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            setattr(cache, name, t)
    with pytest.raises(ValueError):
        make(True).block_table = None
    for name in ("max_seq", "n_slots", "scale_rows", "n_kv_heads", "head_dim", "other"):
        with pytest.raises(AttributeError):
            setattr(cache, name, 1)
    with pytest.raises(AttributeError):
        del cache.mass
    assert addresses(cache) == before and all(getattr(cache, n) is t for n, t in kept.items())


def test_a_copy_has_its_own_tensors_and_struct():
    for paged in (False, True):
        cache = make(paged)
        shallow, deep = copy.copy(cache), copy.deepcopy(cache)
        shallow.mass = None
        assert addresses(cache) == named(cache) and cache.mass is not None
        assert shallow.k is cache.k and deep.k.data_ptr() != cache.k.data_ptr()
        for c in (shallow, deep):
            assert addresses(c) == named(c) and c.max_seq == cache.max_seq and c.n_slots == cache.n_slots


def test_max_seq_of_a_contiguous_cache_is_its_rows():
    c = make()
    args = c.k, c.v, c.k_scale, c.v_scale, 32
    for n in (32, 63, 65, 0):
        with pytest.raises(ValueError, match="max_seq"):
            T.KV8Cache(*args, max_seq=n)
    assert T.KV8Cache(*args, max_seq=64).max_seq == T.KV8Cache(*args).max_seq == 64


def test_one_token_of_rows_of_any_stride(monkeypatch):
    """Strides that no token follows are not looked at: a key beside a value of other rows, rows
    of an odd width."""
    import types
    table, asked = T.make_rope(64), []
    call = lambda *a: asked.append(a) or 0
    monkeypatch.setattr(T, "lib", lambda: types.SimpleNamespace(tri_kv8_append=call, tri_kv8_attention=call, tri_rope=call))
    monkeypatch.setattr(T, "_on_gpu", lambda what, stream, *tensors: 0)
    monkeypatch.setattr(T, "kv8_attention_workspace_size", lambda *a: 256)
    cache, b = make(), T.DeviceBatch([1], [5], [1], device="cpu")
    cfg = T.LayerConfig(n_q_heads=4, n_kv_heads=2, head_dim=64)
    row = torch.zeros(1, 1003, dtype=torch.bfloat16)
    heads = lambda first, n: row.as_strided((1, n, 64), (1003, 64, 1), first)
    k = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    T.kv8_append(cfg, cache, b, k, heads(128, 2))
    T.kv8_attention(cfg, cache, b, heads(0, 4))
    T.rope(table, heads(0, 4), torch.zeros(1, dtype=torch.int32), out=torch.zeros(1, 4, 64, dtype=torch.bfloat16))
    assert asked[0][5] == 128 and asked[1][4] == 256 and asked[2][2] == asked[2][4] == 256
    b2, k2 = T.DeviceBatch([1], [5], [2], device="cpu"), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="one token stride"):
        T.kv8_append(cfg, cache, b2, k2, torch.zeros(2, 4, 64, dtype=torch.bfloat16)[:, :2])
