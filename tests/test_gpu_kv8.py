"""The 8-bit KV cache on the GPU: append, attention, weights and eviction against their
definitions in float64 (tests/kv8_ref.py, which derives the bounds).  Codes, scales,
plans and stamps are compared for equality."""
import numpy as np
import pytest

import kv8_ref
from paper_2606_29629_amd import _lib as T

pytestmark = pytest.mark.gpu


class Shape:
    rms_eps, rope_base, hidden = 1e-6, 1e6, 64

    def __init__(self, hq, hkv, d):
        self.n_q_heads, self.n_kv_heads, self.head_dim = hq, hkv, d


def config(hq, hkv, d):
    return T.make_config(Shape(hq, hkv, d))


def make_cache(cfg, slots, max_seq, fmt="int8", R=32, page=0, seed=0, mass=True, stamp=True,
               junk=True, wide=2.0):
    """A cache full of random codes and scales (rows past a sequence's end are junk that
    nothing may read into a result), pages in a shuffled order with one to spare."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    table, panels, rows = None, slots, max_seq
    if page:
        per = max_seq // page
        panels, rows = slots * per + 1, page
        perm = torch.randperm(panels, generator=torch.Generator().manual_seed(seed))
        table = perm[:slots * per].reshape(slots, per).to(torch.int32).cuda()
    heads, d = cfg.n_kv_heads, cfg.head_dim
    codes, scales = [], []
    for _ in range(2):
        x = torch.randn(panels, heads, rows, d, generator=g, device="cuda")
        if fmt == "int8":
            codes.append((x * 40).round().clamp(-127, 127).to(torch.int8))
        else:
            codes.append((x * 100).clamp(-448, 448).to(torch.float8_e4m3fn))
        e = torch.randn(panels, heads, -(-rows // R), generator=g, device="cuda") * wide
        scales.append(torch.exp2(e.round() - (5 if fmt == "int8" else 7)))
    kw = {}
    if mass:
        kw["mass"] = torch.rand(panels, heads, rows, generator=g, device="cuda") ** 3
    if stamp:
        kw["stamp"] = torch.randint(0, 1 << 20, (panels, heads, rows), generator=g, device="cuda",
                                    dtype=torch.int32)
    return T.KV8Cache(*codes, *scales, R, block_table=table, max_seq=max_seq if page else None, **kw)


def bits(cache):
    import torch
    names = ("k", "v", "k_scale", "v_scale", "mass", "stamp")
    return {n: getattr(cache, n).view(torch.uint8).clone() for n in names
            if getattr(cache, n) is not None}


def same_cache(cache, ref, mtol=None):
    """The cache's logical rows equal the reference's (NaN equal to NaN)."""
    got = kv8_ref.Cache(cache)
    for name in ("k", "v", "ks", "vs", "stamp"):
        a, b = getattr(got, name), getattr(ref, name)
        if a is not None:
            assert np.array_equal(a, b, equal_nan=name in ("ks", "vs")), name
    if got.mass is not None:
        tol = 0 if mtol is None else mtol
        assert (np.abs(got.mass - ref.mass) <= tol).all()


def bf16(*shape, seed, spread=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(*shape, generator=g, device="cuda")
    return (x * torch.exp2(spread * torch.randn(shape[0], 1, 1, generator=g, device="cuda"))).bfloat16()


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


FORMATS = ["int8", "e4m3"]
# slot, cached rows, new tokens
BATCHES = {
    "one": ([0], [0], [1]),
    "steps": ([2, 0, 1], [5, 100, 255], [1, 1, 1]),
    "chunks": ([1, 0, 2], [0, 31, 64], [70, 33, 128]),
    "mixed": ([3, 0, 1, 2], [200, 0, 33, 190], [1, 130, 0, 66]),
}
MAX_SEQ = 256


def run_append(cfg, cache, batch, seed, spread=1.0):
    db = T.DeviceBatch(*batch)
    k = bf16(db.n_tokens, cfg.n_kv_heads, cfg.head_dim, seed=seed, spread=spread)
    v = bf16(db.n_tokens, cfg.n_kv_heads, cfg.head_dim, seed=seed + 1, spread=spread)
    ref = kv8_ref.Cache(cache)
    T.kv8_append(cfg, cache, db, k, v)
    ref.append(db.host, f64(k), f64(v), db.pos.cpu().numpy())
    return db, ref


@pytest.mark.parametrize("name", sorted(BATCHES))
@pytest.mark.parametrize("page", [0, 128])
@pytest.mark.parametrize("R", [32, 64, 128])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_append(d, fmt, R, page, name):
    cfg = config(4, 2, d)
    cache = make_cache(cfg, 4, MAX_SEQ, fmt, R, page, seed=R + d)
    before = bits(cache)
    for c in range(3):  # growing values: the held codes are rounded to a larger scale
        _, ref = run_append(cfg, cache, BATCHES[name], seed=7 + c, spread=3.0 + 2 * c)
        same_cache(cache, ref)
    if page:  # the page of no sequence
        spare = sorted(set(range(cache.k.shape[0])) - set(cache.block_table.flatten().tolist()))
        for n, t in bits(cache).items():
            assert (t[spare] == before[n][spare]).all(), n


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_token_by_token_stays_within_a_step(fmt):
    """What the header promises of a value appended early: all its roundings together
    are under one step of the final scale."""
    cfg = config(1, 1, 64)
    cache = T.KV8Cache.empty(cfg, 1, 128, fmt, stamp=True)
    new = bf16(128, 1, 64, seed=3, spread=0.0)
    import torch
    grow = torch.exp2((torch.arange(128) % 32) / 3.0).cuda()[:, None, None]
    new = (new.float() * grow).bfloat16()
    for t in range(128):
        T.kv8_append(cfg, cache, T.DeviceBatch([0], [t], [1], pos=[t + 9]), new[t:t + 1], new[t:t + 1])
    ref = kv8_ref.Cache(cache)
    x = f64(new)[:, 0]
    got, s = ref.values("k", 0, 128)[0], np.repeat(ref.ks[0, 0], 32)[:, None]
    step = s if fmt == "int8" else s * np.exp2(np.floor(np.log2(np.maximum(np.abs(x / s), 2.0 ** -6))) - 3)
    assert (np.abs(got - x) < step).all()
    assert np.array_equal(ref.stamp[0, 0], np.arange(128) + 9)
    assert np.array_equal(got, ref.values("v", 0, 128)[0])


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_extremes(fmt):
    """The largest and smallest bf16 numbers, zeros, infinity and NaN."""
    import torch
    cfg = config(2, 2, 64)
    cache = T.KV8Cache.empty(cfg, 6, 64, fmt)
    x = torch.zeros(6, 2, 64, device="cuda")
    top = torch.finfo(torch.bfloat16).max
    x[0] = top
    x[1] = 1e-38
    x[2, :, 3] = -2.0 ** -94
    x[3, 0, 5] = float("inf")
    x[4, 1, 6] = float("nan")
    db = T.DeviceBatch(range(6), [0] * 6, [1] * 6)
    ref = kv8_ref.Cache(cache)
    T.kv8_append(cfg, cache, db, x.bfloat16(), x.bfloat16())
    ref.append(db.host, f64(x.bfloat16()), f64(x.bfloat16()), np.zeros(6))
    same_cache(cache, ref)
    assert np.isnan(kv8_ref.Cache(cache).ks[3, 0, 0]) and kv8_ref.Cache(cache).ks[3, 1, 0] > 0
    # a poisoned block stays so until it is begun anew
    one = torch.ones(6, 2, 64, device="cuda").bfloat16()
    for ctx, nan in ((1, True), (0, False)):
        T.kv8_append(cfg, cache, T.DeviceBatch(range(6), [ctx] * 6, [1] * 6), one, one)
        ks = kv8_ref.Cache(cache).ks
        assert np.isnan(ks[3, 0, 0]) == nan and np.isnan(ks[4, 1, 0]) == nan


def test_append_strided_rows_and_skipped_sequences():
    import torch
    cfg = config(4, 2, 64)
    cache = make_cache(cfg, 3, 128, seed=4)
    db = T.DeviceBatch([0, 7, 2, -1], [10, 0, 126, 3], [3, 2, 3, 1])   # bad slot, past the end
    db.max_ctx_len = 100
    rows = torch.randn(db.n_tokens, 8, 64, device="cuda").bfloat16()
    ref = kv8_ref.Cache(cache)
    T.kv8_append(cfg, cache, db, rows[:, 4:6], rows[:, 6:8])
    ref.append(db.host, f64(rows[:, 4:6]), f64(rows[:, 6:8]), db.pos.cpu().numpy())
    same_cache(cache, ref)


# ---------------------------------------------------------------- attention --

ATTEND = {
    "one": ([0], [0], [1]),
    "steps": ([2, 0, 1, 3], [5, 100, 255, 31], [1, 1, 1, 1]),
    "long": ([1, 0], [1999, 700], [1, 1]),
    "chunks": ([1, 0, 2], [0, 31, 64], [70, 33, 128]),
    "far chunk": ([0, 1], [1500, 3], [150, 2]),
    "mixed": ([3, 0, 1, 2], [600, 0, 33, 190], [1, 130, 0, 66]),
    "farther chunk": ([1, 0], [4500, 4300], [19, 1]),
    "many": (list(range(24)), [37 * i % 300 for i in range(24)], [1 + (i % 5) * (i % 2) for i in range(24)]),
}


def run_attention(cfg, cache, batch, seed=11, spread=0.5):
    db = T.DeviceBatch(*batch)
    q = bf16(db.n_tokens, cfg.n_q_heads, cfg.head_dim, seed=seed, spread=spread)
    ref = kv8_ref.Cache(cache)
    out, tol, mass, mtol = ref.attention(db.host, f64(q))
    got, _ = T.kv8_attention(cfg, cache, db, q)
    live = ~np.isnan(out).all((1, 2))
    err = np.abs(f64(got) - out)
    assert (err[live] <= tol[live]).all(), float((err - tol)[live].max())
    ref.mass = mass
    same_cache(cache, ref, mtol)   # and nothing but the mass has changed
    return db, q, got


def attend_cache(cfg, batch, fmt, R=32, page=0, mass=True, seed=5):
    need = max(c + n for c, n in zip(batch[1], batch[2]))
    max_seq = -(-need // 128) * 128
    return make_cache(cfg, max(batch[0]) + 1, max_seq, fmt, R, page, seed=seed, mass=mass)


@pytest.mark.parametrize("name", sorted(ATTEND))
@pytest.mark.parametrize("page", [0, 128])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (7, 1, 128)])
def test_attention(hq, hkv, d, fmt, page, name):
    cfg = config(hq, hkv, d)
    run_attention(cfg, attend_cache(cfg, ATTEND[name], fmt, 64 if page else 32, page), ATTEND[name])


@pytest.mark.parametrize("name", ["steps", "mixed"])
@pytest.mark.parametrize("hq,hkv,d", [(3, 3, 64), (32, 1, 128), (17, 1, 64), (28, 4, 128), (32, 2, 64)])
def test_attention_head_groups(hq, hkv, d, name):
    cfg = config(hq, hkv, d)
    for fmt in FORMATS:
        run_attention(cfg, attend_cache(cfg, ATTEND[name], fmt, 128), ATTEND[name])


@pytest.mark.parametrize("name", ["long", "far chunk"])
def test_attention_without_mass_is_the_same(name):
    import torch
    cfg = config(8, 2, 128)
    cache = attend_cache(cfg, ATTEND[name], "e4m3")
    plain = T.KV8Cache(cache.k, cache.v, cache.k_scale, cache.v_scale, 32)
    db, q, got = run_attention(cfg, cache, ATTEND[name])
    again, _ = T.kv8_attention(cfg, plain, db, q)
    assert torch.equal(got, again)


def test_attention_sharp_scores_and_wide_scales():
    """Scores in the hundreds (weights of one row or two) and value scales 2^40 apart."""
    import torch
    cfg = config(4, 1, 64)
    for name in ("long", "far chunk"):
        cache = attend_cache(cfg, ATTEND[name], "int8", mass=True)
        cache.v_scale.copy_(torch.exp2((torch.randn_like(cache.v_scale) * 20).round().clamp(-60, 60)))
        run_attention(cfg, cache, ATTEND[name], spread=3.0)


def test_attention_smallest_and_largest_scales():
    import torch
    cfg = config(2, 1, 64)
    for e in (-100, 100):
        cache = attend_cache(cfg, ATTEND["mixed"], "e4m3")
        cache.v_scale.fill_(2.0 ** e)
        run_attention(cfg, cache, ATTEND["mixed"])
    cache.k_scale.fill_(2.0 ** -100)   # all scores nearly 0: the mean
    run_attention(cfg, cache, ATTEND["mixed"])
    cache.k_scale.fill_(1.0)
    db = T.DeviceBatch(*ATTEND["mixed"])
    out, _ = T.kv8_attention(cfg, cache, db, torch.zeros(db.n_tokens, 2, 64, device="cuda").bfloat16())
    assert torch.isfinite(out).all()


def test_attention_poison_reaches_its_head_and_sequence_alone():
    """A NaN scale among the visible rows gives NaN there; junk, NaN scales included, in rows
    past the end reaches nothing."""
    import torch
    cfg = config(4, 2, 64)
    for batch in (([0, 1], [100, 60], [1, 1]), ([0, 1], [100, 60], [3, 40])):
        cache = make_cache(cfg, 2, 256, seed=8)
        db = T.DeviceBatch(*batch)
        q = bf16(db.n_tokens, 4, 64, seed=2)
        ref, _ = T.kv8_attention(cfg, cache, db, q)
        for t in (cache.k_scale, cache.v_scale):
            t[:, :, 4:] = float("nan")      # rows from 128 on: past both ends
        out, _ = T.kv8_attention(cfg, cache, db, q)
        assert torch.equal(out, ref)
        for t in (cache.k_scale, cache.v_scale):
            kept = t.clone()
            t[0, 1, 1] = float("nan")       # sequence 0, KV head 1
            out, _ = T.kv8_attention(cfg, cache, db, q)
            n0 = batch[2][0]
            assert torch.isnan(out[:n0, 2:]).all()
            assert torch.equal(out[:n0, :2], ref[:n0, :2]) and torch.equal(out[n0:], ref[n0:])
            t.copy_(kept)


def test_attention_skipped_sequences_and_strided_q():
    """Bad slots and pages outside the pool: those tokens and all other memory stay."""
    import torch
    cfg = config(4, 2, 64)
    cache = make_cache(cfg, 3, 256, seed=6, page=64)
    db = T.DeviceBatch([1, 9, 0, -2], [40, 3, 70, 0], [1, 1, 20, 5])
    rows = torch.randn(db.n_tokens, 8, 64, device="cuda").bfloat16()
    out = torch.full((db.n_tokens, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ref = kv8_ref.Cache(cache)
    want, tol, mass, mtol = ref.attention(db.host, f64(rows[:, :4]))
    T.kv8_attention(cfg, cache, db, rows[:, :4], out=out)
    live = ~np.isnan(want).all((1, 2))
    assert (np.abs(f64(out) - want)[live] <= tol[live]).all() and live.sum() == 21
    assert (out[torch.from_numpy(~live).cuda()] == 7).all()
    ref.mass = mass
    same_cache(cache, ref, mtol)
    # a page of the visible rows outside the pool: unspecified results, nothing touched
    cache.block_table[1, 0] = 1000
    cache.block_table[0, 1] = -5
    before = bits(cache)
    T.kv8_attention(cfg, cache, db, rows[:, :4], out=out)
    k = rows[:, 4:6]
    T.kv8_append(cfg, cache, db, k, k)
    torch.cuda.synchronize()
    after = bits(cache)
    used = [int(p) for p in cache.block_table.flatten().tolist() if 0 <= p < cache.k.shape[0]]
    for p in range(cache.k.shape[0]):
        if p not in used:
            assert all((after[n][p] == before[n][p]).all() for n in before)


@pytest.mark.parametrize("R", [32, 128])
@pytest.mark.parametrize("max_seq", [1, 45, 77, 100])
def test_odd_cache_lengths(max_seq, R):
    """A contiguous cache that ends within a tile and a scale block, filled to its last row."""
    cfg = config(4, 2, 64)
    for fmt in FORMATS:
        cache = make_cache(cfg, 3, max_seq, fmt, R, seed=max_seq)
        batch = ([1, 0, 2], [max_seq - 1, 0, max_seq // 2], [1, max_seq, max_seq - max_seq // 2])
        _, ref = run_append(cfg, cache, batch, seed=5)
        same_cache(cache, ref)
        run_attention(cfg, cache, batch)


def test_rows_behind_the_last_sequence():
    """Tokens that belong to no sequence: their outputs stay, nothing of them is appended."""
    import torch
    cfg = config(4, 2, 64)
    for q, pad in (([1, 1], 5), ([40, 1], 5), ([3, 70], 5), ([1, 3], 2), ([70, 1], 69), ([1, 1], 2)):
        cache = make_cache(cfg, 2, 256, seed=3)
        db = T.DeviceBatch([1, 0], [30, 100], q)
        n, db.n_tokens = db.n_tokens, db.n_tokens + pad
        db.max_q_len = max(db.max_q_len, -(-db.n_tokens // 2))
        db.pos = torch.arange(db.n_tokens, dtype=torch.int32, device="cuda")
        k = bf16(db.n_tokens, 2, 64, seed=1)
        k[n:] = 1e30
        ref = kv8_ref.Cache(cache)
        T.kv8_append(cfg, cache, db, k, k)
        ref.append(db.host, f64(k), f64(k), np.arange(db.n_tokens))
        same_cache(cache, ref)
        x = bf16(db.n_tokens, 4, 64, seed=2)
        out = torch.full_like(x, 5.0)
        want, tol, mass, mtol = ref.attention(db.host, f64(x))
        T.kv8_attention(cfg, cache, db, x, out=out)
        assert (np.abs(f64(out)[:n] - want[:n]) <= tol[:n]).all() and (out[n:] == 5).all()
        ref.mass = mass
        same_cache(cache, ref, mtol)


def test_value_scales_far_apart():
    """A block of zeros (scale 2^-100) beside values of up to 2^8: their rows count in full."""
    cfg = config(4, 2, 64)
    for batch in (([0, 1], [99, 64], [1, 1]), ([0, 1], [99, 64], [3, 40])):
        cache = make_cache(cfg, 2, 256, seed=3)
        cache.v[:, :, :64] = 0
        cache.v_scale[:, :, :2] = 2.0 ** -100
        cache.v_scale[:, :, 2:] = 2.0
        cache.k_scale.fill_(2.0 ** -9)
        run_attention(cfg, cache, batch)


@pytest.mark.parametrize("q", [[1, 1], [90, 1], [2, 64]])
def test_cache_past_32_bits(q):
    """The last slots of a cache whose codes pass 4 GiB, against a cache of those slots alone."""
    import torch
    cfg = config(16, 8, 128)
    slots, max_seq = 34, 131072
    big = T.KV8Cache.empty(cfg, slots, max_seq, "e4m3", 64, mass=True, stamp=True)
    small = make_cache(cfg, 2, 2048, "e4m3", 64, seed=4)
    assert big.k.numel() > 1 << 32
    for name in ("k", "v", "mass", "stamp"):
        a, b = getattr(big, name), getattr(small, name)
        a.view(torch.uint8)[-2:, :, :2048] = b.view(torch.uint8) if a.dim() == 4 else 0
        if a.dim() == 3:
            a[-2:, :, :2048] = b
    for name in ("k_scale", "v_scale"):
        getattr(big, name)[-2:, :, :32] = getattr(small, name)
    outs = []
    for cache, off in ((big, slots - 2), (small, 0)):
        db = T.DeviceBatch([off + 1, off], [1900, 700], q)
        x = bf16(db.n_tokens, 16, 128, seed=2)
        k = bf16(db.n_tokens, 8, 128, seed=3)
        T.kv8_append(cfg, cache, db, k, k)
        out, _ = T.kv8_attention(cfg, cache, db, x)
        plan, _ = T.kv8_select(cfg, cache, db, 512, 4, 64)
        T.kv8_move(cfg, cache, db, plan)
        outs.append((out, plan))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    for name in ("k", "v", "mass", "stamp", "k_scale", "v_scale"):
        a, b = getattr(big, name), getattr(small, name)
        assert torch.equal(a[-2:, :, :b.shape[2]].view(torch.uint8), b.view(torch.uint8)), name


@pytest.mark.parametrize("rows,chunks", [(9000, 20), (5140, 1), (2540, 1)])
def test_many_sequences_with_few_chunks(rows, chunks):
    """More pieces of weight sums than the workgroups that go through them (the groups of 128
    and of 64 rows), all of the sequences' or one chunk's alone."""
    cfg = config(4, 2, 64)
    n = 40
    q = [(60 if chunks == 1 else 2 + i % 3) if i % (n // chunks) == 1 else 1 for i in range(n)]
    ctx = [rows - 7 * i if q[i] > 1 else 30 * i for i in range(n)]
    cache = make_cache(cfg, n, rows + 80, "int8", 64, seed=6)
    run_attention(cfg, cache, (list(range(n))[::-1], ctx, q))


def test_memory_of_the_callers_stream():
    """A workspace that the call allocates and drops comes from its own stream's memory: what
    the current stream allocates right after does not reach into it."""
    import torch
    cfg = config(4, 2, 64)
    n = 200000
    cache = make_cache(cfg, 1, n + 64, "int8", 64, seed=1)
    db = T.DeviceBatch([0], [n - 1], [1])
    want = T.kv8_select(cfg, cache, db, 64 * 1024, 4, 64)
    stream = torch.cuda.Stream()
    for given in (stream, stream.cuda_stream):
        torch.cuda.synchronize()
        got = T.kv8_select(cfg, cache, db, 64 * 1024, 4, 64, stream=given)
        junk = [torch.full((size,), 77, dtype=torch.uint8, device="cuda")
                for size in (T.kv8_select_workspace_size(cfg, cache, db, 64 * 1024),) * 8]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), junk[0]


def test_mixed_batch_on_the_side_stream():
    """A batch whose single tokens may read 192 MiB runs them beside the chunk: the same
    results as the sequences alone, in a graph too, and from two streams at once."""
    import torch
    cfg = config(4, 2, 64)
    max_seq = 300032
    cache = make_cache(cfg, 3, max_seq, "int8", 64, seed=1, stamp=False)
    db = T.DeviceBatch([2, 0, 1], [5000, 200, 3000], [1, 80, 1])
    db.max_ctx_len = 300000                      # a bound: the largest that may come
    assert db.n_seqs * db.max_ctx_len * 2 * 64 * 2 >= 192 << 20
    x = bf16(db.n_tokens, 4, 64, seed=2)
    start, parts, t = cache.mass.clone(), [], 0
    for s, c, n in zip([2, 0, 1], [5000, 200, 3000], [1, 80, 1]):
        parts.append(T.kv8_attention(cfg, cache, T.DeviceBatch([s], [c], [n]), x[t:t + n])[0])
        t += n
    alone, mass = torch.cat(parts), cache.mass.clone()
    close = lambda a, b: (a.float() - b.float()).abs().max() <= 2.0 ** -7 * b.float().abs().max()

    def check(out, m):
        assert close(out, alone) and close(m, mass)

    streams = [torch.cuda.Stream() for _ in range(2)]
    caches = [T.KV8Cache(cache.k, cache.v, cache.k_scale, cache.v_scale, 64, mass=start.clone())
              for _ in streams]
    size = T.kv8_attention_workspace_size(cfg, caches[0], db)
    bufs = [(torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty_like(x)) for _ in streams]
    torch.cuda.synchronize()
    for st, kv, (ws, out) in zip(streams, caches, bufs):       # two calls at once
        T.kv8_attention(cfg, kv, db, x, out=out, workspace=ws, stream=st)
    torch.cuda.synchronize()
    for kv, (_, out) in zip(caches, bufs):
        check(out, kv.mass)
    assert torch.equal(bufs[0][1], bufs[1][1]) and torch.equal(caches[0].mass, caches[1].mass)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=streams[0]):
        T.kv8_attention(cfg, caches[0], db, x, out=bufs[0][1], workspace=bufs[0][0], stream=streams[0])
    for i in range(3):
        for kv, (_, out) in zip(caches, bufs):
            kv.mass.copy_(start)
            out.zero_()
        torch.cuda.synchronize()
        g.replay()
        T.kv8_attention(cfg, caches[1], db, x, out=bufs[1][1], workspace=bufs[1][0], stream=streams[1])
        torch.cuda.synchronize()
        assert torch.equal(bufs[0][1], bufs[1][1]) and torch.equal(caches[0].mass, caches[1].mass), i


def test_attention_repeats_bit_for_bit():
    import torch
    cfg = config(28, 4, 128)
    batch = (list(range(5)), [900, 77, 0, 1500, 3], [1, 1, 150, 90, 1])
    outs = []
    for _ in range(2):
        cache = attend_cache(cfg, batch, "int8", seed=9)
        db = T.DeviceBatch(*batch)
        q = bf16(db.n_tokens, 28, 128, seed=1)
        o, _ = T.kv8_attention(cfg, cache, db, q)
        outs.append((o, cache.mass))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


# ----------------------------------------------------------------- eviction --

EVICT = {
    "short": ([1, 0], [30, 63], [1, 1], 64, 4, 16),
    "cut": ([0, 2, 1], [200, 127, 255], [1, 0, 1], 128, 4, 32),
    "long": ([0, 1], [4999, 900], [1, 100], 2048, 8, 100),
    "longest": ([1, 0, 2], [30001, 16384, 600], [1, 1, 1], 4096, 4, 500),
    "half of long": ([0], [20479], [1], 10240, 0, 10240),
    "nearly all": ([0], [1091], [5], 1088, 0, 0),
    "bad slot": ([5, 0, -1], [100, 200, 3], [1, 1, 1], 32, 1, 31),
}


@pytest.mark.parametrize("name", sorted(EVICT))
@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("stamp", [False, True])
def test_select_and_move(name, page, stamp):
    slot, ctx, q, budget, first, recent = EVICT[name]
    for d, fmt in ((64, "int8"), (128, "e4m3")):
        cfg = config(4, 2, d)
        max_seq = -(-max(c + n for c, n in zip(ctx, q)) // 64) * 64
        if max_seq > 10000 and d == 128:
            continue   # (the host's reference takes its time)
        R = max(r for r in (32, 64, 128) if budget % r == 0 and (page or 64) % r == 0 or r == 32)
        if not page and budget % 128 == 0:
            R = 128
        cache = make_cache(cfg, 3, max_seq, fmt, R, page, seed=budget, stamp=stamp)
        if stamp:   # positions in any order, as after an eviction
            cache.stamp.copy_(cache.stamp % (2 * max_seq))
        db = T.DeviceBatch(slot, ctx, q)
        db.max_ctx_len = max(ctx)
        ref = kv8_ref.Cache(cache)
        want, want_len = ref.select(db.host, budget, first, recent)
        plan, new_len = T.kv8_select(cfg, cache, db, budget, first, recent)
        assert np.array_equal(plan.cpu().numpy(), want)
        assert np.array_equal(new_len.cpu().numpy(), want_len)
        T.kv8_move(cfg, cache, db, plan)
        ref.move(db.host, want)
        same_cache(cache, ref)
        T.kv8_move(cfg, cache, db, plan)   # once more changes nothing
        same_cache(cache, ref)


@pytest.mark.parametrize("rows", [129, 2300, 5000, 9000, 17000])
def test_select_ties_and_strange_weights(rows):
    """Equal weights go to the lower rows; NaN last, infinities and -0 in their order."""
    cfg = config(2, 2, 64)
    cache = make_cache(cfg, 2, -(-rows // 32) * 32, seed=3, stamp=False)
    m = cache.mass
    m[0, 0] = 0.0
    m[0, 1] = (m[0, 1] * 4).floor()
    m[1, 0, 5:90] = float("nan")
    m[1, 0, 100], m[1, 0, 101], m[1, 0, 7] = float("inf"), -1.0, -0.0
    m[1, 1] = -m[1, 1]
    db = T.DeviceBatch([0, 1], [rows - 1, rows - 2], [1, 1])
    ref = kv8_ref.Cache(cache)
    for budget in (32, 96, 128):
        want, _ = ref.select(db.host, budget, 0, 3)
        plan, _ = T.kv8_select(cfg, cache, db, budget, 0, 3)
        assert np.array_equal(plan.cpu().numpy(), want), budget


def test_move_of_poisoned_blocks():
    cfg = config(2, 1, 64)
    cache = make_cache(cfg, 1, 256, "int8", seed=2)
    cache.k_scale[0, 0, 6] = float("nan")
    cache.mass[0, 0, 192:224] = 9.0
    db = T.DeviceBatch([0], [255], [1])
    ref = kv8_ref.Cache(cache)
    plan, _ = T.kv8_select(cfg, cache, db, 64)
    want, _ = ref.select(db.host, 64, 0, 0)
    assert np.array_equal(plan.cpu().numpy(), want)
    T.kv8_move(cfg, cache, db, plan)
    ref.move(db.host, want)
    same_cache(cache, ref)


def test_move_leaves_bad_entries_out():
    import torch
    cfg = config(2, 1, 64)
    cache = make_cache(cfg, 1, 128, seed=2)
    before = bits(cache)
    db = T.DeviceBatch([0], [127], [1])
    plan = torch.full((1, 1, 64), 1 << 30, dtype=torch.int32, device="cuda")
    plan[0, 0, 5:9] = torch.tensor([-1, -(1 << 31), 128, 8], dtype=torch.int32)
    T.kv8_move(cfg, cache, db, plan)
    torch.cuda.synchronize()
    assert all((bits(cache)[n] == before[n]).all() for n in before)


# ------------------------------------------------------------ all as it runs --

@pytest.mark.parametrize("page", [0, 128])
@pytest.mark.parametrize("fmt", FORMATS)
def test_long_context_loop(fmt, page):
    """Prompts, steps and evictions as a serving loop makes them: fused rows rotated in
    place, appended, attended to, and the cache cut back whenever it is past its budget;
    every piece held to its definition on the cache as it stands."""
    import torch
    hq, hkv, d, budget = 14, 2, 64, 128
    cfg, rcfg = config(hq, hkv, d), T.make_rope(64, scaling="turns", factor=4.0, original_len=64)
    table = None
    if page:
        table = torch.randperm(9, generator=torch.Generator().manual_seed(1))[:9].view(3, 3).int().cuda()
    cache = T.KV8Cache.empty(cfg, 3, 384, fmt, 32, mass=True, stamp=True, block_table=table,
                             block_size=page, n_blocks=9 if page else 0)
    slots, ctx, seen = [2, 0, 1], [0, 0, 0], [0, 0, 0]
    freqs = kv8_ref.rope_freqs(64, 1e6, "turns", 4.0, original_len=64)
    for step in range(6):
        q_len = [[140, 1, 33], [1, 1, 1], [1, 70, 1], [1, 1, 120], [90, 1, 1], [1, 1, 1]][step]
        pos = np.concatenate([np.arange(s, s + n) for s, n in zip(seen, q_len)])
        db = T.DeviceBatch(slots, ctx, q_len, pos=pos)
        rows = bf16(db.n_tokens, hq + 2 * hkv, d, seed=step, spread=0.3)
        qk = rows[:, :hq + hkv]
        turned = kv8_ref.rope(f64(qk), pos, freqs)
        T.rope(rcfg, qk, db.pos, out=qk)
        assert (np.abs(f64(qk) - turned) <= 2.0 ** -8 * np.abs(turned) + 2e-6 * np.abs(turned).max()).all()
        ref = kv8_ref.Cache(cache)
        T.kv8_append(cfg, cache, db, rows[:, hq:hq + hkv], rows[:, hq + hkv:])
        ref.append(db.host, f64(rows[:, hq:hq + hkv]), f64(rows[:, hq + hkv:]), pos)
        same_cache(cache, ref)
        out, tol, mass, mtol = ref.attention(db.host, f64(rows[:, :hq]))
        got, _ = T.kv8_attention(cfg, cache, db, rows[:, :hq])
        assert (np.abs(f64(got) - out) <= tol).all()
        ref.mass = mass
        same_cache(cache, ref, mtol)
        ref = kv8_ref.Cache(cache)
        plan, new_len = T.kv8_select(cfg, cache, db, budget, 2, 32)
        want, want_len = ref.select(db.host, budget, 2, 32)
        assert np.array_equal(plan.cpu().numpy(), want)
        T.kv8_move(cfg, cache, db, plan)
        ref.move(db.host, want)
        same_cache(cache, ref)
        ctx, seen = want_len.tolist(), [s + n for s, n in zip(seen, q_len)]
        assert new_len.tolist() == ctx


def test_step_on_another_stream_and_in_graphs():
    """Append, attention and select captured into a graph and replayed between eager
    work; two graphs on workspaces of their own."""
    import torch
    cfg = config(14, 2, 64)
    batch = ([1, 0, 2], [300, 20, 0], [1, 1, 65])
    cache = attend_cache(cfg, batch, "e4m3", seed=12)
    db = T.DeviceBatch(*batch)
    q = bf16(db.n_tokens, 14, 64, seed=3)
    k = bf16(db.n_tokens, 2, 64, seed=4)
    start = cache.mass.clone()
    st = torch.cuda.Stream()

    def step(ws, out, plan, new_len):
        T.kv8_append(cfg, cache, db, k, k, stream=st)
        T.kv8_attention(cfg, cache, db, q, out=out, workspace=ws, stream=st)
        T.kv8_select(cfg, cache, db, 64, 2, 8, plan=plan, new_len=new_len, stream=st)

    def buffers():
        return (torch.empty(T.kv8_attention_workspace_size(cfg, cache, db), dtype=torch.uint8, device="cuda"),
                torch.zeros_like(q), torch.zeros(3, 2, 64, dtype=torch.int32, device="cuda"),
                torch.zeros(3, dtype=torch.int32, device="cuda"))

    eager, sets = buffers(), [buffers(), buffers()]
    torch.cuda.synchronize()
    step(*eager)
    st.synchronize()
    mass = cache.mass.clone()
    graphs = []
    for b in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            step(*b)
        graphs.append(g)
    for i in range(3):
        for g, b in zip(graphs, sets):
            cache.mass.copy_(start)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(b[1], eager[1]) and torch.equal(cache.mass, mass), i
            assert torch.equal(b[2], eager[2]) and torch.equal(b[3], eager[3]), i
            junk = torch.randn(1 << 20, device="cuda") * 3.0
            del junk
            torch.cuda.synchronize()
