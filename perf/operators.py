"""The operators of a long context, as measurable cases: rotary positions, the
8-bit key/value cache (append, attention over it) and its eviction by
accumulated attention weight.

A case names a head layout of the model zoo (LAYERS) and, where there is a
step, its ragged batch as text: space-separated groups COUNTxQ@CTX, COUNT
sequences of Q new tokens after CTX cached ones; Q and CTX may be ranges
LO..HI, spread evenly over the logarithm within the group.

The cache holds one byte per value, and per head and scale_rows rows a scale:
the smallest power of two with which no value leaves the type (127 for int8,
448 for e4m3).  A value is code * scale; a scale only ever grows while rows
are appended, and the codes that were there are rounded once more to it.
"""
import math

import numpy as np
import torch

own = False

LAYERS = {
    "dense": dict(hq=28, hkv=4, d=128),   # the 7B-class layer
    "moe": dict(hq=32, hkv=4, d=128),     # the 128-expert layer
    "talker": dict(hq=14, hkv=2, d=64),
}
BASE = 1e6
BLOCK = 128      # rows of a page where the cache is paged
LEAST = -100     # exponent of the smallest scale


def listed():
    return [
        # one token of one speech stream: all latency
        _rope("rope_token", "talker", 1, 300),
        # partly rotated heads, pairs side by side, a context four times the trained one
        _rope("rope_partial", "moe", 1061, 16000, rotary=64, interleaved=True, scaling="turns",
              factor=4.0, original=8192, f32=True),
        # the benchmark's prefill: 8 prompts of 2048 tokens, far positions
        _rope("rope_prompt", "dense", 16384, 131072, scaling="index", factor=4.0, original=32768),
        # the decode step of a full batch
        _append("append_step", "dense", "64x1@4096", scale_rows=64),
        # ragged prompts, some continued, into a paged cache
        _append("append_prompt", "moe", "5x300..2048@40..900", paged=True),
        # one user's token after a long chat
        _attend("attend_one", "dense", "1x1@5000", "int8"),
        # the decode benchmark: 64 sequences of 4096 tokens
        _attend("attend_batch", "dense", "64x1@4096", "int8", scale_rows=64),
        # the expert layer's decode, paged, the weights summed for an eviction later
        _attend("attend_weighed", "moe", "128x1@2048", "e4m3", paged=True, mass=True),
        # a 512-token chunk at 6144 beside 32 single tokens, weights summed
        _attend("attend_mixed", "dense", "1x512@6144 32x1@1024..8192", "e4m3", mass=True),
        # the benchmark's prefill: 8 prompts of 2048 tokens
        _attend("attend_prompt", "dense", "8x2048@0", "int8"),
        # a batch a few hundred tokens over its budget
        _evict("evict_batch", "dense", "64x1@4351", 4096, first=4, recent=256),
        # a long document cut in half
        _evict("evict_long", "moe", "1x1@131071", 65536, first=64, recent=4096, scale_rows=128),
    ]


def _rope(name, layer, tokens, far, rotary=0, interleaved=False, scaling="none", factor=1.0,
          original=0, f32=False):
    c = dict(op="rope", layer=layer, tokens=tokens, far=far, rotary=rotary or LAYERS[layer]["d"],
             interleaved=interleaved, scaling=scaling, factor=factor, original=original, f32=f32)
    return dict(c, name=name) if name else c


def _append(name, layer, batch, paged=False, scale_rows=32):
    # e4m3: codes come back as the 8-bit floats they are, beside their scales
    c = dict(op="append", layer=layer, batch=batch, fmt="e4m3", paged=paged, mass=True,
             scale_rows=scale_rows)
    return dict(c, name=name) if name else c


def _attend(name, layer, batch, fmt, paged=False, mass=False, scale_rows=32):
    c = dict(op="attend", layer=layer, batch=batch, fmt=fmt, paged=paged, mass=mass,
             scale_rows=scale_rows)
    return dict(c, name=name) if name else c


def _evict(name, layer, batch, budget, first=4, recent=64, paged=False, scale_rows=32):
    c = dict(op="evict", layer=layer, batch=batch, budget=budget, first=first, recent=recent,
             fmt="e4m3", paged=paged, mass=True, scale_rows=scale_rows)
    return dict(c, name=name) if name else c


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    layer = rng.choice(sorted(LAYERS))
    paged, scale_rows = rng.random() < 0.5, rng.choice([32, 64, 128])
    op = rng.choice(["rope", "append", "decode", "decode", "chunk", "mixed", "evict"])
    if op == "rope":
        d = LAYERS[layer]["d"]
        return _rope(None, layer, log(1, 16000), log(1000, 1000000),
                     rotary=rng.choice([d, d // 2, d // 4, 2 * rng.randint(1, d // 2)]),
                     interleaved=rng.random() < 0.5,
                     scaling=rng.choice(["none", "linear", "base", "turns", "index"]),
                     factor=rng.choice([1.5, 2.0, 4.0, 8.0, 40.0]), original=log(2000, 40000),
                     f32=rng.random() < 0.3)
    if op == "append":
        n = log(1, 100)
        q = log(1, max(1, 16000 // n))
        return _append(None, layer, "%dx%d..%d@%d..%d" % (n, -(-q // 3), q, log(1, 100),
                                                          log(100, 4000)), paged, scale_rows)
    fmt, mass = rng.choice(["int8", "e4m3"]), rng.random() < 0.5
    if op == "decode":
        n = log(1, 128)
        ctx = log(40, min(100000, 260000 // n))
        return _attend(None, layer, "%dx1@%d..%d" % (n, max(1, ctx // 20), ctx), fmt, paged, mass,
                       scale_rows)
    if op == "chunk":
        n = rng.randint(1, 5)
        q = log(2, 4000 // n)
        return _attend(None, layer, "%dx%d..%d@%d" % (n, -(-q // 3), q,
                                                      rng.choice([0, log(20, 6000)])),
                       fmt, paged, mass, scale_rows)
    if op == "mixed":
        return _attend(None, layer, "1x%d@%d %dx1@%d..%d" % (
            log(30, 600), log(60, 6000), rng.randint(1, 32), log(30, 500), log(600, 8000)), fmt,
            paged, mass, scale_rows)
    n = log(1, 64)
    ctx = log(600, min(131000, 260000 // n))
    budget = max(scale_rows, int(ctx * rng.uniform(0.3, 0.98)) // scale_rows * scale_rows)
    return _evict(None, layer, "%dx1@%d..%d" % (n, max(1, ctx // 3), ctx), budget,
                  rng.randint(0, 8), log(8, max(9, budget // 2)), paged, scale_rows)


# ---------------------------------------------------------------- the batch --

def _spread(text, n):
    """n values of "V" or "LO..HI" (evenly over the logarithm, largest in the middle)."""
    if ".." not in text:
        return [int(text)] * n
    lo, hi = (int(v) for v in text.split(".."))
    up = [int(round(lo * (hi / lo) ** (i / max(1, n - 1)))) for i in range(n)]
    return up[0::2] + up[1::2][::-1]


def _seqs(case):
    """[(new tokens, cached tokens)] of the step's sequences."""
    out = []
    for group in case["batch"].split():
        n, rest = group.split("x")
        q, ctx = rest.split("@")
        out += list(zip(_spread(q, int(n)), _spread(ctx, int(n))))
    return out


# --------------------------------------------------------------- the inputs --

def _max_seq(case, seqs):
    """Rows of a sequence's slot: its longest, and an eviction's budget (which a sequence may
    lie below), in whole pages."""
    return -(-max(case.get("budget", 0), *(q + c for q, c in seqs)) // BLOCK) * BLOCK


def _inputs(case, seed):
    """Everything a pass reads, from the seed alone."""
    L = LAYERS[case["layer"]]
    hq, hkv, d = L["hq"], L["hkv"], L["d"]
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)

    def normal(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)

    def uniform(*shape):
        return torch.empty(shape, device="cuda").uniform_(generator=g)

    if case["op"] == "rope":
        T = case["tokens"]
        dt = torch.float32 if case["f32"] else torch.bfloat16
        # the fused projection's rows: q heads, k heads, v heads
        qkv = normal(T, hq + 2 * hkv, d, dtype=dt)
        pos = (uniform(1) * (case["far"] - T if case["far"] > T else 1)).to(torch.int32) + \
            torch.arange(T, dtype=torch.int32, device="cuda")
        return dict(x=qkv[:, :hq + hkv], pos=pos)

    seqs, R = _seqs(case), case["scale_rows"]
    n, T = len(seqs), sum(q for q, _ in seqs)
    max_seq = _max_seq(case, seqs)
    slots = [(i * 5 + 2) % n if n % 5 else (i + 2) % n for i in range(n)]  # a fixed permutation
    table, panels, rows = None, n, max_seq
    if case["paged"]:
        per = max_seq // BLOCK
        panels, rows = n * per + 3, BLOCK
        order = torch.randperm(panels, generator=torch.Generator().manual_seed(int(seed)))
        table = order[:n * per].reshape(n, per).to(torch.int32).cuda()
    i = dict(seqs=seqs, slots=slots, max_seq=max_seq, table=table)
    # keys with a few strong channels, values whose size differs from page to page
    loud = 1 + 4 * (uniform(1, hkv, 1, d) > 0.95)
    size = 2.0 ** (2 * normal(panels, hkv, rows // 32, 1, 1))
    for name, times in (("k", loud), ("v", None)):
        x = normal(panels, hkv, rows, d)
        if times is not None:
            x *= times
        else:
            x.view(panels, hkv, rows // 32, 32, d).mul_(size)
        x = x.view(panels, hkv, rows // R, R, d)
        s = _scale(x.abs().amax((3, 4)), case["fmt"])
        i[name + "_scale"] = s
        i[name] = _codes(x / s[..., None, None], case["fmt"]).view(panels, hkv, rows, d)
        del x
    if case["mass"]:
        i["mass"] = 8 * uniform(panels, hkv, rows) ** 6 * (uniform(panels, hkv, rows) > 0.1)
        # the position of the token in each row
        i["stamp"] = torch.full((panels, hkv, rows), -1, dtype=torch.int32, device="cuda")
        at = torch.arange(max_seq, dtype=torch.int32, device="cuda")
        if table is None:
            i["stamp"][:] = at
        else:
            i["stamp"][table.long()] = at.view(1, -1, 1, BLOCK).expand(n, -1, hkv, -1)
    if case["op"] == "append":
        i["k_new"] = (normal(T, hkv, d) * loud[0, :, 0] * 2.0 ** normal(T, 1, 1)).bfloat16()
        i["v_new"] = (normal(T, hkv, d) * 2.0 ** normal(T, 1, 1)).bfloat16()
    if case["op"] == "attend":
        i["q"] = normal(T, hq, d, dtype=torch.bfloat16)
    return i


# ------------------------------------------------------- 8 bits and a scale --

def _scale(amax, fmt):
    """Smallest power of two s with amax <= s * (largest number of the type)."""
    m, e = torch.frexp(amax)
    if fmt == "int8":      # 127 = 0.9921875 * 2^7
        e = e - 7 + (m > 0.9921875).to(e.dtype)
    else:                  # 448 = 0.875 * 2^9
        e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.ldexp(torch.ones_like(amax), e.clamp(min=LEAST))


def _codes(x, fmt):
    return x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)


def _bytes(x):
    return x.view(torch.uint8)


# ------------------------------------------------------------------- a pass --

def _index(i, case):
    """The batch as index tensors on the GPU: per sequence its rows' place in
    the cache, per touched block of the scales its place and rows."""
    R = case["scale_rows"]
    dev = lambda a: torch.tensor(a, device="cuda")
    q, c = dev([q for q, _ in i["seqs"]]), dev([c for _, c in i["seqs"]])
    slot = dev(i["slots"])
    x = dict(q=q, c=c, slot=slot, len=q + c, end=q.cumsum(0), max_len=max(a + b for a, b in i["seqs"]))
    x["start"] = x["end"] - q
    seq, blk = [], []
    for s, (n, ctx) in enumerate(i["seqs"]):
        for b in range(ctx // R, -(-(ctx + n) // R)):
            seq.append(s)
            blk.append(b)
    x["seq"], x["blk"] = dev(seq), dev(blk)
    return x


def _place(i, slot, row):
    """Panel and row within it of the logical rows of slots (broadcast)."""
    if i["table"] is None:
        return slot.expand_as(row), row
    return i["table"][slot, row // BLOCK].long(), row % BLOCK


def prepare(case, seed):
    i = _inputs(case, seed)
    state = dict(case=case, i=i)
    L = LAYERS[case["layer"]]
    if case["op"] == "rope":
        state["out"] = torch.empty(i["x"].shape, dtype=i["x"].dtype, device="cuda")
    else:
        state["x"] = _index(i, case)
        if case["op"] == "attend":
            state["out"] = torch.empty_like(i["q"])
        if case["op"] == "evict":
            # what the rows are chosen by; the cache's own weights and positions move
            i["score"], i["age"] = i["mass"].clone(), i["stamp"].clone()
    if own:
        from paper_2606_29629_amd import _lib as tri
        if case["op"] == "rope":
            state["cfg"] = tri.make_rope(L["d"], rotary_dim=case["rotary"], base=BASE,
                                         interleaved=case["interleaved"], scaling=case["scaling"],
                                         factor=case["factor"], low=1.0, high=32.0,
                                         original_len=case["original"])
            return state

        class Config:
            hidden, n_q_heads, n_kv_heads, head_dim = 64, L["hq"], L["hkv"], L["d"]
            rms_eps, rope_base = 1e-6, BASE

        state["cfg"] = tri.make_config(Config)
        state["batch"] = tri.DeviceBatch(i["slots"], [c for _, c in i["seqs"]],
                                         [q for q, _ in i["seqs"]])

        def cache(mass, stamp):
            return tri.KV8Cache(i["k"], i["v"], i["k_scale"], i["v_scale"], case["scale_rows"],
                                mass=mass, stamp=stamp, block_table=i["table"],
                                max_seq=i["max_seq"])

        state["cache"] = cache(i.get("mass"), i.get("stamp"))
        if case["op"] == "attend":
            state["ws"] = torch.empty(
                tri.kv8_attention_workspace_size(state["cfg"], state["cache"], state["batch"]),
                dtype=torch.uint8, device="cuda")
        if case["op"] == "evict":
            state["scored"] = cache(i["score"], i["age"])
            shape = len(i["seqs"]), L["hkv"], case["budget"]
            state["plan"] = torch.empty(shape, dtype=torch.int32, device="cuda")
            state["new_len"] = torch.empty(shape[0], dtype=torch.int32, device="cuda")
    return state


def run(state):
    case, i = state["case"], state["i"]
    op = case["op"]
    if own:
        from paper_2606_29629_amd import _lib as tri
        if op == "rope":
            return tri.rope(state["cfg"], i["x"], i["pos"], out=state["out"])
        args = state["cfg"], state["cache"], state["batch"]
        if op == "append":
            tri.kv8_append(*args, i["k_new"], i["v_new"])
        elif op == "attend":
            out, _ = tri.kv8_attention(*args, i["q"], out=state["out"], workspace=state["ws"])
            return {"out": out, "mass": i.get("mass")}
        else:
            tri.kv8_select(state["cfg"], state["scored"], state["batch"], case["budget"],
                           case["first"], case["recent"], plan=state["plan"],
                           new_len=state["new_len"])
            tri.kv8_move(*args, state["plan"])
            return dict(_cache_of(i), plan=state["plan"], new_len=state["new_len"])
        return _cache_of(i)
    if op == "rope":
        return _rope_plain(case, i["x"], i["pos"])
    if op == "append":
        _append_plain(case, i, state["x"], "k")
        _append_plain(case, i, state["x"], "v")
        _append_rows(case, i, state["x"])
        return _cache_of(i)
    if op == "attend":
        return {"out": _attend_plain(state), "mass": i.get("mass")}
    plan, new_len = _select_plain(case, i, state["x"])
    _move_plain(case, i, state["x"], plan)
    return dict(_cache_of(i), plan=plan.to(torch.int32), new_len=new_len.to(torch.int32))


def _cache_of(i):
    """The updated cache: its buffers (codes as the 8-bit floats they are)."""
    return {name: i[name] for name in ("k", "v", "k_scale", "v_scale", "mass", "stamp")}


def _freqs(case):
    """Rotary frequencies in double precision."""
    r = case["rotary"]
    base = BASE
    if case["scaling"] == "base" and r > 2:
        base = BASE * case["factor"] ** (r / (r - 2))
    f = base ** (torch.arange(r // 2, dtype=torch.float64, device="cuda") * (-2.0 / r))
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "turns":
        t = ((case["original"] * f / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        f = f * (t + (1 - t) / case["factor"])
    if case["scaling"] == "index":
        def at(turns):
            return r * math.log(case["original"] / (2 * math.pi * turns)) / (2 * math.log(BASE))
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        ramp = ((torch.arange(r // 2, dtype=torch.float64, device="cuda") - lo)
                / max(hi - lo, 0.001)).clamp(0, 1)
        f = f * (1 - ramp) + f / case["factor"] * ramp
    return f


def _rope_plain(case, x, pos):
    r = case["rotary"]
    angle = pos.double()[:, None] * _freqs(case)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _append_plain(case, i, x, name):
    """New rows into the touched blocks of the scales, all blocks at once."""
    R, fmt = case["scale_rows"], case["fmt"]
    codes, scale, new = i[name], i[name + "_scale"], i[name + "_new"]
    row = x["blk"][:, None] * R + torch.arange(R, device="cuda")
    c, q, start = (x[k][x["seq"]][:, None] for k in ("c", "q", "start"))
    held, fresh = row < c, (row >= c) & (row < c + q)
    panel, prow = _place(i, x["slot"][x["seq"]][:, None], row)
    at = panel[:, :1], torch.arange(codes.shape[1], device="cuda"), prow[:, :1] // R
    value = new[(start + row - c).clamp(0, new.shape[0] - 1)].float().transpose(1, 2)
    value = torch.where(fresh[:, None, :, None], value, 0)
    s = _scale(value.abs().amax((2, 3)), fmt)
    before = scale[at]
    s = torch.where(held.any(1)[:, None], torch.maximum(s, before), s)
    raw = _bytes(codes)
    place = panel[:, None], torch.arange(codes.shape[1], device="cuda")[:, None], prow[:, None]
    old = raw[place]
    number = old.view(codes.dtype).float() * (before / s)[..., None, None]
    both = torch.where(held[:, None, :, None], number, value / s[..., None, None])
    write = (held | fresh)[:, None, :, None]
    raw[place] = torch.where(write, _bytes(_codes(both, fmt)), old)
    scale[at] = s


def _append_rows(case, i, x):
    """The new rows' attention weight (none yet) and position."""
    T = int(i["k_new"].shape[0])
    t = torch.arange(T, device="cuda")
    s = torch.searchsorted(x["end"], t, right=True)
    row = x["c"][s] + t - x["start"][s]
    panel, prow = _place(i, x["slot"][s], row)
    i["mass"][panel, :, prow] = 0
    i["stamp"][panel, :, prow] = row.to(torch.int32)[:, None]


def _rows_of(case, i, x, seqs, length):
    """Panel, row and scale block of rows 0 .. length - 1 of some sequences."""
    row = torch.arange(length, device="cuda").expand(seqs.numel(), -1)
    panel, prow = _place(i, x["slot"][seqs][:, None], row)
    return panel, prow, prow // case["scale_rows"]


def _values(case, i, x, seqs, length, name):
    """Cache rows as the float32 values they stand for: [sequences, heads, rows, d]."""
    panel, prow, blk = _rows_of(case, i, x, seqs, length)
    h = torch.arange(i[name].shape[1], device="cuda")[None, :, None]
    codes = _bytes(i[name])[panel[:, None], h, prow[:, None]].view(i[name].dtype)
    return codes.float() * i[name + "_scale"][panel[:, None], h, blk[:, None]][..., None]


def _attend_plain(state):
    """Chunks and single tokens each as one padded batch."""
    i, x = state["i"], state["x"]
    out = state["out"]
    many = [s for s, (q, _) in enumerate(i["seqs"]) if q > 1]
    one = [s for s, (q, _) in enumerate(i["seqs"]) if q == 1]
    if many:
        _attend_part(state, many, out)
    if one:
        _attend_part(state, one, out)
    return out


def _attend_part(state, part, out):
    case, i, x = state["case"], state["i"], state["x"]
    hkv = LAYERS[case["layer"]]["hkv"]
    seqs = torch.tensor(part, device="cuda")
    length = max(sum(i["seqs"][s]) for s in part)
    Q = max(i["seqs"][s][0] for s in part)
    n, d = len(part), out.shape[-1]
    k, v = (_values(case, i, x, seqs, length, name) for name in "kv")
    t = x["start"][seqs][:, None] + torch.arange(Q, device="cuda")
    real = torch.arange(Q, device="cuda") < x["q"][seqs][:, None]
    t = torch.where(real, t, x["start"][seqs][:, None])
    q = i["q"][t].float().view(n, Q, hkv, -1, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    p = (q @ k.transpose(2, 3)).mul_(1 / math.sqrt(d))
    last = x["c"][seqs][:, None] + torch.arange(Q, device="cuda")
    hidden = torch.arange(length, device="cuda") > last[..., None]
    p = p.view(n, hkv, -1, Q, length).masked_fill_(hidden[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    p = p.div_(p.sum(-1, keepdim=True))
    o = (p.view(n, hkv, -1, length) @ v).view(n, hkv, -1, Q, d).permute(0, 3, 1, 2, 4)
    out[t[real]] = o[real].reshape(-1, *out.shape[1:]).to(out.dtype)
    if case["mass"]:
        weight = (p * real[:, None, None, :, None]).sum((2, 3))
        panel, prow, _ = _rows_of(case, i, x, seqs, length)
        there = torch.arange(length, device="cuda") < x["len"][seqs][:, None]
        h = torch.arange(hkv, device="cuda")
        at = panel[there][:, None], h, prow[there][:, None]
        i["mass"][at] += weight.transpose(1, 2)[there]


def _select_plain(case, i, x):
    """Row r of every head holds, after the eviction, what was in row plan[r]."""
    B = case["budget"]
    seqs = torch.arange(len(i["seqs"]), device="cuda")
    L = max(x["max_len"], B)
    panel, prow, _ = _rows_of(case, i, x, seqs, x["max_len"])
    h = torch.arange(i["score"].shape[1], device="cuda")[None, :, None]
    score = i["score"][panel[:, None], h, prow[:, None]]
    stamp = i["age"][panel[:, None], h, prow[:, None]]
    there = (torch.arange(x["max_len"], device="cuda") < x["len"][:, None])[:, None]
    newest = torch.where(there, stamp, -1).amax(-1, keepdim=True)
    kept_anyway = (stamp < case["first"]) | (stamp > newest - case["recent"])
    key = torch.where(kept_anyway, math.inf, score).masked_fill(~there, -math.inf)
    if L > key.shape[-1]:
        key = torch.nn.functional.pad(key, (0, L - key.shape[-1]), value=-math.inf)
    order = key.sort(dim=-1, descending=True, stable=True).indices
    keep = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, order[..., :B], True)
    row = torch.arange(L, device="cuda")
    keep &= row < x["len"][:, None, None]
    movers = torch.where(keep & (row >= B), row, L).sort(-1).values
    low = keep[..., :B]
    hole = ((~low).cumsum(-1) - 1).clamp(min=0)
    full = (x["len"] > B)[:, None, None]
    plan = torch.where(low, row[:B], torch.where(full, movers.gather(-1, hole), -1))
    return plan, x["len"].clamp(max=B)


def _move_plain(case, i, x, plan):
    B, R, fmt = case["budget"], case["scale_rows"], case["fmt"]
    n, hkv = plan.shape[:2]
    h = torch.arange(hkv, device="cuda")[None, :, None]
    there = plan >= 0
    src = plan.clamp(min=0)
    spanel, srow = _place(i, x["slot"][:, None, None], src)
    panel, prow = _place(i, x["slot"][:, None, None], torch.arange(B, device="cuda").expand_as(src))
    at, to = (spanel, h, srow), (panel, h, prow)
    for name in "kv":
        codes, scale = i[name], i[name + "_scale"]
        before = torch.where(there, scale[spanel, h, srow // R], 0)
        s = before.view(n, hkv, -1, R).amax(-1)
        full = there.view(n, hkv, -1, R).any(-1)
        each = s.repeat_interleave(R, -1)
        raw = _bytes(codes)
        number = raw[at].view(codes.dtype).float() * (before / each)[..., None]
        raw[to] = torch.where(there[..., None], _bytes(_codes(number, fmt)), raw[to])
        b = (panel[..., ::R], h, prow[..., ::R] // R)
        scale[b] = torch.where(full, s, scale[b])
    for name in ("mass", "stamp"):
        i[name][to] = torch.where(there, i[name][at], i[name][to])


# -------------------------------------------------------------------- work --

def work(case):
    """One pass: inputs read once, outputs written once; two flops per multiply-add."""
    L = LAYERS[case["layer"]]
    hq, hkv, d = L["hq"], L["hkv"], L["d"]
    if case["op"] == "rope":
        n = case["tokens"] * (hq + hkv)
        return {"bytes": n * d * 2 * (4 if case["f32"] else 2) + 4 * case["tokens"],
                "flops": 3 * n * case["rotary"]}
    seqs, R = _seqs(case), case["scale_rows"]
    T, rows = sum(q for q, _ in seqs), sum(q + c for q, c in seqs)
    per_row = 2 * hkv * (d + 4 / R)
    if case["op"] == "append":
        # the new rows and, in a block begun before, the old codes where the scale grows (half)
        begun = sum(c % R for _, c in seqs)
        return {"bytes": T * (4 * hkv * d + per_row + 8 * hkv) + begun * per_row,
                "flops": 4 * T * hkv * d}
    if case["op"] == "attend":
        pairs = sum(q * c + q * (q + 1) // 2 for q, c in seqs)
        return {"bytes": rows * per_row + 4 * T * hq * d + (8 * rows * hkv if case["mass"] else 0),
                "flops": 4 * d * hq * pairs}
    # every row's weight and position, the plan, and the rows that change place
    B = case["budget"]
    moved = sum((q + c - B) * B / (q + c) for q, c in seqs if q + c > B)
    return {"bytes": 8 * rows * hkv + 4 * hkv * B * len(seqs) + moved * (2 * per_row + 16 * hkv),
            "flops": rows * hkv}


# ------------------------------------------------------ the same in 64 bits --

def _exact_number(x, fmt):
    """x rounded to the type's numbers, ties to even, in float64."""
    if fmt == "int8":
        return torch.round(x)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_scale(amax, fmt):
    top = 127.0 if fmt == "int8" else 448.0
    e = torch.ceil(torch.log2((amax / top).clamp(min=2.0 ** LEAST)))
    e = torch.where(torch.exp2(e - 1) * top >= amax, e - 1, e).clamp(min=LEAST)
    return torch.exp2(torch.where(torch.exp2(e) * top < amax, e + 1, e))


def _exact_rope(case, i):
    r, D = case["rotary"], i["x"].shape[-1]
    f = []
    for j in range(r // 2):
        w = math.exp(-2 * j / r * math.log(BASE))
        if case["scaling"] == "linear":
            w /= case["factor"]
        elif case["scaling"] == "base" and r > 2:
            w *= case["factor"] ** (-2 * j / (r - 2))
        elif case["scaling"] == "turns":
            turns = case["original"] * w / (2 * math.pi)
            t = 1.0 if turns >= 32 else 0.0 if turns <= 1 else (turns - 1) / 31
            w = t * w + (1 - t) * w / case["factor"]
        elif case["scaling"] == "index":
            place = [r / 2 * math.log(case["original"] / (2 * math.pi * b)) / math.log(BASE)
                     for b in (32.0, 1.0)]
            lo, hi = max(0, math.floor(place[0])), min(r - 1, math.ceil(place[1]))
            t = min(1.0, max(0.0, (j - lo) / (hi - lo if hi > lo else 0.001)))
            w = w * (1 - t) + w * t / case["factor"]
        f.append(w)
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                    i["pos"].double()[:, None, None] * torch.tensor(f, dtype=torch.float64,
                                                                  device="cuda"))
    y = i["x"].double().clone()
    first = slice(0, r, 2) if case["interleaved"] else slice(0, r // 2)
    second = slice(1, r, 2) if case["interleaved"] else slice(r // 2, r)
    w = torch.complex(y[..., first], y[..., second]) * z
    y[..., first], y[..., second] = w.real, w.imag
    return y


def _panels(i, slot, rows):
    """[(panel, first row of the panel, first logical row, rows)] of a slot."""
    if i["table"] is None:
        return [(slot, 0, 0, rows)]
    ids = i["table"][slot].tolist()
    return [(ids[r // BLOCK], 0, r, min(BLOCK, rows - r)) for r in range(0, rows, BLOCK)]


def _exact_values(case, i, slot, rows, name):
    """[heads, rows, d] in float64."""
    R, got = case["scale_rows"], []
    for p, _, _, n in _panels(i, slot, rows):
        s = i[name + "_scale"][p].double().repeat_interleave(R, -1)[:, :n, None]
        got.append(i[name][p, :, :n].double() * s)
    return torch.cat(got, 1)


def exact(case, seed):
    i = _inputs(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, i)
    seqs, slots, R, fmt = i["seqs"], i["slots"], case["scale_rows"], case["fmt"]
    if case["op"] == "attend":
        if sum(q * (q + c) for q, c in seqs) * i["q"].shape[1] > 4e9:
            return None
        hkv, d = i["k"].shape[1], i["k"].shape[-1]
        out = torch.empty(i["q"].shape, dtype=torch.float64, device="cuda")
        mass = i["mass"].double().clone() if case["mass"] else None
        t = 0
        for slot, (q, c) in zip(slots, seqs):
            k, v = (_exact_values(case, i, slot, q + c, name) for name in "kv")
            seen = torch.arange(q + c, device="cuda") <= torch.arange(c, c + q, device="cuda")[:, None]
            total = 0
            for g in range(out.shape[1] // hkv):
                at = torch.arange(hkv, device="cuda") * (out.shape[1] // hkv) + g
                s = i["q"][t:t + q, at].double().transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(d)
                p = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
                out[t:t + q, at] = (p @ v).transpose(0, 1)
                total = total + p.sum(1)
            if mass is not None:
                for p, _, r, n in _panels(i, slot, q + c):
                    mass[p, :, :n] += total[:, r:r + n]
            t += q
        return {"out": out, "mass": mass}
    got = {name: i[name].double().clone() for name in ("k", "v", "k_scale", "v_scale", "mass")}
    if case["op"] == "append":
        t = 0
        for slot, (q, c) in zip(slots, seqs):
            ids = None if i["table"] is None else i["table"][slot].tolist()
            for b in range(c // R, (c + q + R - 1) // R):
                lo, hi = max(b * R, c), min(b * R + R, c + q)
                p, r = (slot, b * R) if ids is None else (ids[b * R // BLOCK], b * R % BLOCK)
                for name in "kv":
                    new = i[name + "_new"][t + lo - c:t + hi - c].double().transpose(0, 1)
                    s = _exact_scale(new.abs().amax((1, 2)), fmt)
                    if lo > b * R:
                        s = torch.maximum(s, got[name + "_scale"][p, :, r // R])
                        old = got[name][p, :, r:r + lo - b * R]
                        old *= (got[name + "_scale"][p, :, r // R] / s)[:, None, None]
                        old.copy_(_exact_number(old, fmt))
                    got[name][p, :, r + lo - b * R:r + hi - b * R] = _exact_number(
                        new / s[:, None, None], fmt)
                    got[name + "_scale"][p, :, r // R] = s
                got["mass"][p, :, r + lo - b * R:r + hi - b * R] = 0
            t += q
        return dict(got, stamp=None)
    B, hkv = case["budget"], i["k"].shape[1]
    plan = torch.full((len(seqs), hkv, B), -1, dtype=torch.int64)
    old = {name: i[name].cpu() for name in ("k_scale", "v_scale", "mass")}
    for s, (slot, (q, c)) in enumerate(zip(slots, seqs)):
        places = _panels(i, slot, q + c)
        weight, stamp = (torch.cat([i[name][p, :, :n].cpu() for p, _, _, n in places], 1).numpy()
                         for name in ("mass", "stamp"))
        panel = np.concatenate([np.full(n, p) for p, _, _, n in places])
        prow = np.concatenate([np.arange(n) for _, _, _, n in places])
        for h in range(hkv):
            safe = (stamp[h] < case["first"]) | (stamp[h] > stamp[h].max() - case["recent"])
            rank = np.lexsort((np.arange(q + c), -np.where(safe, np.inf, weight[h])))
            keep = np.sort(rank[:B])
            src = np.arange(min(B, q + c))
            src[np.setdiff1d(src, keep)] = keep[keep >= B]
            plan[s, h, :src.size] = torch.from_numpy(src)
            at, to = (panel[src], prow[src]), (panel[:src.size], prow[:src.size])
            got["mass"][to[0], h, to[1]] = old["mass"][at[0], h, at[1]].double().cuda()
            for name in "kv":
                before = old[name + "_scale"][at[0], h, at[1] // R].numpy()
                block = np.arange(src.size) // R
                scale = np.zeros(block[-1] + 1)
                np.maximum.at(scale, block, before)
                number = i[name][at[0], h, at[1]].double()
                number *= torch.from_numpy(before / scale[block]).cuda()[:, None]
                got[name][to[0], h, to[1]] = _exact_number(number, fmt)
                first = torch.from_numpy(np.unique(block) * R)
                got[name + "_scale"][panel[first], h, prow[first] // R] = torch.from_numpy(scale).cuda()
    return dict(got, plan=None, new_len=None, stamp=None)
