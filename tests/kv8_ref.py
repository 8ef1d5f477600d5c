"""The long-context operators from their definitions, in plain float64 on the host
(test infrastructure: no code shared with the library), and the bounds that a kernel
in the documented precision keeps against them."""
import math

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}


# ------------------------------------------------------------------- rotary --

def rope_freqs(r, base, scaling="none", factor=1.0, low=1.0, high=32.0, original_len=0):
    w = np.array([base ** (-2.0 * i / r) for i in range(r // 2)])
    if scaling == "linear":
        return w / factor
    if scaling == "base" and r > 2:
        b = base * factor ** (r / (r - 2.0))
        return np.array([b ** (-2.0 * i / r) for i in range(r // 2)])
    if scaling == "turns":
        turns = original_len * w / (2 * math.pi)
        t = np.clip((turns - low) / (high - low), 0, 1)
        return w * (t + (1 - t) / factor)
    if scaling == "index":
        at = lambda n: r * math.log(original_len / (2 * math.pi * n)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), r - 1)
        u = np.clip((np.arange(r // 2) - lo) / max(hi - lo, 0.001), 0, 1)
        return w * (1 - u) + w / factor * u
    return w


def rope(x, pos, freqs, interleaved=False, magnitude=1.0):
    """x [tokens, heads, D] float64."""
    r = 2 * len(freqs)
    ang = pos.astype(np.float64)[:, None, None] * freqs
    c, s = magnitude * np.cos(ang), magnitude * np.sin(ang)
    y = x.copy()
    ia = np.arange(0, r, 2) if interleaved else np.arange(r // 2)
    ib = ia + (1 if interleaved else r // 2)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


# ---------------------------------------------------------------- the cache --

def number(x, fmt):
    """x rounded to the type's numbers, ties to even."""
    if fmt == "int8":
        return np.rint(x)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.rint(x / step) * step


def scale_of(amax, fmt):
    """Least power of two s >= 2^-100 with amax <= top * s; NaN for a non-finite amax."""
    if not np.isfinite(amax):
        return math.nan
    e = -100
    if amax > 0:
        e = max(e, math.floor(math.log2(amax / TOP[fmt])) - 1)
    while TOP[fmt] * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


class Cache:
    """Logical rows [slots, heads, max_seq, ...] of a KV8Cache, in float64."""

    def __init__(self, cache):
        import torch
        self.fmt = "int8" if cache.k.dtype == torch.int8 else "e4m3"
        self.R, self.max_seq, self.slots = cache.scale_rows, cache.max_seq, cache.n_slots
        self.table = None if cache.block_table is None else cache.block_table.cpu().numpy()
        self.page = cache.k.shape[2]
        f = lambda t: None if t is None else t.cpu().float().numpy().astype(np.float64)
        self.k, self.v = self.rows(f(cache.k)), self.rows(f(cache.v))
        self.ks, self.vs = self.rows(f(cache.k_scale), self.R), self.rows(f(cache.v_scale), self.R)
        self.mass = None if cache.mass is None else self.rows(f(cache.mass))
        self.stamp = None if cache.stamp is None else self.rows(cache.stamp.cpu().numpy())

    def rows(self, a, per=1):
        if self.table is None:
            return a
        heads, rest = a.shape[1], a.shape[3:]
        out = np.zeros((self.slots, heads, self.max_seq // per) + rest, a.dtype)
        n = self.page // per
        for s in range(self.slots):
            for j, p in enumerate(self.table[s]):
                if 0 <= p < len(a):
                    out[s, :, j * n:(j + 1) * n] = a[p]
        return out

    def values(self, name, slot, n):
        c, s = (self.k, self.ks) if name == "k" else (self.v, self.vs)
        return c[slot, :, :n] * np.repeat(s[slot], self.R, -1)[:, :n, None]

    def append(self, batch, k_new, v_new, pos):
        """k_new, v_new float64 [tokens, heads, D]."""
        t = 0
        for slot, c, q in zip(batch["slot"], batch["ctx_len"], batch["q_len"]):
            t0, t = t, t + q
            if not 0 <= slot < self.slots or c + q > self.max_seq or q == 0:
                continue
            for blk in range(c // self.R, -(-(c + q) // self.R)):
                b0 = blk * self.R
                lo, hi = max(b0, c), min(b0 + self.R, c + q)
                for codes, scales, new in ((self.k, self.ks, k_new), (self.v, self.vs, v_new)):
                    for h in range(codes.shape[1]):
                        x = new[t0 + lo - c:t0 + hi - c, h]
                        s = scale_of(np.abs(x).max(), self.fmt)
                        if lo > b0:
                            old = scales[slot, h, blk]
                            s = math.nan if math.isnan(s) or math.isnan(old) else max(s, old)
                            if s != old:
                                codes[slot, h, b0:lo] = 0 if math.isnan(s) else number(
                                    codes[slot, h, b0:lo] * (old / s), self.fmt)
                        codes[slot, h, lo:hi] = 0 if math.isnan(s) else number(x / s, self.fmt)
                        scales[slot, h, blk] = s
            if self.mass is not None:
                self.mass[slot, :, c:c + q] = 0
            if self.stamp is not None:
                self.stamp[slot, :, c:c + q] = pos[t0:t]

    def attention(self, batch, q):
        """(out, tolerance of out, mass, tolerance of mass) of float64 q [tokens, Hq, D];
        NaN rows in out: tokens of a skipped sequence.

        The bounds, with u = 2^-24 the float32 rounding and n rows: a score is a sum of
        D products, off by at most (D + 8) u sum |q k| / sqrt D =: e (scaling and
        exponent's argument included), which moves every weight by a factor within 1 +-
        2 e; the exponential and the sums of n terms by (n + 64) u; weights rounded to 11
        bits by 2^-11, or where they fall below 2^-14 of the largest weight (times its
        value's scale) by 2^-25 of it, 2^8 more while the running maximum lags; the
        output's rounding is 2^-8 of it.  A weight that is added to the mass may be lost
        whole where it is below 2^-126, float32's least normal number: with a start of zero
        the terms relative to it bound nothing there (exp(-96) is 2^-138 already)."""
        tokens, hq, D = q.shape
        u = 2.0 ** -24
        out, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
        mass = None if self.mass is None else self.mass.copy()
        mtol = None if mass is None else np.zeros_like(mass)
        t = 0
        for slot, c, n_new in zip(batch["slot"], batch["ctx_len"], batch["q_len"]):
            t0, t = t, t + n_new
            if not 0 <= slot < self.slots or c + n_new > self.max_seq or n_new == 0:
                continue
            n = c + n_new
            k, v = self.values("k", slot, n), self.values("v", slot, n)
            vs = np.repeat(self.vs[slot], self.R, -1)[:, :n]
            seen = np.arange(n)[None] <= c + np.arange(n_new)[:, None]
            for head in range(hq):
                h = head // (hq // k.shape[0])
                x = q[t0:t, head]
                s = x @ k[h].T / math.sqrt(D)
                s[~seen] = -np.inf
                with np.errstate(invalid="ignore"):
                    p = np.exp(s - s.max(-1, keepdims=True))
                    p /= p.sum(-1, keepdims=True)
                e = (D + 8) * u * (np.abs(x) @ np.abs(k[h]).T / math.sqrt(D)).max(-1, keepdims=True)
                few = 2 * e + (n + 64) * u
                out[t0:t, head] = p @ v[h]
                top = np.abs(v[h] / np.where(vs[h] == 0, 1, vs[h])[:, None]).max()
                tol[t0:t, head] = (2.0 ** -8 * np.abs(out[t0:t, head])
                                   + (2.0 ** -11 + few) * (p @ np.abs(v[h]))
                                   + n * 2.0 ** -25 * (p * vs[h]).max(-1, keepdims=True) * top)
                if mass is not None:
                    mass[slot, h, :n] += p.sum(0)
                    mtol[slot, h, :n] += (few * p).sum(0)
            if mass is not None:  # and the sums over heads and tokens
                mtol[slot, :, :n] += ((hq // k.shape[0]) * n_new + 2) * (
                    u * mass[slot, :, :n] + 2.0 ** -126)
        return out, tol, mass, mtol

    def select(self, batch, budget, n_first, n_recent):
        seqs = list(zip(batch["slot"], batch["ctx_len"], batch["q_len"]))
        heads = self.k.shape[1]
        plan = np.full((len(seqs), heads, budget), -1, np.int32)
        new_len = np.zeros(len(seqs), np.int32)
        for i, (slot, c, q) in enumerate(seqs):
            n = c + q
            if not 0 <= slot < self.slots or n > self.max_seq:
                continue
            new_len[i] = min(n, budget)
            for h in range(heads):
                stamp = np.arange(n) if self.stamp is None else self.stamp[slot, h, :n]
                m = self.mass[slot, h, :n]
                newest = max(stamp) if n else 0
                rank = sorted(range(n), key=lambda r: (
                    not (stamp[r] < n_first or stamp[r] > newest - n_recent),
                    np.isnan(m[r]), 0.0 if np.isnan(m[r]) else -m[r], r))
                # (protected rows compare equal: by row)
                safe = [r for r in rank if stamp[r] < n_first or stamp[r] > newest - n_recent]
                rank = sorted(safe) + [r for r in rank if r not in set(safe)]
                keep = set(rank[:budget])
                movers = iter(sorted(r for r in keep if r >= budget))
                for r in range(min(n, budget)):
                    plan[i, h, r] = r if r in keep else next(movers)
        return plan, new_len

    def move(self, batch, plan):
        budget = plan.shape[-1]
        for i, slot in enumerate(batch["slot"]):
            if not 0 <= slot < self.slots:
                continue
            for h in range(plan.shape[1]):
                src = plan[i, h]
                for codes, scales in ((self.k, self.ks), (self.v, self.vs)):
                    new, old = codes[slot, h].copy(), scales[slot, h].copy()
                    for b in range(budget // self.R):
                        rows = np.arange(b * self.R, (b + 1) * self.R)
                        frm = src[rows]
                        ok = frm >= 0
                        if not ok.any() or (frm[ok] == rows[ok]).all():
                            continue
                        s = np.max(old[frm[ok] // self.R])   # (NaN if any is)
                        scales[slot, h, b] = s
                        for r, f in zip(rows[ok], frm[ok]):
                            new[r] = 0 if math.isnan(s) else number(
                                codes[slot, h, f] * (old[f // self.R] / s), self.fmt)
                    codes[slot, h] = new
                ok = np.nonzero(src >= 0)[0]
                for a in (self.mass, self.stamp):
                    if a is not None:
                        a[slot, h, ok] = a[slot, h, src[ok]].copy()
