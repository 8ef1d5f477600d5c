"""Moves by plans that a caller made: rows left out beside rows that move.  A row that is left
out is one that stays where it is, so the definition is that of the plan with such entries
filled in (tests/kv8_ref.py: codes, scales, weights and stamps compared for equality)."""
import numpy as np
import pytest

import kv8_ref
from paper_2606_29629_amd import _lib as T
from test_gpu_kv8 import config, make_cache, same_cache

pytestmark = pytest.mark.gpu

BUDGET, MAX_SEQ = 256, 512


def plans(heads, bad_row=None):
    """Per 64 rows: one mover beside rows left out; movers, rows left out and rows that stay;
    nothing; movers only.  bad_row: a row whose page is outside the pool."""
    rng = np.random.default_rng(heads)
    rows = np.arange(BUDGET)
    plan = np.tile(rows, (heads, 1))
    out = [-1, -(1 << 31), MAX_SEQ, (1 << 31) - 1]
    for h in range(heads):
        free = iter(rng.permutation(np.arange(BUDGET, MAX_SEQ - 128)))  # (the last page may be outside)
        plan[h, :64] = rng.choice(out, 64)
        plan[h, 3 + h] = next(free)
        for r in range(64, 128):
            plan[h, r] = [r, rng.choice(out), -1][r % 3] if r % 9 else next(free)
        if bad_row is not None:
            plan[h, 70], plan[h, 150] = bad_row, bad_row
        plan[h, 192:] = [next(free) for _ in range(64)]
    stay = (plan < 0) | (plan >= MAX_SEQ) | (plan == bad_row)
    return plan.astype(np.int32), np.where(stay, rows, plan).astype(np.int32)


@pytest.mark.parametrize("page", [0, 128])
@pytest.mark.parametrize("R", [32, 64, 128])
@pytest.mark.parametrize("d,fmt", [(64, "int8"), (128, "e4m3")])
def test_rows_left_out_beside_movers(d, fmt, R, page):
    import torch
    cfg = config(4, 2, d)
    cache = make_cache(cfg, 2, MAX_SEQ, fmt, R, page, seed=R + d, wide=3.0)
    bad = None
    if page:
        cache.block_table[:, -1] = torch.tensor([1 << 20, -7], dtype=torch.int32)
        bad = MAX_SEQ - 5
    db = T.DeviceBatch([1, 0], [MAX_SEQ - 1] * 2, [1, 1])
    plan, filled = (np.stack([a, a]) for a in plans(2, bad))
    for poison in (False, True):
        if poison:  # a block of rows left out that is NaN: so is what moves into it
            panel = 1 if not page else int(cache.block_table[1, 0])
            cache.k_scale[panel, 0, 0] = float("nan")
        ref = kv8_ref.Cache(cache)
        T.kv8_move(cfg, cache, db, torch.from_numpy(plan).cuda())
        ref.move(db.host, filled)
        same_cache(cache, ref)
