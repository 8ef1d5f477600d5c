"""Weight sums beside a query that is not finite: its token's weights are NaN for the rows that
the token sees, its KV head's alone, and nothing for the rows behind it.  Compared bit for bit
with the call in which that query is zero."""
import pytest

from paper_2606_29629_amd import _lib as T
from test_gpu_kv8 import attend_cache, bf16, config

pytestmark = pytest.mark.gpu

CASES = {  # heads, batch, the token and query head in question
    "short": ((4, 2, 64), ([0, 1], [100, 60], [3, 40]), 12, 1),
    "chunks": ((7, 1, 128), ([1, 0, 2], [0, 31, 64], [70, 33, 128]), 5, 6),
    "far": ((4, 2, 64), ([0, 1], [1500, 3], [150, 2]), 77, 3),
    "large": ((28, 4, 128), (list(range(8)), [0, 40, 7, 900, 0, 1, 64, 65], [300] * 8), 1010, 15),
    "beside steps": ((8, 2, 128), ([3, 0, 1, 2], [600, 0, 33, 190], [1, 130, 1, 66]), 20, 2),
    "many": ((4, 2, 64), (list(range(40)), [9000 - 9 * i if i == 20 else 30 * i for i in range(40)],
                          [60 if i == 20 else 1 for i in range(40)]), 25, 0),
}


@pytest.mark.parametrize("value", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_rows_behind_a_poisoned_query(name, value):
    import torch
    (hq, hkv, d), batch, token, head = CASES[name]
    cfg = config(hq, hkv, d)
    db = T.DeviceBatch(*batch)
    s = int((db.cu_q.cpu() <= token).sum()) - 1
    last = batch[1][s] + token - int(db.cu_q[s])              # the last row that the token sees
    assert batch[2][s] > 1 and last + 1 < batch[1][s] + batch[2][s]
    q = bf16(db.n_tokens, hq, d, seed=2)
    outs, masses = [], []
    for v in (0.0, float(value)):
        cache = attend_cache(cfg, batch, "int8", seed=9)
        q[token, head] = v
        out, _ = T.kv8_attention(cfg, cache, db, q)
        outs.append(out)
        masses.append(cache.mass)
    slot, h = batch[0][s], head // (hq // hkv)
    assert torch.isnan(outs[1][token, head]).all() and torch.isnan(masses[1][slot, h, :last + 1]).all()
    outs[1][token, head], masses[1][slot, h, :last + 1] = outs[0][token, head], masses[0][slot, h, :last + 1]
    assert torch.equal(outs[1], outs[0]) and torch.equal(masses[1], masses[0])
    assert torch.isfinite(masses[1]).all()
