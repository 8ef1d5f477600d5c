"""tri_rope against its definition in float64.

Bound: the table's angle is reduced in double precision and taken to sin and cos in
float32, the rotation is two float32 products and a sum: 8 u (|a| + |b|) m covers them,
u = 2^-24 (4 u for the table: half a step of the angle in half turns, at most 1/2 * pi u,
one of the function, one of the magnitude; 2 u for product and sum; the rest spare);
frequencies are double, good to 1e-15, times positions up to 1e6 and the float32 base,
factor, low and high as given: 1e-8.  Then half a step of the output type."""
import numpy as np
import pytest

import kv8_ref
from paper_2606_29629_amd import _lib as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
KINDS = {
    "none": dict(),
    "linear": dict(factor=4.0),
    "base": dict(factor=8.0),
    "turns": dict(factor=8.0, original_len=8192, low=1.0, high=4.0),
    "index": dict(factor=40.0, original_len=4096, low=1.0, high=32.0, magnitude=1.375),
}


def check(x, y, pos, rotary, base=1e6, interleaved=False, scaling="none", magnitude=1.0, **kw):
    import torch
    x64 = x.double().cpu().numpy()
    ref = kv8_ref.rope(x64, pos.cpu().numpy(), kv8_ref.rope_freqs(rotary, base, scaling, **kw),
                       interleaved, magnitude)
    got = y.double().cpu().numpy()
    r = rotary
    ia = np.arange(0, r, 2) if interleaved else np.arange(r // 2)
    ib = ia + (1 if interleaved else r // 2)
    size = np.zeros_like(x64)
    size[..., ia] = size[..., ib] = np.abs(x64[..., ia]) + np.abs(x64[..., ib])
    tol = (8 * U + 1e-8) * magnitude * size
    if y.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) - tol).max())
    assert np.array_equal(got[..., r:], x64[..., r:])


@pytest.mark.parametrize("tokens", [1, 2, 7, 1000])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "inter"])
@pytest.mark.parametrize("d,rotary,heads", [(128, 128, 32), (64, 64, 16), (128, 32, 3), (80, 20, 5),
                                            (256, 256, 2), (6, 2, 1), (64, 62, 4)])
def test_layouts(d, rotary, heads, interleaved, tokens):
    import torch
    g = torch.Generator(device="cuda").manual_seed(d + rotary + tokens)
    for dt in (torch.bfloat16, torch.float32):
        x = torch.randn(tokens, heads, d, generator=g, device="cuda").to(dt)
        pos = torch.randint(-1000, 1000000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
        y = T.rope(T.make_rope(d, rotary, interleaved=interleaved), x, pos)
        check(x, y, pos, rotary, interleaved=interleaved)


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("d,rotary", [(128, 128), (64, 32), (64, 2)])
def test_scaled(kind, d, rotary):
    import torch
    x = torch.randn(65, 4, d, device="cuda")
    pos = torch.arange(65, dtype=torch.int32, device="cuda") * 1999
    y = T.rope(T.make_rope(d, rotary, base=5e5, scaling=kind, **KINDS[kind]), x, pos)
    check(x, y, pos, rotary, base=5e5, scaling=kind, **KINDS[kind])


@pytest.mark.parametrize("shift", [0, 1, 4])
def test_strided_rows_in_place_and_their_neighbours(shift):
    """The q and k heads of fused rows turned in place, at an odd element offset too:
    the v heads and the rows around stay as they were."""
    import torch
    hq, hkv, d, n = 6, 2, 64, 33
    flat = torch.randn((n + 2) * (hq + 2 * hkv) * d + 8, device="cuda").bfloat16()
    rows = flat[shift:shift + (n + 2) * (hq + 2 * hkv) * d].view(n + 2, hq + 2 * hkv, d)
    before = flat.clone()
    x = rows[1:-1, :hq + hkv]
    x0 = x.clone()
    pos = torch.arange(n, dtype=torch.int32, device="cuda") + 5
    T.rope(T.make_rope(d), x, pos, out=x)
    check(x0, x, pos, d)
    x.copy_(x0)
    assert torch.equal(flat, before)
    # and to a plain tensor
    y = T.rope(T.make_rope(d, 48, interleaved=True), x, pos)
    check(x0, y, pos, 48, interleaved=True)
    assert torch.equal(flat, before)


def test_position_zero_copies_bit_for_bit():
    import torch
    x = torch.randn(3, 2, 64, device="cuda").bfloat16()
    x[0, 0, 0], x[1, 1, 40] = float("inf"), -0.0
    y = T.rope(T.make_rope(64, 32), x, torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert torch.equal(y[..., 32:], x[..., 32:]) and torch.equal(y[1:], x[1:])


def test_other_stream_and_graph():
    import torch
    x = torch.randn(70, 16, 64, device="cuda").bfloat16()
    pos = torch.arange(70, dtype=torch.int32, device="cuda")
    cfg = T.make_rope(64)
    ref = T.rope(cfg, x, pos)
    out = torch.zeros_like(x)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    T.rope(cfg, x, pos, out=out, stream=st)
    st.synchronize()
    assert torch.equal(out, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        T.rope(cfg, x, pos, out=out, stream=st)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
