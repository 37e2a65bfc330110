"""The norms around the layer (pre_norm, post_norm) against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import decode_ref as R
from paper_2607_04164_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


# one thread's worth, ragged chunks, each thread count of a row and its edges, the largest
SIZES = [(1, 8), (3, 16), (5, 264), (2, 512), (1, 520), (1, 2048), (7, 2056), (1030, 264), (1100, 2048), (1025, 4096),
         (1024, 4104), (9, 4104), (3, 16384), (2, 16392), (3, 32768)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SIZES)
def test_pre_norm(T, d, dtype):
    rng = np.random.default_rng(T * 7 + d)
    x, w = R.rand(rng, (T, d), 1.5, dtype), R.rand(rng, (d,), 1.0, dtype)
    x[T // 2] = 0  # an empty row: zeros, not NaN
    for weight in (w, None):
        out = B.pre_norm(x.cuda(), None if weight is None else weight.cuda(), EPS)
        want = R.np64(x) * R.inv_rms(R.np64(x), EPS) * (1.0 if weight is None else R.np64(weight))
        R.assert_rounded(out, want, R.SUM * np.abs(want), dtype, f"T={T} d={d} {dtype}")
    y = x.cuda()
    assert B.pre_norm(y, w.cuda(), EPS, out=y) is y  # in place
    assert torch.equal(y, B.pre_norm(x.cuda(), w.cuda(), EPS))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("norm,nxt", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("T,d", [(1, 2048), (5, 264), (1030, 520), (3, 16392)])
def test_post_norm(T, d, norm, nxt, gate, dtype):
    rng = np.random.default_rng(T + d)
    x, y = R.rand(rng, (T, d), 2.0, dtype), R.rand(rng, (T, d), 0.4, dtype)
    wp, wn = R.rand(rng, (d,), 1.0, dtype), R.rand(rng, (d,), 1.0, dtype)
    shape = {"none": None, "channel": (d,), "token": (T, 1), "full": (T, d)}[gate]
    g = None if shape is None else R.rand(rng, shape, 1.0, "f32" if gate == "token" else dtype)
    y[T // 2] = 0
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    r, a = B.post_norm(cu(y), cu(x), norm, w_post=cu(wp) if norm else None, gate=cu(g), res_scale=0.75,
                       next_norm=nxt, w_next=cu(wn) if nxt else None, eps=EPS)
    n64 = lambda t: None if t is None else R.np64(t)  # noqa: E731
    want, er, wa, ea = R.post_ref(R.np64(y), R.np64(x), norm, n64(wp), n64(g), 0.75, n64(wn), EPS)
    R.assert_rounded(r, want, er, dtype, "r")
    assert (a is not None) == nxt
    if nxt:
        R.assert_rounded(a, wa, ea, dtype, "a")


def test_post_norm_in_place_and_weightless():
    rng = np.random.default_rng(3)
    x, y = R.rand(rng, (37, 1032), 1.0, "bf16").cuda(), R.rand(rng, (37, 1032), 1.0, "bf16").cuda()
    g = R.rand(rng, (37, 1032), 1.0, "bf16").cuda()
    r, a = B.post_norm(y, x, True, gate=g, next_norm=True)
    x2, y2 = x.clone(), y.clone()
    r2, a2 = B.post_norm(y2, x2, True, gate=g, next_norm=True, out=x2, out_next=y2)
    assert r2 is x2 and a2 is y2 and torch.equal(r, r2) and torch.equal(a, a2)
    want, er, wa, ea = R.post_ref(R.np64(y), R.np64(x), True, None, R.np64(g), 1.0, None, 1e-6)
    R.assert_rounded(r, want, er, "bf16", "r")
    R.assert_rounded(a, wa, ea, "bf16", "a")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [264, 2048, 16392])
def test_large_and_small_rows(d, dtype):
    """Rows whose squares leave fp32: too large (the sum is taken again, scaled down) and too small (eps decides)."""
    rng = np.random.default_rng(d)
    x = R.rand(rng, (6, d), 1.0, "f32")
    scale = torch.tensor([1e30, 1e19, 3e18, 1e-30, 1e-19, 1.0])[:, None]
    x = (x * scale).to(R.TORCH[dtype])
    out = B.pre_norm(x.cuda(), None, 1e-6)
    x64 = R.np64(x)
    want = x64 * R.inv_rms(x64, 1e-6)
    R.assert_rounded(out, want, R.SUM * np.abs(want), dtype, "large and small rows")


def test_norm_stream_and_graph():
    """On another stream, and captured: replays give the eager bits with eager work between them."""
    rng = np.random.default_rng(5)
    T, d = 33, 2048
    x, y = R.rand(rng, (T, d), 1.0, "bf16").cuda(), R.rand(rng, (T, d), 1.0, "bf16").cuda()
    r, a = B.post_norm(y, x, True, next_norm=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r1, a1 = torch.empty_like(r), torch.empty_like(a)
    B.post_norm(y, x, True, next_norm=True, out=r1, out_next=a1, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(r, r1) and torch.equal(a, a1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.post_norm(y, x, True, next_norm=True, out=r1, out_next=a1)
    for k in range(3):
        y.copy_(R.rand(rng, (T, d), 1.0, "bf16"))
        r1.zero_(), a1.zero_()
        want = B.post_norm(y, x, True, next_norm=True)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(r1, want[0]) and torch.equal(a1, want[1]), f"replay {k}"


# (T, d) for the splits of a row that SIZES has not
PRE_SPLITS = [(1030, 1024), (2, 12296), (2, 24584)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", PRE_SPLITS)
def test_pre_norm_row_splits(T, d, dtype):
    rng = np.random.default_rng(T + d)
    x, w = R.rand(rng, (T, d), 1.5, dtype), R.rand(rng, (d,), 1.0, dtype)
    want = R.np64(x) * R.inv_rms(R.np64(x), EPS) * R.np64(w)
    R.assert_rounded(B.pre_norm(x.cuda(), w.cuda(), EPS), want, R.SUM * np.abs(want), dtype, f"T={T} d={d} {dtype}")


# (T, d) for every number of threads a row and chunks a thread that a post_norm can take
POST_SPLITS = [(5, 200), (1030, 256), (1030, 1032), (1024, 512), (3, 1032), (4, 2056), (5, 4104), (3, 8200), (2, 12296), (3, 24584), (2, 32768)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", POST_SPLITS)
def test_post_norm_row_splits(T, d, dtype):
    rng = np.random.default_rng(T + d)
    x, y, g = (R.rand(rng, (T, d), s, dtype) for s in (2.0, 0.4, 1.0))
    wp, wn = R.rand(rng, (d,), 1.0, dtype), R.rand(rng, (d,), 1.0, dtype)
    r, a = B.post_norm(y.cuda(), x.cuda(), True, w_post=wp.cuda(), gate=g.cuda(), res_scale=0.75, next_norm=True,
                       w_next=wn.cuda(), eps=EPS)
    n64 = R.np64
    want, er, wa, ea = R.post_ref(n64(y), n64(x), True, n64(wp), n64(g), 0.75, n64(wn), EPS)
    R.assert_rounded(r, want, er, dtype, "r")
    R.assert_rounded(a, wa, ea, dtype, "a")


def test_rows_near_the_largest_value_in_fp32():
    """A row of +-c: every step is exact but the reciprocal of the root and the product with it (the sum of squares
    has 14 + 8 bits), so the result is +-1 within two roundings, however large c is."""
    for c in [m * e for m in (103 / 64, 108 / 64, 111 / 64, 115 / 64) for e in (2.0 ** 127, 2.0 ** 100, 1.0)]:
        sign = 1.0 - 2.0 * (torch.arange(256, device="cuda") % 3 == 0)
        x = (sign * c).float()[None].expand(3, -1).contiguous()
        zero = torch.zeros_like(x)
        outs = [B.pre_norm(x, None, 1e-12), B.post_norm(x, zero, True, eps=1e-12)[0],
                B.post_norm(zero, x, False, next_norm=True, eps=1e-12)[1]]
        for out in outs:
            assert bool(((out * sign - 1).abs() <= 2 * 2.0 ** -24).all()), f"{c}: {(out * sign - 1).abs().max()}"
    # small values beside a large one, which is most of the sum: its square, the quotient, the root, the reciprocal and
    # the product, half a step each (the sum's other terms are below 2^-24 of it)
    x = torch.full((2, 256), 1e-12, device="cuda")
    x[:, 7] = 3.1e38
    x[:, 8:40] = torch.logspace(-14, 30, 32, device="cuda")
    want = R.np64(x) * R.inv_rms(R.np64(x), 0.0)
    for out in (B.pre_norm(x, None, 1e-12), B.post_norm(torch.zeros_like(x), x, False, next_norm=True, eps=1e-12)[1]):
        # (results below 2^-126 keep fewer bits)
        assert (np.abs(R.np64(out) - want) <= 4 * 2.0 ** -24 * np.abs(want) + 2.0 ** -149).all()
