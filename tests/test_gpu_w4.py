"""Products with 4-bit weights and the quantizer, against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import decode_ref as R
from paper_2607_04164_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def _w4(t, K, group):
    return B.W4(t[0].cuda(), t[1].cuda(), None if t[2] is None else t[2].cuda(), K=K, group=group)


def _sum_error(K, group):
    """Rounding of one output's sums, relative to the sum of its terms' magnitudes (w4_magnitude): a group's
    chain of additions, then the groups', each step at most 2^-23."""
    return (group + -(-K // group) + 8) * 2.0 ** -23


def _segments(rng, rows, n, first=0):
    cut = np.sort(rng.integers(0, rows + 1, n - 1))
    return np.concatenate([[0], cut, [rows]]).astype(np.int32) + first


def _check(y, want, err, rows, what):
    got = R.np64(y)[rows]
    assert np.isfinite(got).all(), what
    tol = R.HALF["bf16"] * (np.abs(want) + err) + err
    assert (np.abs(got - want) <= tol).all(), f"{what}: {float((np.abs(got - want) / np.maximum(tol, 1e-300)).max())}"
    # the sums are far below the one rounding: over all values the error is that of a rounding (at most half a step)
    if want.size and np.linalg.norm(want):
        assert np.linalg.norm(got - want) <= R.HALF["bf16"] * np.linalg.norm(want), what


# rows that end inside a tile of 16 and a pass of 32, K that ends inside a chunk, a group and 32 columns, N inside a tile
CASES = [(1, 1, 8, 8), (1, 1, 4096, 1408), (1, 17, 24, 264), (1, 65, 72, 136), (3, 7, 40, 128), (5, 130, 16, 1408),
         (8, 64, 256, 2048), (4, 300, 56, 40), (60, 48, 176, 352),
         (1, 3, 24, 4096), (2, 150, 40, 2048), (1, 33, 16, 8192)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("n,rows,N,K", CASES)
def test_w4_matmul(n, rows, N, K, group, zeros):
    rng = np.random.default_rng(n * 1000 + rows + K)
    t = R.w4_random(rng, n, N, K, group, zeros)
    offs = _segments(rng, rows, n) if n > 1 else np.array([0, rows], np.int32)
    m = rows // 3 + 1
    a = R.rand(rng, (m, K), 1.0, "bf16")
    src = rng.integers(0, m, rows).astype(np.int32)
    w64, mag, a64 = R.w4_values(*t, K, group), R.w4_magnitude(*t, K, group), R.np64(a)[src]
    w = _w4(t, K, group)
    gathered = B.w4_matmul(torch.from_numpy(offs).cuda(), a.cuda(), w, a_rows=torch.from_numpy(src).cuda())
    plain = B.w4_matmul(torch.from_numpy(offs).cuda(), a[src.astype(np.int64)].contiguous().cuda(), w)
    assert torch.equal(gathered, plain)
    for s in range(n):
        sl = slice(offs[s], offs[s + 1])
        err = _sum_error(K, group) * np.abs(a64[sl]) @ mag[s].T
        _check(gathered, a64[sl] @ w64[s].T, err, sl, f"segment {s}")


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("n,rows,f,d", [(1, 1, 24, 40), (1, 1, 1408, 2048), (4, 33, 200, 264), (8, 250, 72, 1408)])
def test_w4_ffn(n, rows, f, d, group, zeros):
    rng = np.random.default_rng(rows + f)
    tg, tu = (R.w4_random(rng, n, f, d, group, zeros) for _ in range(2))
    td = R.w4_random(rng, n, d, f, group, zeros)
    offs = _segments(rng, rows, n) if n > 1 else np.array([0, rows], np.int32)
    a = R.rand(rng, (rows, d), 1.0, "bf16")
    wg, wu, wd = _w4(tg, d, group), _w4(tu, d, group), _w4(td, f, group)
    o = torch.from_numpy(offs).cuda()
    y, h = B.w4_ffn(o, a.cuda(), wg, wu, wd)
    assert torch.equal(h, B.w4_gate_up(o, a.cuda(), wg, wu))
    a64, h64 = R.np64(a), R.np64(h)
    e = _sum_error(d, group)
    for s in range(n):
        sl = slice(offs[s], offs[s + 1])
        g, u = a64[sl] @ R.w4_values(*tg, d, group)[s].T, a64[sl] @ R.w4_values(*tu, d, group)[s].T
        eg = e * np.abs(a64[sl]) @ R.w4_magnitude(*tg, d, group)[s].T
        eu = e * np.abs(a64[sl]) @ R.w4_magnitude(*tu, d, group)[s].T
        want = R.silu(g) * u
        # |silu'| <= 1.1; exp, reciprocal and products of silu within 2^-20
        err = 1.1 * np.abs(u) * eg + (np.abs(R.silu(g)) + 1.1 * eg) * eu + 2.0 ** -20 * np.abs(want)
        _check(h, want, err, sl, f"h of segment {s}")
        # y from the h that the call stored
        _check(y, h64[sl] @ R.w4_values(*td, f, group)[s].T,
               _sum_error(f, group) * np.abs(h64[sl]) @ R.w4_magnitude(*td, f, group)[s].T, sl, f"y of segment {s}")


def test_rows_of_no_segment_stay_as_they_are():
    rng = np.random.default_rng(2)
    n, N, K, rows = 3, 40, 160, 90
    t = R.w4_random(rng, n, N, K, 32, True)
    a = R.rand(rng, (rows, K), 1.0, "bf16").cuda()
    y = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    B.w4_matmul(torch.tensor([5, 20, 20, 61], dtype=torch.int32, device="cuda"), a, _w4(t, K, 32), y=y)
    assert bool((y[:5] == 7).all()) and bool((y[61:] == 7).all())
    w64 = R.w4_values(*t, K, 32)
    np.testing.assert_allclose(R.np64(y)[20:61], R.np64(a)[20:61] @ w64[2].T, rtol=0.01, atol=0.01)
    # offsets past the capacity or out of order touch nothing outside, and empty calls nothing at all
    y.fill_(7.0)
    B.w4_matmul(torch.tensor([90, 90, 90, 500], dtype=torch.int32, device="cuda"), a, _w4(t, K, 32), y=y)
    assert bool((y == 7).all())
    assert B.w4_matmul(torch.zeros(4, dtype=torch.int32, device="cuda"), a[:0], _w4(t, K, 32)).shape == (0, N)


def test_source_rows_out_of_range_are_clamped():
    rng = np.random.default_rng(4)
    t = R.w4_random(rng, 1, 32, 64, 64, False)
    a = R.rand(rng, (4, 64), 1.0, "bf16").cuda()
    rows = torch.tensor([-5, 0, 3, 1000], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    y = B.w4_matmul(off, a, _w4(t, 64, 64), a_rows=rows)
    want = B.w4_matmul(off, a, _w4(t, 64, 64), a_rows=rows.clamp(0, 3))
    assert torch.equal(y, want)


def test_extreme_codes_scales_and_zeros():
    """All codes 0 and 15, scale 0 and large, zero points past the codes; one hot activation row."""
    K, N, group = 256, 16, 64
    codes = torch.zeros((1, N, 128), dtype=torch.uint8)
    codes[:, 1::2] = 0xFF
    scales = torch.tensor([0.0, 1.0, -2.0, 1e30]).to(torch.bfloat16).repeat(1, N, 1)
    zeros = torch.tensor([3, 0, 15, 255], dtype=torch.uint8).repeat(1, N, 1)
    a = torch.zeros((5, K), dtype=torch.bfloat16)
    for i, k in enumerate((0, 63, 64, 191, 255)):
        a[i, k] = 1.0
    y = B.w4_matmul(torch.tensor([0, 5], dtype=torch.int32, device="cuda"), a.cuda(),
                    _w4((codes, scales, zeros), K, group))
    want = R.np64(a) @ R.w4_values(codes, scales, zeros, K, group)[0].T
    np.testing.assert_allclose(R.np64(y), want, rtol=2.0 ** -8)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(40, 264), (40, 1408), (72, 40)])
def test_a_row_with_nan_scales_is_the_only_one(N, K, group):
    """Also where a unit of columns ends inside the row, so that the next row's scales are loaded with it."""
    rng = np.random.default_rng(N + K + group)
    t = R.w4_random(rng, 2, N, K, group, True)
    a = R.rand(rng, (60, K), 1.0, "bf16").cuda()
    off = torch.tensor([0, 20, 60], dtype=torch.int32, device="cuda")
    clean = B.w4_matmul(off, a, _w4(t, K, group))
    scales = t[1].clone()
    scales[0, 5] = float("nan")
    scales[1, 0] = float("inf")
    scales[1, N - 1] = float("nan")
    y = B.w4_matmul(off, a, _w4((t[0], scales, t[2]), K, group))
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[:20, 5] = True
    bad[20:, 0] = True
    bad[20:, N - 1] = True
    assert not torch.isfinite(y[bad].float()).any()
    assert torch.equal(y[~bad], clean[~bad])


def quantize_ref(w32, group, zeros):
    """The quantizer's definition, element by element in fp32."""
    n, N, K = w32.shape
    ng, pitch = -(-K // group), 16 * (-(-K // 32))
    codes = np.full((n, N, 2 * pitch), 8, np.int64)
    scales, zps = np.zeros((n, N, ng), np.float32), np.zeros((n, N, ng), np.uint8)
    for g in range(ng):
        v = w32[:, :, g * group:min(K, (g + 1) * group)]
        lo, hi = np.minimum(v.min(-1), 0), np.maximum(v.max(-1), 0)
        s = ((hi - lo) / np.float32(15) if zeros else np.maximum(hi, -lo) / np.float32(7)).astype(np.float32)
        s = torch.from_numpy(s).to(torch.bfloat16).float().numpy()
        safe = np.where(s > 0, s, np.float32(1))
        z = np.clip(np.rint(-lo / safe), 0, 15) if zeros else np.full(s.shape, 8.0)
        if zeros:
            z = np.where(s > 0, z, 0)
        q = np.where(s[..., None] > 0, np.rint(v / safe[..., None]), 0) + z[..., None]
        codes[:, :, g * group:g * group + v.shape[-1]] = np.clip(q, 0 if zeros else 1, 15)
        scales[:, :, g], zps[:, :, g] = s, z
    packed = (codes[:, :, 0::2] | (codes[:, :, 1::2] << 4)).astype(np.uint8)
    return packed, scales, zps


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,N,K", [(1, 3, 8), (2, 5, 40), (1, 16, 256), (3, 7, 1408)])
def test_w4_quantize(n, N, K, group, zeros, dtype):
    rng = np.random.default_rng(K + group)
    w = R.rand(rng, (n, N, K), 0.02, dtype)
    w[0, 0, :] = 0  # groups of zeros
    w[0, N - 1] = w[0, N - 1].abs()  # one-sided groups
    q = B.w4_quantize(w.cuda(), group, zeros)
    codes, scales, zps = quantize_ref(w.float().numpy(), group, zeros)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    assert np.array_equal(q.scales.float().cpu().numpy(), scales)
    if zeros:
        assert np.array_equal(q.zeros.cpu().numpy(), zps)
    else:
        assert q.zeros is None
    # a code is at most half a step off (the bf16 scale moves the ends by 2^-8 of 7 or 15 steps)
    back = R.w4_values(q.codes, q.scales, q.zeros, K, group)
    step = np.repeat(scales.astype(np.float64), group, axis=2)[:, :, :K]
    assert (np.abs(back - R.np64(w)) <= (0.5 + (1.0 if zeros else 0.0) * 0.5 + 15 * 2.0 ** -8) * step + 1e-30).all()


def test_w4_graph_and_stream():
    rng = np.random.default_rng(9)
    n, rows, f, d = 4, 40, 96, 256
    tg, tu, td = (R.w4_random(rng, n, *s, 64, True) for s in ((f, d), (f, d), (d, f)))
    ws = _w4(tg, d, 64), _w4(tu, d, 64), _w4(td, f, 64)
    o = torch.from_numpy(_segments(rng, rows, n)).cuda()
    a = R.rand(rng, (rows, d), 1.0, "bf16").cuda()
    y, h = B.w4_ffn(o, a, *ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y1, h1 = torch.zeros_like(y), torch.zeros_like(h)
    B.w4_ffn(o, a, *ws, y=y1, h=h1, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y, y1) and torch.equal(h, h1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.w4_ffn(o, a, *ws, y=y1, h=h1)
    for k in range(3):
        a.copy_(R.rand(rng, (rows, d), 1.0, "bf16"))
        want = B.w4_ffn(o, a, *ws)
        y1.zero_(), h1.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y1, want[0]) and torch.equal(h1, want[1]), f"replay {k}"


def test_weights_of_another_device_are_refused():
    rng = np.random.default_rng(8)
    w = _w4(R.w4_random(rng, 1, 32, 32, 32, False), 32, 32)
    a, off = R.rand(rng, (2, 32), 1.0, "bf16").cuda(), torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    w.device += 1
    for call in (lambda: B.w4_matmul(off, a, w), lambda: B.w4_gate_up(off, a, w, w), lambda: B.w4_ffn(off, a, w, w, w)):
        with pytest.raises(ValueError, match="4-bit weights are on GPU"):
            call()


@pytest.mark.parametrize("n,rows", [(65, 64), (200, 300), (256, 1000)])
def test_more_segments_than_lanes(n, rows):
    rng = np.random.default_rng(n)
    N, K, group = 24, 72, 32
    t = R.w4_random(rng, n, N, K, group, True)
    offs = _segments(rng, rows, n)
    offs[n // 2:] = offs[n // 2]  # the second half's rows belong to the last segment
    offs[n] = rows
    a = R.rand(rng, (rows, K), 1.0, "bf16")
    y = B.w4_matmul(torch.from_numpy(offs).cuda(), a.cuda(), _w4(t, K, group))
    w64, mag, a64 = R.w4_values(*t, K, group), R.w4_magnitude(*t, K, group), R.np64(a)
    for s in range(n):
        sl = slice(offs[s], offs[s + 1])
        _check(y, a64[sl] @ w64[s].T, _sum_error(K, group) * np.abs(a64[sl]) @ mag[s].T, sl, f"segment {s}")


def test_more_passes_than_a_launch_has():
    """160 segments of a row and 2^20 columns: 16384 blocks of columns, of which a launch holds 128 passes."""
    n, N, K, group = 160, 1 << 20, 8, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    codes = torch.randint(0, 256, (n, N, 16), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((n, N, 1), generator=g, device="cuda") + 0.5).to(torch.bfloat16)
    a = torch.randn((n, K), generator=g, device="cuda").to(torch.bfloat16)
    y = B.w4_matmul(torch.arange(n + 1, dtype=torch.int32, device="cuda"), a, B.W4(codes, scales, K=K, group=group))
    cols = torch.cat([torch.arange(40), torch.arange(40, N - 40, N // 41), torch.arange(N - 40, N)]).cuda()
    t = codes[:, cols].cpu(), scales[:, cols].cpu(), None
    w64, mag, a64 = R.w4_values(*t, K, group), R.w4_magnitude(*t, K, group), R.np64(a)
    part = y[:, cols]
    for s in range(n):
        sl = slice(s, s + 1)
        _check(part, a64[sl] @ w64[s].T, _sum_error(K, group) * np.abs(a64[sl]) @ mag[s].T, sl, f"segment {s}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_quantize_of_a_range_past_the_largest_value(group, dtype):
    """max - min is infinite in fp32, the scale is not."""
    K = 264
    rng = np.random.default_rng(group)
    w = R.rand(rng, (1, 6, K), 1.0, dtype)
    w[0, :, 3::group], w[0, :, 5::group] = 3.0e38, -2.5e38
    w[0, 1] *= -1
    q = B.w4_quantize(w.cuda(), group, True)
    assert bool(torch.isfinite(q.scales).all())
    w64, s, back = R.np64(w), R.np64(q.scales), R.w4_values(q.codes, q.scales, q.zeros, K, group)
    ng = -(-K // group)
    span = np.stack([np.maximum(v.max(-1), 0) - np.minimum(v.min(-1), 0)
                     for v in (w64[..., g * group:(g + 1) * group] for g in range(ng))], -1) / 15
    # rounded to bf16 from a value with the roundings of a difference and a quotient
    assert (np.abs(s - span) <= (R.HALF["bf16"] + 2 * R.HALF["f32"]) * span).all()
    step = np.repeat(s, group, axis=2)[:, :, :K]
    assert (np.abs(back - w64) <= (1.0 + 15 * 2.0 ** -8) * step).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("zeros", [False, True], ids=["sym", "zeros"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [8, 200, 384])
def test_w4_quantize_marks_groups_that_are_not_finite(K, group, zeros, dtype):
    """A NaN or infinite weight makes its group's scale NaN; every other group is as without it."""
    rng = np.random.default_rng(K + group)
    w = R.rand(rng, (2, 9, K), 0.02, dtype)
    clean = B.w4_quantize(w.cuda(), group, zeros)
    ng = -(-K // group)
    bad = np.zeros((2, 9, ng), bool)
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"), float("nan"))):
        for row, k in ((2 * i, (7 * i + 3) % K), (2 * i, K - 1), (2 * i + 1, K // 2)):
            w[i % 2, row, k] = v
            bad[i % 2, row, k // group] = True
    q = B.w4_quantize(w.cuda(), group, zeros)
    back, was = (R.w4_values(t.codes, t.scales, t.zeros, K, group) for t in (q, clean))
    cols = np.repeat(bad, group, axis=2)[:, :, :K]
    assert np.isnan(back[cols]).all() and np.array_equal(back[~cols], was[~cols])
    assert bool((q.codes[..., -(-K // 2):] == 0x88).all())  # (padding)


def _same_beyond(got, want, what):
    """Infinities and NaN where they belong."""
    for f in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(f(got), f(want)), f"{what}: {f.__name__}"


# (n, rows, N, K): one tile of columns a wave, and four
BEYOND = [(1, 5, 40, 264), (3, 40, 72, 512), (8, 60, 2048, 264), (8, 60, 2048, 256)]


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("n,rows,N,K", BEYOND)
def test_activations_whose_sums_leave_fp32(n, rows, N, K, group, zeros):
    """Finite products of activations near the largest value, whose sums with the codes + 16 would be infinite,
    and infinite activations: what the definition gives. Rows beside them are as they would be alone."""
    rng = np.random.default_rng(rows + K)
    t = R.w4_random(rng, n, N, K, group, zeros)
    offs = _segments(rng, rows, n) if n > 1 else np.array([0, rows], np.int32)
    a = R.rand(rng, (rows, K), 1.0, "bf16")
    off, w = torch.from_numpy(offs).cuda(), _w4(t, K, group)
    clean = B.w4_matmul(off, a.cuda(), w)
    kind = np.arange(rows) % 5  # 0: as it was
    for r in range(rows):
        k = rng.choice(K, 4, replace=False)
        if kind[r] == 1:
            a[r, k[0]] = 3.3e38 * (-1) ** r
        elif kind[r] == 2:  # a sum that cancels
            a[r, k[0]], a[r, k[1]], a[r, k[2]] = 3.0e38, 3.0e38, -3.0e38
        elif kind[r] == 3:
            a[r, k[0]] = float("inf") * (-1) ** r
        elif kind[r] == 4:
            a[r, k[3]] = float("nan") if r % 2 else float("inf")
    y = B.w4_matmul(off, a.cuda(), w)
    keep = torch.from_numpy(kind == 0).cuda()
    assert torch.equal(y[keep], clean[keep])
    with np.errstate(invalid="ignore"):
        for s in range(n):
            rs = np.arange(offs[s], offs[s + 1])
            w64, mag = R.w4_values(*t, K, group)[s], R.w4_magnitude(*t, K, group)[s]
            finite = rs[kind[rs] < 3]
            a64 = R.np64(a)[finite]
            _check(y, a64 @ w64.T, _sum_error(K, group) * np.abs(a64) @ mag.T, finite, f"segment {s}")
            rest = rs[kind[rs] >= 3]
            want = (R.np64(a)[rest][:, None, :] * w64[None]).sum(-1)
            _same_beyond(R.np64(y)[rest], want, f"segment {s}")


@pytest.mark.parametrize("n,rows,f,d", [(2, 9, 40, 264), (8, 70, 1024, 264)])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True)])
def test_hidden_values_whose_sums_leave_fp32(n, rows, f, d, group, zeros):
    """gate_up of large activations, and a product of the infinite h that it stored."""
    rng = np.random.default_rng(rows + f)
    tg, tu = (R.w4_random(rng, n, f, d, group, zeros) for _ in range(2))
    td = R.w4_random(rng, n, d, f, group, zeros)
    tu[1][:, 1::2, 0] = 0  # every second hidden value has no part of the large activation in its factor
    offs = _segments(rng, rows, n)
    a = R.rand(rng, (rows, d), 1.0, "bf16")
    a[::2, 3] = 3.0e38
    off = torch.from_numpy(offs).cuda()
    y, h = B.w4_ffn(off, a.cuda(), _w4(tg, d, group), _w4(tu, d, group), _w4(td, f, group))
    a64, h64, y64 = R.np64(a), R.np64(h), R.np64(y)
    e = _sum_error(d, group)
    with np.errstate(invalid="ignore", over="ignore"):
        for s in range(n):
            sl = slice(offs[s], offs[s + 1])
            wg, wu, wd = (R.w4_values(*t, K, group)[s] for t, K in ((tg, d), (tu, d), (td, f)))
            g, u = a64[sl] @ wg.T, a64[sl] @ wu.T
            eg = e * np.abs(a64[sl]) @ R.w4_magnitude(*tg, d, group)[s].T
            eu = e * np.abs(a64[sl]) @ R.w4_magnitude(*tu, d, group)[s].T
            want = R.silu(g) * u
            # (a product past the type's largest value, by more than its error, is infinite)
            err = 1.1 * np.abs(u) * eg + (np.abs(R.silu(g)) + 1.1 * eg) * eu + 2.0 ** -20 * np.abs(want)
            tol = R.HALF["bf16"] * (np.abs(want) + err) + err
            past = np.abs(want) - tol > float(torch.finfo(torch.bfloat16).max)
            assert past.any() or sl.stop - sl.start < 2
            assert np.array_equal(h64[sl][past], np.sign(want[past]) * np.inf)
            sure = np.abs(want) + tol < float(torch.finfo(torch.bfloat16).max)
            assert (np.abs(h64[sl] - want)[sure] <= tol[sure]).all()
            hs = h64[sl]
            wanty = (hs[:, None, :] * wd[None]).sum(-1)
            fin = np.isfinite(hs).all(-1)
            _same_beyond(y64[sl][~fin], wanty[~fin], f"segment {s}")
            tol = _sum_error(f, group) * np.abs(hs[fin]) @ R.w4_magnitude(*td, f, group)[s].T
            tol = R.HALF["bf16"] * (np.abs(wanty[fin]) + tol) + tol
            assert (np.abs(y64[sl][fin] - wanty[fin]) <= tol).all()


def test_outputs_are_memory_of_the_calls_stream():
    """A call on another stream than the current one writes no memory that the current stream may still read."""
    rng = np.random.default_rng(12)
    w = _w4(R.w4_random(rng, 2, 64, 64, 32, False), 64, 32)
    a, off = R.rand(rng, (8, 64), 1.0, "bf16").cuda(), torch.tensor([0, 5, 8], dtype=torch.int32, device="cuda")
    calls = {"matmul": lambda s: (B.w4_matmul(off, a, w, stream=s),), "gate_up": lambda s: (B.w4_gate_up(off, a, w, w, stream=s),),
             "ffn": lambda s: B.w4_ffn(off, a, w, w, w, stream=s), "pre": lambda s: (B.pre_norm(a, stream=s),),
             "post": lambda s: B.post_norm(a, a, next_norm=True, stream=s),
             "quantize": lambda s: (lambda q: (q.codes, q.scales, q.zeros))(B.w4_quantize(a[None], 32, True, stream=s))}
    for name, call in calls.items():
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        outs = call(s)
        torch.cuda.synchronize()
        want = call(None)
        for got, w0 in zip(outs, want):
            assert torch.equal(got, w0), name
            seg, = (g for g in torch.cuda.memory_snapshot()
                    if g["address"] <= got.data_ptr() < g["address"] + g["total_size"])
            assert seg["stream"] == s.cuda_stream, name


# (n, rows, N, K): at least 256 blocks of four tiles a wave; rows that end a tile of 16 and a pass of 32, K in whole
# units and not, units that the eight waves do not share evenly, the last tile of columns cut
FOUR_TILES = [(8, 250, 4096, 2048), (4, 100, 4096, 4360), (6, 96, 2808, 4096), (1, 16, 16384, 264), (1, 32, 8200, 512),
              (1, 64, 5464, 40), (3, 7, 8192, 264)]
# the same rows for one tile a wave
ONE_TILE = [(1, 16, 264, 2048), (1, 32, 136, 8200), (1, 64, 40, 4360), (1, 33, 64, 4096)]


@pytest.mark.parametrize("group,zeros", [(32, True), (32, False), (64, True), (64, False), (128, True), (128, False)])
@pytest.mark.parametrize("n,rows,N,K", FOUR_TILES + ONE_TILE)
def test_w4_matmul_by_tiles(n, rows, N, K, group, zeros):
    rng = np.random.default_rng(rows + N + K)
    t = R.w4_random(rng, n, N, K, group, zeros)
    offs = _segments(rng, rows, n) if n > 1 else np.array([0, rows], np.int32)
    a = R.rand(rng, (rows, K), 1.0, "bf16")
    y = B.w4_matmul(torch.from_numpy(offs).cuda(), a.cuda(), _w4(t, K, group))
    # (some of the columns: the first and last tiles, and every 37th)
    cols = np.unique(np.concatenate([np.arange(min(N, 80)), np.arange(0, N, 37), np.arange(max(N - 80, 0), N)]))
    part = y[:, torch.from_numpy(cols).cuda()]
    tc = t[0][:, cols], t[1][:, cols], None if t[2] is None else t[2][:, cols]
    w64, mag, a64 = R.w4_values(*tc, K, group), R.w4_magnitude(*tc, K, group), R.np64(a)
    for s in range(n):
        sl = slice(offs[s], offs[s + 1])
        _check(part, a64[sl] @ w64[s].T, _sum_error(K, group) * np.abs(a64[sl]) @ mag[s].T, sl, f"segment {s}")


# (n, rows, f, d): gate_up with four tiles a wave
FFN_FOUR_TILES = [(8, 250, 1408, 2048), (8, 200, 1400, 2312), (4, 130, 1408, 4096), (6, 60, 1416, 264), (1, 64, 5464, 264)]


@pytest.mark.parametrize("group,zeros", [(32, True), (32, False), (64, True), (64, False), (128, True), (128, False)])
@pytest.mark.parametrize("n,rows,f,d", FFN_FOUR_TILES)
def test_w4_ffn_by_tiles(n, rows, f, d, group, zeros):
    rng = np.random.default_rng(rows + f + d)
    tg, tu = (R.w4_random(rng, n, f, d, group, zeros) for _ in range(2))
    td = R.w4_random(rng, n, d, f, group, zeros)
    offs = _segments(rng, rows, n) if n > 1 else np.array([0, rows], np.int32)
    m = rows // 4 + 1
    a = R.rand(rng, (m, d), 1.0, "bf16")
    src = rng.integers(0, m, rows).astype(np.int32)
    y, h = B.w4_ffn(torch.from_numpy(offs).cuda(), a.cuda(), _w4(tg, d, group), _w4(tu, d, group), _w4(td, f, group),
                    a_rows=torch.from_numpy(src).cuda())
    a64, h64 = R.np64(a)[src], R.np64(h)
    hc = np.unique(np.concatenate([np.arange(min(f, 70)), np.arange(0, f, 29), np.arange(max(f - 70, 0), f)]))
    yc = np.unique(np.concatenate([np.arange(min(d, 70)), np.arange(0, d, 29), np.arange(max(d - 70, 0), d)]))
    pick = lambda t, c: (t[0][:, c], t[1][:, c], None if t[2] is None else t[2][:, c])  # noqa: E731
    wg, mg = R.w4_values(*pick(tg, hc), d, group), R.w4_magnitude(*pick(tg, hc), d, group)
    wu, mu = R.w4_values(*pick(tu, hc), d, group), R.w4_magnitude(*pick(tu, hc), d, group)
    wd, md = R.w4_values(*pick(td, yc), f, group), R.w4_magnitude(*pick(td, yc), f, group)
    hp, yp = h[:, torch.from_numpy(hc).cuda()], y[:, torch.from_numpy(yc).cuda()]
    e = _sum_error(d, group)
    for s in range(n):
        sl = slice(offs[s], offs[s + 1])
        g, u = a64[sl] @ wg[s].T, a64[sl] @ wu[s].T
        eg, eu = e * np.abs(a64[sl]) @ mg[s].T, e * np.abs(a64[sl]) @ mu[s].T
        want = R.silu(g) * u
        err = 1.1 * np.abs(u) * eg + (np.abs(R.silu(g)) + 1.1 * eg) * eu + 2.0 ** -20 * np.abs(want)
        _check(hp, want, err, sl, f"h of segment {s}")
        _check(yp, h64[sl] @ wd[s].T, _sum_error(f, group) * np.abs(h64[sl]) @ md[s].T, sl, f"y of segment {s}")
