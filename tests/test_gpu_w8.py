"""Rows in 8 bits and the grouped products with them, against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2607_04164_amd import binding as B

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8   # one rounding to bf16, relative
F32 = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def rounded64(x):
    """The quantizer's definition in 64 bits: (codes, scales) of the rows of x [.., K]. The scale is fp32's own
    quotient; x / scale in 64 bits tells every tie, since x - scale (code + 1/2) is 0 or at least 2^-32 of x."""
    v = x.double()
    m = v.abs().amax(dim=-1)
    s = (m / 127.0).float().double()
    s = torch.where(s < 2.0 ** -120, torch.zeros_like(s), s)
    ok = torch.isfinite(v).all(dim=-1)
    s = torch.where(ok, s, torch.full_like(s, float("nan")))
    q = torch.round(v / s[..., None])
    return torch.where((s > 0)[..., None], q, torch.zeros_like(q)), s


def weights(g, n, N, K, std=None):
    """Random codes and scales; the padding holds what must not matter: the activations' padding is zeros."""
    P = B.w8_row_bytes(K)
    codes = torch.randint(-127, 128, (n, N, P), generator=g, device="cuda", dtype=torch.int8)
    scales = (torch.rand((n, N), generator=g, device="cuda") + 0.5) * (std or 1.0 / (73.0 * np.sqrt(K)))
    return B.W8(codes, scales, K=K)


def segments(seed, rows, n, first=0):
    if n == 1:
        return np.array([first, first + rows], np.int32)
    cut = np.sort(np.random.default_rng(seed).integers(0, rows + 1, n - 1))
    return (np.concatenate([[0], cut, [rows]]) + first).astype(np.int32)


def products64(q, s, offs, w):
    """[rows, N] in 64 bits from the rows' codes and scales (rows of no segment: 0). The sums are whole numbers
    below 2^53: exact."""
    n, N, K = w.shape
    y = torch.zeros((q.shape[0], N), dtype=torch.float64, device="cuda")
    for i in range(n):
        b, e = int(offs[i]), int(offs[i + 1])
        if e > b:
            y[b:e] = (q[b:e] @ w.codes[i, :, :K].double().t()) * s[b:e, None] * w.scales[i].double()[None]
    return y


def check_product(y, want, what):
    """The sum to fp32, two products, one rounding to bf16."""
    err = (y.double() - want).abs()
    tol = want.abs() * (BF16 + 4 * F32)
    assert bool(torch.isfinite(y.float()).all()), what
    assert bool((err <= tol).all()), (what, float((err / tol.clamp(min=1e-300)).max()))


def check_hidden(h, gate, up, what):
    """silu(g) u: g and u are off by 3 roundings each, so e^-g by 3|g| more, and exp (its argument's rounding |g|, its
    own), sum, reciprocal (two) and the products add 10; then bf16."""
    want = gate * torch.sigmoid(gate) * up
    tol = want.abs() * (BF16 + (4 * gate.abs() + 16) * F32) + 1e-37
    err = (h.double() - want).abs()
    assert bool((err <= tol).all()), (what, float((err / tol).max()))


# ---------------------------------------------------------------------------
# the quantizer

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 8), (3, 40), (5, 128), (7, 136), (64, 1024), (33, 1048), (6, 2048), (9, 4096),
                                    (4, 8192), (5, 8200), (3, 16384), (2, 20008), (2, 131072), (3001, 264), (600, 2048)])
def test_quantize(rows, K, dtype):
    g = gen(rows * 7 + K)
    x = randn(g, rows, K, dtype=dtype) * torch.exp(2 * torch.randn((rows, 1), generator=g, device="cuda")).to(dtype)
    x[0] = 0
    if rows > 2:
        x[1] = x[1].abs()
        x[2, K - 1] = 1000.0
    q = B.a8_quantize(x)
    want, s = rounded64(x)
    assert torch.equal(q.scales.double(), s)
    assert torch.equal(q.codes[:, :K].double(), want)
    assert not q.codes[:, K:].any()
    again = B.A8(torch.full_like(q.codes, 99), torch.full_like(q.scales, 99.0), K=K)
    assert B.a8_quantize(x, out=again) is again
    assert torch.equal(again.codes, q.codes) and torch.equal(again.scales, q.scales)
    if rows % 3 == 0:  # the same rows as a weight stack
        w = B.w8_quantize(x.view(3, rows // 3, K))
        assert torch.equal(w.codes.view_as(q.codes), q.codes) and torch.equal(w.scales.view(-1), q.scales)


@pytest.mark.parametrize("rows,K", [((1 << 26) + 5, 8), ((1 << 24) + 3, 1032)])
def test_quantize_more_workgroups_than_a_grid_dimension_holds(rows, K):
    """Rows of one power of two each, and its half: codes 127 and -64 (fp32's 1/127 is below 1/127, so just past -63.5)."""
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    exponent = (torch.arange(rows, device="cuda") % 7).to(torch.bfloat16)
    x[:, 0], x[:, K - 1] = torch.exp2(exponent), -torch.exp2(exponent) / 2
    q = B.a8_quantize(x)
    assert torch.equal(q.scales, torch.exp2(exponent.float()) / 127)
    assert bool((q.codes[:, 0] == 127).all()) and bool((q.codes[:, K - 1] == -64).all())
    for part in (slice(0, 9), slice((1 << 24) - 4, (1 << 24) + 4), slice(rows - 9, rows)):
        assert int(q.codes[part].ne(0).sum()) == 2 * q.codes[part].shape[0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_quantize_ties_go_to_even(dtype):
    """Scale 1 (a row whose largest is 127) and powers of two beside it: every half is a tie."""
    half = torch.arange(-126.5, 127, 1.0, device="cuda")
    half = half[half.abs() < 64] if dtype is torch.bfloat16 else half  # (halves that bf16 holds)
    x = torch.cat([half, torch.tensor([127.0, -127.0], device="cuda")])
    x = torch.cat([x, torch.zeros(-x.numel() % 8, device="cuda")])
    rows = torch.stack([x, -x, x * 2.0 ** 40, x * 2.0 ** -40]).to(dtype)
    q = B.a8_quantize(rows)
    assert torch.equal(q.scales, torch.tensor([1.0, 1.0, 2.0 ** 40, 2.0 ** -40], device="cuda"))
    want, _ = rounded64(rows)
    assert torch.equal(q.codes[:, :x.numel()].double(), want)
    assert bool((q.codes[0, :half.numel()] % 2 == 0).all())


def test_quantize_near_ties():
    """fp32 values on either side of half a step, for scales with full significands."""
    g = gen(5)
    top = torch.rand((64, 1), generator=g, device="cuda") * 100 + 1
    s = (top.double() / 127).float()
    code = torch.arange(0, 126, device="cuda").float()
    mid = ((code.double() + 0.5)[None] * s.double()).float()
    up = torch.nextafter(mid, torch.full_like(mid, 1e30))
    down = torch.nextafter(mid, torch.zeros_like(mid))
    x = torch.cat([top, -top, mid, -mid, up, -up, down, -down], dim=1)
    x = torch.cat([x, torch.zeros((64, -x.shape[1] % 8), device="cuda")], dim=1).contiguous()
    q, (want, scales) = B.a8_quantize(x), rounded64(x)
    assert torch.equal(q.scales.double(), scales)
    assert torch.equal(q.codes[:, :x.shape[1]].double(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("K", [8, 264, 2056, 20008])
def test_quantize_extremes(K, dtype):
    g = gen(K)
    x = randn(g, 12, K, dtype=dtype)
    x[0, 3] = float("nan")
    x[1, K - 1] = float("inf")
    x[2, 0] = -float("inf")
    x[3] = 0
    x[4] = torch.finfo(dtype).max
    x[5] = -torch.finfo(dtype).max
    x[6] = x[6] * 1e-37     # scale below 2^-120
    x[7] = x[7] * 2.0 ** -100
    x[8] = torch.finfo(dtype).smallest_normal
    x[9, :] = 0
    x[9, K // 2] = -1.0
    q, (want, s) = B.a8_quantize(x), rounded64(x)
    assert torch.equal(torch.isnan(q.scales), torch.isnan(s))
    assert torch.isnan(q.scales[:3]).all() and not torch.isnan(q.scales[3:]).any()
    assert torch.equal(q.scales[3:].double(), s[3:])
    assert torch.equal(q.codes[:, :K].double(), want)
    assert float(q.scales[6]) == 0 and float(q.scales[7]) > 0 and float(q.scales[8]) == 0


# ---------------------------------------------------------------------------
# products

# few rows on both of their kernels; large tiles whole and half, with and without the VAR kernel; K of one K-step and
# of many, N inside a tile, rows that end inside one
CASES = [(1, 1, 8, 8), (1, 1, 4096, 1408), (1, 17, 24, 264), (3, 7, 40, 128), (5, 130, 16, 1408), (8, 64, 256, 2048),
         (60, 48, 176, 352), (60, 300, 1408, 256), (1, 64, 2816, 2048), (4, 12, 4096, 14336), (15, 40, 1408, 2048),
         (1, 9, 136, 2816),
         (1, 65, 72, 136), (5, 777, 1000, 1048), (3, 700, 264, 64), (2, 3000, 264, 520), (1, 1000, 8, 8),
         (7, 2000, 136, 384), (1, 800, 1032, 128),
         # large tiles: whole ones, and half ones for short segments; K of one K-step, N and rows inside a tile
         (1, 9000, 1032, 136), (15, 6000, 520, 264), (40, 20000, 136, 40), (3, 40000, 72, 8), (2, 9000, 264, 1400)]


@pytest.mark.parametrize("n,rows,N,K", CASES)
def test_w8_matmul(n, rows, N, K):
    g = gen(n * 1000 + rows + K)
    w = weights(g, n, N, K)
    offs = segments(rows + K, rows, n)
    m = rows // 3 + 1
    a = randn(g, m, K)
    src = torch.randint(0, m, (rows,), generator=g, device="cuda", dtype=torch.int32)
    o = torch.from_numpy(offs).cuda()
    q, s = rounded64(a)
    want = products64(q[src.long()], s[src.long()], offs, w)
    y = B.w8_matmul(o, a, w, a_rows=src)
    check_product(y, want, "gathered")
    assert torch.equal(B.w8_matmul(o, a[src.long()].contiguous(), w), y)
    a8 = B.a8_quantize(a)
    assert torch.equal(B.w8_matmul(o, a8, w, a_rows=src), y)
    ws = B.new_w8_workspace(m, K, "cuda")
    assert torch.equal(B.w8_matmul(o, a, w, a_rows=src, workspace=ws), y)


@pytest.mark.parametrize("n,rows,f,d", [(1, 1, 24, 40), (1, 1, 1408, 2048), (4, 33, 200, 264), (8, 250, 72, 1408),
                                        (15, 4, 1408, 2048), (3, 500, 136, 128), (2, 2000, 392, 264), (5, 900, 520, 72),
                                        (2, 9000, 392, 264), (15, 9000, 520, 72)])
def test_w8_ffn(n, rows, f, d):
    g = gen(rows + f)
    wg, wu, wd = weights(g, n, f, d), weights(g, n, f, d), weights(g, n, d, f)
    offs = segments(rows, rows, n)
    o = torch.from_numpy(offs).cuda()
    a = randn(g, rows, d)
    y, h = B.w8_ffn(o, a, wg, wu, wd)
    assert torch.equal(h, B.w8_gate_up(o, a, wg, wu))
    assert torch.equal(y, B.w8_matmul(o, h, wd))
    q, s = rounded64(a)
    check_hidden(h, products64(q, s, offs, wg), products64(q, s, offs, wu), "h")
    # y from the h that the call stored
    q, s = rounded64(h)
    check_product(y, products64(q, s, offs, wd), "y")
    # gathered, the activations rounded before, a workspace of the caller's
    src = torch.randperm(rows, generator=g, device="cuda").int()
    back = torch.empty_like(a)
    back[src.long()] = a
    ws = B.new_w8_workspace(rows, d, "cuda", rows_cap=rows, d_ff=f)
    for x in (back, B.a8_quantize(back)):
        y1, h1 = B.w8_ffn(o, x, wg, wu, wd, a_rows=src, workspace=ws)
        assert torch.equal(y1, y) and torch.equal(h1, h)


@pytest.mark.parametrize("n,rows,N,K", [(1, 4000, 1032, 8192), (4, 9000, 520, 14336), (15, 9000, 520, 14336),
                                        (2, 257, 264, 20000)])
def test_split_tiles_have_the_same_bits(n, rows, N, K):
    """K long enough that the last tiles' K loops are split over the workgroups."""
    g = gen(K)
    w, w1 = weights(g, n, N, K), weights(g, n, N, K)
    offs = segments(rows, rows, n)
    o = torch.from_numpy(offs).cuda()
    a = B.a8_quantize(randn(g, rows, K))
    whole, split = (B.new_w8_workspace(0, K, "cuda", split=s) for s in (False, True))
    assert split.numel() > whole.numel() + (64 << 20)
    y = B.w8_matmul(o, a, w, workspace=whole)
    q, s = a.codes[:, :K].double(), a.scales.double()
    check_product(y, products64(q, s, offs, w), "whole")
    assert torch.equal(B.w8_matmul(o, a, w, workspace=split), y)
    h = B.w8_gate_up(o, a, w, w1, workspace=whole)
    assert torch.equal(B.w8_gate_up(o, a, w, w1, workspace=split), h)
    check_hidden(h, products64(q, s, offs, w), products64(q, s, offs, w1), "gated")


@pytest.mark.parametrize("rows,first,last", [(90, 5, 61), (2000, 300, 1500), (20000, 300, 15000)])
def test_rows_of_no_segment_stay_as_they_are(rows, first, last):
    g = gen(rows)
    n, d, f = 3, 160, 136
    offs = np.array([first, first + 15, first + 15, last], np.int32)
    o = torch.from_numpy(offs).cuda()
    wg, wu, wd = weights(g, n, f, d), weights(g, n, f, d), weights(g, n, d, f)
    a = randn(g, rows, d)
    a[first - 1], a[last] = float("nan"), float("inf")
    y = torch.full((rows, d), 7.0, dtype=torch.bfloat16, device="cuda")
    h = torch.full((rows, f), 7.0, dtype=torch.bfloat16, device="cuda")
    B.w8_ffn(o, a, wg, wu, wd, y=y, h=h)
    for t in (y, h):
        assert bool((t[:first] == 7).all()) and bool((t[last:] == 7).all())
    q, s = rounded64(h)
    check_product(y[first:last], products64(q, s, offs, wd)[first:last], "y")
    y.fill_(7.0)
    B.w8_matmul(torch.tensor([rows, rows, rows, rows + 500], dtype=torch.int32, device="cuda"), a, wu,
                y=torch.empty((rows, f), dtype=torch.bfloat16, device="cuda"))
    B.w8_matmul(torch.tensor([rows, rows, rows, rows + 500], dtype=torch.int32, device="cuda"), h, wd, y=y)
    assert bool((y == 7).all())
    none = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    assert B.w8_matmul(none, a[:0], wu).shape == (0, f)
    B.w8_matmul(none, h, wd, y=y)
    assert bool((y == 7).all())


@pytest.mark.parametrize("rows", [4, 300, 60000])
def test_source_rows_out_of_range_are_clamped(rows):
    g = gen(rows)
    w = weights(g, 1, 32, 64)
    a = randn(g, 4, 64)
    src = torch.tensor([-5, 0, 3, 1000], dtype=torch.int32, device="cuda").repeat(rows // 4)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    assert torch.equal(B.w8_matmul(off, a, w, a_rows=src), B.w8_matmul(off, a, w, a_rows=src.clamp(0, 3)))


@pytest.mark.parametrize("rows", [5, 400, 40000])
def test_values_that_are_not_finite_stay_in_their_rows_and_channels(rows):
    g = gen(rows)
    n, d, f = 2, 264, 72
    offs = segments(1, rows, n)
    offs[1] = 2
    o = torch.from_numpy(offs).cuda()
    a = randn(g, rows, d)
    wd = randn(g, n, f, d) * 0.05
    clean = B.w8_matmul(o, a, B.w8_quantize(wd))
    a[1, 7], a[rows - 1, d - 1] = float("nan"), -float("inf")
    wd[0, 5, 0], wd[1, f - 1, d - 1] = float("inf"), float("nan")
    y = B.w8_matmul(o, a, B.w8_quantize(wd))
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[1], bad[rows - 1], bad[:2, 5], bad[2:, f - 1] = True, True, True, True
    assert bool(torch.isnan(y[bad].float()).all()) and torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("rows", [3, 300, 60000])
def test_scales_far_apart(rows):
    """Scales near both ends of fp32 whose products, or whose products with the sum, would leave it on the way."""
    K, N = 128, 8
    a = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    a[0, :] = 1e38
    a[1, :] = 2.0 ** -112
    a[2, :] = 1.0
    codes = torch.full((1, N, 128), 127, dtype=torch.int8, device="cuda")
    scales = torch.tensor([[2.0 ** -120, 2.0 ** -60, 1e-30, 1.0, 2.0 ** 60, 1e30, 0.0, 2.0 ** -100]], device="cuda")
    w = B.W8(codes, scales, K=K)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    y = B.w8_matmul(off, a, w)
    q, s = rounded64(a)
    want = products64(q, s, [0, rows], w)
    fits = want.abs() < torch.finfo(torch.bfloat16).max
    assert bool(fits[1:].all()) and not bool(fits[0].all())
    assert bool(torch.isposinf(y[~fits].float()).all())
    # (below the smallest normal value a rounding is an absolute one)
    tol = want.abs() * (BF16 + 4 * F32) + 2.0 ** -133
    assert bool(((y.double() - want).abs() <= tol)[fits].all())


@pytest.mark.parametrize("rows", [3, 300, 60000])
@pytest.mark.parametrize("given", [False, True], ids=["a", "a8"])
def test_scales_far_apart_of_either_sign(rows, given):
    """Scales may be negative where the codes were made elsewhere: their sizes say which product is formed first."""
    K, N = 128, 8
    a = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    a[0, :] = 127 * 2.0 ** -100
    a[1, :] = 127 * 2.0 ** 110
    a[2, :] = 127.0
    codes = torch.full((1, N, 128), 127, dtype=torch.int8, device="cuda")
    scales = torch.tensor([[-2.0 ** 110, -2.0 ** -100, 2.0 ** 110, 2.0 ** -120, -2.0 ** 60, -1.5, -0.0, -2.0 ** -126]],
                          device="cuda")
    w = B.W8(codes, scales, K=K)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    q, s = rounded64(a)
    if given:
        a = B.A8(q.to(torch.int8), s.float() * torch.tensor([-1.0, 1.0, -1.0] + [1.0] * (rows - 3), device="cuda"), K=K)
        s = a.scales.double()
    y = B.w8_matmul(off, a, w)
    want = products64(q, s, [0, rows], w)
    fits = want.abs() < torch.finfo(torch.bfloat16).max
    assert bool(fits[0].all()) and fits[1].tolist() == [False, True, False, True, False, False, True, True]
    assert torch.equal(y[~fits].double(), torch.sign(want[~fits]) * float("inf"))
    # (the sum and the scales are powers of two but for 127^2 128 and 1.5: fp32 holds every product, the rounding to bf16 is
    # the only one; below the smallest normal value it is an absolute one)
    assert bool(((y.double() - want).abs() <= want.abs() * BF16 + 2.0 ** -133)[fits].all())


@pytest.mark.parametrize("rows", [3, 300, 60000])
def test_gated_scales_far_apart(rows):
    """Activations of 2^70 and of 2^-60 beside ordinary ones, weights that bring them back."""
    K, N = 128, 16
    g = gen(rows)
    a = randn(g, rows, K)
    a[0] *= 2.0 ** 70
    a[1] *= 2.0 ** -60
    wg, wu = weights(g, 1, N, K), weights(g, 1, N, K)
    wg.scales[0, :4] *= 2.0 ** -72
    wu.scales[0, :4] *= 2.0 ** -66
    wg.scales[0, 4:8] *= 2.0 ** 58
    wu.scales[0, 4:8] *= 2.0 ** 62
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    h = B.w8_gate_up(off, a, wg, wu)
    q, s = rounded64(a)
    gate, up = products64(q, s, [0, rows], wg), products64(q, s, [0, rows], wu)
    inside = (gate.abs() < 2.0 ** 120) & (up.abs() < 2.0 ** 120) & ((gate * up).abs() < 2.0 ** 120)
    assert bool(inside[0, :4].all()) and bool(inside[1, :8].all()) and not bool(inside[0].all())
    big = torch.where(inside, gate, torch.zeros_like(gate)), torch.where(inside, up, torch.zeros_like(up))
    check_hidden(torch.where(inside, h, torch.zeros_like(h)), *big, "h")


@pytest.mark.parametrize("n,rows,N,K", [(1, 3, 264, 1048), (5, 777, 1000, 1048), (15, 6000, 520, 264), (1, 4000, 1032, 8192)])
def test_negative_scales(n, rows, N, K):
    """Every product with one scale negated is the product negated, on each kernel."""
    g = gen(rows + N)
    w = weights(g, n, N, K)
    o = torch.from_numpy(segments(rows, rows, n)).cuda()
    a8 = B.a8_quantize(randn(g, rows, K))
    ws = B.new_w8_workspace(0, K, "cuda")
    y = B.w8_matmul(o, a8, w, workspace=ws)
    sign = torch.where(torch.rand(w.scales.shape, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    col = torch.repeat_interleave(sign, torch.diff(o.long()), dim=0, output_size=rows)
    row = torch.where(torch.rand((rows,), generator=g, device="cuda") < 0.5, -1.0, 1.0)
    back = B.w8_matmul(o, B.A8(a8.codes, a8.scales * row, K=K), B.W8(w.codes, w.scales * sign, K=K), workspace=ws)
    assert torch.equal(back.float(), y.float() * col * row[:, None])


@pytest.mark.parametrize("n,rows,d", [(2, 5, 256), (3, 60, 264), (2, 9000, 392)])
def test_the_output_in_place_of_the_activations(n, rows, d):
    g = gen(d)
    f = 136
    ws = weights(g, n, f, d), weights(g, n, f, d), weights(g, n, d, f)
    o = torch.from_numpy(segments(rows, rows, n)).cuda()
    a = randn(g, rows, d)
    y, h = B.w8_ffn(o, a, *ws)
    y1, h1 = B.w8_ffn(o, a, *ws, y=a)
    assert y1 is a and torch.equal(a, y) and torch.equal(h, h1)


@pytest.mark.parametrize("n,rows", [(65, 64), (200, 300), (256, 20000), (256, 90000)])
def test_more_segments_than_lanes(n, rows):
    g = gen(n)
    N, K = 24, 72
    w = weights(g, n, N, K)
    offs = segments(n, rows, n)
    offs[n // 2:] = offs[n // 2]  # the second half's rows belong to the last segment
    offs[n] = rows
    a = randn(g, rows, K)
    y = B.w8_matmul(torch.from_numpy(offs).cuda(), a, w)
    check_product(y, products64(*rounded64(a), offs, w), "y")


def test_largest_sums():
    """K of 131072 codes of 127 and -127: 2.1e9, near the end of int32."""
    K = B.W8_MAX_K
    for rows in (2, 130):
        a = torch.ones((rows, K), dtype=torch.bfloat16, device="cuda")
        a[1] = -1.0
        codes = torch.full((1, 16, K), 127, dtype=torch.int8, device="cuda")
        codes[0, 1] = -127
        w = B.W8(codes, torch.ones((1, 16), device="cuda"), K=K)
        off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        y = B.w8_matmul(off, a, w, workspace=B.new_w8_workspace(rows, K, "cuda"))
        check_product(y, products64(*rounded64(a), [0, rows], w), f"{rows} rows")


@pytest.mark.parametrize("given", [False, True], ids=["a", "a8"])
def test_most_segments_of_the_widest_matrices(given):
    """256 segments of 2^20 columns (34 GB of codes): 2^24 workgroups of 16 columns are more threads than one dimension of
    a grid has."""
    g = gen(20)
    n, N, K, rows = 256, 1 << 20, 64, 6
    codes = torch.empty((n, N, 128), dtype=torch.int8, device="cuda")
    at = [0, 1, 131, 255]
    codes[at] = torch.randint(-127, 128, (len(at), N, 128), generator=g, device="cuda", dtype=torch.int8)
    w = B.W8(codes, torch.rand((n, N), generator=g, device="cuda") + 0.5, K=K)
    offs = np.zeros(n + 1, np.int32)
    for i, e in zip(at, (1, 3, 5, 6)):
        offs[i + 1:] = e
    a = randn(g, rows, K)
    q, s = rounded64(a)
    y = B.w8_matmul(torch.from_numpy(offs).cuda(), B.a8_quantize(a) if given else a, w)
    check_product(y, products64(q, s, offs, w), "y")


@pytest.mark.parametrize("n,rows,f,d", [(3, 9, 96, 256), (4, 40, 96, 256), (3, 9000, 520, 136)])
def test_stream_and_graph(n, rows, f, d):
    g = gen(9)
    ws = weights(g, n, f, d), weights(g, n, f, d), weights(g, n, d, f)
    o = torch.from_numpy(segments(rows, rows, n)).cuda()
    a = randn(g, rows, d)
    space = B.new_w8_workspace(rows, d, "cuda", rows_cap=rows, d_ff=f)
    y, h = B.w8_ffn(o, a, *ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y1, h1 = torch.zeros_like(y), torch.zeros_like(h)
    torch.cuda.synchronize()
    B.w8_ffn(o, a, *ws, y=y1, h=h1, stream=s)
    y2, h2 = B.w8_ffn(o, a, *ws, stream=s)
    torch.cuda.synchronize()
    for t, want in ((y1, y), (h1, h), (y2, y), (h2, h)):
        assert torch.equal(t, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.w8_ffn(o, a, *ws, y=y1, h=h1, workspace=space)
    for k in range(4):
        a.copy_(randn(g, rows, d))
        want = B.w8_ffn(o, a, *ws)
        y1.zero_(), h1.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y1, want[0]) and torch.equal(h1, want[1]), f"replay {k}"


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    g = gen(4)
    n, rows, f, d = 4, 600, 264, 520
    ws = weights(g, n, f, d), weights(g, n, f, d), weights(g, n, d, f)
    o = torch.from_numpy(segments(1, rows, n)).cuda()
    xs = [randn(g, rows, d) for _ in range(2)]
    want = [B.w8_ffn(o, x, *ws) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got = [B.w8_ffn(o, x, *ws, stream=s) for x, s in zip(xs, streams)]
    torch.cuda.synchronize()
    for (y, h), (y1, h1) in zip(want, got):
        assert torch.equal(y, y1) and torch.equal(h, h1)


def test_rows_of_another_device_are_refused():
    g = gen(8)
    w, a = weights(g, 1, 32, 32), randn(g, 2, 32)
    off = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    a8 = B.a8_quantize(a)
    w.device += 1
    for call in (lambda: B.w8_matmul(off, a, w), lambda: B.w8_gate_up(off, a, w, w), lambda: B.w8_ffn(off, a, w, w, w),
                 lambda: B.w8_matmul(off, a8, w)):
        with pytest.raises(ValueError, match="8-bit rows are on GPU"):
            call()


def test_argument_refusals():
    g = gen(3)
    w, a = weights(g, 2, 32, 64), randn(g, 6, 64)
    off = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    rows = torch.zeros(4, dtype=torch.int32, device="cuda")
    bad = [
        lambda: B.w8_matmul(off, a.float(), w), lambda: B.w8_matmul(off, a[:, :56].contiguous(), w),
        lambda: B.w8_matmul(off[:2], a, w), lambda: B.w8_matmul(off.long(), a, w), lambda: B.w8_matmul(off, a.t(), w),
        lambda: B.w8_matmul(off, a, w, a_rows=rows.long()), lambda: B.w8_matmul(off, a[:0], w, a_rows=rows),
        lambda: B.w8_matmul(off, a.cpu(), w), lambda: B.w8_matmul(off, a, w, y=torch.empty(6, 24, device="cuda")),
        lambda: B.w8_gate_up(off, a, w, weights(g, 2, 40, 64)), lambda: B.w8_ffn(off, a, w, w, w),
        lambda: B.w8_matmul(off, a, w, workspace=torch.empty(16, dtype=torch.uint8)),
        lambda: B.W8(w.codes, w.scales, K=200), lambda: B.W8(w.codes, w.scales[:, :8], K=64),
        lambda: B.W8(w.codes.to(torch.uint8), w.scales, K=64), lambda: B.W8(w.codes[0], w.scales[0], K=64),
        lambda: B.A8(w.codes, w.scales, K=64), lambda: B.w8_quantize(a), lambda: B.a8_quantize(a[:, :60].contiguous()),
        lambda: B.a8_quantize(a.half()), lambda: B.a8_quantize(a, out=B.a8_quantize(a[:2].contiguous()))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    # memory shared with the input, a workspace that is too small
    y = a.view(-1)[:6 * 32].view(6, 32)
    with pytest.raises(B.BmoeError, match="UNSUPPORTED"):
        B.w8_matmul(off, a, w, y=y)
    with pytest.raises(B.BmoeError, match="WORKSPACE"):
        B.w8_matmul(off, a, w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
