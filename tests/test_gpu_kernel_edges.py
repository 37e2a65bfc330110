"""Edges of the kernels' tiles and of the rules that pick a kernel, against
the CPU oracle (needs an MI355X): remainders, empty and one-row segments, the
smallest sizes, and the sizes on either side of a rule. Tolerances are those
of gpu_util."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
from gpu_util import TOL, assert_close_rows, assert_gates, desc_of, dev_tensor, host_f32, to_storage  # noqa: F401
from paper_2607_04164_amd import binding as B
from paper_2607_04164_amd import workload as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def ffn_case(sizes, cap, d, f, dtype, seed, n_tokens=None):
    """Random segments: offsets, storage-format arrays and the oracle's (y, h).
    n_tokens: the rows are gathered from that many tokens."""
    r = np.random.default_rng(seed)
    n = len(sizes)
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    N = int(offsets[-1])
    x = to_storage(r.standard_normal((n_tokens or cap, d)).astype(np.float32), dtype)
    rows = r.integers(0, n_tokens, cap).astype(np.int32) if n_tokens else None
    ws = [to_storage((r.standard_normal(s) / np.sqrt(d)).astype(np.float32), dtype)
          for s in ((n, f, d), (n, f, d), (n, d, f))]
    wide = (lambda a: a) if dtype == "f32" else W.bf16_bits_to_f32
    a = wide(x if rows is None else x[rows])
    y, h = oracle.ffn(offsets, a[:max(N, 1)], *(wide(t) for t in ws), want_h=True)
    return offsets, N, x, rows, ws, y, h


def check_ffn(sizes, cap, d, f, dtype, seed=0, n_tokens=None, workspace=None, split_min_idle=None):
    offsets, N, x, rows, ws, y, h = ffn_case(sizes, cap, d, f, dtype, seed, n_tokens)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    yg = torch.full((cap, d), -5.0, dtype=dt, device="cuda")
    hg = torch.full((cap, f), -5.0, dtype=dt, device="cuda")
    offs, w = torch.from_numpy(offsets).cuda(), [dev_tensor(t, dtype) for t in ws]
    if rows is None:
        B.ffn(offs, dev_tensor(x, dtype), *w, y=yg, h=hg, workspace=workspace, split_min_idle=split_min_idle)
    else:
        B.ffn_gather(offs, torch.from_numpy(rows).cuda(), dev_tensor(x, dtype), *w, y=yg, h=hg, workspace=workspace)
    torch.cuda.synchronize()
    assert_close_rows(host_f32(hg[:N]), h, dtype, "h")
    assert_close_rows(host_f32(yg[:N]), y, dtype, "y")
    assert bool((yg[N:] == -5.0).all()) and bool((hg[N:] == -5.0).all()), "rows past the last segment are not written"


F32_FFN = [
    # (segment sizes, spare rows, d, d_ff, tokens gathered from): one K unit
    # for eight waves, tiles of exactly 32 rows and columns, remainders of 8
    # columns and 1 row, more segments than a wave has lanes
    ((1,), 0, 8, 8, None),
    ((32, 0, 33, 31), 4, 72, 40, None),
    ((64, 5), 0, 264, 104, 20),
    (tuple(i % 4 for i in range(70)), 9, 32, 64, 11),
    ((200, 0, 1), 55, 512, 32, None),
]


@pytest.mark.parametrize("sizes,spare,d,f,tokens", F32_FFN, ids=[f"seg{len(c[0])}-d{c[2]}-f{c[3]}" for c in F32_FFN])
def test_f32_ffn_tiles(sizes, spare, d, f, tokens):
    check_ffn(sizes, sum(sizes) + spare, d, f, "f32", n_tokens=tokens)


@pytest.mark.parametrize("T,d,E,k", [(1, 8, 1, 1), (17, 24, 8, 2), (16, 264, 16, 4), (33, 72, 17, 3), (50, 40, 200, 9)])
def test_f32_route(T, d, E, k):
    """The fp32 gate: one and several blocks of 16 experts, a last half unit of d, ragged token tiles."""
    cfg = W.LayerConfig("f32route", T=T, d=d, E=E, top_k=k, G=max(1, E // 2), d_ff=8, dtype="f32", zipf_s=1.0)
    L = W.make_layer(cfg, 4, with_weights=False)
    ref = oracle.route(L.f32("x"), L.f32("w_router"), L.bias, L.e2g, k, 0)
    got = B.route(desc_of(cfg), dev_tensor(L.x, "f32"), dev_tensor(L.w_router, "f32"), torch.from_numpy(L.bias).cuda(),
                  torch.from_numpy(L.e2g).cuda(), want_logits=True)
    torch.cuda.synchronize()
    zerr = np.abs(got["logits"].cpu().numpy().astype(np.float64) - ref["logits"]).max()
    assert zerr < B.ROUTE_RECHECK_GAP / 4, f"fp32 logit error {zerr:.3e}"
    for key in ("topk_idx", "slot_group"):
        assert np.array_equal(got[key].cpu().numpy(), ref[key]), key
    assert_gates(got["topk_w"].cpu().numpy(), ref["topk_w"], "topk_w")
    assert_gates(got["slot_gate"].cpu().numpy(), ref["slot_gate"], "slot_gate")


def ffn_workspace():
    return torch.empty(B.workspace_bytes(B.make_desc(1, 64, 1, 1, 1, 64), B.STAGE_FFN), dtype=torch.uint8, device="cuda")


TILE_FFN = [
    # (segment sizes, rows_cap, d, d_ff, tokens gathered from), above the skinny
    # kernels' size: tails on either side of half a 256-row tile, segments of a
    # half tile only, column remainders
    ((128, 129, 256, 257, 1, 0, 384, 385), 1600, 320, 192, None),
    # ragged K of few rows (one round of workgroups): the register-staged tiles
    ((128, 127, 512, 1), 800, 136, 176, None),
    ((300, 64), 400, 184, 200, 150),
    ((130, 700), 900, 168, 136, None),
    ((513, 40, 0, 200), 800, 152, 144, 300),
    ((250, 255, 3), 600, 312, 248, None),
    # the same with empty segments, so that the rows are few per segment: the
    # persistent kernel with ragged last K-steps of 8 to 56 columns, three
    # K-steps and more
    ((128, 127, 512, 1) + (0,) * 5, 800, 136, 304, None),
    ((300, 64) + (0,) * 3, 400, 184, 328, 150),
    ((130, 700) + (0,) * 8, 900, 168, 264, None),
    ((513, 40, 0, 200) + (0,) * 6, 800, 152, 280, 300),
    ((250, 255, 3) + (0,) * 6, 600, 312, 376, None),
    # and for so many segments that the register-staged tiles might not be one round: three K-steps in down
    ((200, 129) + (3,) * 19 + (0,) * 110, 8400, 512, 136, None),
    # whole tiles only (768 rows per segment of capacity), a column remainder of
    # 48 in gate/up (a tensor-parallel share)
    ((1000, 0, 513, 1), 4096, 320, 176, None),
    # more half tiles than workgroups: 60 segments x 5 column tiles of gate/up
    (tuple(1 + (37 * i) % 128 for i in range(60)), 5000, 128, 584, None),
    # whole tiles and half tiles in the same round, half tiles in the next
    (tuple([256] * 20 + [100] * 30), 8400, 192, 1160, None),
    # ragged K too short for the copies: the register-staged tiles, of 128 rows,
    # then of 256 rows in one of the GEMMs
    ((200, 130), 400, 72, 104, None),
    ((2600, 0, 257, 1), 5000, 72, 1024, 3000),
    ((4000, 255), 7000, 1032, 120, None),
    ((300, 1, 0, 129), 450, 120, 88, 200),
]


# with the split threshold at zero and the workspace, where a K is whole K-steps
# (a ragged K is never split; ffn_gather takes no threshold)
TILE_RUNS = [(c, False) for c in TILE_FFN] + [(c, True) for c in TILE_FFN if c[4] is None and min(c[2] % 64, c[3] % 64) == 0]


@pytest.mark.parametrize("case,stream_k", TILE_RUNS,
                         ids=[f"seg{len(c[0])}-d{c[2]}-f{c[3]}{'-stream_k' if k else ''}" for c, k in TILE_RUNS])
def test_ffn_tile_heights_and_ragged_k(case, stream_k):
    sizes, cap, d, f, tokens = case
    assert cap > 64 * len(sizes) and sum(sizes) <= cap
    if stream_k:
        check_ffn(sizes, cap, d, f, "bf16", 1, None, ffn_workspace(), 0)
    else:
        check_ffn(sizes, cap, d, f, "bf16", 1, tokens)


def test_ffn_tails_of_wide_weights():
    """Half tiles read their segment's weights again: past 256 MB of that, the
    tails of segments with whole tiles stay whole while segments of at most 128
    rows keep half tiles. Against fp32 products of the same bf16 values."""
    sizes, d, f = (300, 350, 60, 270, 380, 128), 4096, 4160
    assert sum(s > 256 and 0 < s % 256 <= 128 for s in sizes) * 2 * d * f * 2 > 256 << 20
    n, cap = len(sizes), sum(sizes) + 40
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(cap, d, generator=gen, device="cuda").bfloat16()
    wg, wu = ((torch.randn(n, f, d, generator=gen, device="cuda") / d ** 0.5).bfloat16() for _ in range(2))
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    h = torch.full((cap, f), -5.0, dtype=torch.bfloat16, device="cuda")
    B.ffn_gate_up(offsets, x, wg, wu, h=h)
    beg = 0
    for s, rows in enumerate(sizes):
        a = x[beg:beg + rows].float()
        want = torch.nn.functional.silu(a @ wg[s].float().t()) * (a @ wu[s].float().t())
        assert_close_rows(host_f32(h[beg:beg + rows]), want.cpu().numpy(), "bf16", f"h of segment {s}")
        beg += rows
    assert bool((h[beg:] == -5.0).all())


# the persistent kernel; the register-staged tiles; the 16-column kernel
@pytest.mark.parametrize("part,K,rows", [("up", 456, 150), ("up", 520, 700), ("down", 648, 150), ("down", 696, 700),
                                         ("up", 200, 150), ("down", 176, 150), ("up", 72, 150), ("down", 120, 150),
                                         ("up", 328, 10), ("down", 72, 10)])
def test_ffn_infinite_weights_ragged_k(part, K, rows):
    """An infinite weight in the last 64-column step of a ragged K: the step's
    padding must not turn it into NaN (0 * inf). Exact inputs (one-hot rows and
    small integers), so the expected sums are exact."""
    N, n = 136, 2
    r = np.random.default_rng(K)
    # (two segments; the skinny kernels' capacity ends at 64 rows per segment)
    offsets = torch.tensor([0, rows, 2 * rows], dtype=torch.int32, device="cuda")
    a = torch.from_numpy(r.integers(1, 4, (2 * rows, K)).astype(np.float32))
    w = torch.from_numpy(r.integers(-2, 3, (n, N, K)).astype(np.float32))
    tail = K // 64 * 64
    w[0, 3, tail + 1], w[1, 5, tail], w[0, 130, K - 1] = float("inf"), float("-inf"), float("inf")
    want = torch.cat([a[s * rows:(s + 1) * rows].double() @ w[s].double().t() for s in range(n)])
    ab, wb = a.bfloat16().cuda(), w.bfloat16().cuda()
    if part == "down":
        got = B.ffn_down(offsets, ab, wb)
    else:
        # gate columns of 64 so that silu is the identity: h = 64 * up
        gate = torch.zeros_like(w)
        gate[:, :, 0] = 64.0
        one = a.clone()
        one[:, 0] = 1.0
        want = 64.0 * torch.cat([one[s * rows:(s + 1) * rows].double() @ w[s].double().t() for s in range(n)])
        got = B.ffn_gate_up(offsets, one.bfloat16().cuda(), gate.bfloat16().cuda(), wb)
    torch.cuda.synchronize()
    got = got.double().cpu()
    inf = want.isinf()
    assert int(inf.sum()) == 3 * rows
    assert torch.equal(got[inf], want[inf])
    # finite sums are whole numbers below 2^24, rounded once to bf16
    assert torch.equal(got[~inf], want[~inf].float().bfloat16().double())


_FEW30 = tuple(1 + i % 5 for i in range(30))

SKINNY = [
    # (segment sizes, spare rows, d, d_ff, tokens gathered from); capacity of at
    # most 64 rows per segment. The 16-column kernel in both GEMMs:
    ((1,), 0, 8, 8, None),                                # K below one pair, half a column tile
    ((16, 17, 33, 65) + (0,) * 8, 3, 256, 72, None),      # every row-tile count, two and three passes
    ((15, 0, 48, 1), 0, 1032, 40, 30),                    # K = whole pairs + 8 columns, gathered
    ((1, 0, 3), 0, 2184, 1096, None),                     # gate/up: two batches and a tail; down: six pairs, a tail
    ((2, 17), 2, 136, 1608, 9),                           # down: two batches of four pairs and a tail
    # 30 segments of 1 to 5 rows: in gate/up, then in down (K one pair), the
    # second round of the ring kernel's workgroups or (640 columns) not
    (_FEW30, 6, 128, 832, None), (_FEW30, 6, 128, 640, None), (_FEW30, 5, 832, 64, 40), (_FEW30, 5, 640, 64, 40),
    # a quarter of the CUs in gate/up: under it, under it with more empty segments, past it
    ((30, 20, 14) + (0,) * 13, 0, 192, 192, None), ((30, 20, 14) + (0,) * 14, 0, 192, 192, None),
    ((30, 20, 14) + (0,) * 19, 0, 192, 192, None),
    # the other two kernels (down of 24 and 328 columns: the 16-column one): more
    # segments than lanes, some empty; ragged K; two and three passes; K of 4 and
    # 6 chunks
    ((16, 17, 32, 33, 64, 65, 0), 3, 256, 72, None),
    (tuple((7 * i) % 5 for i in range(100)), 20, 64, 24, 40),
    (tuple(1 + i % 3 for i in range(60)), 40, 320, 328, None),
    (tuple(3 * (i % 4) for i in range(70)), 100, 256, 384, 50),
    ((70, 0, 64, 129) + (1,) * 60, 300, 192, 320, None),
]


@pytest.mark.parametrize("sizes,spare,d,f,tokens", SKINNY, ids=[f"seg{len(c[0])}-d{c[2]}-f{c[3]}" for c in SKINNY])
def test_skinny_ffn(sizes, spare, d, f, tokens):
    cap = sum(sizes) + spare
    assert cap <= 64 * len(sizes)
    check_ffn(sizes, cap, d, f, "bf16", 2, tokens)


ROUTE = [
    # (experts, d, top_k, tokens): rings of the waves' own with fewer chunks than
    # waves, more chunks than slots, ragged token tiles of 16 (up to 4096 tokens)
    # and 32, one and four blocks of experts, picks past the register list; then
    # both sides of their rules (d not whole chunks, more experts, more tokens:
    # x straight into registers for d of 512, 1024 and 2048, the shared ring with
    # 16, 32 and 64 tokens per workgroup)
    (9, 64, 2, 40), (64, 64, 5, 17), (3, 320, 2, 33), (16, 192, 3, 4130), (40, 576, 9, 4110), (17, 2112, 4, 4096),
    (60, 2048, 4, 1), (12, 72, 3, 300), (65, 256, 4, 300), (33, 512, 3, 8193), (16, 640, 16, 50),
    (33, 1024, 5, 8200), (60, 512, 9, 8200), (30, 72, 3, 200), (16, 640, 3, 8200), (40, 320, 2, 8300), (12, 128, 2, 16400),
    (40, 192, 2, 16390),
]


@pytest.mark.parametrize("E,d,k,T", ROUTE, ids=[f"E{c[0]}-d{c[1]}-k{c[2]}-T{c[3]}" for c in ROUTE])
def test_route_paths(E, d, k, T):
    cfg = W.LayerConfig("rpath", T=T, d=d, E=E, top_k=k, G=max(1, E // 2), d_ff=64, dtype="bf16", zipf_s=1.0,
                        norm_topk=k % 2)
    L = W.make_layer(cfg, 6, with_weights=False)
    ref = oracle.route(L.f32("x"), L.f32("w_router"), L.bias, L.e2g, k, cfg.norm_topk)
    got = B.route(desc_of(cfg), dev_tensor(L.x, "bf16"), dev_tensor(L.w_router, "bf16"), torch.from_numpy(L.bias).cuda(),
                  torch.from_numpy(L.e2g).cuda(), want_logits=True)
    torch.cuda.synchronize()
    zerr = np.abs(got["logits"].cpu().numpy().astype(np.float64) - ref["logits"]).max()
    assert zerr < B.ROUTE_RECHECK_GAP / 4, f"fp32 logit error {zerr:.3e}"
    for key in ("topk_idx", "slot_group"):
        assert np.array_equal(got[key].cpu().numpy(), ref[key]), key
    assert_gates(got["topk_w"].cpu().numpy(), ref["topk_w"], "topk_w")
    assert_gates(got["slot_gate"].cpu().numpy(), ref["slot_gate"], "slot_gate")


@pytest.mark.parametrize("E,d,T", [(64, 2048, 16384), (33, 1024, 9000), (60, 512, 12289)])
def test_route_two_workgroups_per_cu_repeats(E, d, T):
    """x straight into registers, two workgroups per CU: the same bits on every
    call, alone and beside copies on another stream, and logits within a quarter
    of the gap of their float64 values."""
    gen = torch.Generator(device="cuda").manual_seed(E)
    x = torch.randn(T, d, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(E, d, generator=gen, device="cuda") / d ** 0.5).bfloat16()
    e2g = (torch.arange(E, device="cuda", dtype=torch.int32) % 16).contiguous()
    desc = B.make_desc(T, d, E, 6, 16, 64)
    first = B.route(desc, x, w, None, e2g, want_logits=True)
    z = x.double() @ w.double().t()
    assert float((first["logits"].double() - z).abs().max()) < B.ROUTE_RECHECK_GAP / 4
    side, a, b = torch.cuda.Stream(), torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), None
    side.wait_stream(torch.cuda.current_stream())
    runs = []
    for i in range(12):
        if i >= 6:
            with torch.cuda.stream(side):
                b = a.clone()
        runs.append(B.route(desc, x, w, None, e2g, want_logits=True))
    torch.cuda.synchronize()
    for i, r in enumerate(runs):
        for k, v in first.items():
            assert torch.equal(r[k], v), (i, k)
    del b


def test_most_segments_of_the_widest_matrices():
    """256 segments of 2^20 columns: as 2^24 workgroups of 16 columns they are more threads than one dimension of a
    grid has."""
    g = torch.Generator(device="cuda").manual_seed(20)
    n, d, f, rows = 256, 1 << 20, 24, 6
    w = torch.empty((n, d, f), dtype=torch.bfloat16, device="cuda")
    at, ends = [0, 1, 131, 255], (1, 3, 5, 6)
    offs = np.zeros(n + 1, np.int32)
    for i, e in zip(at, ends):
        w[i] = torch.randn((d, f), generator=g, device="cuda").to(torch.bfloat16)
        offs[i + 1:] = e
    h = torch.randn((rows, f), generator=g, device="cuda").to(torch.bfloat16)
    y = B.ffn_down(torch.from_numpy(offs).cuda(), h, w)
    for i, b, e in zip(at, (0, *ends), ends):
        want, size = h[b:e].double() @ w[i].double().t(), h[b:e].double().abs() @ w[i].double().abs().t()
        # products of bf16 values are exact in fp32; their sum in any order, then one rounding to bf16
        assert bool(((y[b:e].double() - want).abs() <= want.abs() * 2.0 ** -8 + size * (f + 1) * 2.0 ** -24).all()), i
