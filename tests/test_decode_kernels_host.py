"""Which kernels the decode-side calls launch, seen without a GPU: every one that is built is run by the cases of the
GPU tests, and cases that are meant for a kernel reach it."""
import re
import shutil

import pytest

import test_gpu_few as F
import test_gpu_norm as N
import test_gpu_w4 as Q
from launch_record import PTR, kernels, record, struct
from paper_2607_04164_amd import binding as B

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler for the recording runtime")
GROUPS = (32, 64, 128)
FAR = 1 << 40  # outputs


def ptrs(n):
    return [["p", PTR]] * n


def ints(*v):
    return [["i", i] for i in v]


def few_call(case, dtype, group, zeros, **device):
    d = F.desc_of(case, dtype)
    m = B._Matrix(PTR, PTR if group else None, PTR if zeros else None)
    w = B._FewWeights(w_router=PTR, bias=PTR, e2g=PTR, gate=m, up=m, down=m, gate_sh=m, up_sh=m, down_sh=m, group=group)
    return {"fn": "brownout_moe_few", "args": [struct(d), struct(w), *ptrs(7), ["z", 1 << 40], ["p", 0]], **device}


def w4(group, zeros=False):
    return struct(B._W4Struct(PTR, PTR, PTR if zeros else None, group))


def matmul_call(n, rows, N_, K, group, **device):
    return {"fn": "brownout_moe_w4_matmul",
            "args": [*ints(1, n, rows, N_, K), ["p", PTR], ["p", 0], ["i", 0], ["p", PTR], w4(group), ["p", FAR], ["p", 0]],
            **device}


def gate_up_call(n, rows, f, d, group, **device):
    return {"fn": "brownout_moe_w4_gate_up",
            "args": [*ints(1, n, rows, d, f), ["p", PTR], ["p", 0], ["i", 0], ["p", PTR], w4(group), w4(group),
                     ["p", FAR], ["p", 0]], **device}


def quantize_call(dtype, group):
    return {"fn": "brownout_moe_w4_quantize", "args": [*ints(dtype, 1, 8, 64, group), *ptrs(4), ["p", 0]]}


def pre_call(T, d, dtype):
    return {"fn": "brownout_moe_pre_norm", "args": [*ints(dtype, T, d), ["f", 1e-6], *ptrs(2), ["p", FAR], ["p", 0]]}


def post_call(T, d, dtype):
    return {"fn": "brownout_moe_post_norm",
            "args": [*ints(dtype, T, d), ["f", 1e-6], ["i", 1], ["f", 1.0], ["i", 3], *ptrs(4), ["p", FAR], ["p", PTR],
                     ["p", 2 * FAR], ["p", 0]]}


def launched(calls, tmp_path):
    res = record(calls, tmp_path)
    assert all(status == 0 for status, _ in res)
    return [ls for _, ls in res]


def test_every_kernel_is_run_by_a_test_case(tmp_path):
    calls = [few_call(c, *fmt) for c in F.CASES.values() for fmt in F.FORMATS]
    calls += [few_call(dict(T=T, d=96, E=10, top_k=3, G=5, f=48, fs=24), *fmt) for T in range(1, 17) for fmt in F.FORMATS[:3]]
    calls += [matmul_call(*c, g) for c in Q.CASES + Q.FOUR_TILES + Q.ONE_TILE for g in GROUPS]
    calls += [gate_up_call(*c, g) for c in Q.FFN_FOUR_TILES for g in GROUPS]
    # test_w4_ffn, test_w4_layer_of_any_size
    calls += [gate_up_call(*c) for c in ((1, 1, 1408, 2048, 32), (1, 1, 24, 40, 32), (1, 1, 1408, 2048, 64),
                                         (1, 1, 24, 40, 64), (1, 1, 1408, 2048, 128), (1, 1, 24, 40, 128))]
    calls += [quantize_call(t, g) for t in (0, 1) for g in GROUPS]
    calls += [pre_call(T, d, t) for T, d in N.SIZES + N.PRE_SPLITS for t in (0, 1)]
    calls += [post_call(T, d, t) for T, d in N.POST_SPLITS + [(1, 2048), (5, 264), (1030, 520), (3, 16392)] for t in (0, 1)]
    ran = {name for ls in launched(calls, tmp_path) for name, _ in ls}
    built = {k for k in kernels(tmp_path) if re.search(r"few_|w4_|_norm_kernel", k)}
    assert len(built) > 70
    assert not built - ran, "\n".join(sorted(built - ran))


@pytest.mark.parametrize("group", GROUPS)
def test_cases_of_four_tiles_reach_them(group, tmp_path):
    for n, rows, N_, K in Q.FOUR_TILES:
        ((name, grid),), = launched([matmul_call(n, rows, N_, K, group)], tmp_path)
        assert f"w4_gemm_kernel<1, 4, {group}, {'true' if K % 256 else 'false'}>" in name
        assert grid[0] * grid[1] >= 256
    for n, rows, N_, K in Q.ONE_TILE:
        ((name, _),), = launched([matmul_call(n, rows, N_, K, group)], tmp_path)
        assert f"w4_gemm_kernel<1, 1, {group}, {'true' if K % 256 else 'false'}>" in name
    for n, rows, f, d in Q.FFN_FOUR_TILES:
        ((name, grid),), = launched([gate_up_call(n, rows, f, d, group)], tmp_path)
        assert f"w4_gemm_kernel<2, 4, {group}, {'true' if d % 256 else 'false'}>" in name
        assert grid[0] * grid[1] >= 256
    hidden = [few_call(F.CASES[c], "bf16", group, True) for c in ("whole-units-past-lds-9", "whole-units-past-lds-16")]
    for ls in launched(hidden, tmp_path):
        assert [n for n, _ in ls if f"few_up_kernel<bmoe::(anonymous namespace)::FmtW4<{group}>, 2, false, false>" in n]
        assert [n for n, _ in ls if f"few_down_kernel<bmoe::(anonymous namespace)::FmtW4<{group}>, false, false>" in n]


def test_choices_follow_the_cu_count(tmp_path):
    """On half of the chip (128 CUs) the splits and tiles are chosen for half as many workgroups, and more CUs than the
    workspace is for change nothing."""
    case = dict(T=1, d=2048, E=60, top_k=4, G=15, f=1408)
    up, down = "few_up_kernel<bmoe::(anonymous namespace)::FmtPlain<unsigned short>, {}, false", "few_down_kernel"
    for i, (cus, tiles, ups, downs) in enumerate(((256, 2, 176, 768), (128, 1, 256, 384), (304, 2, 176, 768))):
        ls, = launched([few_call(case, "bf16", 0, False, cus=cus, device=20 + i)], tmp_path)
        (_, (u, g)), (_, (dn, h)) = [(n, x) for n, x in enumerate(ls) if "few_logits" not in x[0]]
        assert up.format(tiles) in u and g[0] == ups and down in dn and h[0] == downs
    # 200 blocks of four tiles
    one, four = (launched([matmul_call(1, 5, 12800, 512, 64, cus=c, device=30 + i)], tmp_path)[0][0][0]
                 for i, c in enumerate((256, 128)))
    assert "w4_gemm_kernel<1, 1, 64" in one and "w4_gemm_kernel<1, 4, 64" in four
