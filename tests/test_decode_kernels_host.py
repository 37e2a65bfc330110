"""Which kernels the decode-side calls launch, seen without a GPU: test cases that are meant for a kernel reach it."""
import shutil

import pytest

import test_gpu_few as F
import test_gpu_w4 as Q
from launch_record import PTR, record, struct
from paper_2607_04164_amd import binding as B

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler for the recording runtime")
GROUPS = (32, 64, 128)


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
            "args": [*ints(1, n, rows, N_, K), ["p", PTR], ["p", 0], ["i", 0], ["p", PTR], w4(group), ["p", 2 * PTR], ["p", 0]],
            **device}


def gate_up_call(n, rows, f, d, group, **device):
    return {"fn": "brownout_moe_w4_gate_up",
            "args": [*ints(1, n, rows, d, f), ["p", PTR], ["p", 0], ["i", 0], ["p", PTR], w4(group), w4(group),
                     ["p", 2 * PTR], ["p", 0]], **device}


def launched(calls, tmp_path):
    res = record(calls, tmp_path)
    assert all(status == 0 for status, _ in res)
    return [ls for _, ls in res]


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
