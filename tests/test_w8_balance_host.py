"""Refusals of the 8-bit and balance calls on the host: every call here fails validation or is an empty no-op, so
nothing is enqueued. And the kernels that the cases of the GPU tests reach."""
import ctypes
import os
import re
import shutil

import pytest

from launch_record import PTR, ffn_part, kernels, record, struct
from paper_2607_04164_amd import binding as B

OK, NULL, SHAPE, ALIGN, UNSUP, WS = 0, 1, 2, 3, 5, 6
A = 0x10000  # aligned, never read
Y = 0x40000000  # outputs, apart from the inputs
ODD = 0x10008


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_header_constants():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "brownout_moe.h")).read()
    assert int(re.search(r"#define BMOE_W8_MAX_K (\d+)", text).group(1)) == B.W8_MAX_K
    assert int(re.search(r"#define BMOE_BALANCE_ZERO_BYTES (\d+)", text).group(1)) == B.BALANCE_ZERO_BYTES
    assert [B.w8_row_bytes(K) for K in (8, 128, 136, 4096)] == [128, 128, 256, 4096]


def rows8(codes=A, scales=A):
    return ctypes.byref(B._W8Struct(codes, scales))


def quantize(lib, **kw):
    a = dict(dtype=1, rows=4, K=64, x=A, codes=Y, scales=2 * Y)
    a.update(kw)
    return lib.brownout_moe_w8_quantize(*(a[n] for n in ("dtype", "rows", "K", "x", "codes", "scales")), None)


@pytest.mark.parametrize("kw,code", [
    ({"dtype": 2}, UNSUP), ({"rows": -1}, SHAPE), ({"rows": (1 << 30) + 1}, SHAPE), ({"K": 0}, SHAPE), ({"K": 12}, SHAPE),
    ({"K": 131080}, SHAPE), ({"x": None}, NULL), ({"codes": None}, NULL), ({"scales": None}, NULL), ({"x": ODD}, ALIGN),
    ({"codes": ODD}, ALIGN), ({"scales": ODD}, ALIGN), ({"codes": A}, UNSUP), ({"codes": A + 496}, UNSUP),
    ({"scales": A + 16}, UNSUP), ({"scales": Y + 496}, UNSUP), ({"rows": 0, "x": None}, OK)])
def test_quantize_refusals(lib, kw, code):
    assert quantize(lib, **kw) == code


MATMUL = ("dtype", "n", "rows", "N", "K", "off", "src", "m", "a", "a8", "w", "y", "ws", "bytes")


def matmul(lib, **kw):
    a = dict(dtype=1, n=2, rows=8, N=32, K=64, off=A, src=None, m=0, a=A, a8=None, w=rows8(), y=Y, ws=2 * Y,
             bytes=1 << 20)
    a.update(kw)
    return lib.brownout_moe_w8_matmul(*(a[n] for n in MATMUL), None)


@pytest.mark.parametrize("kw,code", [
    ({"dtype": 0}, UNSUP), ({"dtype": 7}, UNSUP), ({"n": 0}, SHAPE), ({"n": 257}, SHAPE), ({"rows": -1}, SHAPE),
    ({"rows": (1 << 30) + 1}, SHAPE), ({"N": 0}, SHAPE), ({"N": 20}, SHAPE), ({"N": (1 << 20) + 8}, SHAPE),
    ({"K": 4}, SHAPE), ({"K": 131080}, SHAPE), ({"off": None}, NULL), ({"a": None}, NULL), ({"w": None}, NULL),
    ({"y": None}, NULL), ({"w": rows8(codes=None)}, NULL), ({"w": rows8(scales=None)}, NULL),
    ({"a": None, "a8": rows8(scales=None)}, NULL), ({"a8": rows8()}, UNSUP), ({"a": ODD}, ALIGN), ({"y": Y + 8}, ALIGN),
    ({"w": rows8(codes=ODD)}, ALIGN), ({"w": rows8(scales=ODD)}, ALIGN), ({"a": None, "a8": rows8(codes=ODD)}, ALIGN),
    ({"src": A, "m": 0}, SHAPE), ({"src": A, "m": 1 << 25, "K": 128}, SHAPE), ({"src": A, "m": (1 << 30) + 1}, SHAPE),
    ({"y": A}, UNSUP), ({"y": A + 1008}, UNSUP), ({"a": None, "a8": rows8(), "y": A}, UNSUP),
    ({"a": None, "a8": rows8(codes=4 * Y, scales=Y + 496)}, UNSUP), ({"ws": None}, WS), ({"bytes": 1279}, WS),
    ({"ws": 2 * Y + 128}, ALIGN), ({"rows": 0, "a": None, "off": None, "w": None, "y": None, "ws": None}, OK)])
def test_matmul_refusals(lib, kw, code):
    assert matmul(lib, **kw) == code


def ffn(lib, **kw):
    a = dict(dtype=1, n=2, rows=8, d=64, f=32, off=A, src=None, m=0, a=A, a8=None, wg=rows8(), wu=rows8(), wd=rows8(),
             h=Y, y=2 * Y, ws=3 * Y, bytes=1 << 20)
    a.update(kw)
    return lib.brownout_moe_w8_ffn(*(a[n] for n in ("dtype", "n", "rows", "d", "f", "off", "src", "m", "a", "a8", "wg",
                                                    "wu", "wd", "h", "y", "ws", "bytes")), None)


def gate_up(lib, **kw):
    a = dict(dtype=1, n=2, rows=8, d=64, f=32, off=A, src=None, m=0, a=A, a8=None, wg=rows8(), wu=rows8(), h=Y,
             ws=3 * Y, bytes=1 << 20)
    a.update(kw)
    return lib.brownout_moe_w8_gate_up(*(a[n] for n in ("dtype", "n", "rows", "d", "f", "off", "src", "m", "a", "a8",
                                                        "wg", "wu", "h", "ws", "bytes")), None)


@pytest.mark.parametrize("kw,code", [
    ({"dtype": 0}, UNSUP), ({"f": 131080}, SHAPE), ({"d": 131080}, SHAPE), ({"f": 12}, SHAPE), ({"wg": None}, NULL),
    ({"wu": None}, NULL), ({"h": None}, NULL), ({"wu": rows8(codes=ODD)}, ALIGN), ({"h": Y + 8}, ALIGN), ({"h": A}, UNSUP),
    ({"bytes": 255}, WS), ({"ws": None}, WS)])
def test_ffn_refusals(lib, kw, code):
    # (as a hidden size of 131080 is only a product's width)
    if kw != {"f": 131080}:
        assert gate_up(lib, **kw) == code
    assert ffn(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    ({"wd": None}, NULL), ({"y": None}, NULL), ({"wd": rows8(scales=None)}, NULL), ({"y": Y}, UNSUP), ({"y": ODD}, ALIGN),
    ({"a": None, "a8": rows8(), "ws": None}, WS), ({"rows": 0, "a": None, "y": None, "h": None, "ws": None, "wu": None}, OK)])
def test_ffn_down_refusals(lib, kw, code):
    assert ffn(lib, **kw) == code


def test_workspace_sizes(lib):
    size = lambda *a: lib.bmoe_w8_workspace_bytes(*a, 0)  # noqa: E731
    assert size(0, 64, 100, 0) == 0
    assert size(3, 64, 100, 0) == 512 + 256
    assert size(3, 64, 100, 264) == 100 * 384 + 512  # (the hidden rows take the place of the input's)
    assert size(1 << 20, 14336, 8, 264) == (1 << 20) * (14336 + 4)
    assert size(-1, 64, 1, 1) == 0 and size(1, 64, 1, 131080) == 0 and size(1, 4, 1, 8) == 0


def bal(lib, **kw):
    a = dict(T=100, E=12, k=2, G=12, z=A, idx=A, valid=None, e2g=None, losses=Y, counts=2 * Y, prob=3 * Y, ws=4 * Y,
             bytes=1 << 30)
    a.update(kw)
    return lib.brownout_moe_balance(*(a[n] for n in ("T", "E", "k", "G", "z", "idx", "valid", "e2g", "losses", "counts",
                                                     "prob", "ws", "bytes")), None)


@pytest.mark.parametrize("kw,code", [
    ({"T": -1}, SHAPE), ({"E": 0}, SHAPE), ({"E": 257, "G": 257}, SHAPE), ({"k": 0}, SHAPE), ({"k": 17}, SHAPE),
    ({"G": 3}, SHAPE), ({"G": 0, "e2g": A}, SHAPE), ({"G": 257, "e2g": A}, SHAPE), ({"T": 1 << 30, "k": 4}, SHAPE),
    ({"z": None}, NULL), ({"idx": None}, NULL), ({"losses": None}, NULL), ({"counts": None}, NULL), ({"prob": None}, NULL),
    ({"z": A + 2}, ALIGN), ({"losses": Y + 1}, ALIGN), ({"e2g": A + 2}, ALIGN), ({"prob": A}, UNSUP),
    ({"losses": A + 4796}, UNSUP), ({"counts": 3 * Y + 44}, UNSUP), ({"valid": 3 * Y + 40}, UNSUP),
    ({"T": 5000, "ws": None}, WS), ({"T": 5000, "bytes": 100}, WS), ({"T": 5000, "ws": 4 * Y + 4}, ALIGN),
    ({"T": 0, "z": None, "losses": None}, OK)])
def test_balance_refusals(lib, kw, code):
    assert bal(lib, **kw) == code


def grad(lib, **kw):
    a = dict(T=100, E=12, k=2, G=12, z=A, valid=None, e2g=None, counts=2 * Y, d=3 * Y, dz=Y)
    a.update(kw)
    return lib.brownout_moe_balance_grad(*(a[n] for n in ("T", "E", "k", "G", "z", "valid", "e2g", "counts", "d", "dz")),
                                         None)


@pytest.mark.parametrize("kw,code", [
    ({"T": -1}, SHAPE), ({"E": 300}, SHAPE), ({"k": 0}, SHAPE), ({"G": 5}, SHAPE), ({"z": None}, NULL),
    ({"counts": None}, NULL), ({"d": None}, NULL), ({"dz": None}, NULL), ({"dz": Y + 2}, ALIGN), ({"dz": A + 4}, UNSUP),
    ({"dz": 2 * Y + 48}, UNSUP), ({"dz": 3 * Y + 4}, UNSUP), ({"valid": Y + 4799}, UNSUP),
    ({"T": 0, "z": None, "dz": None}, OK)])
def test_balance_grad_refusals(lib, kw, code):
    assert grad(lib, **kw) == code


# ---------------------------------------------------------------------------
# the kernels that the calls reach

needs_recorder = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler for the recording runtime")


def ints(*v):
    return [["i", i] for i in v]


def w8(codes=PTR):
    return struct(B._W8Struct(codes, PTR))


def product(n, rows, N, K, gated=False, ws=1 << 36, a8=False, **device):
    far = ["p", 1 << 40]
    a = [["p", 0], w8()] if a8 else [["p", PTR], ["p", 0]]
    args = [*ints(1, n, rows, *((K, N) if gated else (N, K))), ["p", PTR], ["p", 0], ["i", 0], *a, w8()]
    args += ([w8()] if gated else []) + [far, ["p", 1 << 41], ["z", ws], ["p", 0]]
    return {"fn": f"brownout_moe_w8_{'gate_up' if gated else 'matmul'}", "args": args, **device}


def launched(calls, tmp_path):
    res = record(calls, tmp_path)
    assert all(status == 0 for status, _ in res)
    return [ls for _, ls in res]


@needs_recorder
def test_every_kernel_is_run_by_a_test_case(tmp_path):
    import test_gpu_balance as TB
    import test_gpu_w8 as T8
    calls = [product(*c, a8=a8) for c in T8.CASES for a8 in (False, True)]
    # test_w8_ffn, test_split_tiles_have_the_same_bits
    calls += [product(n, rows, f, d, True) for n, rows, f, d in [
        (1, 1, 1408, 2048), (8, 250, 72, 1408), (1, 1, 24, 40), (2, 9000, 392, 264), (15, 9000, 520, 72), (4, 33, 200, 264),
        (4, 9000, 520, 14336)]]
    calls += [product(1, 1, 1408, 2048, True, a8=True), product(4, 9000, 520, 14336)]
    calls += [{"fn": "brownout_moe_w8_quantize", "args": [*ints(t, rows, K), ["p", PTR], ["p", 1 << 40], ["p", 1 << 41],
                                                          ["p", 0]]}
              for t in (0, 1) for rows, K in ((1, 8), (600, 2048), (9, 4096), (4, 8192), (2, 20008))]
    for T, E, k in TB.SIZES:
        calls += [{"fn": "brownout_moe_balance", "args": [*ints(T, E, k, E), ["p", PTR + 4], ["p", PTR], ["p", 0], ["p", 0],
                                                          ["p", 1 << 40], ["p", 1 << 41], ["p", 1 << 42], ["p", 1 << 43],
                                                          ["z", 1 << 30], ["p", 0]]},  # (test_rows_off_16_byte_chunks)
                  {"fn": "brownout_moe_balance", "args": [*ints(T, E, k, E), ["p", PTR], ["p", PTR], ["p", 0], ["p", 0],
                                                          ["p", 1 << 40], ["p", 1 << 41], ["p", 1 << 42], ["p", 1 << 43],
                                                          ["z", 1 << 30], ["p", 0]]},
                  {"fn": "brownout_moe_balance_grad", "args": [*ints(T, E, k, E), ["p", PTR], ["p", 0], ["p", 0], ["p", PTR],
                                                               ["p", PTR], ["p", 1 << 40], ["p", 0]]}]
    ran = {name for ls in launched(calls, tmp_path) for name, _ in ls}
    built = {k for k in kernels(tmp_path) if re.search(r"OpI8|q8_|balance_", k)}
    assert len(built) >= 30
    assert not built - ran, "\n".join(sorted(built - ran))


@needs_recorder
def test_product_choice(tmp_path):
    """Very few rows round their activations themselves; few rows, and more where the large tiles would leave the CUs
    idle, take the weight-streaming kernels; else the large tiles (half ones where segments are short), with the
    fixup where there is room for it and K is long."""
    few, skinny, whole, half = "few8_kernel", "skinny_", "grouped_gemm_dma_kernel<false, false", "grouped_gemm_dma_kernel<false, true"
    cases = [((15, 4, 2048, 1408), [few]), ((1, 2, 512, 4096), [few]), ((1, 3, 512, 4096), ["q8_", skinny]),
             ((2, 4, 512, 4096), [few]), ((2, 5, 512, 4096), ["q8_", skinny]), ((4, 16, 512, 1024), [few]),
             ((1, 17, 512, 128), ["q8_", skinny]), ((4, 256, 4096, 4096), ["q8_", skinny]),
             # both sides of the estimate
             ((1, 1536, 2048, 1408), ["q8_", skinny]), ((4, 1200, 2048, 1408), ["q8_", skinny]),
             ((15, 1200, 2048, 1408), ["q8_", half]), ((4, 2400, 2048, 1408), ["q8_", half]),
             ((4, 600, 4096, 4096), ["q8_", skinny]), ((4, 4800, 4096, 4096), ["q8_", whole]),
             ((1, 192, 4096, 14336), ["q8_", skinny]), ((1, 384, 4096, 14336), ["q8_", half, "fixup"]),
             ((1, 4000, 1032, 8192), ["q8_", whole, "fixup"]), ((1, 40000, 1032, 6144), ["q8_", whole])]
    for case, want in cases:
        ls, = launched([product(*case)], tmp_path)
        assert [w for w, (name, _) in zip(want, ls) if w in name] == want and len(ls) == len(want), (case, ls)
    # activations that are rounded already, no room for a split
    assert len(launched([product(15, 4, 2048, 1408, a8=True)], tmp_path)[0]) == 1
    assert len(launched([product(1, 4000, 1032, 8192, a8=True, ws=0)], tmp_path)[0]) == 1
    # a source too large for the few-row copies' 32-bit offsets
    ls, = launched([product(256, 256 * 64, 64, 131072, a8=True)], tmp_path)
    assert "grouped_gemm_dma_kernel" in ls[0][0]


@needs_recorder
def test_largest_sizes_are_launched(tmp_path):
    """The widest matrices of the most segments: no dimension of a grid holds 2^32 threads (the runtime refuses them)."""
    sizes = [(256, rows, N, K) for rows in (1, 16, 200, 20000) for N in ((1 << 20) - 8, 1 << 20) for K in (8, 128, 4096)]
    sizes += [(1, 1 << 30, 64, 128), (256, 1 << 30, 8, 8), (256, 16384, 1 << 20, 131072)]
    calls = [product(*c, gated=gated, a8=a8, ws=1 << 44) for c in sizes for gated in (False, True) for a8 in (False, True)]
    calls += [{"fn": "brownout_moe_w8_quantize", "args": [*ints(t, 1 << 30, K), ["p", PTR], ["p", 1 << 50], ["p", 1 << 55],
                                                          ["p", 0]]} for t in (0, 1) for K in (8, 4096, 131072)]
    # a narrow matrix with a long K, where the few-row tiles are taken for any number of rows (gathered from few)
    for rows in (1 << 25, (1 << 30) - 64, 1 << 30):
        c = product(1, rows, 8, 12800, a8=True, ws=0)
        c["args"][6:8] = [["p", PTR], ["i", 100]]
        calls.append(c)
    # bf16, on the same kernels
    calls += [ffn_part("down", 256, rows, 1 << 20, f) for rows in (1, 16, 200) for f in (8, 64, 4096)]
    calls += [ffn_part("up", 256, rows, d, 1 << 20) for rows in (1, 16, 200) for d in (8, 512, 4096)]
    for c, ls in zip(calls, launched(calls, tmp_path)):
        assert ls, c


@needs_recorder
def test_choice_follows_the_cu_count(tmp_path):
    """On half of the chip the few-row tiles take twice the rounds."""
    names = [launched([product(4, 1200, 2048, 1408, cus=c, device=40 + i)], tmp_path)[0][1][0]
             for i, c in enumerate((256, 128))]
    assert "skinny_dma" in names[0] and "grouped_gemm" in names[1]
