"""Refusals of the decode-side calls on the host: every call here fails validation or is an empty no-op, so
nothing is enqueued."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2607_04164_amd import binding as B

OK, NULL, SHAPE, ALIGN, UNSUP, WS = 0, 1, 2, 3, 5, 6
A = 0x10000  # aligned, never read
ODD = 0x10008


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_header_constants():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "brownout_moe.h")).read()
    assert int(re.search(r"#define BMOE_FEW_MAX_TOKENS (\d+)", text).group(1)) == B.FEW_MAX_TOKENS
    assert int(re.search(r"#define BMOE_NORM_MAX_D (\d+)", text).group(1)) == B.NORM_MAX_D
    for name, v in (("NONE", B.GATE_NONE), ("CHANNEL", B.GATE_CHANNEL), ("TOKEN", B.GATE_TOKEN), ("FULL", B.GATE_FULL)):
        assert int(re.search(rf"BMOE_GATE_{name} = (\d+)", text).group(1)) == v
    assert B.w4_row_bytes(8) == 16 and B.w4_row_bytes(32) == 16 and B.w4_row_bytes(40) == 32


def pre(lib, **kw):
    a = dict(dtype=1, T=4, d=64, eps=1e-6, x=A, w=A, out=A, **{})
    a.update(kw)
    return lib.brownout_moe_pre_norm(*(a[n] for n in ("dtype", "T", "d", "eps", "x", "w", "out")), None)


@pytest.mark.parametrize("kw,code", [
    ({"dtype": 2}, UNSUP), ({"T": -1}, SHAPE), ({"d": 12}, SHAPE), ({"d": 0}, SHAPE), ({"d": 32776}, SHAPE),
    ({"eps": 0.0}, SHAPE), ({"eps": 2.0}, SHAPE), ({"eps": float("nan")}, SHAPE), ({"x": None}, NULL),
    ({"out": None}, NULL), ({"x": ODD}, ALIGN), ({"w": ODD}, ALIGN), ({"out": ODD}, ALIGN), ({"T": 0, "x": None}, OK)])
def test_pre_norm_refusals(lib, kw, code):
    assert pre(lib, **kw) == code


def post(lib, **kw):
    a = dict(dtype=0, T=4, d=64, eps=1e-6, norm=1, rho=1.0, mode=0, y=A, x=A, wp=A, gate=None, r=A, wn=None, a=None)
    a.update(kw)
    return lib.brownout_moe_post_norm(*(a[n] for n in ("dtype", "T", "d", "eps", "norm", "rho", "mode", "y", "x", "wp",
                                                       "gate", "r", "wn", "a")), None)


@pytest.mark.parametrize("kw,code", [
    ({"dtype": -1}, UNSUP), ({"T": -5}, SHAPE), ({"d": 40000}, SHAPE), ({"eps": -1.0}, SHAPE), ({"norm": 2}, UNSUP),
    ({"mode": 4}, UNSUP), ({"mode": -1}, UNSUP), ({"rho": float("inf")}, SHAPE), ({"rho": float("nan")}, SHAPE),
    ({"y": None}, NULL), ({"x": None}, NULL), ({"r": None}, NULL), ({"mode": 1}, NULL), ({"mode": 0, "gate": A}, UNSUP),
    ({"norm": 0}, UNSUP), ({"wn": A}, UNSUP), ({"a": A}, UNSUP), ({"a": ODD}, ALIGN), ({"mode": 3, "gate": ODD}, ALIGN),
    ({"mode": 2, "gate": 0x10002}, ALIGN), ({"y": ODD}, ALIGN), ({"T": 0, "y": None}, OK)])
def test_post_norm_refusals(lib, kw, code):
    assert post(lib, **kw) == code


def w4s(codes=A, scales=A, zeros=None, group=64):
    return B._W4Struct(codes, scales, zeros, group)


def matmul(lib, w=None, **kw):
    a = dict(dtype=1, n=2, rows=5, N=16, K=64, off=A, a_rows=None, m=0, a=A, y=A)
    a.update(kw)
    w = w4s() if w is None else w
    ref = None if w is False else ctypes.byref(w)
    return lib.brownout_moe_w4_matmul(*(a[n] for n in ("dtype", "n", "rows", "N", "K", "off", "a_rows", "m", "a")), ref,
                                      a["y"], None)


@pytest.mark.parametrize("kw,code", [
    ({"dtype": 0}, UNSUP), ({"n": 0}, SHAPE), ({"n": 257}, SHAPE), ({"rows": -1}, SHAPE), ({"N": 12}, SHAPE),
    ({"K": 4}, SHAPE), ({"K": (1 << 20) + 8}, SHAPE), ({"off": None}, NULL),
    ({"a": None}, NULL), ({"y": None}, NULL), ({"w": False}, NULL), ({"a_rows": A, "m": 0}, SHAPE), ({"a": ODD}, ALIGN),
    ({"y": ODD}, ALIGN), ({"w": w4s(codes=None)}, NULL), ({"w": w4s(scales=None)}, NULL), ({"w": w4s(group=16)}, UNSUP),
    ({"w": w4s(codes=ODD)}, ALIGN), ({"w": w4s(scales=0x10001)}, ALIGN), ({"rows": 0, "a": None}, OK)])
def test_w4_matmul_refusals(lib, kw, code):
    assert matmul(lib, **kw) == code


@pytest.mark.parametrize("wu,wd,code", [
    (w4s(group=32), w4s(), UNSUP), (w4s(zeros=A), w4s(), UNSUP), (None, w4s(), NULL), (w4s(), None, NULL),
    (w4s(), w4s(group=7), UNSUP)])
def test_w4_ffn_refusals(lib, wu, wd, code):
    ref = lambda w: None if w is None else ctypes.byref(w)  # noqa: E731
    st = lib.brownout_moe_w4_ffn(1, 2, 5, 64, 32, A, None, 0, A, ctypes.byref(w4s()), ref(wu), ref(wd), A, A, None)
    assert st == code
    if wd is not None and wu is not None and wd.group == 64:
        assert lib.brownout_moe_w4_gate_up(1, 2, 5, 64, 32, A, None, 0, A, ctypes.byref(w4s()), ref(wu), A, None) == code


def test_w4_outputs_are_not_their_inputs(lib):
    assert matmul(lib, a=A, y=A) == UNSUP
    ref, other = ctypes.byref(w4s()), A + 4096
    gate_up = lambda a, h: lib.brownout_moe_w4_gate_up(1, 2, 5, 64, 64, A, None, 0, a, ref, ref, h, None)  # noqa: E731
    ffn = lambda a, h, y: lib.brownout_moe_w4_ffn(1, 2, 5, 64, 64, A, None, 0, a, ref, ref, ref, h, y, None)  # noqa: E731
    assert gate_up(A, A) == UNSUP
    assert ffn(A, A, other) == UNSUP and ffn(A, other, other) == UNSUP


@pytest.mark.parametrize("kw,code", [
    ({"dtype": 3}, UNSUP), ({"group": 16}, UNSUP), ({"n": 0}, SHAPE), ({"N": 0}, SHAPE), ({"K": 12}, SHAPE),
    ({"w": None}, NULL), ({"codes": None}, NULL), ({"scales": None}, NULL), ({"w": ODD}, ALIGN), ({"codes": ODD}, ALIGN),
    ({"scales": 0x10001}, ALIGN)])
def test_w4_quantize_refusals(lib, kw, code):
    a = dict(dtype=1, n=1, N=4, K=64, group=32, w=A, codes=A, scales=A, zeros=None)
    a.update(kw)
    assert lib.brownout_moe_w4_quantize(*(a[n] for n in ("dtype", "n", "N", "K", "group", "w", "codes", "scales",
                                                         "zeros")), None) == code


def few(lib, group=0, desc=None, ws_bytes=None, weights=None, **kw):
    d = B.make_desc(T=4, d=64, E=8, top_k=2, G=4, d_ff=32, d_ff_shared=16).replace(**(desc or {}))
    m = B._Matrix(A, A if group else None, None)
    w = B._FewWeights(w_router=A, bias=None, e2g=A, gate=m, up=m, down=m, gate_sh=m, up_sh=m, down_sh=m, group=group)
    for n, v in (weights or {}).items():
        setattr(w, n, v)
    a = dict(x=A, idx=A, tw=A, sg=A, sgate=A, out=A, ws=A)
    a.update(kw)
    size = B.workspace_bytes(d, B.STAGE_FEW) if ws_bytes is None else ws_bytes
    ref = None if weights is False else ctypes.byref(w)
    return lib.brownout_moe_few(ctypes.byref(d), ref, *(a[n] for n in ("x", "idx", "tw", "sg", "sgate", "out", "ws")), size,
                                None)


@pytest.mark.parametrize("kw,code", [
    ({"desc": {"T": 17}}, SHAPE), ({"desc": {"T": -1}}, SHAPE), ({"desc": {"E": 0}}, SHAPE),
    ({"group": 16}, UNSUP), ({"group": 64, "desc": {"dtype": 0}}, UNSUP), ({"x": None}, NULL), ({"idx": None}, NULL),
    ({"tw": None}, NULL), ({"sg": None}, NULL), ({"sgate": None}, NULL), ({"out": None}, NULL),
    ({"weights": {"w_router": None}}, NULL), ({"weights": {"e2g": None}}, NULL), ({"x": ODD}, ALIGN), ({"out": ODD}, ALIGN),
    ({"weights": {"w_router": ODD}}, ALIGN), ({"weights": {"down": B._Matrix(None, None, None)}}, NULL),
    ({"weights": {"down_sh": B._Matrix(None, None, None)}}, NULL), ({"weights": {"up": B._Matrix(ODD, None, None)}}, ALIGN),
    ({"weights": {"up": B._Matrix(A, A, None)}}, UNSUP), ({"weights": {"up": B._Matrix(A, None, A)}}, UNSUP),
    ({"group": 64, "weights": {"up": B._Matrix(A, None, None)}}, NULL),
    ({"group": 64, "weights": {"up": B._Matrix(A, A, A)}}, UNSUP),
    ({"group": 64, "weights": {"up": B._Matrix(A, 0x10001, None)}}, ALIGN),
    ({"ws": None}, WS), ({"ws_bytes": 8}, WS), ({"ws": 0x10010}, ALIGN), ({"weights": False}, NULL),
    ({"desc": {"T": 0}, "x": None, "ws": None}, OK)])
def test_few_refusals(lib, kw, code):
    assert few(lib, **kw) == code


def test_few_workspace_size():
    d = B.make_desc(T=4, d=64, E=8, top_k=2, G=4, d_ff=32, d_ff_shared=16)
    # logits, counters, partial sums of 4 column tiles, hidden values
    assert B.workspace_bytes(d, B.STAGE_FEW) == 256 + 256 + 4 * 8 * 1024 + (4 * 2 * 32 + 4 * 16) * 4
    assert B.workspace_bytes(d.replace(T=17), B.STAGE_FEW) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    for call in (lambda: B.pre_norm(x), lambda: B.post_norm(x, x), lambda: B.w4_quantize(x[None]),
                 lambda: B.W4(torch.zeros((1, 8, 16), dtype=torch.uint8), x, K=32, group=32)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        B.W4(None, None, K=32, group=48)
    with pytest.raises(ValueError):
        B.W4(None, None, K=12, group=32)


def test_reference_unpacks_known_codes():
    """The reference's reading of the format on a row written out by hand."""
    import decode_ref as R
    codes = torch.zeros((1, 1, 32), dtype=torch.uint8)
    codes[0, 0, 0], codes[0, 0, 19] = 0x3A, 0xF0  # columns 0: 10, 1: 3, 38: 0, 39: 15
    scales = torch.tensor([[[2.0, 0.5]]]).to(torch.bfloat16)
    zeros = torch.tensor([[[1, 4]]], dtype=torch.uint8)
    v = R.w4_values(codes, scales, zeros, 40, 32)[0, 0]
    assert v[0] == 18.0 and v[1] == 4.0 and v[2] == -2.0 and v[38] == -2.0 and v[39] == 5.5 and v[37] == -2.0
    assert np.array_equal(R.w4_values(codes, scales, None, 40, 32)[0, 0, :2], [4.0, -10.0])


class Far(torch.Tensor):
    """A tensor of GPU 0 with a size and no memory."""

    @staticmethod
    def __new__(cls, *shape, dtype=torch.bfloat16):
        return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=dtype, device="cuda:0")

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise AssertionError(f"{func} on a tensor without memory")


def test_sizes_past_32_bits_are_refused(monkeypatch):
    """The C calls take int32: 2^32 + 5 rows would arrive as 5."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    n = 2 ** 32 + 5
    x = Far(n, 8)
    w = B.W4(Far(1, 8, 16, dtype=torch.uint8), Far(1, 8, 1), K=8, group=32)
    off, rows, u8 = Far(2, dtype=torch.int32), Far(n, dtype=torch.int32), torch.uint8
    calls = (lambda: B.pre_norm(x, out=x), lambda: B.post_norm(x, x, out=x), lambda: B.w4_quantize(Far(1, n, 8)),
             lambda: B.w4_matmul(off, x, w, y=x), lambda: B.w4_matmul(off, Far(3, 8), w, a_rows=rows, y=x),
             lambda: B.w4_gate_up(off, x, w, w, h=x), lambda: B.w4_ffn(off, x, w, w, w, h=x, y=x),
             lambda: B.W4(Far(1, n, 16, dtype=u8), Far(1, n, 1), K=8, group=32))
    for call in calls:
        with pytest.raises(ValueError, match=f"size of {n}"):
            call()


ELSEWHERE = 1 << 40


@pytest.mark.parametrize("T,kw", [(4, dict(out=A + 128)), (4, dict(x=A + 384)), (4, dict(x=ELSEWHERE, w=A + 512 - 16)),
                                  (2, dict(x=ELSEWHERE, w=A)), (1, dict(x=ELSEWHERE, w=A + 64))])
def test_pre_norm_refuses_shared_memory(lib, T, kw):
    """T rows of 64 bf16 at A: an output that begins inside its input or reaches the weights."""
    assert pre(lib, T=T, **{"w": None, **kw}) == UNSUP


@pytest.mark.parametrize("kw", [
    dict(r=A + 256), dict(x=A + 256), dict(y=A + 16), dict(wp=A), dict(wp=A + 256), dict(mode=1, gate=A + 256),
    dict(mode=2, gate=A + 1020), dict(mode=3, gate=A + 16), dict(a=A + 768), dict(a=ELSEWHERE, wn=A + 512),
    dict(a=ELSEWHERE, wn=ELSEWHERE + 256), dict(r=ELSEWHERE, a=A + 16), dict(r=ELSEWHERE, a=A, mode=2, gate=A)])
def test_post_norm_refuses_shared_memory(lib, kw):
    """Four rows of 64 fp32 at A."""
    assert post(lib, **{"wp": None, **kw}) == UNSUP


def test_w4_products_refuse_shared_memory(lib):
    """Five rows of 64 and 16 bf16: outputs that begin inside the input, or end there."""
    for a, y in ((A, A + 512), (A + 144, A), (A + 16, A)):
        assert matmul(lib, a=a, y=y) == UNSUP
    # gathered rows: a has m of them
    assert matmul(lib, a=A, y=A + 8 * 128 - 16, a_rows=ELSEWHERE, m=8) == UNSUP
    ref = ctypes.byref(w4s())
    ffn = lambda a, h, y: lib.brownout_moe_w4_ffn(1, 2, 5, 64, 64, A, None, 0, a, ref, ref, ref, h, y, None)  # noqa: E731
    assert lib.brownout_moe_w4_gate_up(1, 2, 5, 64, 64, A, None, 0, A, ref, ref, A + 624, None) == UNSUP
    assert ffn(A, A + 16, ELSEWHERE) == UNSUP and ffn(ELSEWHERE, A, A + 624) == UNSUP
