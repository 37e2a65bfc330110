"""The few-token layer, layers with 4-bit weights, and a residual block around them, against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import decode_ref as R
from gpu_util import assert_gates
from paper_2607_04164_amd import binding as B

pytestmark = pytest.mark.gpu

CASES = {
    "one": dict(T=1, d=256, E=8, top_k=2, G=4, f=512),
    "sixteen": dict(T=16, d=512, E=60, top_k=4, G=15, f=352),
    "smallest": dict(T=1, d=8, E=1, top_k=1, G=1, f=8),
    "odd": dict(T=5, d=264, E=7, top_k=3, G=3, f=200, fs=72, norm=1),
    "all-segments": dict(T=16, d=128, E=256, top_k=16, G=256, f=24, fs=40),
    "one-segment": dict(T=9, d=136, E=12, top_k=6, G=1, f=88),
    "wide-hidden": dict(T=3, d=64, E=8, top_k=2, G=4, f=2048, norm=1),
    "wide-model": dict(T=2, d=2048, E=16, top_k=4, G=8, f=40, fs=16),
    "shared-wider": dict(T=7, d=192, E=20, top_k=5, G=6, f=56, fs=488),
    "whole-units-9": dict(T=9, d=1024, E=60, top_k=4, G=15, f=256, fs=128),
    "whole-units-8": dict(T=8, d=1024, E=24, top_k=6, G=20, f=384, norm=1),
    "many-items": dict(T=4, d=1024, E=64, top_k=8, G=32, f=288),
    "many-items-odd": dict(T=5, d=200, E=64, top_k=8, G=40, f=296, fs=24),
    "wider-than-lds": dict(T=16, d=2056, E=8, top_k=1, G=4, f=40),
    "few-columns": dict(T=13, d=40, E=33, top_k=7, G=11, f=16),
    # d and d_ff in whole units, and more tokens than their LDS copies hold
    "whole-units-past-lds-9": dict(T=9, d=4096, E=8, top_k=2, G=4, f=512, norm=1),
    "whole-units-past-lds-16": dict(T=16, d=4096, E=8, top_k=2, G=4, f=512, fs=256),
}
FORMATS = [("bf16", 0, False), ("f32", 0, False), ("bf16", 32, False), ("bf16", 64, True), ("bf16", 128, False),
           ("bf16", 128, True)]
IDS = ["bf16", "f32", "w4-32", "w4-64-zeros", "w4-128", "w4-128-zeros"]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def to_gpu(c, case, group):
    """Device weights of a case, and x."""
    K = {"w_gate": case["d"], "w_up": case["d"], "w_down": case["f"], "w_gate_sh": case["d"], "w_up_sh": case["d"],
         "w_down_sh": case.get("fs", 0)}
    w = {}
    for name, t in c.items():
        if isinstance(t, tuple):
            w[name] = B.W4(t[0].cuda(), t[1].cuda(), None if t[2] is None else t[2].cuda(), K=K[name], group=group)
        else:
            w[name] = t.cuda()
    return w, w.pop("x")


def desc_of(case, dtype):
    return B.make_desc(case["T"], case["d"], case["E"], case["top_k"], case["G"], case["f"], case.get("fs", 0),
                       case.get("norm", 0), dtype)


def reference(c, vals, case):
    sh = tuple(vals[n] for n in ("w_gate_sh", "w_up_sh", "w_down_sh")) if case.get("fs") else None
    return R.few_ref(c["x"].float().numpy(), c["w_router"].float().numpy(), c["bias"].numpy(), c["e2g"].numpy(),
                     tuple(vals[n] for n in ("w_gate", "w_up", "w_down")), case["top_k"], case.get("norm", 0), sh)


def check(layer, out, ref, dtype, what):
    r = layer.bufs["route"]
    for n in ("topk_idx", "slot_group"):
        assert np.array_equal(r[n].cpu().numpy(), ref[n]), f"{what}: {n}"
    for n in ("topk_w", "slot_gate"):
        assert_gates(r[n].cpu().numpy(), ref[n], f"{what}: {n}")
    R.assert_few(out, ref, dtype, what)


@pytest.mark.parametrize("dtype,group,zeros", FORMATS, ids=IDS)
@pytest.mark.parametrize("name", list(CASES))
def test_few(name, dtype, group, zeros):
    case = CASES[name]
    c, vals = R.make_case(11, dtype=dtype, group=group, zeros=zeros, **case)
    w, x = to_gpu(c, case, group)
    layer = B.LayerForward(desc_of(case, dtype), w, few_tokens=True)
    layer.ws.fill_(0xFF)  # NaN in every hidden value that is not written
    out = layer(x)
    check(layer, out, reference(c, vals, case), dtype, name)
    first = out.clone()
    layer.ws.fill_(0xFF)
    assert torch.equal(layer(x), first)


@pytest.mark.parametrize("dtype,group,zeros", FORMATS[:3], ids=IDS[:3])
def test_every_token_count(dtype, group, zeros):
    for T in range(1, 17):
        case = dict(T=T, d=96, E=10, top_k=3, G=5, f=48, fs=24)
        c, vals = R.make_case(T, dtype=dtype, group=group, zeros=zeros, **case)
        w, x = to_gpu(c, case, group)
        layer = B.LayerForward(desc_of(case, dtype), w, few_tokens=True)
        check(layer, layer(x), reference(c, vals, case), dtype, f"T={T}")


@pytest.mark.parametrize("dtype,group,zeros", [f for f in FORMATS if f[0] == "bf16"], ids=[i for i in IDS if i != "f32"])
@pytest.mark.parametrize("T", [3, 11])
def test_more_columns_than_the_chip_holds(T, dtype, group, zeros):
    """16392 output columns: too many tiles for workgroups to share one, and activations past the LDS."""
    case = dict(T=T, d=16392, E=4, top_k=2, G=2, f=72, fs=8)
    c, vals = R.make_case(17, dtype=dtype, group=group, zeros=zeros, **case)
    w, x = to_gpu(c, case, group)
    layer = B.LayerForward(desc_of(case, dtype), w, few_tokens=True)
    layer.ws.fill_(0xFF)
    check(layer, layer(x), reference(c, vals, case), dtype, f"T={T}")


def test_ties_and_masked_experts():
    """Equal router rows (the lower index wins) and experts masked by the lowest bias, fewer left than top_k."""
    case = dict(T=6, d=128, E=12, top_k=5, G=4, f=64)
    c, vals = R.make_case(3, **case)
    c["w_router"][:] = c["w_router"][0]
    c["bias"][:] = 0
    w, x = to_gpu(c, case, 0)
    layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)
    check(layer, layer(x), reference(c, vals, case), "bf16", "ties")
    assert np.array_equal(layer.bufs["route"]["topk_idx"].cpu().numpy(), np.tile(np.arange(5), (6, 1)))
    c, vals = R.make_case(4, **case)
    c["bias"][3:] = torch.finfo(torch.float32).min
    w, x = to_gpu(c, case, 0)
    layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)
    check(layer, layer(x), reference(c, vals, case), "bf16", "masked")


def test_tokens_do_not_mix():
    """An infinite weight reaches only the tokens that call its segment, a NaN token only itself."""
    case = dict(T=8, d=64, E=6, top_k=1, G=6, f=48)
    c, vals = R.make_case(21, **case)
    ref = reference(c, vals, case)
    g0 = ref["slot_group"][0, 0]
    hit = (ref["slot_group"] == g0).any(axis=1)
    assert hit.any() and not hit.all()
    c["w_down"][g0, 5, 7] = float("inf")
    w, x = to_gpu(c, case, 0)
    layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)
    out = layer(x).float().cpu().numpy()
    assert not np.isfinite(out[hit, 5]).any() and np.isfinite(out[~hit]).all()
    c, vals = R.make_case(21, **case)
    w, x = to_gpu(c, case, 0)
    layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)
    clean = layer(x).clone()
    x[3] = float("nan")
    out = layer(x)
    keep = [t for t in range(8) if t != 3]
    assert torch.equal(out[keep], clean[keep])


@pytest.mark.parametrize("dtype,group,zeros", FORMATS[:3], ids=IDS[:3])
@pytest.mark.parametrize("fs", [0, 72])
def test_experts_of_no_segment(dtype, group, zeros, fs):
    """Experts that the map sends nowhere give nothing: one segment of four left, then none, so that the output
    is the shared experts' or zero."""
    case = dict(T=6, d=136, E=8, top_k=3, G=4, f=48, fs=fs)
    for left in (1, 0):
        c, vals = R.make_case(31, dtype=dtype, group=group, zeros=zeros, **case)
        c["e2g"][c["e2g"] >= left] = -1
        w, x = to_gpu(c, case, group)
        layer = B.LayerForward(desc_of(case, dtype), w, few_tokens=True)
        layer.ws.fill_(0xFF)
        out = layer(x)
        ref = reference(c, vals, case)
        ref["slot_gate"] = np.where(ref["slot_group"] >= 0, ref["slot_gate"], 0)  # as the route kernels write it
        check(layer, out, ref, dtype, f"{left} left")
        if not left and not fs:
            assert not out.any()


@pytest.mark.parametrize("E,G", [(12, 5), (200, 30)])
@pytest.mark.parametrize("T", [4, 16])
def test_map_entries_out_of_range(T, E, G):
    """An entry outside [0, G), whatever its bits, sends its expert nowhere, as brownout_moe_route takes it."""
    case = dict(T=T, d=128, E=E, top_k=6, G=G, f=40)
    wild = [-2, -100, -65536, -(2 ** 31), G, 300, 65535, 65536, 65537 + G, 70000, 131073, 2 ** 31 - 1]
    c, vals = R.make_case(41, zipf=0.0, **case)
    # every second of the experts that are picked most often
    first = reference(c, vals, case)
    order = np.argsort(-np.bincount(first["topk_idx"].ravel(), minlength=E), kind="stable")
    for i, e in enumerate(order[:2 * len(wild):2]):
        c["e2g"][int(e)] = wild[i % len(wild)]
    w, x = to_gpu(c, case, 0)
    desc = desc_of(case, "bf16")
    layer = B.LayerForward(desc, w, few_tokens=True)
    layer.ws.fill_(0xFF)
    out = layer(x)
    want = B.route(desc, x, w["w_router"], w["bias"], w["e2g"])
    c["e2g"][(c["e2g"] < 0) | (c["e2g"] >= G)] = -1
    ref = reference(c, vals, case)
    ref["slot_gate"] = np.where(ref["slot_group"] >= 0, ref["slot_gate"], 0)
    assert (ref["slot_group"] < 0).any() and (ref["slot_group"] >= 0).any()
    check(layer, out, ref, "bf16", "map")
    for n in ("topk_idx", "slot_group"):
        assert torch.equal(layer.bufs["route"][n], want[n]), n
    for n in ("topk_w", "slot_gate"):
        assert_gates(layer.bufs["route"][n].cpu().numpy(), want[n].cpu().numpy(), n)


@pytest.mark.parametrize("T", [5, 12])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, True)])
def test_nan_scales_do_not_spread(T, group, zeros):
    """A row of NaN scales reaches one output column of the tokens that call its segment, and units that end
    inside a row (200 columns) take nothing of the next row."""
    case = dict(T=T, d=264, E=6, top_k=1, G=6, f=200, fs=72)
    c, vals = R.make_case(21, group=group, zeros=zeros, **case)
    ref = reference(c, vals, case)
    w, x = to_gpu(c, case, group)
    layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)
    clean = layer(x).float().cpu().numpy()
    g0 = ref["slot_group"][0, 0]
    hit = (ref["slot_group"] == g0).any(axis=1)
    assert hit.any() and not hit.all()
    c["w_down"][1][g0, 7] = float("nan")
    w, x = to_gpu(c, case, group)
    out = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)(x).float().cpu().numpy()
    assert np.isnan(out[hit, 7]).all()
    bad = np.zeros_like(out, dtype=bool)
    bad[hit, 7] = True
    assert np.array_equal(out[~bad], clean[~bad])
    c, vals = R.make_case(21, group=group, zeros=zeros, **case)
    c["w_gate"][1][g0, 9] = float("nan")  # a hidden column of the callers, so all of their outputs
    w, x = to_gpu(c, case, group)
    out = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)(x).float().cpu().numpy()
    assert np.isnan(out[hit]).all() and np.array_equal(out[~hit], clean[~hit])


def test_same_as_the_four_calls():
    """Routing bit for bit, the output within both paths' rounding: the four calls round h, y and out (three
    roundings of at most 2^-8, each at random), this path once."""
    case = dict(T=16, d=512, E=60, top_k=4, G=15, f=352, fs=176)
    c, _ = R.make_case(8, **case)
    w, x = to_gpu(c, case, 0)
    few, four = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True), B.LayerForward(desc_of(case, "bf16"), w)
    a, b = few(x), four(x)
    for n in ("topk_idx", "slot_group"):
        assert torch.equal(few.bufs["route"][n], four.bufs["route"][n])
    for n in ("topk_w", "slot_gate"):
        assert_gates(few.bufs["route"][n].cpu().numpy(), four.bufs["route"][n].cpu().numpy(), n)
    assert np.linalg.norm(R.np64(a) - R.np64(b)) <= 4 * 2.0 ** -8 * np.linalg.norm(R.np64(b))


@pytest.mark.parametrize("T,fs", [(1, 0), (40, 72), (300, 0)])
def test_w4_layer_of_any_size(T, fs):
    """LayerForward with 4-bit weights on the dispatch path. Its h and y are rounded to bf16 on the way: 2^-8 of
    each, with random signs, beside the output's own rounding."""
    case = dict(T=T, d=256, E=12, top_k=3, G=5, f=200, fs=fs)
    c, vals = R.make_case(T, group=64, zeros=True, **case)
    w, x = to_gpu(c, case, 64)
    layer = B.LayerForward(desc_of(case, "bf16"), w)
    out = R.np64(layer(x))
    ref = reference(c, vals, case)
    rms = np.sqrt((ref["out"] ** 2).mean(axis=1, keepdims=True))
    tol = 2.0 ** -8 * np.abs(ref["out"]) + 5 * 2 * 2.0 ** -8 * rms
    assert (np.abs(out - ref["out"]) <= tol).all()
    assert np.linalg.norm(out - ref["out"]) <= 3 * 2.0 ** -8 * np.linalg.norm(ref["out"])
    # stage by stage as in one call
    layer.route(x), layer.dispatch(x)
    h = layer.ffn_gate_up(x=x).clone()
    y = layer.ffn_down().clone()
    n = int(layer.bufs["dispatch"]["offsets"][-1])
    y2, h2 = layer.ffn(x=x)
    assert torch.equal(h[:n], h2[:n]) and torch.equal(y[:n], y2[:n])


@pytest.mark.parametrize("dtype,group,zeros", FORMATS[:4], ids=IDS[:4])
def test_residual_block(dtype, group, zeros):
    """Two blocks in a row, the first handing its normed output on; every stage against 64 bits on the
    values that the stage before stored."""
    case = dict(T=6, d=264, E=10, top_k=3, G=4, f=96, fs=40)
    rng = np.random.default_rng(1)
    x = R.rand(rng, (6, 264), 2.0, dtype).cuda()
    given = None
    for i in range(2):
        c, vals = R.make_case(30 + i, dtype=dtype, group=group, zeros=zeros, **case)
        w, _ = to_gpu(c, case, group)
        layer = B.LayerForward(desc_of(case, dtype), w, few_tokens=True)
        norms = {n: R.rand(rng, (264,), 1.0, dtype).cuda() for n in ("w_pre", "w_post", "gate")}
        if i == 0:
            norms["w_next"] = R.rand(rng, (264,), 1.0, dtype).cuda()
        block = B.ResidualBlock(layer, norms, res_scale=0.9, next_norm=i == 0)
        r, a_next = block(x, given)
        a = block.bufs["a"] if given is None else given
        if given is None:
            want = R.np64(x) * R.inv_rms(R.np64(x), 1e-6) * R.np64(norms["w_pre"])
            R.assert_rounded(a, want, R.SUM * np.abs(want), dtype, "a")
        c["x"] = a.cpu()
        ref = reference(c, vals, case)
        check(layer, layer.bufs["out"], ref, dtype, f"block {i}")
        wn = norms.get("w_next")
        want, er, wa, ea = R.post_ref(R.np64(layer.bufs["out"]), R.np64(x), True, R.np64(norms["w_post"]),
                                      R.np64(norms["gate"]), 0.9, None if wn is None else R.np64(wn), 1e-6)
        R.assert_rounded(r, want, er, dtype, "r")
        if i == 0:
            R.assert_rounded(a_next, wa, ea, dtype, "a'")
        x, given = r, a_next
    assert given is None


@pytest.mark.parametrize("dtype,group,zeros", FORMATS[:3], ids=IDS[:3])
def test_few_graph_and_streams(dtype, group, zeros):
    """A captured block step replayed with new inputs and eager work between; two layers on two streams at once."""
    case = dict(T=4, d=256, E=16, top_k=4, G=8, f=176, fs=48)
    c, _ = R.make_case(5, dtype=dtype, group=group, zeros=zeros, **case)
    w, x = to_gpu(c, case, group)
    layer, other = (B.LayerForward(desc_of(case, dtype), w, few_tokens=True) for _ in range(2))
    xs = [R.rand(np.random.default_rng(i), (4, 256), 1.0, dtype).cuda() for i in range(3)]
    want = [other(v).clone() for v in xs]
    block = B.ResidualBlock(layer, next_norm=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block(x)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r, a = block(x, x)  # x as its own normed input: the layer sees it as it is
    for k in range(4):
        x.copy_(xs[k % 3])
        layer.bufs["out"].zero_()
        other(xs[(k + 1) % 3])
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.bufs["out"], want[k % 3]), f"replay {k}"
        eager = B.post_norm(want[k % 3], xs[k % 3], True, next_norm=True)
        assert torch.equal(r, eager[0]) and torch.equal(a, eager[1]), f"replay {k}"
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        p = layer(xs[0])
        q = other(xs[1], stream=side)
        torch.cuda.synchronize()
        assert torch.equal(p, want[0]) and torch.equal(q, want[1])


def test_another_device_is_refused():
    case = CASES["one"]
    c, _ = R.make_case(5, group=32, **case)
    w, x = to_gpu(c, case, 32)
    layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)
    layer._few_device += 1
    with pytest.raises(ValueError, match="the layer on GPU"):
        layer(x)
    w["w_up"].device += 1
    with pytest.raises(ValueError, match="4-bit weights are on GPU"):
        B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)


def _hidden_then_out(x, slots, vals):
    """One token's output from hidden values held in fp32, where they can be infinite; slots: (segment, gate, shared)."""
    out = np.zeros(len(x))
    with np.errstate(all="ignore"):
        for g, gate, sh in slots:
            wg, wu, wd = (vals[n + "_sh" * sh][g] for n in ("w_gate", "w_up", "w_down"))
            h = (R.silu(wg @ x) * (wu @ x) * np.float64(gate)).astype(np.float32).astype(np.float64)
            out += (wd * h).sum(1)
    return out


@pytest.mark.parametrize("T", [3, 8, 16])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("fs", [0, 72])
def test_sums_that_leave_fp32(T, group, zeros, fs):
    """4-bit layers: activations and hidden values near the largest value, whose sums with the codes + 16 would be
    infinite; then infinite hidden values. Tokens beside them are as they would be alone. (In one of the cases a
    hidden value of the shared experts is past the largest value already with one large factor: -3.427e38.)"""
    case = dict(T=T, d=264, E=6, top_k=2, G=3, f=200, fs=fs)
    c, vals = R.make_case(51, group=group, zeros=zeros, **case)
    K = {"w_gate": 264, "w_up": 264, "w_down": 200, "w_gate_sh": 264, "w_up_sh": 264, "w_down_sh": fs}
    names = ["w_gate", "w_up"] + (["w_gate_sh", "w_up_sh"] if fs else [])
    c["w_router"][:, 0] = 0
    for n in names:
        c[n][1][:, :, 0] = 0  # columns of the first group: only in the hidden columns below
    for n in names:
        c[n][0][:, 5, 0] |= 15  # (code 15 in column 0)
        if zeros:
            c[n][2][:, 5, 0] = 8
    for n in names[::2]:
        c[n][1][:, 5, 0] = 0.05  # a large factor of one hidden column, the other one stays as it is
    w, x = to_gpu(c, case, group)
    clean = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)(x).clone()
    hot = np.arange(T) % 3 == 1
    c["x"][torch.from_numpy(hot), 0] = 3.0e38
    x64, finite = R.np64(c["x"]), 0
    for factors in (1, 2):
        if factors == 2:
            for n in names[1::2]:
                c[n][1][:, 5, 0] = 0.05
        for n in vals:
            vals[n] = R.w4_values(*c[n], K[n], group)
        with np.errstate(all="ignore"):
            ref = reference(c, vals, case)
        w, x = to_gpu(c, case, group)
        layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=True)
        layer.ws.fill_(0xFF)
        out = layer(x)
        o64 = R.np64(out)
        for t in np.flatnonzero(hot):
            slots = [(g, gate, 0) for g, gate in zip(ref["slot_group"][t], ref["slot_gate"][t]) if g >= 0]
            want = _hidden_then_out(x64[t], slots + ([(0, 1.0, 1)] if fs else []), vals)
            if np.isfinite(want).all():
                assert factors == 1 and np.abs(want).max() > 1e35
                R.assert_few(out[t:t + 1], {"out": ref["out"][t:t + 1]}, "bf16", f"token {t}")
                finite += 1
                continue
            assert not np.isfinite(want).any()
            for f in (np.isnan, np.isposinf, np.isneginf):
                assert np.array_equal(f(o64[t]), f(want)), f"token {t}: {f.__name__}"
        keep = torch.from_numpy(~hot).cuda()
        if factors == 1:
            assert torch.equal(out[keep], clean[keep])
    assert finite >= hot.sum() - 1


@pytest.mark.parametrize("dtype,group,zeros", FORMATS[:3], ids=IDS[:3])
def test_gate_keeps_a_hidden_value_finite(dtype, group, zeros):
    """silu(g) u past the largest value, times the token's gate below it: the hidden value, so the output, is finite."""
    case = dict(T=3, d=64, E=4, top_k=2, G=4, f=24)
    c, vals = R.make_case(7, dtype=dtype, group=group, zeros=zeros, zipf=0.0, **case)
    c["w_router"][:, :32] = 0
    c["x"][:, :32] = 0
    c["x"][1, 0], c["x"][1, 1] = 2.0 ** 127, 4.0
    for n, k in (("w_gate", 0), ("w_up", 1)):
        if group:
            codes, scales, _ = c[n]
            codes[:, 5, :16] = 0x88
            codes[:, 5, 0] = 0x8A if k == 0 else 0xA8  # two steps in column k, none beside it
            scales[:, 5, 0] = 0.5
            codes[:, :5, 0], codes[:, 6:, 0] = 0x88, 0x88
            vals[n] = R.w4_values(*c[n], 64, group)
        else:
            c[n][:, :, :2] = 0
            c[n][:, 5, :32] = 0
            c[n][:, 5, k] = 1.0
            vals[n] = R.np64(c[n])
    with np.errstate(over="ignore"):
        ref = reference(c, vals, case)
    g, gate = ref["slot_group"][1], ref["slot_gate"][1]
    x = R.np64(c["x"])[1]
    big = [(R.silu(vals["w_gate"][s] @ x) * (vals["w_up"][s] @ x))[5] for s in g]
    w, x = to_gpu(c, case, group)
    layer = B.LayerForward(desc_of(case, dtype), w, few_tokens=True)
    assert any(b > 3.41e38 for b in big) and all(abs(b * y) < 3.3e38 for b, y in zip(big, gate))
    check(layer, layer(x), ref, dtype, "gate")


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("device", ["cpu", "cuda:1"])
def test_buffers_on_another_device_are_refused(device, few):
    case = CASES["one"]
    c, _ = R.make_case(5, group=32, **case)
    w, _ = to_gpu(c, case, 32)
    with pytest.raises(ValueError, match="buffers would be on"):
        B.LayerForward(desc_of(case, "bf16"), w, device=device, few_tokens=few)
    for same in ("cuda", "cuda:0", torch.device("cuda", 0)):
        B.LayerForward(desc_of(case, "bf16"), w, device=same, few_tokens=few)


@pytest.mark.parametrize("few", [True, False])
def test_calls_from_another_device_are_refused(few, monkeypatch):
    """The parts of a 4-bit layer too: with x on another GPU, and with another GPU the current one."""
    case = dict(T=4, d=64, E=6, top_k=2, G=3, f=40, fs=24)
    c, _ = R.make_case(5, group=32, **case)
    w, x = to_gpu(c, case, 32)
    layer = B.LayerForward(desc_of(case, "bf16"), w, few_tokens=few)
    want = layer(x).clone()
    parts = [] if few else [lambda: layer.route(x), lambda: layer.dispatch(x), lambda: layer.ffn(x=x),
                            lambda: layer.ffn_gate_up(x=x), lambda: layer.shared(x), lambda: layer.shared_fork(x)]
    layer._few_device += 1
    for call in (lambda: layer(x), *parts):
        with pytest.raises(ValueError, match="the layer on GPU"):
            call()
    layer._few_device -= 1
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        side = torch.cuda.Stream(device=0)
        for call in (lambda: layer(x), lambda: layer(x, side), *parts, *([] if few else [layer.ffn_down, layer.combine])):
            with pytest.raises(ValueError, match="the layer on GPU"):
                call()
    assert torch.equal(layer(x), want)


@pytest.mark.parametrize("group,zeros", [(32, True), (128, False)])
def test_w4_layer_graph(group, zeros):
    """The four calls of a 4-bit layer with shared experts on their own stream, captured: replays give the eager bits."""
    case = dict(T=24, d=256, E=12, top_k=3, G=5, f=200, fs=72)
    c, _ = R.make_case(61, group=group, zeros=zeros, **case)
    w, x = to_gpu(c, case, group)
    layer, other = (B.LayerForward(desc_of(case, "bf16"), w) for _ in range(2))
    xs = [R.rand(np.random.default_rng(i), (24, 256), 1.0, "bf16").cuda() for i in range(3)]
    want = [other(v).clone() for v in xs]
    layer(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = layer(x)
    for k in range(4):
        x.copy_(xs[k % 3])
        out.zero_()
        other(xs[(k + 1) % 3])
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k % 3]), f"replay {k}"
