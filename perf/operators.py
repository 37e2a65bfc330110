"""The decode-side operators, as cases that can be timed and compared.

Three operators that a decode step of this layer runs together:

* ``few``: a whole grouped MoE layer for 1 to 16 tokens (gate, map, the
  reached segments' SwiGLU FFNs, the gate-weighted sum, shared experts), its
  weights in the layer's type or in 4 bits with group scales;
* ``w4_matmul`` / ``w4_ffn``: products of grouped rows with 4-bit weights;
* ``pre_norm`` / ``post_norm``: the RMS norms before and after the layer, the
  latter with its gate, the residual stream and the next block's norm.

4-bit weights of a matrix [n, N, K]: codes [n, N, 16 ceil(K/32)] uint8 (byte b
of a row: column 2b in the low four bits, 2b+1 in the high four; the bytes past
K/2 are padding), scales [n, N, ceil(K/group)] bf16, zeros the same shape in
uint8 or none (8): w = scale * (code - zero).

``own`` False computes plain torch expressions of these definitions; True makes
the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

__all__ = ["listed", "draw", "prepare", "run", "work", "exact"]

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _few(name, T, d, E, top_k, G, d_ff, *, dtype="bf16", zipf=1.2, norm=0, shared=0, group=0, zeros=False):
    """group 0: weights in dtype; else 4-bit weights with that group."""
    return {"name": name, "kind": "few", "T": T, "d": d, "E": E, "top_k": top_k, "G": G, "d_ff": d_ff,
            "dtype": dtype, "zipf": zipf, "norm": norm, "shared": shared, "group": group, "zeros": zeros}


def _w4(name, kind, rows, n, N, K, group, zeros, gather=False):
    return {"name": name, "kind": kind, "rows": rows, "n": n, "N": N, "K": K, "group": group, "zeros": zeros,
            "gather": gather, "dtype": "bf16"}


def _post(name, T, d, gate, *, norm=True, after=True, dtype="bf16"):
    """gate: none, channel ([d]), token ([T, 1], fp32) or full ([T, d]); after: the next block's norm in the same pass."""
    return {"name": name, "kind": "post_norm", "T": T, "d": d, "gate": gate, "norm": norm, "next": after,
            "dtype": dtype}


def listed():
    return [
        # one request's next token on the fine-grained layer: latency
        _few("few_1", 1, 2048, 60, 4, 15, 1408),
        # a small decode batch that reaches most of the segments
        _few("few_16", 16, 2048, 60, 4, 15, 1408),
        # a few requests with shared experts and heavy skew
        _few("few_shared_4", 4, 2048, 64, 6, 16, 1408, zipf=1.5, shared=2816),
        # wide experts, Mixtral-shaped: two requests
        _few("few_wide_2", 2, 4096, 8, 2, 4, 14336, zipf=1.0, norm=1),
        # the fp32 layer a program checks its numerics with, at odd sizes
        _few("few_f32_3", 3, 264, 7, 3, 3, 200, dtype="f32", shared=72),
        # one token with 4-bit experts
        _few("few_w4_1", 1, 2048, 60, 4, 15, 1408, group=128),
        # six tokens, wide 4-bit experts with zero points
        _few("few_w4_wide_6", 6, 4096, 8, 2, 4, 14336, zipf=1.0, norm=1, group=64, zeros=True),
        # one row through one 4-bit matrix: the smallest product
        _w4("w4_matvec_1", "w4_matmul", 1, 1, 4096, 4096, 128, False),
        # the grouped FFN of a decode step in 4 bits, ragged segments, gathered rows
        _w4("w4_ffn_decode", "w4_ffn", 250, 8, 1408, 2048, 32, True, gather=True),
        # one token past a block: the smallest norm
        _post("post_norm_1", 1, 2048, "channel"),
        # the norm before a block, odd rows and width, fp32
        {"name": "pre_norm_f32", "kind": "pre_norm", "T": 1001, "d": 4104, "dtype": "f32"},
        # prefill: every stream of the block boundary in one pass
        _post("post_norm_8192", 8192, 2048, "full"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["few", "few", "few", "few_w4", "few_w4", "w4_matmul", "w4_ffn", "pre_norm", "post_norm"])
    if kind in ("few", "few_w4"):
        E = rng.choice([8, 60, 64, rng.randint(4, 128)])
        k = min(E, rng.choice([1, 2, 4, 6, 8]))
        G = rng.randint(max(1, E // 8), min(E, 32))
        d, f = 8 * _log(rng, 32, 512), 8 * _log(rng, 16, 512)
        w4 = kind == "few_w4"
        c = _few("", _log(rng, 1, 16), d, E, k, G, f, zipf=round(rng.uniform(0.5, 1.5), 2), norm=rng.randint(0, 1),
                 dtype="bf16" if w4 or rng.random() < 0.8 else "f32", shared=rng.choice([0, 0, 8 * rng.randint(8, 352)]),
                 group=rng.choice([32, 64, 128]) if w4 else 0, zeros=w4 and rng.random() < 0.5)
    elif kind in ("w4_matmul", "w4_ffn"):
        n = rng.choice([1, rng.randint(2, 32)])
        c = _w4("", kind, _log(rng, 1, 32 * n), n, 8 * _log(rng, 16, 512), 8 * _log(rng, 16, 512),
                rng.choice([32, 64, 128]), rng.random() < 0.5, rng.random() < 0.5)
    elif kind == "pre_norm":
        c = {"name": "", "kind": kind, "T": _log(rng, 1, 8192), "d": 8 * _log(rng, 32, 640),
             "dtype": rng.choice(["bf16", "bf16", "f32"])}
    else:
        c = _post("", _log(rng, 1, 6144), 8 * _log(rng, 32, 256), rng.choice(["none", "channel", "token", "full"]),
                  norm=rng.random() < 0.7, after=rng.random() < 0.7, dtype=rng.choice(["bf16", "bf16", "f32"]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs

def _randn(gen, shape, std, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype).mul_(std)


def _w4_weights(gen, n, N, K, group, zeros, std):
    """Codes of roughly normal weights (clipped at about 2.5 deviations), scales that vary by group."""
    pitch, ng = 16 * -(-K // 32), -(-K // group)
    q = torch.randn((n, N, 2 * pitch), generator=gen, device="cuda", dtype=torch.bfloat16)
    q = q.mul_(3.0).add_(8.0).round_().clamp_(0, 15).to(torch.uint8)
    codes = q[:, :, 0::2] | (q[:, :, 1::2] << 4)
    scales = (torch.rand((n, N, ng), generator=gen, device="cuda") + 0.5).mul_(std / 3.0).to(torch.bfloat16)
    z = torch.randint(6, 11, (n, N, ng), generator=gen, device="cuda", dtype=torch.uint8) if zeros else None
    return {"codes": codes, "scales": scales, "zeros": z, "K": K, "group": group}


def _matrix(case, gen, n, N, K, std):
    if case["group"]:
        return _w4_weights(gen, n, N, K, case["group"], case["zeros"], std)
    return _randn(gen, (n, N, K), std, _DT[case["dtype"]])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    dt, kind = _DT[case["dtype"]], case["kind"]
    s = {"case": case}
    if kind == "few":
        T, d, E, k, G, f, fs = (case[n] for n in ("T", "d", "E", "top_k", "G", "d_ff", "shared"))
        std = 1.0 / math.sqrt(d)
        e2g = np.empty(E, np.int32)
        e2g[rng.permutation(E)] = (np.arange(E) * G) // E
        q = (1.0 + rng.permutation(E)) ** -case["zipf"]
        s["x"] = _randn(gen, (T, d), 1.0, dt)
        w = {"w_router": _randn(gen, (E, d), std, dt), "e2g": torch.from_numpy(e2g).cuda(),
             "bias": torch.from_numpy(np.log(q / q.sum()).astype(np.float32)).cuda(),
             "w_gate": _matrix(case, gen, G, f, d, std), "w_up": _matrix(case, gen, G, f, d, std),
             "w_down": _matrix(case, gen, G, d, f, std)}
        if fs:
            w.update(w_gate_sh=_matrix(case, gen, 1, fs, d, std), w_up_sh=_matrix(case, gen, 1, fs, d, std),
                     w_down_sh=_matrix(case, gen, 1, d, fs, std))
        s["w"] = w
    elif kind in ("w4_matmul", "w4_ffn"):
        n, N, K, rows = case["n"], case["N"], case["K"], case["rows"]
        cut = np.sort(rng.integers(0, rows + 1, n - 1)) if n > 1 else np.zeros(0, np.int64)
        s["offsets"] = torch.from_numpy(np.concatenate([[0], cut, [rows]]).astype(np.int32)).cuda()
        m = -(-rows // 4) if case["gather"] else rows
        s["a_rows"] = torch.from_numpy(rng.integers(0, m, rows).astype(np.int32)).cuda() if case["gather"] else None
        s["a"] = _randn(gen, (m, K), 1.0, dt)
        std = 1.0 / math.sqrt(K)
        if kind == "w4_matmul":
            s["w"] = (_matrix(case, gen, n, N, K, std),)
            s["out"] = (torch.empty((rows, N), dtype=dt, device="cuda"),)
        else:
            s["w"] = (_matrix(case, gen, n, N, K, std), _matrix(case, gen, n, N, K, std),
                      _matrix(case, gen, n, K, N, std))
            s["out"] = (torch.empty((rows, K), dtype=dt, device="cuda"), torch.empty((rows, N), dtype=dt, device="cuda"))
    else:
        T, d = case["T"], case["d"]
        # a residual stream whose channels differ in size, as trained ones do
        s["x"] = (torch.randn((T, d), generator=gen, device="cuda")
                  * torch.exp(torch.randn((d,), generator=gen, device="cuda"))).to(dt)
        s["w"] = (1.0 + 0.2 * torch.randn((d,), generator=gen, device="cuda")).to(dt)
        s["out"] = torch.empty((T, d), dtype=dt, device="cuda")
        if kind == "post_norm":
            s["y"] = _randn(gen, (T, d), 0.3, dt)
            s["w_post"] = (1.0 + 0.2 * torch.randn((d,), generator=gen, device="cuda")).to(dt) if case["norm"] else None
            shape = {"none": None, "channel": (d,), "token": (T, 1), "full": (T, d)}[case["gate"]]
            s["gate"] = None if shape is None else _randn(gen, shape, 0.5, torch.float32 if case["gate"] == "token" else dt)
            s["res_scale"] = 0.875
            s["out_next"] = torch.empty((T, d), dtype=dt, device="cuda") if case["next"] else None
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that serves these weights keeps between calls."""
    from paper_2607_04164_amd import binding as B
    case = s["case"]
    wrap = lambda w: B.W4(w["codes"], w["scales"], w["zeros"], K=w["K"], group=w["group"]) if isinstance(w, dict) else w  # noqa: E731
    if case["kind"] == "few":
        desc = B.make_desc(case["T"], case["d"], case["E"], case["top_k"], case["G"], case["d_ff"], case["shared"],
                           case["norm"], case["dtype"])
        s["layer"] = B.LayerForward(desc, {n: wrap(w) for n, w in s["w"].items()}, few_tokens=True)
    elif case["kind"] in ("w4_matmul", "w4_ffn"):
        s["w4"] = tuple(wrap(w) for w in s["w"])


EPS = 1e-6


def run(state):
    if own:
        return _run_own(state)
    return {"few": _plain_few, "w4_matmul": _plain_w4, "w4_ffn": _plain_w4, "pre_norm": _plain_pre,
            "post_norm": _plain_post}[state["case"]["kind"]](state)


def _run_own(s):
    from paper_2607_04164_amd import binding as B
    kind = s["case"]["kind"]
    if kind == "few":
        out = s["layer"](s["x"])
        return {"out": out, **s["layer"].bufs["route"]}
    if kind == "w4_matmul":
        return {"y": B.w4_matmul(s["offsets"], s["a"], s["w4"][0], a_rows=s["a_rows"], y=s["out"][0])}
    if kind == "w4_ffn":
        y, h = B.w4_ffn(s["offsets"], s["a"], *s["w4"], a_rows=s["a_rows"], y=s["out"][0], h=s["out"][1])
        return {"y": y, "h": h}
    if kind == "pre_norm":
        return {"a": B.pre_norm(s["x"], s["w"], EPS, out=s["out"])}
    r, a = B.post_norm(s["y"], s["x"], s["case"]["norm"], w_post=s["w_post"], gate=s["gate"], res_scale=s["res_scale"],
                       next_norm=s["case"]["next"], w_next=s["w"] if s["case"]["next"] else None, eps=EPS,
                       out=s["out"], out_next=s["out_next"])
    return {"r": r, "a": a} if s["case"]["next"] else {"r": r}


# ---------------------------------------------------------------------------
# the plain forms

def _weights(w):
    """A weight stack in fp32: widened, or the values its 4-bit codes stand for."""
    if not isinstance(w, dict):
        return w.float()
    codes = torch.stack([w["codes"] & 15, w["codes"] >> 4], dim=-1).flatten(-2)[..., :w["K"]].float()
    spread = lambda t: t.float().repeat_interleave(w["group"], dim=-1)[..., :w["K"]]  # noqa: E731
    return (codes - (spread(w["zeros"]) if w["zeros"] is not None else 8.0)) * spread(w["scales"])


def _pick(w, idx):
    """The stack's matrices idx."""
    if not isinstance(w, dict):
        return w[idx]
    return {**w, "codes": w["codes"][idx], "scales": w["scales"][idx],
            "zeros": None if w["zeros"] is None else w["zeros"][idx]}


def _silu(g):
    return g / (1.0 + torch.exp(-g))


def _plain_few(s):
    case, w, x = s["case"], s["w"], s["x"]
    T, k, G = case["T"], case["top_k"], case["G"]
    z = x.double() @ w["w_router"].double().t() + w["bias"].double()
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    z32 = z.float()
    p = torch.exp(z32 - z32.amax(dim=1, keepdim=True))
    p = (p / p.sum(dim=1, keepdim=True)).gather(1, order)
    if case["norm"]:
        p = p / p.sum(dim=1, keepdim=True)
    g = w["e2g"].long()[order]
    same = g[:, :, None] == g[:, None, :]  # [T, slot, other slot]
    first = ~(same & torch.ones(k, k, dtype=torch.bool, device=x.device).tril(-1)).any(dim=2)
    group = torch.where(first, g, torch.full_like(g, -1))
    gate = torch.where(first, (same * p[:, None, :]).sum(dim=2), torch.zeros_like(p))
    xf = x.float()
    if T * k < G:  # only the picked matrices
        a = xf.repeat_interleave(k, dim=0)[:, :, None]
        idx = g.reshape(-1)
        h = _silu(torch.matmul(_weights(_pick(w["w_gate"], idx)), a)) * torch.matmul(_weights(_pick(w["w_up"], idx)), a)
        y = torch.matmul(_weights(_pick(w["w_down"], idx)), h).view(T, k, -1)
        out = (y * p[:, :, None]).sum(dim=1)
    else:  # every matrix on every token, weighted by the gates (zero for the segments a token does not call)
        gates = torch.zeros((T, G), device=x.device).scatter_add_(1, g, p)
        h = _silu(torch.matmul(xf, _weights(w["w_gate"]).transpose(1, 2))) * torch.matmul(
            xf, _weights(w["w_up"]).transpose(1, 2))
        y = torch.matmul(h, _weights(w["w_down"]).transpose(1, 2))
        out = (y * gates.t()[:, :, None]).sum(dim=0)
    if case["shared"]:
        h = _silu(xf @ _weights(w["w_gate_sh"])[0].t()) * (xf @ _weights(w["w_up_sh"])[0].t())
        out = out + h @ _weights(w["w_down_sh"])[0].t()
    return {"out": out.to(x.dtype), "topk_idx": order.int(), "topk_w": p, "slot_group": group.int(),
            "slot_gate": gate}


def _rows_by_matrix(s):
    """(rows of a, their segment) in row order."""
    a = s["a"] if s["a_rows"] is None else s["a"][s["a_rows"].long()]
    row = torch.arange(a.shape[0], device=a.device)
    return a.float(), (s["offsets"][1:].long()[None, :] <= row[:, None]).sum(dim=1)


def _grouped(a, seg, w):
    """Row r times the transpose of matrix seg[r]."""
    wf = _weights(w)
    n = wf.shape[0]
    if n == 1:
        return a @ wf[0].t()
    # every matrix on every row, then each row's own
    return torch.matmul(a, wf.transpose(1, 2))[seg, torch.arange(a.shape[0], device=a.device)]


def _plain_w4(s):
    a, seg = _rows_by_matrix(s)
    dt = s["a"].dtype
    if s["case"]["kind"] == "w4_matmul":
        return {"y": _grouped(a, seg, s["w"][0]).to(dt)}
    h = _silu(_grouped(a, seg, s["w"][0])) * _grouped(a, seg, s["w"][1])
    return {"y": _grouped(h, seg, s["w"][2]).to(dt), "h": h.to(dt)}


def _rms(v):
    return v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + EPS)


def _plain_pre(s):
    return {"a": (_rms(s["x"].float()) * s["w"].float()).to(s["x"].dtype)}


def _plain_post(s):
    case, dt = s["case"], s["x"].dtype
    y = s["y"].float()
    if case["norm"]:
        y = _rms(y) * s["w_post"].float()
    if s["gate"] is not None:
        y = y * s["gate"].float()
    r = s["x"].float() * s["res_scale"] + y
    if not case["next"]:
        return {"r": r.to(dt)}
    return {"r": r.to(dt), "a": (_rms(r) * s["w"].float()).to(dt)}


# ---------------------------------------------------------------------------
# what a pass cannot do without

def _matrix_bytes(case, N, K):
    if not case["group"]:
        return (2 if case["dtype"] == "bf16" else 4) * N * K
    return N * (K / 2 + (3 if case["zeros"] else 2) * -(-K // case["group"]))


def _reached(case):
    """Segments with at least one call, and calls, on average over routing draws: logits are the
    bias plus N(0, 1)."""
    rng = np.random.default_rng(0)
    T, E, k, G = case["T"], case["E"], case["top_k"], case["G"]
    hit = calls = 0.0
    for _ in range(32):
        q = (1.0 + rng.permutation(E)) ** -case["zipf"]
        e2g = np.empty(E, np.int64)
        e2g[rng.permutation(E)] = (np.arange(E) * G) // E
        picks = e2g[np.argsort(-(np.log(q) + rng.standard_normal((T, E))), axis=1)[:, :k]]
        called = np.zeros((T, G), bool)
        np.put_along_axis(called, picks, True, axis=1)
        hit += called.any(axis=0).sum() / 32
        calls += called.sum() / 32
    return hit, calls


def work(case):
    es, kind = 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind == "few":
        T, d, E, k, f, fs = (case[n] for n in ("T", "d", "E", "top_k", "d_ff", "shared"))
        hit, calls = _reached(case)
        return {"bytes": es * (2 * T * d + E * d) + 8 * E + 16 * T * k
                + hit * (2 * _matrix_bytes(case, f, d) + _matrix_bytes(case, d, f))
                + (2 * _matrix_bytes(case, fs, d) + _matrix_bytes(case, d, fs) if fs else 0),
                "flops": 2.0 * T * E * d + 6.0 * calls * d * f + 6.0 * T * d * fs}
    if kind in ("w4_matmul", "w4_ffn"):
        rows, n, N, K = case["rows"], case["n"], case["N"], case["K"]
        used = n * (1.0 - (1.0 - 1.0 / n) ** rows) if n > 1 else 1.0  # segments that get rows
        m = -(-rows // 4) if case["gather"] else rows
        if kind == "w4_matmul":
            return {"bytes": used * _matrix_bytes(case, N, K) + es * (m * K + rows * N), "flops": 2.0 * rows * N * K}
        return {"bytes": used * (2 * _matrix_bytes(case, N, K) + _matrix_bytes(case, K, N))
                + es * (m * K + rows * (K + N)), "flops": 6.0 * rows * N * K}
    T, d = case["T"], case["d"]
    if kind == "pre_norm":
        return {"bytes": es * (2 * T * d + d), "flops": 4.0 * T * d}
    gate = {"none": 0, "channel": es * d, "token": 4 * T, "full": es * T * d}[case["gate"]]
    return {"bytes": es * ((3 + case["next"]) * T * d + (case["norm"] + case["next"]) * d) + gate,
            "flops": 4.0 * T * d * (1 + case["norm"] + case["next"])}


# ---------------------------------------------------------------------------
# the definitions in 64 bits, element by element where that is short

def _dense64(w, i):
    """Matrix i of a stack."""
    if not isinstance(w, dict):
        return w[i].double()
    K, c = w["K"], w["codes"][i].to(torch.int32)
    q = torch.empty((c.shape[0], 2 * c.shape[1]), dtype=torch.float64, device=c.device)
    q[:, 0::2], q[:, 1::2] = (c % 16).double(), torch.div(c, 16, rounding_mode="floor").double()
    out = torch.empty((c.shape[0], K), dtype=torch.float64, device=c.device)
    for j in range(w["scales"].shape[2]):
        a, b = j * w["group"], min(K, (j + 1) * w["group"])
        zero = w["zeros"][i, :, j].double()[:, None] if w["zeros"] is not None else 8.0
        out[:, a:b] = w["scales"][i, :, j].double()[:, None] * (q[:, a:b] - zero)
    return out


def _expert64(a, wg, wu, wd, i):
    """(h, y) of one SwiGLU expert."""
    g = a @ _dense64(wg, i).t()
    h = g * torch.sigmoid(g) * (a @ _dense64(wu, i).t())
    return h, h @ _dense64(wd, i).t()


def _exact_few(s):
    case, w, x = s["case"], s["w"], s["x"].double()
    T, k = case["T"], case["top_k"]
    z = (x @ w["w_router"].double().t() + w["bias"].double()).cpu().numpy()
    e2g = w["e2g"].cpu().numpy()
    idx, tw = np.zeros((T, k), np.int32), np.zeros((T, k))
    group, gate = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        idx[t] = sorted(range(case["E"]), key=lambda e: (-z[t, e], e))[:k]
        p = np.exp(z[t] - z[t].max())
        tw[t] = p[idx[t]] / (p[idx[t]].sum() if case["norm"] else p.sum())
        slot_of = {}
        for i in range(k):
            r = int(e2g[idx[t, i]])
            if r not in slot_of:
                slot_of[r] = i
                group[t, i] = r
            gate[t, slot_of[r]] += tw[t, i]
    out = torch.zeros_like(x)
    for r in sorted(set(group[group >= 0].tolist())):
        tok, slot = np.nonzero(group == r)
        y = _expert64(x[tok.tolist()], w["w_gate"], w["w_up"], w["w_down"], r)[1]
        out[tok.tolist()] += torch.from_numpy(gate[tok, slot]).to(out.device)[:, None] * y
    if case["shared"]:
        out += _expert64(x, w["w_gate_sh"], w["w_up_sh"], w["w_down_sh"], 0)[1]
    return {"out": out, "topk_idx": idx, "topk_w": tw, "slot_group": group, "slot_gate": gate}


def _exact_w4(s):
    case = s["case"]
    rows, offs = case["rows"], s["offsets"].cpu().tolist()
    src = list(range(rows)) if s["a_rows"] is None else s["a_rows"].cpu().tolist()
    y = torch.zeros(s["out"][0].shape, dtype=torch.float64, device="cuda")
    h = torch.zeros(s["out"][-1].shape, dtype=torch.float64, device="cuda")
    for i in range(case["n"]):
        b, e = offs[i], offs[i + 1]
        if b == e:
            continue
        a = s["a"][src[b:e]].double()
        if case["kind"] == "w4_matmul":
            y[b:e] = a @ _dense64(s["w"][0], i).t()
        else:
            h[b:e], y[b:e] = _expert64(a, *s["w"], i)
    return {"y": y} if case["kind"] == "w4_matmul" else {"y": y, "h": h}


def _exact_norm(s):
    case, x = s["case"], s["x"].double()
    unit = lambda v: v / torch.sqrt((v * v).sum(dim=1, keepdim=True) / v.shape[1] + EPS)  # noqa: E731
    if case["kind"] == "pre_norm":
        return {"a": unit(x) * s["w"].double()}
    y = s["y"].double()
    if case["norm"]:
        y = unit(y) * s["w_post"].double()
    if case["gate"] != "none":
        g = s["gate"].double()
        y = g * y
    r = s["res_scale"] * x + y
    return {"r": r, "a": unit(r) * s["w"].double()} if case["next"] else {"r": r}


def exact(case, seed):
    s = prepare(case, seed)
    return {"few": _exact_few, "w4_matmul": _exact_w4, "w4_ffn": _exact_w4, "pre_norm": _exact_norm,
            "post_norm": _exact_norm}[case["kind"]](s)
