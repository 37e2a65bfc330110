"""64-bit numpy references of the decode-side operators, and random inputs for them.

Everything is float64 from the exact values of the inputs; nothing here is shared with the library.
"""
from __future__ import annotations

import numpy as np
import torch

import oracle
from paper_2607_04164_amd import workload as W

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # relative error of one rounding
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def np64(t: torch.Tensor) -> np.ndarray:
    return t.detach().to(torch.float64).cpu().numpy()


def rand(rng, shape, std, dtype) -> torch.Tensor:
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(TORCH[dtype])


# ---- 4-bit weights

def w4_random(rng, n, N, K, group, zeros, std=None):
    """(codes, scales, zeros or None) as CPU tensors; padding bytes are random (they must not matter)."""
    std = 1.0 / np.sqrt(K) if std is None else std
    pitch, ng = 16 * (-(-K // 32)), -(-K // group)
    codes = torch.from_numpy(rng.integers(0, 256, (n, N, pitch)).astype(np.uint8))
    scales = torch.from_numpy(((0.5 + rng.random((n, N, ng))) * std / 4.6).astype(np.float32)).to(torch.bfloat16)
    z = torch.from_numpy(rng.integers(0, 16, (n, N, ng)).astype(np.uint8)) if zeros else None
    return codes, scales, z


def w4_values(codes, scales, zeros, K, group) -> np.ndarray:
    """[n, N, K] float64: column k is scale * (code - zero), one column at a time."""
    c, s = codes.cpu().numpy().astype(np.int64), np64(scales)
    z = np.full(s.shape, 8.0) if zeros is None else zeros.cpu().numpy().astype(np.float64)
    out = np.empty(c.shape[:2] + (K,))
    for k in range(K):
        q = (c[:, :, k // 2] >> (4 * (k % 2))) & 15
        out[:, :, k] = s[:, :, k // group] * (q - z[:, :, k // group])
    return out


def w4_magnitude(codes, scales, zeros, K, group) -> np.ndarray:
    """|scale| * (32 + code + zero) per column: what the rounding of a group's sums goes by (its terms
    are code + 16 and zero + 16)."""
    c, s = codes.cpu().numpy().astype(np.int64), np.abs(np64(scales))
    z = np.full(s.shape, 8.0) if zeros is None else zeros.cpu().numpy().astype(np.float64)
    out = np.empty(c.shape[:2] + (K,))
    for k in range(K):
        q = (c[:, :, k // 2] >> (4 * (k % 2))) & 15
        out[:, :, k] = s[:, :, k // group] * (32 + q + z[:, :, k // group])
    return out


def silu(g):
    return g / (1.0 + np.exp(-g))


# ---- the layer

def few_ref(x, w_router, bias, e2g, w, top_k, norm, w_sh=None):
    """Outputs of the layer in float64. x, w_router: fp32 arrays of the exact inputs; w, w_sh: (gate, up, down)
    float64 stacks."""
    r = oracle.route(x, w_router, bias, e2g, top_k, norm)
    T = x.shape[0]
    x = x.astype(np.float64)
    out = np.zeros_like(x)
    for t in range(T):
        for i in range(top_k):
            g = r["slot_group"][t, i]
            if g >= 0:
                h = silu(w[0][g] @ x[t]) * (w[1][g] @ x[t])
                out[t] += np.float64(r["slot_gate"][t, i]) * (w[2][g] @ h)
    if w_sh is not None:
        h = silu(x @ w_sh[0][0].T) * (x @ w_sh[1][0].T)
        out += h @ w_sh[2][0].T
    return {"out": out, **r}


def assert_few(out, ref, dtype, what=""):
    """out against the float64 output. Beside its one rounding (HALF of the value) an output carries the errors
    of the hidden values (2^-17 of each in bf16 layers, from their two parts) and of fp32 sums; both enter the
    down product with random signs, so their sum is about that share of the row's rms: five deviations of
    2^-17 + 2^-17 stay under 2^-13 of the rms. In fp32 layers the sums' error is about 2^-24 sqrt(terms / 3) of
    the rms in each of the three products, 2^-17 with five deviations at the sizes tested here (up to 2048
    terms and 16 experts)."""
    out, want = np64(out), ref["out"]
    assert np.isfinite(out).all(), what
    rms = np.sqrt((want ** 2).mean(axis=1, keepdims=True))
    tol = HALF[dtype] * np.abs(want) + {"bf16": 2.0 ** -13, "f32": 2.0 ** -17}[dtype] * rms
    worst = float((np.abs(out - want) / np.maximum(tol, 1e-300)).max())
    assert worst <= 1.0, f"{what}: {worst:.3f} of the tolerance"


# ---- norms

def inv_rms(v, eps):
    return 1.0 / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)


SUM = 64 * 2.0 ** -24  # fp32 sum of squares over a row: at most 64 terms a thread and 10 levels of a tree, halved by the root


def post_ref(y, x, norm, w_post, gate, rho, w_next, eps):
    """(r, bound of r's error before its rounding, a, bound of a's error before its rounding)."""
    n = y * inv_rms(y, eps) * (1.0 if w_post is None else w_post) if norm else y
    gn = n if gate is None else gate * n
    r = rho * x + gn
    er = SUM * (np.abs(rho * x) + np.abs(gn))
    inv = inv_rms(r, eps)
    w = 1.0 if w_next is None else w_next
    a = r * inv * w
    spread = np.sqrt((er * er).mean(axis=1, keepdims=True)) * inv
    ea = np.abs(inv * w) * er + np.abs(a) * (SUM + spread)
    return r, er, a, ea


def assert_rounded(got, want, err, dtype, what):
    """got: want rounded once to dtype, from a value at most err off."""
    got = np64(got)
    tol = HALF[dtype] * (np.abs(want) + err) + err + 1e-42
    bad = np.abs(got - want) > tol
    assert np.isfinite(got).all(), what
    assert not bad.any(), f"{what}: {int(bad.sum())} values off, first at {np.argwhere(bad)[0]}"


# ---- layers of random weights

def make_case(seed, T, d, E, top_k, G, f, fs=0, norm=0, dtype="bf16", group=0, zeros=False, zipf=1.0):
    """Inputs of one few-token layer: CPU tensors, and the float64 weights they stand for."""
    rng = np.random.default_rng(seed)
    e2g = W.balanced_map(rng.permutation(E), E, G)
    bias = W.zipf_bias(rng.permutation(E), zipf)
    std = 1.0 / np.sqrt(d)
    c = {"x": rand(rng, (T, d), 1.0, dtype), "w_router": rand(rng, (E, d), std, dtype),
         "bias": torch.from_numpy(bias), "e2g": torch.from_numpy(e2g)}
    vals = {}

    def matrix(name, n, N, K):
        if group:
            t = w4_random(rng, n, N, K, group, zeros, std)
            c[name], vals[name] = t, w4_values(*t, K, group)
        else:
            c[name] = rand(rng, (n, N, K), std, dtype)
            vals[name] = np64(c[name])

    matrix("w_gate", G, f, d), matrix("w_up", G, f, d), matrix("w_down", G, d, f)
    if fs:
        matrix("w_gate_sh", 1, fs, d), matrix("w_up_sh", 1, fs, d), matrix("w_down_sh", 1, d, fs)
    return c, vals
