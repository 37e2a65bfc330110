"""Expert products in 8-bit integers and the router's balance loss, as cases that can be timed and compared.

* ``w8_matmul`` / ``w8_ffn``: products of grouped rows with weights held in 8
  bits, on the activations rounded to 8 bits token by token;
* ``balance`` / ``balance_step``: how evenly the router's picks fall on the
  experts (or their groups), the z loss and the per-expert counts; the step
  with the gradient by the logits.

8-bit rows: codes of a matrix [.., K] are [.., P] int8, P = 128 ceil(K/128), the
bytes past K zero, with one fp32 scale for each row: x = scale * code. A row's
scale is max|x| / 127, its codes round(x / scale), to nearest even.

``own`` False computes plain torch expressions of these definitions; True makes
the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

__all__ = ["listed", "draw", "prepare", "run", "work", "exact"]


def _w8(name, kind, rows, n, N, K, gather=False):
    """rows of n segments, matrices [N, K] (the FFN: d_ff = N, d = K); gather: four rows read one token on average."""
    return {"name": name, "kind": kind, "rows": rows, "n": n, "N": N, "K": K, "gather": gather}


def _bal(name, kind, T, E, k, G=0, padded=False):
    """G: groups of the map, 0 for the experts themselves; padded: a quarter of the tokens does not count."""
    return {"name": name, "kind": kind, "T": T, "E": E, "k": k, "G": G, "padded": padded}


def listed():
    return [
        # one row through one matrix: the smallest product
        _w8("w8_matvec_1", "w8_matmul", 1, 1, 4096, 4096),
        # a few hundred rows in ragged segments, sizes that fill no tile
        _w8("w8_matmul_ragged", "w8_matmul", 777, 5, 1000, 1048),
        # a prompt through one wide matrix: matrix cores only
        _w8("w8_matmul_4096", "w8_matmul", 4096, 1, 14336, 4096),
        # one token, top-4, on the fine-grained layer's segments: latency
        _w8("w8_ffn_token", "w8_ffn", 4, 15, 1408, 2048, gather=True),
        # a decode step: the weights stream once
        _w8("w8_ffn_decode", "w8_ffn", 250, 8, 1408, 2048, gather=True),
        # prefill on fine-grained experts
        _w8("w8_ffn_fine", "w8_ffn", 30000, 15, 1408, 2048, gather=True),
        # prefill, Mixtral-shaped
        _w8("w8_ffn_mixtral", "w8_ffn", 8192, 4, 14336, 4096, gather=True),
        # the counts and losses of one decode step
        _bal("balance_64", "balance", 64, 64, 6),
        # a training batch with padding, balanced over the united experts
        _bal("balance_fine_8192", "balance", 8192, 60, 4, G=15, padded=True),
        # a long batch over the most experts the router takes
        _bal("balance_131072", "balance", 131072, 256, 8),
        # odd sizes, forward and gradient
        _bal("balance_step_1001", "balance_step", 1001, 7, 2, padded=True),
        # a training step of the layer with heavy skew, over its groups
        _bal("balance_step_16384", "balance_step", 16384, 64, 6, G=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["w8_matmul", "w8_ffn", "w8_ffn", "balance", "balance_step"])
    if kind in ("w8_matmul", "w8_ffn"):
        n = rng.choice([1, 4, rng.randint(2, 32)])
        N, K = 8 * _log(rng, 16, 1792), 8 * _log(rng, 16, 768)
        while n * N * K > 2.3e8:  # (what the largest listed case holds)
            n -= 1
        rows = min(_log(rng, 1, 1024 * n), max(1, int(4.8e11 / (N * K))))
        c = _w8("", kind, rows, n, N, K, rng.random() < 0.5)
    else:
        E = rng.choice([8, 60, 64, 128, rng.randint(2, 256)])
        k = min(E, rng.choice([1, 2, 4, 6, 8]))
        c = _bal("", kind, _log(rng, 1, 65536), E, k, rng.choice([0, rng.randint(1, E)]), rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs

def _pitch(K):
    return 128 * -(-K // 128)


def _weights(gen, n, N, K):
    """Codes of normal weights (four deviations to the largest), scales that vary by channel."""
    w = torch.zeros((n, N, _pitch(K)), dtype=torch.int8, device="cuda")
    q = torch.randn((n, N, K), generator=gen, device="cuda", dtype=torch.bfloat16)
    w[:, :, :K] = q.mul_(32.0).round_().clamp_(-127, 127).to(torch.int8)
    scale = (torch.rand((n, N), generator=gen, device="cuda") + 0.5).mul_(1.0 / (32.0 * math.sqrt(K)))
    return {"codes": w, "scales": scale, "K": K}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    s = {"case": case}
    if case["kind"] in ("w8_matmul", "w8_ffn"):
        n, N, K, rows = case["n"], case["N"], case["K"], case["rows"]
        cut = np.sort(rng.integers(0, rows + 1, n - 1)) if n > 1 else np.zeros(0, np.int64)
        offsets = np.concatenate([[0], cut, [rows]])
        s["offsets"] = torch.from_numpy(offsets.astype(np.int32)).cuda()
        s["longest"] = int(np.diff(offsets).max())
        m = -(-rows // 4) if case["gather"] else rows
        s["a_rows"] = torch.from_numpy(rng.integers(0, m, rows).astype(np.int32)).cuda() if case["gather"] else None
        # normed activations whose channels differ in size, as trained ones do
        s["a"] = (torch.randn((m, K), generator=gen, device="cuda")
                  * torch.exp(0.5 * torch.randn((K,), generator=gen, device="cuda"))).to(torch.bfloat16)
        new = lambda cols: torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")  # noqa: E731
        if case["kind"] == "w8_matmul":
            s["w"], s["out"] = (_weights(gen, n, N, K),), (new(N),)
        else:
            s["w"] = (_weights(gen, n, N, K), _weights(gen, n, N, K), _weights(gen, n, K, N))
            s["out"] = (new(K), new(N))
    else:
        T, E, k, G = (case[x] for x in ("T", "E", "k", "G"))
        q = (1.0 + rng.permutation(E)) ** -1.2  # a Zipf law over the experts
        z = torch.randn((T, E), generator=gen, device="cuda") + torch.from_numpy(np.log(q / q.sum())).float().cuda()
        s["logits"] = z
        s["topk_idx"] = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k].int().contiguous()
        s["valid"] = (torch.rand((T,), generator=gen, device="cuda") >= 0.25).to(torch.uint8) if case["padded"] else None
        s["e2g"] = None
        if G:
            e2g = np.empty(E, np.int32)
            e2g[rng.permutation(E)] = (np.arange(E) * G) // E
            s["e2g"] = torch.from_numpy(e2g).cuda()
        s["d_losses"] = torch.tensor([1e-2, 1e-3], device="cuda")  # the weights of the two losses
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that serves these weights, or trains this router, keeps between calls."""
    from paper_2607_04164_amd import binding as B
    case = s["case"]
    if case["kind"] in ("w8_matmul", "w8_ffn"):
        s["w8"] = tuple(B.W8(w["codes"], w["scales"], K=w["K"]) for w in s["w"])
        s["ws"] = B.new_w8_workspace(s["a"].shape[0], case["K"], "cuda", rows_cap=case["rows"],
                                     d_ff=case["N"] if case["kind"] == "w8_ffn" else 0)
    else:
        s["ws"] = B.new_balance_workspace(case["T"], case["E"], "cuda")
        s["bufs"] = B.new_balance_buffers(case["E"], "cuda")
        s["d_logits"] = torch.empty_like(s["logits"]) if case["kind"] == "balance_step" else None


def run(state):
    if own:
        return _run_own(state)
    return _plain_w8(state) if state["case"]["kind"] in ("w8_matmul", "w8_ffn") else _plain_balance(state)


def _run_own(s):
    from paper_2607_04164_amd import binding as B
    case, kind = s["case"], s["case"]["kind"]
    if kind == "w8_matmul":
        return {"y": B.w8_matmul(s["offsets"], s["a"], s["w8"][0], a_rows=s["a_rows"], y=s["out"][0], workspace=s["ws"])}
    if kind == "w8_ffn":
        y, h = B.w8_ffn(s["offsets"], s["a"], *s["w8"], a_rows=s["a_rows"], y=s["out"][0], h=s["out"][1],
                        workspace=s["ws"])
        return {"y": y, "h": h}
    over = {"valid": s["valid"], "e2g": s["e2g"], "G": case["G"] or None}
    o = B.balance(s["logits"], s["topk_idx"], out=s["bufs"], workspace=s["ws"], **over)
    got = {n: o[n] for n in ("losses", "counts", "prob")}
    if kind == "balance_step":
        got["d_logits"] = B.balance_grad(s["logits"], o["counts"], case["k"], s["d_losses"], out=s["d_logits"], **over)
    return got


# ---------------------------------------------------------------------------
# the plain forms

def _rounded(v):
    """Rows in 8 bits: (codes as numbers, scales). In 64 bits: quotients next to a border."""
    v = v.double()
    scale = (v.abs().amax(dim=1, keepdim=True) / 127.0).float()
    q = torch.round(v / torch.where(scale > 0, scale, torch.ones_like(scale)).double()).clamp_(-127, 127)
    return q.float(), scale


def _grouped(q, scale, s, w):
    """Row r times the transpose of its segment's matrix: the segments as one padded batch."""
    first, end = s["offsets"][:-1].long(), s["offsets"][1:].long()
    rows = q.shape[0]
    row = torch.arange(rows, device=q.device)
    seg = (end[None, :] <= row[:, None]).sum(dim=1)
    at = (first[:, None] + torch.arange(s["longest"], device=q.device)[None, :]).clamp_(max=rows - 1)
    m = w["codes"][:, :, :w["K"]].float()
    y = torch.matmul(q[at], m.transpose(1, 2))[seg, row - first[seg]]
    return y * scale * w["scales"][seg]


def _plain_w8(s):
    q, scale = _rounded(s["a"])
    if s["a_rows"] is not None:
        q, scale = q[s["a_rows"].long()], scale[s["a_rows"].long()]
    if s["case"]["kind"] == "w8_matmul":
        return {"y": _grouped(q, scale, s, s["w"][0]).to(torch.bfloat16)}
    g = _grouped(q, scale, s, s["w"][0])
    h = (g / (1.0 + torch.exp(-g)) * _grouped(q, scale, s, s["w"][1])).to(torch.bfloat16)
    return {"y": _grouped(*_rounded(h), s, s["w"][2]).to(torch.bfloat16), "h": h}


def _plain_balance(s):
    case, z = s["case"], s["logits"]
    T, E, k = case["T"], case["E"], case["k"]
    on = (s["valid"] != 0) if s["valid"] is not None else torch.ones(T, dtype=torch.bool, device=z.device)
    count = torch.zeros(E + 1, dtype=torch.int64, device=z.device)
    count.scatter_add_(0, s["topk_idx"].long().flatten(), on.long()[:, None].expand(T, k).flatten())
    count[E] = on.sum()
    V = count[E].clamp(min=1).double()
    top = z.amax(dim=1, keepdim=True)
    x = torch.exp(z - top)
    total = x.sum(dim=1, keepdim=True)
    p, lse = x / total, top + torch.log(total)
    prob = (p * on[:, None]).sum(dim=0, dtype=torch.float64) / V
    share = count[:E].double()
    G = E
    if s["e2g"] is not None:
        G, e2g = case["G"], s["e2g"].long()
        share = torch.zeros(G, dtype=torch.float64, device=z.device).scatter_add_(0, e2g, share)[e2g]
    share = share / (k * V)
    losses = torch.stack([G * (share * prob).sum(), (lse.double()[:, 0].square() * on).sum() / V])
    got = {"losses": losses.float(), "counts": count.int(), "prob": prob.float()}
    if case["kind"] == "balance_step":
        b, a = s["d_losses"].double() / V
        f = (G * b * share).float()
        d = p * (f - (f * p).sum(dim=1, keepdim=True) + (2.0 * a).float() * lse)
        got["d_logits"] = d * on[:, None]
    return got


# ---------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind in ("w8_matmul", "w8_ffn"):
        rows, n, N, K = case["rows"], case["n"], case["N"], case["K"]
        used = n * (1.0 - (1.0 - 1.0 / n) ** rows) if n > 1 else 1.0  # segments that get rows
        m = -(-rows // 4) if case["gather"] else rows
        index = 4 * rows if case["gather"] else 0
        if kind == "w8_matmul":
            return {"bytes": used * N * (K + 4) + 2 * (m * K + rows * N) + index, "flops": 2.0 * rows * N * K}
        return {"bytes": used * (2 * N * (K + 4) + K * (N + 4)) + 2 * (m * K + rows * (K + N)) + index,
                "flops": 6.0 * rows * N * K}
    T, E, k = case["T"], case["E"], case["k"]
    read = 4 * T * E + 4 * T * k + (T if case["padded"] else 0) + (4 * E if case["G"] else 0) + 8 * E + 12
    if kind == "balance":
        return {"bytes": read, "flops": 8.0 * T * E}
    return {"bytes": read + 4 * T * E, "flops": 14.0 * T * E}


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def _codes64(v):
    """[rows, K] in 64 bits -> (codes, scales) of its rows."""
    largest = torch.maximum(v.max(dim=1).values, -v.min(dim=1).values)
    scales = (largest / 127).to(torch.float32).to(torch.float64)
    codes = torch.zeros_like(v)
    live = scales > 0
    t = v[live] / scales[live][:, None]
    low = torch.floor(t)
    up = ((t - low) > 0.5) | (((t - low) == 0.5) & (low % 2 != 0))
    codes[live] = low + up.double()
    return codes, scales


def _exact_w8(s):
    case = s["case"]
    rows, offs = case["rows"], s["offsets"].cpu().tolist()
    src = s["a_rows"].cpu().tolist() if s["a_rows"] is not None else list(range(rows))
    qa, sa = _codes64(s["a"].double())
    outs = [torch.zeros(o.shape, dtype=torch.float64, device="cuda") for o in s["out"]]

    def times(q, scale, w, i):
        return (q @ w["codes"][i, :, :w["K"]].double().t()) * scale[:, None] * w["scales"][i].double()[None, :]

    for i in range(case["n"]):
        b, e = offs[i], offs[i + 1]
        if b == e:
            continue
        q, scale = qa[src[b:e]], sa[src[b:e]]
        if case["kind"] == "w8_matmul":
            outs[0][b:e] = times(q, scale, s["w"][0], i)
            continue
        g = times(q, scale, s["w"][0], i)
        h = g * torch.sigmoid(g) * times(q, scale, s["w"][1], i)
        outs[1][b:e] = h
        # (the hidden values are held in bf16, then rounded to 8 bits)
        qh, sh = _codes64(h.to(torch.bfloat16).double())
        outs[0][b:e] = times(qh, sh, s["w"][2], i)
    return {"y": outs[0]} if case["kind"] == "w8_matmul" else {"y": outs[0], "h": outs[1]}


def _exact_balance(s):
    case = s["case"]
    E, k, G = case["E"], case["k"], case["G"] or case["E"]
    keep = np.ones(case["T"], bool) if s["valid"] is None else s["valid"].cpu().numpy() != 0
    z = s["logits"].cpu().numpy().astype(np.float64)
    e2g = np.arange(E) if s["e2g"] is None else s["e2g"].cpu().numpy()
    V = int(keep.sum())
    counts = np.bincount(s["topk_idx"].cpu().numpy()[keep].ravel(), minlength=E)
    lse = np.log(np.exp(z).sum(axis=1))  # (logits of a few units)
    p = np.exp(z - lse[:, None])
    n = max(V, 1)
    prob = p[keep].sum(axis=0) / n
    F = np.bincount(e2g, weights=counts, minlength=G) / (k * n)
    P = np.bincount(e2g, weights=prob, minlength=G)
    got = {"losses": np.array([G * (F * P).sum(), (lse[keep] ** 2).sum() / n]),
           "counts": np.append(counts, V).astype(np.int32), "prob": prob}
    if case["kind"] == "balance_step":
        b, a = s["d_losses"].cpu().numpy().astype(np.float64)
        # d p_e / d z_j = p_e ([e = j] - p_j), so the balance loss gives p_j (w_j - sum of w_e p_e), w the losses' slopes by p
        slope = b * G / n * F[e2g] + a * 2.0 / n * lse[:, None]  # (the z loss: d lse / d z_j = p_j)
        d = p * (slope - ((b * G / n * F[e2g]) * p).sum(axis=1, keepdims=True))
        got["d_logits"] = d * keep[:, None]
    return got


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_w8(s) if case["kind"] in ("w8_matmul", "w8_ffn") else _exact_balance(s)
