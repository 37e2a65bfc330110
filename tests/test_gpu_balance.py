"""The router's balance: counts, losses and their gradient, against 64 bits and differences."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2607_04164_amd import binding as B

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()


def make(seed, T, E, k, *, padded=True, spread=2.0):
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal((T, E)) * spread).astype(np.float32)
    idx = np.argsort(-z, axis=1, kind="stable")[:, :k].astype(np.int32)
    valid = (rng.random(T) < 0.75).astype(np.uint8) if padded else None
    return z, idx, valid


def losses64(z, idx, valid, e2g, G, k):
    """(losses, counts, prob, p, lse) from the definition, row by row in 64 bits; -inf is an expert of probability 0."""
    T, E = z.shape
    z = z.astype(np.float64)
    keep = np.ones(T, bool) if valid is None else valid != 0
    p, lse = np.zeros((T, E)), np.zeros(T)
    for t in np.nonzero(keep)[0]:
        top = z[t].max()
        if top == -np.inf:
            continue
        x = np.exp(z[t] - top)
        p[t], lse[t] = x / x.sum(), top + np.log(x.sum())
    picks = idx[keep].ravel()
    counts = np.bincount(picks[(picks >= 0) & (picks < E)], minlength=E)
    n = max(int(keep.sum()), 1)
    prob = p.sum(axis=0) / n
    F = np.zeros(G)
    inside = [(e, g) for e, g in enumerate(e2g) if 0 <= g < G]
    for e, g in inside:
        F[g] += counts[e] / (k * n)
    f = np.zeros(E)
    for e, g in inside:
        f[e] = F[g]
    losses = np.array([G * (f * prob).sum(), (lse ** 2).sum() / n])
    return losses, np.append(counts, int(keep.sum())), prob, p, lse, f, n


def grad64(d, G, p, lse, f, n, keep):
    slope = d[0] * G / n * f
    out = p * (slope - (p @ slope)[:, None]) + d[1] * 2 / n * lse[:, None] * p
    out[~keep] = 0
    return out


def row_error(z):
    """Relative rounding of a row's p: its logits' differences (rounded once, and e^x has their size as its
    derivative), the sum over E in any order, exp, reciprocal and products: a step 2^-24 each."""
    z = np.where(np.isfinite(z), z, 0.0)
    return (2 * (z.max(axis=1) - z.min(axis=1)) + z.shape[1] + 12) * F32


def device(*arrays):
    return [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


# one workgroup and several, each lane layout and its edges, more tokens than a round
SIZES = [(1, 1, 1), (1, 2, 1), (3, 7, 2), (64, 8, 2), (17, 16, 4), (65, 17, 3), (64, 64, 6), (513, 60, 4), (600, 65, 1),
         (1001, 128, 8), (777, 129, 16), (2049, 256, 8), (20000, 4, 2), (40000, 64, 6), (9001, 131, 5), (20011, 256, 3)]


@pytest.mark.parametrize("grouped", [False, True], ids=["experts", "groups"])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_losses_and_gradient(T, E, k, grouped):
    z, idx, valid = make(T + E, T, E, k, padded=T % 2 == 1)
    rng = np.random.default_rng(E)
    G = max(1, E // 3) if grouped else E
    e2g = rng.integers(0, G, E).astype(np.int32) if grouped else np.arange(E)
    if grouped and E > 4:
        e2g[[1, 3]] = -1, G  # experts of no group
    want = losses64(z, idx, valid, e2g, G, k)
    zd, id_, vd, gd = device(z, idx, valid, e2g if grouped else None)
    o = B.balance(zd, id_, valid=vd, e2g=gd, G=G if grouped else None)
    assert np.array_equal(o["counts"].cpu().numpy(), want[1])
    keep = np.ones(T, bool) if valid is None else valid != 0
    worst = row_error(z[keep]).max() if keep.any() else 0.0
    # a lane adds its tokens one by one, then a workgroup its waves
    adds = (T / 64 + 32) * F32
    got = {n: t.double().cpu().numpy() for n, t in o.items()}
    assert (np.abs(got["prob"] - want[2]) <= want[2] * (worst + adds + F32)).all()
    assert abs(got["losses"][0] - want[0][0]) <= want[0][0] * (worst + adds + 2 * F32)
    # lse: the logarithm's argument (its sum), itself and the addition, by the sizes of both; then a square
    size = np.abs(z).max() + np.log(E) + 1
    assert abs(got["losses"][1] - want[0][1]) <= 2 * size * (worst + 8 * size * F32) + want[0][1] * (adds + 4 * F32)
    d = np.array([0.7, -0.3], np.float32)
    dz = B.balance_grad(zd, o["counts"], k, torch.from_numpy(d).cuda(), valid=vd, e2g=gd, G=G if grouped else None)
    exact = grad64(d.astype(np.float64), G, *want[3:], keep)
    p, lse, f, n = want[3:]
    terms = p * (abs(d[0]) * G / n * (f + (p @ f)[:, None]) + abs(d[1]) * 2 / n * (np.abs(lse)[:, None] + size))
    assert (np.abs(dz.double().cpu().numpy() - exact) <= terms * (3 * worst + (E + 16) * F32) + 1e-44).all()
    if valid is not None:
        assert not dz[torch.from_numpy(valid == 0).cuda()].any()
    again = zd.clone()
    assert B.balance_grad(again, o["counts"], k, torch.from_numpy(d).cuda(), valid=vd, e2g=gd, G=G if grouped else None,
                          out=again) is again
    assert torch.equal(again, dz)


def test_gradient_by_differences():
    """Of the losses in 64 bits with the counts held: the gradient is theirs."""
    T, E, k, G = 5, 6, 2, 3
    z, idx, _ = make(3, T, E, k, padded=False)
    valid = np.array([1, 0, 1, 1, 1], np.uint8)
    e2g = np.array([0, 1, 2, 0, 1, 2], np.int32)
    d = np.array([0.5, 0.25], np.float32)
    zd, id_, vd, gd, dd = device(z, idx, valid, e2g, d)
    counts = B.balance(zd, id_, valid=vd, e2g=gd, G=G)["counts"]
    dz = B.balance_grad(zd, counts, k, dd, valid=vd, e2g=gd, G=G).double().cpu().numpy()
    step = 1e-4
    for t in range(T):
        for e in range(E):
            side = []
            for s in (step, -step):
                y = z.astype(np.float64).copy()
                y[t, e] += s
                side.append(losses64_of(y, idx, valid, e2g, G, k) @ d.astype(np.float64))
            # third derivatives are a few units: the difference is off by step^2, the kernel by fp32
            assert abs((side[0] - side[1]) / (2 * step) - dz[t, e]) <= 20 * step ** 2 + 1e-6


def losses64_of(z, idx, valid, e2g, G, k):
    return losses64(z, idx, valid, e2g, G, k)[0]


def test_even_picks_and_probabilities_give_one():
    T, E, k = 60, 12, 2
    z = torch.zeros((T, E), device="cuda")
    idx = torch.arange(T * k, device="cuda").view(T, k).remainder(E).int()
    o = B.balance(z, idx)
    assert abs(float(o["losses"][0]) - 1) <= 16 * F32
    assert abs(float(o["losses"][1]) - np.log(E) ** 2) <= 32 * F32 * np.log(E) ** 2
    assert o["counts"].tolist() == [T * k // E] * E + [T]
    assert float(B.balance_grad(z, o["counts"], k, torch.tensor([1.0, 0.0], device="cuda")).abs().max()) <= 4 * F32 / T


@pytest.mark.parametrize("T", [40, 900, 3000])
def test_masks_and_infinities(T):
    """Tokens that do not count may hold anything; -inf is an expert of probability 0; a row of nothing else adds
    nothing; picks outside the experts pick nothing."""
    E, k, G = 20, 3, 5
    z, idx, valid = make(T, T, E, k)
    valid[:4] = 0
    z[0], z[1], z[2] = np.nan, np.inf, -np.inf
    idx[3] = 9999
    valid[4:8] = 1
    z[4, :E - 1] = -np.inf
    z[5] = -np.inf
    z[6, ::2] = -np.inf
    z[7, 3] = -200.0
    idx[6] = [-1, E, 2]
    idx[7] = 4  # the same expert in every slot
    e2g = (np.arange(E) % G).astype(np.int32)
    want = losses64(z, idx, valid, e2g, G, k)
    zd, id_, vd, gd = device(z, idx, valid, e2g)
    o = B.balance(zd, id_, valid=vd, e2g=gd, G=G)
    assert np.array_equal(o["counts"].cpu().numpy(), want[1])
    tol = (2 * 16.0 + E + T / 64 + 64) * F32  # (the finite logits span less than 16, or their p is below 1e-80)
    np.testing.assert_allclose(o["prob"].double().cpu().numpy(), want[2], rtol=tol)
    np.testing.assert_allclose(o["losses"].double().cpu().numpy(), want[0], rtol=4 * tol)
    d = torch.tensor([1.0, 0.5], device="cuda")
    dz = B.balance_grad(zd, o["counts"], k, d, valid=vd, e2g=gd, G=G).double().cpu().numpy()
    exact = grad64(np.array([1.0, 0.5]), G, *want[3:], valid != 0)
    assert np.isfinite(dz).all() and not dz[:4].any() and not dz[5].any() and not dz[6, ::2].any()
    p, lse, f, n = want[3:]
    terms = p * (G / n * (f + (p @ f)[:, None]) + 1.0 / n * (np.abs(lse)[:, None] + 12))
    assert (np.abs(dz - exact) <= terms * 4 * tol + 1e-44).all()
    # a value that is not a number in a token that counts shows
    z[4, 0] = np.nan
    zd, = device(z)
    o = B.balance(zd, id_, valid=vd, e2g=gd, G=G)
    assert bool(torch.isnan(o["losses"]).all()) and np.array_equal(o["counts"].cpu().numpy(), want[1])
    dz = B.balance_grad(zd, o["counts"], k, d, valid=vd, e2g=gd, G=G)
    assert bool(torch.isnan(dz[4]).all()) and bool(torch.isfinite(dz[5:]).all())


@pytest.mark.parametrize("T", [1, 64, 4000])
def test_no_token_counts(T):
    z, idx, _ = make(1, T, 9, 2)
    zd, id_, vd = device(z, idx, np.zeros(T, np.uint8))
    o = B.balance(zd, id_, valid=vd)
    assert not o["losses"].any() and not o["counts"].any() and not o["prob"].any()
    assert not B.balance_grad(zd, o["counts"], 2, torch.ones(2, device="cuda"), valid=vd).any()


def test_large_logits():
    """Spans past where e^x is 0, and values near the end of fp32's."""
    z = np.zeros((6, 5), np.float32)
    z[0] = [0, -50, -103, -104, -1000]
    z[1] = [3e38, -3e38, 0, 0, 0]
    z[2] = [1e4, 1e4 - 1, 0, 0, 0]
    z[3] = -1e4
    z[4] = [-3e38] * 5
    z[5] = [88, 0, -88, 1, 2]
    idx = np.zeros((6, 1), np.int32)
    for rows in ([0, 2, 3, 5], [1, 4]):
        zd, id_ = device(z[rows], idx[rows])
        o = B.balance(zd, id_)
        want = losses64(z[rows], idx[rows], None, np.arange(5), 5, 1)
        np.testing.assert_allclose(o["prob"].double().cpu().numpy(), want[2], rtol=1e-6, atol=1e-30)
        np.testing.assert_allclose(float(o["losses"][0]), want[0][0], rtol=1e-6)
        with np.errstate(over="ignore"):
            z2 = np.float32(want[0][1])
        assert float(o["losses"][1]) == z2 or abs(float(o["losses"][1]) / z2 - 1) <= 1e-6


@pytest.mark.parametrize("T,E,k", [(70, 8, 2), (900, 60, 4), (300, 128, 2), (700, 256, 8)])
def test_rows_off_16_byte_chunks(T, E, k):
    """E a multiple of four, the logits (or the gradient) a view that starts between 16-byte chunks: another path, the
    same definition."""
    z, idx, valid = make(T, T, E, k)
    zd, id_, vd = device(z, idx, valid)
    off = torch.empty(T * E + 1, device="cuda")[1:].view(T, E).copy_(zd)
    d = torch.tensor([0.3, 0.2], device="cuda")
    a, b = B.balance(zd, id_, valid=vd), B.balance(off, id_, valid=vd)
    assert torch.equal(a["counts"], b["counts"])
    # (either is off by what test_losses_and_gradient allows)
    tol = 2 * (row_error(z).max() + (T / 64 + 34) * F32)
    torch.testing.assert_close(a["prob"], b["prob"], rtol=tol, atol=0)
    torch.testing.assert_close(a["losses"], b["losses"], rtol=4 * tol, atol=0)
    g = B.balance_grad(zd, a["counts"], k, d, valid=vd)
    size = float(g.abs().max())
    for src, dst in ((off, None), (zd, torch.empty(T * E + 1, device="cuda")[1:].view(T, E))):
        torch.testing.assert_close(B.balance_grad(src, a["counts"], k, d, valid=vd, out=dst), g, rtol=0, atol=8 * tol * size)


@pytest.mark.parametrize("T", [7, 900, 5000])
def test_squares_past_fp32(T):
    """The sum of the squares leaves fp32, their mean does not."""
    z = torch.full((T, 12), 1.5e19, device="cuda")
    idx = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    lse = float(np.float32(1.5e19))  # (log 12 is far below its last bit)
    assert abs(float(B.balance(z, idx)["losses"][1]) / lse ** 2 - 1) <= 2 * F32


# 65536 (E <= 16) and 16384 tokens a round of 256 workgroups: 2048 rounds and some, or 128; sums of two levels
@pytest.mark.parametrize("T,E", [((1 << 27) + 77, 2), ((1 << 25) + 5, 17), ((1 << 21) + 3, 100), ((1 << 21) + 1, 251)])
def test_long_batches_add_as_well_as_short_ones(T, E):
    """A lane takes thousands of tokens; what it adds in fp32 is bounded all the same. Rows alike, so that every
    rounding of a running sum would go the same way for long."""
    row = np.zeros(E, np.float32)
    row[0], row[1] = (3.0, 0.0) if E == 2 else (5.0, 2.0)
    z = torch.from_numpy(row).cuda().expand(T, E).contiguous()
    idx = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    valid = torch.ones(T, dtype=torch.uint8, device="cuda")
    valid[::1001] = 0
    o = B.balance(z, idx, valid=valid)
    want = losses64(row[None], np.zeros((1, 1), np.int32), None, np.arange(E), E, 1)
    V = T - -(-T // 1001)
    assert o["counts"].tolist() == [V] + [0] * (E - 1) + [V]
    # fp32 sums of a lane up to 32 tokens, rounded once more; over 4 or 16 lanes' tokens and 16 waves; rounded where
    # they are put away, twice, and at the end
    tol = row_error(row[None])[0] + (32 + 1 + 4 + 16 + 3) * F32
    np.testing.assert_allclose(o["prob"].double().cpu().numpy(), want[2], rtol=tol, atol=0)
    got = o["losses"].double().cpu().numpy()
    assert abs(got[0] / want[0][0] - 1) <= tol + F32
    # (lse: the sum's error relative to its argument, its own roundings by its size, and the square)
    size = float(want[4][0]) + 1
    assert abs(got[1] - want[0][1]) <= 2 * size * (row_error(row[None])[0] + 8 * size * F32) + want[0][1] * 4 * F32


def test_results_do_not_depend_on_the_run():
    z, idx, valid = make(2, 30000, 60, 4)
    zd, id_, vd = device(z, idx, valid)
    ws, bufs = B.new_balance_workspace(30000, 60, "cuda"), B.new_balance_buffers(60, "cuda")
    first = {n: t.clone() for n, t in B.balance(zd, id_, valid=vd).items()}
    for fill in (0, 255):
        ws[B.BALANCE_ZERO_BYTES:].fill_(fill)
        for _ in range(20):
            o = B.balance(zd, id_, valid=vd, out=bufs, workspace=ws)
            assert o["losses"] is bufs["losses"]
            for n in first:
                assert torch.equal(o[n], first[n]), n
            assert not ws[:B.BALANCE_ZERO_BYTES].any()
    # a workspace of more tokens
    few = {n: t.clone() for n, t in B.balance(zd[:9000], id_[:9000], valid=vd[:9000]).items()}
    B.balance(zd[:9000], id_[:9000], valid=vd[:9000], out=bufs, workspace=ws)
    assert all(torch.equal(bufs[n], few[n]) for n in few)


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    sets = [device(*make(i, 20000 + i, 60, 4)) for i in range(2)]
    want = [{n: t.clone() for n, t in B.balance(z, i, valid=v).items()} for z, i, v in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [B.new_balance_workspace(z.shape[0], 60, "cuda") for z, _, _ in sets]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [B.balance(z, i, valid=v, workspace=w, stream=s) for (z, i, v), w, s in zip(sets, spaces, streams)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(a[n], b[n]) for n in b)


@pytest.mark.parametrize("T", [100, 5000])
def test_autograd(T):
    z, idx, valid = make(T, T, 24, 3)
    e2g = (np.arange(24) % 7).astype(np.int32)
    zd, id_, vd, gd = device(z, idx, valid, e2g)
    # the router's own product in front, as a program trains it
    x = torch.randn((T, 16), device="cuda")
    w = torch.randn((24, 16), device="cuda", requires_grad=True)
    logits = x @ w.t() + zd
    losses, counts, prob = B.balance_loss(logits, id_, valid=vd, e2g=gd, G=7)
    assert not counts.requires_grad and not prob.requires_grad
    c = torch.tensor([0.01, 0.001], device="cuda")
    (losses * c).sum().backward()
    direct = B.balance_grad(logits.detach(), counts, 3, c, valid=vd, e2g=gd, G=7)
    torch.testing.assert_close(w.grad, direct.t() @ x, rtol=1e-5, atol=1e-7)
    # one of the two losses, twice through the same leaf
    leaf = zd.clone().requires_grad_()
    losses, _, _ = B.balance_loss(leaf, id_, valid=vd, e2g=gd, G=7)
    losses[1].backward()
    one = leaf.grad.clone()
    assert torch.equal(one, B.balance_grad(zd, counts_of(zd, id_, vd), 3, torch.tensor([0.0, 1.0], device="cuda"),
                                           valid=vd, e2g=gd, G=7))
    losses, _, _ = B.balance_loss(leaf, id_, valid=vd, e2g=gd, G=7)
    losses[1].backward()
    assert torch.equal(leaf.grad, one + one)
    # no tokens
    empty = torch.zeros((0, 24), device="cuda", requires_grad=True)
    losses, counts, _ = B.balance_loss(empty, id_[:0])
    losses.sum().backward()
    assert not losses.any() and not counts.any() and empty.grad.shape == (0, 24)


def counts_of(z, idx, valid):
    return B.balance(z, idx, valid=valid)["counts"]


@pytest.mark.parametrize("T", [200, 3000])
def test_stream_and_graph(T):
    z, idx, valid = make(T, T, 60, 4)
    zd, id_, vd = device(z, idx, valid)
    d = torch.tensor([0.1, 0.2], device="cuda")
    want = B.balance(zd, id_, valid=vd)
    dz = B.balance_grad(zd, want["counts"], 4, d, valid=vd)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    o = B.balance(zd, id_, valid=vd, stream=s)
    g = B.balance_grad(zd, o["counts"], 4, d, valid=vd, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(g, dz) and all(torch.equal(o[n], want[n]) for n in want)
    bufs, ws, out = B.new_balance_buffers(60, "cuda"), B.new_balance_workspace(T, 60, "cuda"), torch.empty_like(zd)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.balance(zd, id_, valid=vd, out=bufs, workspace=ws)
        B.balance_grad(zd, bufs["counts"], 4, d, valid=vd, out=out)
    for rep in range(4):
        zd.normal_()
        want = B.balance(zd, id_, valid=vd)
        dz = B.balance_grad(zd, want["counts"], 4, d, valid=vd)
        for t in (*bufs.values(), out):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, dz) and all(torch.equal(bufs[n], want[n]) for n in want), f"replay {rep}"
        assert not ws[:B.BALANCE_ZERO_BYTES].any()


def test_argument_refusals():
    z, idx, valid = make(1, 30, 12, 2)
    zd, id_, vd = device(z, idx, valid)
    e2g = torch.zeros(12, dtype=torch.int32, device="cuda")
    c, d = B.balance(zd, id_)["counts"], torch.ones(2, device="cuda")
    bad = [lambda: B.balance(zd.double(), id_), lambda: B.balance(zd, id_.long()), lambda: B.balance(zd[:, :11], id_),
           lambda: B.balance(zd, id_[:29]), lambda: B.balance(zd, id_, valid=vd.bool()), lambda: B.balance(zd, id_, e2g=e2g),
           lambda: B.balance(zd, id_, G=3), lambda: B.balance(zd, id_, e2g=e2g[:4], G=3), lambda: B.balance(zd.cpu(), id_),
           lambda: B.balance(zd, id_, out={"prob": c}), lambda: B.balance_grad(zd, c[:12], 2, d),
           lambda: B.balance_grad(zd, c, 2, d[:1]), lambda: B.balance_grad(zd, c, 2, d, out=torch.empty(30, 11, device="cuda")),
           lambda: B.balance_loss(zd[0], id_)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    with pytest.raises(B.BmoeError, match="SHAPE"):
        B.balance_grad(zd, c, 17, d)
    with pytest.raises(B.BmoeError, match="UNSUPPORTED"):
        B.balance(zd, id_, out={"prob": zd.view(-1)[:12]})
    big = torch.zeros((5000, 12), device="cuda")
    with pytest.raises(B.BmoeError, match="WORKSPACE"):
        B.balance(big, torch.zeros((5000, 2), dtype=torch.int32, device="cuda"),
                  workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
