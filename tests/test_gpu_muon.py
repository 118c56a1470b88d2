"""The Muon step against the 64-bit oracle.

Tolerance of X: the roundings of a step, each independent, carried through the following steps.  In
the singular basis of X (its singular values s_i, p(s) = a s + b s^3 + c s^5) a step multiplies the
symmetric part of a change's entry (i, j) by (p(s_i) - p(s_j)) / (s_i - s_j), the antisymmetric one by
(p(s_i) + p(s_j)) / (s_i + s_j) and what is outside X's row space by p(s_i) / s_i; energies (squares) are
carried, spread evenly over the entries where they arise:
    X rounded:  (h / 3^(1/2) |X|)^2,  h = 2^-11 or, with pairs, 2^-22
    A, B:       likewise, and fp32 sums of K products, whose roundings on the matrix cores may all
                point one way: K / 16 2^-24 |A| (twice that with pairs, which add three products)
    into X:     dX_ij = dB_ij s_j,  dB_ij = (b + c (s_i^2 + s_j^2)) dA_ij + that of B = a + b A + c A^2
The test allows four times the root of that energy.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_amd as P
from oracle import training as O
from tests._util import host, say

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
V = 2.0 ** -24
SHAPES = [(1, 1), (1, 40), (40, 1), (3, 5), (16, 64), (64, 64), (63, 65), (65, 63), (128, 128), (129, 127), (130, 300), (300, 130),
          (16, 768), (768, 16), (257, 256), (384, 513)]


def tolerance(u, pairs, steps=5):
    """How far X may be from the oracle's, in the Frobenius norm."""
    h, (a, b, c) = 2.0 ** (-22 if pairs else -11) / np.sqrt(3), O.NS
    u = np.asarray(u, np.float64)
    S, L = sorted(u.shape)
    s = np.linalg.svd(u, compute_uv=False)
    s = s / np.linalg.norm(s)
    kl, ks = ((2 if pairs else 1) * max(1.0, k / 16) * V for k in (L, S))
    p = lambda x: a * x + b * x ** 3 + c * x ** 5  # noqa: E731
    even = lambda e: (e / (S * L)) * np.ones((S, S))  # noqa: E731
    sym = anti = even((h + 2 * V) ** 2) / 2
    rest = (h + 2 * V) ** 2 / (S * L) * (L - S) * np.ones(S)
    for _ in range(steps):
        x, y = s[:, None], s[None, :]
        lam = s ** 2
        poly = b * lam + c * lam ** 2
        gs = a + b * (x * x + x * y + y * y) + c * (x ** 4 + x ** 3 * y + x * x * y * y + x * y ** 3 + y ** 4)
        ga = a + b * (x * x - x * y + y * y) + c * (x ** 4 - x ** 3 * y + x * x * y * y - x * y ** 3 + y ** 4)
        dA = (h ** 2 + kl ** 2) * (lam ** 2).sum() / S ** 2
        dB = (b + c * (x * x + y * y)) ** 2 * dA + (h ** 2 * ((a + poly) ** 2).sum() + (ks * c) ** 2 * (lam ** 4).sum()) / S ** 2
        into = dB * y * y
        new = (h ** 2 + ks ** 2) * (p(s) ** 2).sum()
        sym, anti = (e * g * g + into / 2 + even(new) / 2 for e, g in ((sym, gs), (anti, ga)))
        rest = rest * (a + b * lam + c * lam ** 2) ** 2 + new / (S * L) * (L - S)
        s = np.abs(p(s))
    return 4 * np.sqrt(sym.sum() + anti.sum() + rest.sum())


def matrix(r, rows, cols, kind="plain"):
    x = r.standard_normal((rows, cols))
    if kind == "low":   # a few large directions beside small ones
        k = max(1, min(rows, cols) // 16)
        x = 0.1 * x + r.standard_normal((rows, k)) @ r.standard_normal((k, cols))
    return x * 1e-3


class Model:
    def __init__(self, seed, shapes, p=F32, g=F32, master=False, zero=False, shift=0):
        r = np.random.default_rng(seed)

        def put(x, dtype):
            buf = torch.zeros(x.size + shift, dtype=dtype, device="cuda")
            buf[shift:] = torch.from_numpy(x.reshape(-1)).cuda().to(dtype)
            return buf[shift:].view(x.shape)
        w = [r.standard_normal(s) * (0.0 if zero else 0.1) for s in shapes]
        self.p, self.master = [put(x, p) for x in w], [put(x, F32) for x in w] if master else None
        self.g = [put(matrix(r, *s, "low" if j % 2 else "plain"), g) for j, s in enumerate(shapes)]
        self.m = [put(matrix(r, *s), F32) for s in shapes]
        self.was = [(host((self.master or self.p)[j].double()), host(self.g[j].double()), host(self.m[j].double()))
                    for j in range(len(shapes))]

    def plan(self, **kw):
        return P.MuonTensors(self.p, self.g, self.m, master=self.master, **kw)


@pytest.mark.parametrize("pairs", [False, True], ids=["f16", "pairs"])
@pytest.mark.parametrize("nesterov", [False, True])
def test_update(pairs, nesterov):
    """The update itself: weights of zero, a rate of -1."""
    gs = torch.full((1,), 0.37, device="cuda")
    M = Model(1, SHAPES, zero=True)
    say(f"case: muon update pairs={pairs}")
    P.attr_muon_step(M.plan(), -1.0, momentum=0.9, nesterov=nesterov, pairs=pairs, grad_scale=gs)
    for j, s in enumerate(SHAPES):
        w, g, m = M.was[j]
        f = float(gs)
        _, nm, x = O.muon(w, g, m, -1.0, 0.9, nesterov, grad_scale=f)
        mu, one = np.float32(0.9), np.float32(1.0 - 0.9)
        got_m = m.astype(np.float32) * mu + (g.astype(np.float32) * np.float32(f)) * one
        assert np.array_equal(host(M.m[j]), got_m), s
        u = 0.9 * nm + 0.1 * g * f if nesterov else nm
        off, tol = np.linalg.norm(host(M.p[j]) - x), tolerance(u, pairs)
        say(s, "off by", off / np.linalg.norm(x), "of", tol / np.linalg.norm(x))
        assert off <= tol, (s, off, tol)


@pytest.mark.parametrize("p,g,master", [(F32, F32, False), (F32, BF16, False), (BF16, BF16, True), (BF16, F32, False),
                                        (F16, F16, True), (F16, F16, False)])
def test_weights(p, g, master):
    """The step of the weights in fp32 from that update, rounded once, at any alignment."""
    shapes = [(70, 30), (16, 200), (30, 70), (0, 5), (1, 9), (200, 200)]
    for shift in (0, 1):
        kw = dict(weight_decay=[0.1 * (j % 3) for j in range(6)], lr_scale=[1.0 + j for j in range(6)])
        M, Z = Model(4, shapes, p, g, master, shift=shift), Model(4, shapes, F32, g, zero=True)
        pairs = p == F32 or master
        P.attr_muon_step(M.plan(**kw), 0.02)
        P.attr_muon_step(Z.plan(), -1.0, pairs=pairs)
        for j, s in enumerate(shapes):
            rate = 0.02 * kw["lr_scale"][j]
            lr, lr_wd = np.float32(rate), np.float32(rate * np.float32(kw["weight_decay"][j]).astype(np.float64))
            w = M.was[j][0].astype(np.float32)
            want = w - w * lr_wd - host(Z.p[j]) * lr
            got = M.master[j] if master else M.p[j]
            assert torch.equal(got, torch.from_numpy(want).cuda().to(got.dtype)), (s, shift)
            assert not master or torch.equal(M.p[j], got.to(p))
            assert torch.equal(M.m[j], Z.m[j])


@pytest.mark.parametrize("steps", [1, 2, 7])
def test_steps(steps):
    shapes = [(40, 90), (200, 64)]
    M = Model(6, shapes, zero=True)
    P.attr_muon_step(M.plan(), -1.0, momentum=0.0, steps=steps)
    for j in range(2):
        x = O.newton_schulz(M.was[j][1], steps)
        assert np.linalg.norm(host(M.p[j]) - x) <= tolerance(M.was[j][1], True, steps)


def test_larger_matrices():
    """Several tiles each way, and their products' longer sums; singular values near one."""
    for shape in ((1030, 520), (640, 1537), (1100, 1030), (1025, 1800)):
        M = Model(8, [shape], zero=True)
        N = Model(8, [shape], zero=True)
        P.attr_muon_step(M.plan(), -1.0)
        P.attr_muon_step(N.plan(), -1.0, pairs=False)
        w, g, m = M.was[0]
        _, nm, x = O.muon(w, g, m, -1.0)
        u = 0.95 * nm + 0.05 * g
        n = np.linalg.norm(x)
        fine, coarse = (np.linalg.norm(host(t.p[0]) - x) for t in (M, N))
        say(f"case: muon {shape} off by {fine / n} with pairs, {coarse / n} without")
        assert fine <= tolerance(u, True) and coarse <= tolerance(u, False) and fine < coarse / 50
        s = np.linalg.svd(host(M.p[0].double()), compute_uv=False)
        assert s.max() < 1.21 and np.median(s) > 0.68


@pytest.mark.parametrize("shape", [(5000, 65), (65, 1024), (130, 4100), (9001, 70), (1024, 5000), (2100, 1100), (8193, 64),
                                   (40, 9000), (20000, 7)])
@pytest.mark.parametrize("pairs", [False, True], ids=["f16", "pairs"])
def test_long_matrices(shape, pairs):
    """The products over the longer side, divided among workgroups; the same bits again, and a second
    matrix of other values beside it."""
    M = Model(13, [shape, shape], zero=True)
    P.attr_muon_step(M.plan(), -1.0, pairs=pairs)
    for j in range(2):
        w, g, m = M.was[j]
        _, nm, x = O.muon(w, g, m, -1.0)
        off, tol = np.linalg.norm(host(M.p[j]) - x), tolerance(0.95 * nm + 0.05 * g, pairs)
        say(f"case: muon {shape} {j} off by {off / np.linalg.norm(x)} of {tol / np.linalg.norm(x)}")
        assert off <= tol
    N = Model(13, [shape, shape], zero=True)
    P.attr_muon_step(N.plan(), -1.0, pairs=pairs)
    assert all(torch.equal(a, b) for a, b in zip(M.p, N.p))


def test_many_matrices_of_many_shapes():
    """More shapes than a launch takes groups, more matrices than a table's launch; each as alone."""
    r = np.random.default_rng(3)
    shapes = [(int(a), int(b)) for a, b in r.integers(1, 70, (40, 2))] * 3 + [(8, 8)] * 100
    M = Model(11, shapes, zero=True)
    P.attr_muon_step(M.plan(), -1.0)
    for j in list(range(0, 120, 7)) + [120, 170, 219]:
        A = Model(11, shapes, zero=True)
        one = P.MuonTensors([A.p[j]], [A.g[j]], [A.m[j]])
        P.attr_muon_step(one, -1.0)
        assert torch.equal(A.p[j], M.p[j]) and torch.equal(A.m[j], M.m[j]), shapes[j]


def test_edges():
    """Zero updates, infinities and NaN, huge and tiny gradients: each matrix on its own."""
    n = 6
    g = [torch.randn(20, 30, device="cuda") for _ in range(n)]
    g[0].zero_()
    g[1][3, 4], g[2][5, 6] = float("nan"), float("inf")
    g[3] *= 1e34
    g[4] *= 1e-36
    p = [torch.ones(20, 30, device="cuda") for _ in range(n)]
    m = [torch.zeros(20, 30, device="cuda") for _ in range(n)]
    P.attr_muon_step(P.MuonTensors(p, g, m, weight_decay=0.5), 0.1, momentum=0.5)
    assert torch.equal(p[0], torch.full_like(p[0], 1 - np.float32(0.05)))
    assert torch.isnan(p[1]).all() and torch.isnan(p[2]).all()
    for j in (3, 4, 5):
        want = O.muon(np.ones((20, 30)), host(g[j].double()), np.zeros((20, 30)), 0.1, 0.5, weight_decay=0.5)[0]
        # tiny gradients: u has fewer bits near the end of fp32's range (1e-36: 2^-149 / 1e-36 = 1.4e-9)
        assert np.abs(host(p[j]) - want).max() < 1e-5, j


def test_the_same_bits_again_captured_and_on_another_stream():
    shapes = [(33, 70), (128, 40)]
    M, W = Model(2, shapes), Model(2, shapes)
    a, b = M.plan(), W.plan()
    side, ws = torch.cuda.Stream(), P.Workspace()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.attr_muon_step(a, 0.02, ws=ws)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        P.attr_muon_step(a, 0.02, ws=ws)
    P.attr_muon_step(b, 0.02)
    for k in range(3):
        for t, s in zip(M.g, W.g):
            t.normal_()
            s.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        P.attr_muon_step(b, 0.02)
        torch.cuda.synchronize()
        for x, y in zip(M.p + M.m, W.p + W.m):
            assert torch.equal(x, y), k


def test_plan_refusals():
    t = lambda *s, d=F32: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
    with pytest.raises(ValueError, match="shape"):
        P.MuonTensors([t(4, 5)], [t(5, 4)], [t(4, 5)])
    with pytest.raises(ValueError, match="contiguous"):
        P.MuonTensors([t(5, 4).t()], [t(4, 5)], [t(4, 5)])
    with pytest.raises(ValueError, match="float32"):
        P.MuonTensors([t(4, 5)], [t(4, 5)], [t(4, 5, d=BF16)])
    with pytest.raises(ValueError, match="contiguous"):
        P.MuonTensors([t(4)], [t(4)], [t(4)])
    x = t(4, 5)
    with pytest.raises(ValueError, match="overlap"):
        P.MuonTensors([x], [x], [t(4, 5)])
    with pytest.raises(ValueError, match="overlap"):
        P.MuonTensors([t(4, 5), t(4, 5)], [t(4, 5), t(4, 5)], [x, x])
    P.MuonTensors([t(4, 5), t(4, 5)], [x, x], [t(4, 5), t(4, 5)])   # one gradient twice is only read
    with pytest.raises(ValueError, match="entries"):
        P.MuonTensors([t(4, 5)], [t(4, 5)], [t(4, 5)], lr_scale=[1.0, 2.0])
    plan = P.MuonTensors([t(4, 5)], [t(4, 5)], [t(4, 5)])
    with pytest.raises(P.AttrError, match="steps"):
        P.attr_muon_step(plan, 0.1, steps=17)
    with pytest.raises(P.AttrError, match="momentum"):
        P.attr_muon_step(plan, 0.1, momentum=1.0)
    with pytest.raises(P.AttrError, match="lr"):
        P.attr_muon_step(plan, float("nan"))
    with pytest.raises(ValueError, match="grad_scale"):
        P.attr_muon_step(plan, 0.1, grad_scale=t(1, d=BF16))


def test_autograd_sees_the_step():
    w = torch.randn(6, 6, device="cuda", requires_grad=True)
    loss = (w * w).sum()
    with torch.no_grad():
        P.attr_muon_step(P.MuonTensors([w.detach()], [torch.randn(6, 6, device="cuda")], [torch.zeros(6, 6, device="cuda")]), 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


@pytest.mark.parametrize("p,master", [(F32, False), (BF16, True), (F16, False)])
def test_a_factor_of_the_update_alone(p, master):
    """x (1 - lr wd) - lr f X: the decay is the rate's, whatever the matrix's shape scales the update by.
    Roundings, in half steps of 2^-24: lr f and wd / f one each, lr wd one, then two products and two
    differences; of the weight once more where it has 16 bits."""
    shapes, f, lr, wd, rate = [(70, 30), (30, 70), (200, 90)], [12.8, 0.3, (200 / 90) ** 0.5], 0.02, 0.5, [1.0, 2.0, 0.7]
    M, Z = Model(4, shapes, p, F32, master), Model(4, shapes, F32, F32, zero=True)
    P.attr_muon_step(M.plan(weight_decay=wd, lr_scale=rate, update_scale=f), lr)
    P.attr_muon_step(Z.plan(), -1.0, pairs=p == F32 or master)
    for j, s in enumerate(shapes):
        w, x, r = M.was[j][0], host(Z.p[j].double()), lr * rate[j]
        want = w * (1 - r * wd) - r * f[j] * x
        tol = V * (5 * np.abs(w) * r * wd + 4 * np.abs(r * f[j] * x) + 2 * (np.abs(w) + np.abs(want)))
        got = M.master[j] if master else M.p[j]
        tol = tol + {F32: 0.0, F16: 2.0 ** -11}[got.dtype] * (np.abs(want) + tol) + (2.0 ** -25 if got.dtype == F16 else 0.0)
        assert (np.abs(host(got.double()) - want) <= tol).all(), s
        assert not master or torch.equal(M.p[j], got.to(p))


def test_factors_that_are_refused():
    t = [torch.zeros(4, 5, device="cuda") for _ in range(3)]
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(ValueError, match="update_scale"):
            P.MuonTensors([t[0]], [t[1]], [t[2]], update_scale=bad)
    with pytest.raises(ValueError, match="entries"):
        P.MuonTensors([t[0]], [t[1]], [t[2]], update_scale=[1.0, 2.0])


# ----------------------------------------------------------------------------
# 256 x 256 tiles (shorter sides from 1024, 128 such tiles of A's in a call), rounds, special values
# ----------------------------------------------------------------------------
LARGE = [(1025, 1100), (1100, 1025)] * 5      # 15 tiles of A's each: 150


@pytest.mark.parametrize("pairs", [False, True], ids=["f16", "pairs"])
def test_large_tiles(pairs):
    """Sides that end inside a tile, both ways round; the same bits again."""
    say(f"case: muon tiles of 256, pairs={pairs}")
    M, N = Model(15, LARGE, zero=True), Model(15, LARGE, zero=True)
    P.attr_muon_step(M.plan(), -1.0, pairs=pairs)
    P.attr_muon_step(N.plan(), -1.0, pairs=pairs)
    for j in (0, 1, 2, 9):
        w, g, m = M.was[j]
        _, nm, x = O.muon(w, g, m, -1.0)
        off, tol = np.linalg.norm(host(M.p[j]) - x), tolerance(0.95 * nm + 0.05 * g, pairs)
        say(f"case: muon {LARGE[j]} {j} off by {off / np.linalg.norm(x)} of {tol / np.linalg.norm(x)}")
        assert off <= tol
    for a, b in zip(M.p + M.m, N.p + N.m):
        assert torch.equal(a, b)


@pytest.mark.parametrize("p,g,master", [(F32, F32, False), (BF16, BF16, True), (BF16, BF16, False), (F16, F32, False)])
def test_large_tiles_weights(p, g, master):
    """The step of the weights from that update, rounded once, between aligned places too."""
    for shift in (0, 1):
        say(f"case: muon tiles of 256, weights {p} shift={shift}")
        M, Z = Model(16, LARGE, p, g, master, shift=shift), Model(16, LARGE, F32, g, zero=True)
        pairs = p == F32 or master
        P.attr_muon_step(M.plan(weight_decay=0.1), 0.02)
        P.attr_muon_step(Z.plan(), -1.0, pairs=pairs)
        lr, lr_wd = np.float32(0.02), np.float32(0.02 * np.float64(np.float32(0.1)))
        for j in (0, 1, 9):
            w = M.was[j][0].astype(np.float32)
            want = w - w * lr_wd - host(Z.p[j]) * lr
            got = M.master[j] if master else M.p[j]
            assert torch.equal(got, torch.from_numpy(want).cuda().to(got.dtype)), j
            assert not master or torch.equal(M.p[j], got.to(p))
            assert torch.equal(M.m[j], Z.m[j])


class Many:
    """n matrices of one shape and zero weights, gradients of normal values in one buffer."""

    def __init__(self, n, shape, seed=21):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.g = torch.empty((n,) + shape, device="cuda", dtype=BF16).normal_(generator=gen)
        self.p, self.m = (torch.zeros((n,) + shape, device="cuda") for _ in range(2))

    def plan(self, n=None):
        return P.MuonTensors(list(self.p[:n]), list(self.g[:n]), list(self.m[:n]))

    def check(self, j, pairs):
        g = host(self.g[j].double()) * (1.0 - 0.5)
        x = O.newton_schulz(g)
        off, tol = np.linalg.norm(host(self.p[j]) - x), tolerance(g, pairs)
        say(f"case: muon matrix {j} off by {off / np.linalg.norm(x)} of {tol / np.linalg.norm(x)}")
        assert off <= tol, j


@pytest.mark.parametrize("n,last,shape,pairs", [(48, 1, (1030, 4200), False), (24, 1, (4200, 1030), True),
                                                (460, 4, (70, 1100), False), (460, 4, (1100, 70), True)])
def test_rounds(n, last, shape, pairs):
    """More matrices than are worked on together: the last round has one of 256-tiles, or four of one
    128-tile each, which share out their rows; the same bits again."""
    say(f"case: muon {n} of {shape} pairs={pairs}")
    M, N = Many(n, shape), Many(n, shape)
    size = [P.attr_muon_step_workspace_size(M.plan(k), pairs) for k in (n - last - 1, n - last, n)]
    assert size[0] < size[1] == size[2]    # the last ones take a round of their own
    for t in (M, N):
        P.attr_muon_step(t.plan(), -1.0, momentum=0.5, nesterov=False, pairs=pairs)
    assert torch.equal(M.p, N.p) and torch.equal(M.m, M.g.float() * 0.5)
    for j in (0, n - 2, n - 1):
        M.check(j, pairs)


def test_many_shapes_of_tiles():
    """More shapes than a launch takes groups, matrices of one and of several tiles: each as alone."""
    shapes = [(66 + 5 * j, 70 + 17 * (j * 7 % 23)) for j in range(22)] * 2
    for pairs in (False, True):
        M = Model(17, shapes, zero=True)
        P.attr_muon_step(M.plan(), -1.0, pairs=pairs)
        for j in range(0, 44, 5):
            A = Model(17, shapes, zero=True)
            P.attr_muon_step(P.MuonTensors([A.p[j]], [A.g[j]], [A.m[j]]), -1.0, pairs=pairs)
            assert torch.equal(A.p[j], M.p[j]) and torch.equal(A.m[j], M.m[j]), shapes[j]


@pytest.mark.parametrize("pairs", [False, True], ids=["f16", "pairs"])
@pytest.mark.parametrize("shape", [(130, 200), (300, 70), (1030, 1100)])
def test_special_values_on_tiles(shape, pairs):
    """A zero update, NaN and infinities, huge and tiny gradients, one entry, one direction: each
    matrix on its own, on tiles of 128 and of 256."""
    say(f"case: muon special values {shape} pairs={pairs}")
    r = np.random.default_rng(5)
    g = [matrix(r, *shape) * 1e3 for _ in range(9)]
    g[0][:] = 0
    g[1][-1, -1], g[2][0, 3], g[3][7, 0] = np.nan, np.inf, -np.inf
    g[4] *= 1e34
    g[5] *= 1e-34
    g[6][:] = 0
    g[6][shape[0] - 2, shape[1] - 1] = 3.0
    g[7] = np.outer(g[7][:, 0], g[7][0])
    gt = [torch.from_numpy(x).float().cuda() for x in g]
    for w in (0.0, 1.0):
        p, m = [torch.full(shape, w, device="cuda") for _ in g], [torch.zeros(shape, device="cuda") for _ in g]
        P.attr_muon_step(P.MuonTensors(p, gt, m, weight_decay=0.5 * w), -1.0 + 1.1 * w, momentum=0.5, pairs=pairs)
        assert torch.equal(p[0], torch.full_like(p[0], float(w - w * np.float32(0.05)) if w else 0.0))
        assert all(torch.isnan(p[j]).all() for j in (1, 2, 3))
        if w:
            assert all(torch.isfinite(p[j]).all() for j in (4, 5, 6, 7, 8))
            continue
        for j in (4, 5, 6, 7, 8):
            u = host(gt[j].double())    # X does not depend on its length
            # an update near the end of fp32's range: 2^-149 / 1e-34 = 1.4e-11 of it
            off, tol = np.linalg.norm(host(p[j]) - O.newton_schulz(u)), tolerance(u, pairs)
            say(j, "off by", off, "of", tol)
            assert off <= tol, j


@pytest.mark.parametrize("pairs", [False, True], ids=["f16", "pairs"])
@pytest.mark.parametrize("shape", [(1 << 20, 64), (65, 1 << 20), (1, 1 << 20)])
def test_longest_sides(shape, pairs):
    """The longest sides that are taken, of a thin matrix and of one tile's."""
    say(f"case: muon {shape} pairs={pairs}")
    M = Many(1, shape)
    P.attr_muon_step(M.plan(), -1.0, momentum=0.5, nesterov=False, pairs=pairs)
    M.check(0, pairs)
