"""Embedding and layer norm of token rows, and their gradients, against the 64-bit oracle.

Tolerances, u = 2^-24.  A sum of n fp32 terms in any order is off by less than n u of their
magnitudes' sum; a row's sum over its threads has at most 8 NV + 22 additions after one another
(NV <= 4 vectors of 8 a thread, 6 across a wave, 16 waves): 64.  Rounding to a 16-bit type adds half a step.
"""
import numpy as np
import pytest
import torch

import paper_2606_11660_amd as P
from oracle import training as O
from tests._util import host, say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
K = 64
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF = {F32: 0.0, BF16: 2.0 ** -8, F16: 2.0 ** -11}   # half a step of 8 and 11 significant bits, relative
LEAST = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}  # and of subnormal values


def near(got, want, tol, dtype):
    got = host(got.double()) if isinstance(got, torch.Tensor) else got
    tol = tol + HALF[dtype] * (np.abs(want) + tol) + LEAST[dtype]
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], np.broadcast_to(tol, want.shape)[bad][:3])


class Batch:
    """Rows of n examples: slots, or packed with gaps; `shift` elements into wider rows."""

    def __init__(self, n, T, packed, seed, ragged=True):
        r = self.r = np.random.default_rng(seed)
        self.n, self.T = n, T
        self.length = r.integers(0, T + 1, n) if ragged else np.full(n, T)
        if ragged:
            self.length[0] = T
            self.length[-1] = 0 if n > 1 else T
        self.offset = None
        self.rows = n * T
        if packed:
            order = r.permutation(n)   # examples in another order than their rows, a row between them
            self.offset = np.zeros(n, np.int64)
            at = 1
            for i in order:
                self.offset[i] = at
                at += self.length[i] + 1
            self.rows = at
        self.slots = O.row_slots(n, T, self.rows, self.offset, self.length)

    def c(self):
        return P.ExampleRows(self.n, self.T, None if self.offset is None else torch.from_numpy(self.offset).cuda(),
                             torch.from_numpy(self.length.astype(np.int32)).cuda())

    def put(self, x, dtype, pad=0, shift=0):
        """x's rows on the device, NaN in the padding rows and in `pad` columns behind each row."""
        x = np.array(x, np.float64)
        inside = np.zeros(len(x), bool)
        inside[[row for _, row, ok in self.slots if ok]] = True
        x[~inside] = np.nan
        wide = torch.full((x.shape[0] * (x.shape[1] + pad) + shift,), float("nan"), dtype=dtype, device="cuda")
        v = wide[shift:].view(x.shape[0], x.shape[1] + pad)[:, :x.shape[1]]
        v.copy_(torch.from_numpy(x).cuda())
        return v

    def empty(self, d, dtype, pad=0, shift=0):
        wide = torch.full((self.rows * (d + pad) + shift,), 77.0, dtype=dtype, device="cuda")
        return wide[shift:].view(self.rows, d + pad)[:, :d], wide

    def untouched(self, out, d, pad):
        """Rows that are not written, and the columns behind each row."""
        v, wide = out
        shift = wide.numel() - self.rows * (d + pad)
        whole = host(wide.float())[shift:].reshape(self.rows, d + pad)
        assert (host(wide.float())[:shift] == 77).all() and (whole[:, d:] == 77).all()
        written = {row for _, row, _ in self.slots}
        rest = [i for i in range(self.rows) if i not in written]
        assert (whole[rest] == 77).all()


# ----------------------------------------------------------------------------
# embedding
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("d", [1, 2, 63, 130, 512, 513, 769, 2048, 4100])
@pytest.mark.parametrize("table,out", [(F32, BF16), (BF16, BF16), (F16, F32), (BF16, F16)])
def test_embed(d, table, out):
    for packed, scale, pad, shift in ((False, 1.0, 0, 0), (True, 1.7, 3, 1)):
        say(f"case: embed d={d} {table}->{out} packed={packed}")
        V = 37
        B = Batch(5, 7, packed, d)
        tab = torch.randn(V, d + pad, device="cuda").to(table)[:, :d]
        token = B.r.integers(0, V, B.rows)
        token[B.r.random(B.rows) < 0.2] = -1
        token[B.slots[0][1]] = V
        token[B.slots[1][1]] = 2 ** 40
        o = B.empty(d, out, pad, shift)
        P.attr_embed(tab, torch.from_numpy(token).cuda(), o[0], scale=scale, rows=B.c())
        want = O.embed(host(tab.double()), token, scale, B.slots)
        rows = sorted(want)
        w = np.stack([want[i] for i in rows])
        near(o[0][rows], w, 2 * U * np.abs(w), out)   # the scale's fp32 value, the product
        B.untouched(o, d, pad)


def test_embed_without_rows():
    tab, token = torch.randn(11, 40, device="cuda"), torch.tensor([[3, 10], [0, 11]], device="cuda")
    out = torch.full((2, 2, 40), 5.0, device="cuda")
    P.attr_embed(tab, token, out)
    assert torch.equal(out[0], tab[[3, 10]]) and torch.equal(out[1, 0], tab[0]) and (out[1, 1] == 0).all()


def back_case(V, d, dout, table, B, token, accumulate, scale, pad=0, shift=0):
    g = B.put(B.r.standard_normal((B.rows, d)), dout, pad, shift)
    wide = torch.full((V * (d + pad) + shift,), 77.0, dtype=table, device="cuda")
    dt = wide[shift:].view(V, d + pad)[:, :d]
    was = np.zeros((V, d))
    if accumulate:
        dt.copy_(torch.from_numpy(B.r.standard_normal((V, d))).cuda())
        was = host(dt.double())
    tok = torch.from_numpy(token).cuda()
    P.attr_embed_backward(g, tok, dt, scale=scale, accumulate=accumulate, rows=B.c())
    want, size, count = O.embed_backward(host(g.double()), token, V, scale, B.slots)
    tol = (count[:, None] + 3) * U * size + 2 * U * np.abs(was)
    if accumulate:
        assert np.array_equal(host(dt.double())[count == 0], was[count == 0])
    near(dt, want + was, tol, table)
    assert (wide[:shift] == 77).all()
    if pad:
        assert (wide[shift:].view(V, d + pad)[:, d:] == 77).all()
    return dt


@pytest.mark.parametrize("d", [1, 64, 65, 256, 257, 769, 1500])
@pytest.mark.parametrize("dout,table", [(BF16, F32), (F32, F32), (F16, F16), (BF16, BF16)])
def test_embed_backward(d, dout, table):
    for V, n, T, packed, accumulate in ((1, 3, 9, False, False), (5, 9, 40, True, False), (300, 6, 50, False, True),
                                        (2000, 7, 33, True, True)):
        say(f"case: embed backward d={d} {dout}->{table} V={V} packed={packed} accumulate={accumulate}")
        B = Batch(n, T, packed, d + V)
        token = B.r.integers(-1, V + 1, B.rows)
        back_case(V, d, dout, table, B, token, accumulate and table == F32, 1.0 if packed else 1.3, 3 if packed else 0,
                  1 if packed else 0)


@pytest.mark.parametrize("V", [1, 1023, 1024, 40000, 2 ** 20 + 5])
def test_embed_backward_long(V):
    """More tokens than one workgroup sorts: one token's rows past many parts, every digit's pass."""
    d = 8
    for n, T in ((1, 16384), (1, 16385), (7, 4099)):
        say(f"case: embed backward long V={V} n={n} T={T}")
        B = Batch(n, T, False, V, ragged=n > 1)
        token = np.where(B.r.random(B.rows) < 0.4, V // 2, B.r.integers(0, V, B.rows))
        first = back_case(V, d, F32, F32, B, token, False, 1.0)
        B.r = np.random.default_rng(5)
        a = back_case(V, d, F32, F32, B, token, False, 1.0).clone()
        B.r = np.random.default_rng(5)
        assert torch.equal(a, back_case(V, d, F32, F32, B, token, False, 1.0)) and first.shape == a.shape


def test_embed_backward_order():
    """A token's rows are added in the order of their slots: 1 + 2^-24 + 2^-24 is 1, the other way round 1 + 2^-23."""
    for rows, want in (([1.0, U, U], 1.0), ([U, U, 1.0], 1.0 + 2 * U)):
        token = torch.tensor([4, 2, 4, 1, 4], device="cuda")
        g = torch.tensor([rows[0], 9.0, rows[1], 9.0, rows[2]], device="cuda")[:, None].repeat(1, 3)
        dt = torch.empty(6, 3, device="cuda")
        P.attr_embed_backward(g, token, dt)
        assert (dt[4] == want).all() and (dt[[0, 3, 5]] == 0).all()


def test_embed_backward_nothing():
    dt = torch.full((9, 5), 3.0, device="cuda")
    none, tok = torch.empty(0, 5, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    P.attr_embed_backward(none, tok, dt, accumulate=True)
    assert (dt == 3).all()
    P.attr_embed_backward(none, tok, dt)
    assert (dt == 0).all()
    g, tok = torch.full((4, 5), float("nan"), device="cuda"), torch.tensor([0, 1, 2, 3], device="cuda")
    dt.fill_(3)
    P.attr_embed_backward(g, tok, dt, rows=P.ExampleRows(2, 2, length=torch.zeros(2, dtype=torch.int32, device="cuda")))
    assert (dt == 0).all()
    P.attr_embed_backward(g, torch.full((4,), 9, device="cuda"), dt.fill_(3), accumulate=True)
    assert (dt == 3).all()


# ----------------------------------------------------------------------------
# layer norm
# ----------------------------------------------------------------------------
WIDTHS = [1, 2, 7, 8, 511, 512, 513, 769, 1024, 1500, 2048, 2056, 4096, 5000, 8192, 8199, 16384, 16400, 32768]


def stat_tolerances(x, eps):
    """How far the mean may be, and (relative) 1/std."""
    size = np.abs(x).mean(1)
    dm = (K + 1) * U * size
    var = x.var(1)
    off = (dm + U * size) ** 2  # the mean's error and the differences' rounding, squared
    rel = ((K + 6) * U * var + off + 2 * np.sqrt(var) * U * size) / (var + eps)
    return dm, rel / 2 + 4 * U


@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm(d):
    kinds = [(F32, F32, F32), (BF16, BF16, BF16), (F32, BF16, F32), (F16, F16, F32), (BF16, F32, F16), (F16, BF16, BF16)]
    for j, (xt, yt, wt) in enumerate(kinds if d < 3000 else kinds[d % 3::3]):
        packed, pad, shift = bool(j & 1), (0, 3)[j & 1], (0, 1)[j & 1]
        say(f"case: layer norm d={d} {xt}->{yt} w={wt} packed={packed}")
        B = Batch(4, 5, packed, d + j)
        x = B.put(B.r.standard_normal((B.rows, d)) * np.exp(B.r.standard_normal((B.rows, 1))) + 2 * B.r.standard_normal((B.rows, 1)),
                  xt, pad, shift)
        w, b = (torch.from_numpy(B.r.standard_normal(d)).cuda().to(wt) for _ in range(2))
        if j == 4:
            b = None
        if j == 5:
            w = None
        y = B.empty(d, yt, pad, shift)
        mean, rstd = (torch.full((B.rows,), 77.0, device="cuda") for _ in range(2))
        eps = 1e-5 if j < 3 else 1e-2
        P.attr_layer_norm(x, y[0], w, b, eps, mean, rstd, rows=B.c())
        inside = [row for _, row, ok in B.slots if ok]
        pads = [row for _, row, ok in B.slots if not ok]
        xs = host(x.double())[inside]
        wn, bn = (1.0 if w is None else host(w.double())), (0.0 if b is None else host(b.double()))
        got = [O.layer_norm(row, wn, bn, eps) for row in xs]
        want, m, r = np.stack([g[0] for g in got]), np.array([g[1] for g in got]), np.array([g[2] for g in got])
        dm, dr = stat_tolerances(xs, eps)
        near(mean[inside], m, dm, F32)
        near(rstd[inside], r, dr * r, F32)
        unit = np.abs((xs - m[:, None]) * r[:, None])
        tol = np.abs(wn) * (r[:, None] * (dm[:, None] + U * np.abs(xs)) + unit * (dr[:, None] + 4 * U)) + 2 * U * (np.abs(want) + np.abs(bn))
        near(y[0][inside], want, tol, yt)
        assert (y[0][pads] == 0).all() and (mean[pads] == 0).all() and (rstd[pads] == 0).all()
        B.untouched(y, d, pad)


def test_layer_norm_rows_at_their_edges():
    """One value, equal values, large means, infinities and NaN: a row's own only; in place."""
    d = 600
    x = torch.randn(8, d, device="cuda")
    x[1] = 3.0
    x[2] += 1e4
    x[3, 5], x[4, 7] = float("inf"), float("nan")
    x[5] *= 1e25     # squares pass fp32's range
    x[6] = 0
    x[7] *= 1e-25
    keep = x.clone()
    mean, rstd = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    P.attr_layer_norm(x, x, eps=1e-5, mean=mean, rstd=rstd)
    assert torch.isnan(x[3]).all() and torch.isnan(x[4]).all()
    fine = [0, 2]
    want = np.stack([O.layer_norm(host(keep[i].double()))[0] for i in fine])
    size = np.array([np.abs(host(keep[i])).mean() for i in fine])[:, None]
    near(x[fine], want, (K + 8) * U * (size / host(keep[fine].double()).std(1)[:, None] + np.abs(want)) * 2, F32)
    assert (x[1] == 0).all() and (x[6] == 0).all() and (x[5] == 0).all() and (rstd[5] == 0).all()
    assert torch.isfinite(x[7]).all() and abs(float(rstd[6]) - 1e-5 ** -0.5) < 1e-4 * 1e-5 ** -0.5
    one = torch.tensor([[5.0], [-2.0]], device="cuda", dtype=BF16)
    P.attr_layer_norm(one, one, bias=torch.ones(1, device="cuda"))
    assert (one == 1).all()


def backward_case(B, d, xt, yt, wt, per_example, accumulate, pad=0, shift=0, in_place=None, joined=False):
    x = B.put(B.r.standard_normal((B.rows, d)) + B.r.standard_normal((B.rows, 1)), xt, pad, shift)
    dy = B.put(B.r.standard_normal((B.rows, d)), yt, pad, shift)
    w = None if wt is None else torch.from_numpy(1 + 0.3 * B.r.standard_normal(d)).cuda().to(wt)
    inside = [(i, row) for i, row, ok in B.slots if ok]
    rows = [row for _, row in inside]
    xs, ds = host(x.double()), host(dy.double())
    mean, rstd = (torch.full((B.rows,), float("nan"), device="cuda") for _ in range(2))
    if rows:
        mean[rows] = torch.from_numpy(xs[rows].mean(1)).float().cuda()
        rstd[rows] = torch.from_numpy(1 / np.sqrt(xs[rows].var(1) + 1e-5)).float().cuda()
    units = B.n if per_example else 1
    grads = torch.full((units, 2 * d + 5), 0.5 if accumulate else 77.0, device="cuda")
    if joined:
        dw, db = grads[:, 2:2 + d], grads[:, 3 + d:3 + 2 * d]
    else:
        dw, db = (torch.full((units, d), 0.5 if accumulate else 77.0, device="cuda") for _ in range(2))
    dx = B.empty(d, xt, pad, shift)
    out = {None: dx[0], "x": x, "dy": dy}[in_place]
    P.attr_layer_norm_backward(dy, x, mean, rstd, w, out, dw if per_example else dw[0], db if per_example else db[0],
                               per_example=per_example, accumulate=accumulate, rows=B.c())
    m, r, wn = host(mean.double()), host(rstd.double()), 1.0 if w is None else host(w.double())
    sums = np.zeros((4, units, d))
    for i, row in inside:
        want, tw, tb = O.layer_norm_backward(ds[row], xs[row], m[row], r[row], wn)
        j = i if per_example else 0
        sums[:, j] += tw, tb, np.abs(tw), np.abs(tb)
        unit, e = np.abs((xs[row] - m[row]) * r[row]), np.abs(ds[row] * wn)
        tol = r[row] * ((K + 4) * U * e.mean() + 4 * U * e + unit * ((K + 10) * U * (e * unit).mean()))
        near(out[row], want, tol, xt)
    n = max(1, len(rows)) + 6
    base = 0.5 if accumulate else 0.0
    near(dw, sums[0] + base, n * U * sums[2] + U, F32)
    near(db, sums[1] + base, n * U * sums[3] + U, F32)
    if in_place is None:
        B.untouched(dx, d, pad)
        pads = [row for _, row, ok in B.slots if not ok]
        assert (dx[0][pads] == 0).all()
    if joined:
        rest = torch.cat([grads[:, :2], grads[:, 2 + d:3 + d], grads[:, 3 + 2 * d:]], 1)
        assert (rest == (0.5 if accumulate else 77)).all()


@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm_backward(d):
    kinds = [(F32, F32, F32), (BF16, BF16, BF16), (F32, BF16, F32), (F16, F16, None), (BF16, F32, F16)]
    for j, (xt, yt, wt) in enumerate(kinds if d < 3000 else kinds[d % 2::2]):
        say(f"case: layer norm backward d={d} x={xt} dy={yt} w={wt}")
        backward_case(Batch(4, 5, bool(j & 1), d + j), d, xt, yt, wt, j % 3 == 1, j > 2, (0, 3)[j & 1], (0, 1)[j & 1])


@pytest.mark.parametrize("d", [40, 769, 2304])
def test_layer_norm_backward_many_rows(d):
    """Many chunks, joined; examples of one and of many chunks; gradients that are columns of wider rows."""
    for n, T, packed, per_example in ((3, 300, False, True), (40, 3, True, True), (1, 999, False, False), (6, 170, True, False)):
        say(f"case: layer norm backward d={d} n={n} T={T} per_example={per_example}")
        backward_case(Batch(n, T, packed, d + n), d, F32, F32, F32, per_example, n == 3, joined=per_example)


@pytest.mark.parametrize("d", [100, 3000, 20000])
def test_layer_norm_backward_in_place(d):
    for where in ("x", "dy"):
        backward_case(Batch(3, 4, where == "x", d), d, BF16, BF16, F32, False, False, in_place=where)


def test_layer_norm_backward_parts():
    """Each of its outputs alone gives the same bits."""
    d, n = 300, 50
    x, dy = torch.randn(n, d, device="cuda"), torch.randn(n, d, device="cuda")
    mean, rstd = x.mean(1), 1 / (x.var(1, correction=0) + 1e-5).sqrt()
    new = lambda: (torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda"))  # noqa: E731
    dx, dw, db = new()
    P.attr_layer_norm_backward(dy, x, mean, rstd, None, dx, dw, db)
    for keep in range(8):
        got = new()
        give = [t if keep >> k & 1 else None for k, t in enumerate(got)]
        P.attr_layer_norm_backward(dy, x, mean, rstd, None, *give)
        for k, (a, b) in enumerate(zip(got, (dx, dw, db))):
            assert not keep >> k & 1 or torch.equal(a, b)


def test_layer_norm_backward_nothing():
    e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    dw, db = torch.full((7,), 3.0, device="cuda"), torch.full((7,), 3.0, device="cuda")
    P.attr_layer_norm_backward(e(0, 7), e(0, 7), e(0), e(0), None, e(0, 7), dw, db, accumulate=True)
    assert (dw == 3).all() and (db == 3).all()
    P.attr_layer_norm_backward(e(0, 7), e(0, 7), e(0), e(0), None, e(0, 7), dw, db)
    assert (dw == 0).all() and (db == 0).all()
    dw = torch.full((2, 7), 3.0, device="cuda")
    x = torch.full((4, 7), float("nan"), device="cuda")
    P.attr_layer_norm_backward(x, x.clone(), x[:, 0].contiguous(), x[:, 0].contiguous(), None, None, dw, per_example=True,
                               rows=P.ExampleRows(2, 2, length=torch.tensor([-3, 0], dtype=torch.int32, device="cuda")))
    assert (dw == 0).all()


def test_gradient_against_differences():
    """The kernels' own differences in fp32: a step h moves <y, c> by h <dx, v>."""
    torch.manual_seed(3)
    n, d, h = 6, 96, 1e-2
    x, c, v = (torch.randn(n, d, device="cuda") for _ in range(3))
    w, b, vw, vb = (torch.randn(d, device="cuda") for _ in range(4))

    def f(t):
        y = torch.empty_like(x)
        P.attr_layer_norm(x + t * v, y, w + t * vw, b + t * vb)
        return float((y.double() * c).sum())
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    P.attr_layer_norm(x, y, w, b, mean=mean, rstd=rstd)
    dx, dw, db = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    P.attr_layer_norm_backward(c, x, mean, rstd, w, dx, dw, db)
    want = float((dx.double() * v).sum() + (dw.double() * vw).sum() + (db.double() * vb).sum())
    got = (8 * (f(h) - f(-h)) - (f(2 * h) - f(-2 * h))) / (12 * h)   # to fourth order
    # fp32 values of |y c| ~ 1, 600 of them, over 2 h: 600^(1/2) 2^-23 / h ~ 3e-4; the fifth derivative times h^4: 1e-6
    assert abs(got - want) < 2e-3 * max(1.0, abs(want)), (got, want)


def test_offsets_past_32_bits():
    """Rows whose elements lie past 2^32 bytes and 2^31 elements from the first."""
    d, far = 512, 2 ** 31 // 512 + 3
    x = torch.zeros(far + 2, d, dtype=BF16, device="cuda")
    x[far:] = torch.randn(2, d, device="cuda").to(BF16)
    B = P.ExampleRows(1, 2, torch.tensor([far], device="cuda"), torch.tensor([2], dtype=torch.int32, device="cuda"))
    y = torch.zeros(far + 2, d, dtype=BF16, device="cuda")
    mean, rstd = torch.zeros(far + 2, device="cuda"), torch.zeros(far + 2, device="cuda")
    P.attr_layer_norm(x, y, mean=mean, rstd=rstd, rows=B)
    want = np.stack([O.layer_norm(r)[0] for r in host(x[far:].double())])
    near(y[far:], want, 200 * U * np.ones_like(want), BF16)
    assert (y[:far] == 0).all()
    dx = torch.zeros_like(x)
    P.attr_layer_norm_backward(y, x, mean, rstd, None, dx, rows=B)
    assert (dx[:far] == 0).all() and torch.isfinite(dx[far:]).all() and (dx[far:] != 0).any()
    del dx
    token = torch.zeros(far + 2, dtype=torch.int64, device="cuda")
    token[far + 1] = far
    P.attr_embed(x, token, y.zero_(), rows=B)
    assert torch.equal(y[far + 1], x[far]) and (y[:far + 1] == 0).all()
    dt = x.zero_()
    P.attr_embed_backward(y, token, dt, rows=B)
    assert torch.equal(dt[far], y[far + 1]) and (dt[:far] == 0).all()


def test_rows_outside_the_tensors():
    """Offsets before the first row and past the last: those rows are neither read nor written."""
    d, n_rows = 24, 10
    x = torch.randn(n_rows, d, device="cuda")
    B = P.ExampleRows(4, 4, torch.tensor([-2, 8, 2 ** 62, -2 ** 63], device="cuda"))
    y = torch.full_like(x, 7.0)
    mean, rstd = torch.full((n_rows,), 7.0, device="cuda"), torch.full((n_rows,), 7.0, device="cuda")
    P.attr_layer_norm(x, y, mean=mean, rstd=rstd, rows=B)
    assert (y[2:8] == 7).all() and (y[:2] != 7).all() and (y[8:] != 7).all()
    dx, dw = torch.full_like(x, 7.0), torch.empty(4, d, device="cuda")
    P.attr_layer_norm_backward(x, x.clone(), mean, rstd, None, dx, dw, per_example=True, rows=B)
    assert (dx[2:8] == 7).all() and (dx[:2] != 7).all() and (dw[2:] == 0).all() and (dw[:2] != 0).any(1).all()
    dt = torch.empty(3, d, device="cuda")
    P.attr_embed_backward(x, torch.ones(n_rows, dtype=torch.int64, device="cuda"), dt, rows=B)
    assert torch.allclose(dt[1], x[[0, 1, 8, 9]].sum(0), atol=1e-5) and (dt[[0, 2]] == 0).all()


def test_types_that_are_not_taken():
    x = torch.zeros(4, 8, dtype=torch.float64, device="cuda")
    with pytest.raises(TypeError, match="float64"):
        P.attr_layer_norm(x, x.float())
    with pytest.raises(TypeError, match="float64"):
        P.attr_embed(x, torch.zeros(2, dtype=torch.int64, device="cuda"), x[:2].float())


def test_captured_and_on_another_stream():
    """Replays with eager work between them, two graphs on one workspace, another stream."""
    d, n, V = 700, 300, 50
    torch.manual_seed(1)
    x, dy = torch.randn(n, d, device="cuda"), torch.randn(n, d, device="cuda")
    token = torch.randint(0, V, (n,), device="cuda")
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dt, out = torch.empty(V, d, device="cuda"), torch.empty(n, d, device="cuda")
    side, ws = torch.cuda.Stream(), P.Workspace()

    def norm():
        P.attr_layer_norm(x, y, mean=mean, rstd=rstd)
        P.attr_layer_norm_backward(dy, x, mean, rstd, None, dx, dw, db, ws=ws)

    def emb():
        P.attr_embed(dt, token, out)
        P.attr_embed_backward(dy, token, dt, ws=ws)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        norm(), emb()
    side.synchronize()
    graphs = []
    for f in (norm, emb):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            f()
        graphs.append(g)
    for k in range(4):
        x.normal_(), dy.normal_()
        token.random_(0, V)
        dt.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw, db, dt)]
        norm(), emb()
        torch.cuda.synchronize()
        for a, b in zip(got, (y, dx, dw, db, dt)):
            assert torch.equal(a, b), k


def _each_call(wide):
    """Every call once, with all that it may be given; wide: rows that are columns of wider ones."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    n, T, d, V = 5, 9, 40, 23
    pad = 3 if wide else 0

    def rand(*s, dtype=F32):
        return torch.randn(*s[:-1], s[-1] + pad, generator=gen, device="cuda").to(dtype)[..., :s[-1]]
    where = P.ExampleRows(n, T, length=torch.tensor([9, 3, 0, 9, 1], dtype=torch.int32, device="cuda"))
    token = torch.randint(-1, V + 1, (n * T,), generator=gen, device="cuda")
    x, dy, w, b = rand(n * T, d, dtype=BF16), rand(n * T, d), rand(d, dtype=F16).contiguous(), rand(d, dtype=F16).contiguous()
    out, y, dx = rand(n, T, d) if not wide else rand(n * T, d), rand(n * T, d), rand(n * T, d, dtype=BF16)
    dt, dw, db = rand(V, d), rand(n, d), rand(n, d)
    mean, rstd = torch.zeros(n * T, device="cuda"), torch.zeros(n * T, device="cuda")
    P.attr_embed(rand(V, d, dtype=F16), token, out, scale=1.5, rows=where)
    P.attr_embed_backward(dy, token, dt, scale=0.7, accumulate=True, rows=where)
    P.attr_layer_norm(x, y, w, b, 1e-3, mean, rstd, rows=where)
    P.attr_layer_norm_backward(dy, x, mean, rstd, w, dx, dw, db, per_example=True, accumulate=True, rows=where)
    e = torch.empty(n * T, d, device="cuda")
    P.attr_layer_norm(x, e)
    return out, dt, y, mean, rstd, dx, dw, db, e


@pytest.mark.parametrize("wide", [False, True])
def test_native_checks_and_python_ones_make_the_same_calls(monkeypatch, wide):
    taken = []
    native = P._native_rows_call()
    monkeypatch.setattr(P, "_native_rows", lambda *a: taken.append(native(*a)) or taken[-1])
    a = _each_call(wide)
    assert taken.count(0) >= 4 and None not in taken    # 4: a workspace that had to grow
    monkeypatch.setattr(P, "_native_rows", lambda *a: None)
    for s, t in zip(a, _each_call(wide)):
        assert torch.equal(s, t)


def test_refusals_on_the_gpu():
    t = lambda *s, d=F32: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
    x, m, tok = t(4, 8), t(4), t(4, d=torch.int64)
    calls = [(lambda: P.attr_layer_norm(x, t(5, 8)), "y must"), (lambda: P.attr_layer_norm(x, t(4, 8), t(7)), "8 elements"),
             (lambda: P.attr_layer_norm(x, t(4, 8), t(8), t(8, d=BF16)), "one type"),
             (lambda: P.attr_layer_norm(x, t(4, 8), mean=t(3)), "mean"), (lambda: P.attr_layer_norm(x, t(4, 8).cpu()), "GPU"),
             (lambda: P.attr_layer_norm(x.t(), x.t()), "contiguous last"),
             (lambda: P.attr_layer_norm(x, t(4, 8), rows=P.ExampleRows(3, 2)), "need"),
             (lambda: P.attr_layer_norm(x, t(4, 8), rows=P.ExampleRows(2, 2, length=t(2))), "length"),
             (lambda: P.attr_embed(t(5, 9), tok, x), "table"), (lambda: P.attr_embed(t(5, 8), tok[:3], x), "token"),
             (lambda: P.attr_embed(t(5, 8), tok.int(), x), "token"), (lambda: P.attr_embed(t(5, 8), tok.cpu(), x), "GPU"),
             (lambda: P.attr_embed_backward(x, tok, t(5, 7)), "dtable"),
             (lambda: P.attr_layer_norm_backward(x, x, m, None), "forward"),
             (lambda: P.attr_layer_norm_backward(x, x, m, m, dx=t(4, 8, d=BF16)), "type"),
             (lambda: P.attr_layer_norm_backward(x, x, m, m, dweight=t(1, 8)), "dweight"),
             (lambda: P.attr_layer_norm_backward(x, x, m, m, dbias=t(8, d=BF16)), "dbias"),
             (lambda: P.attr_layer_norm_backward(x, x, m, m, dbias=t(3, 8), per_example=True, rows=P.ExampleRows(2, 2)), "dbias")]
    for f, match in calls:
        with pytest.raises(ValueError, match=match):
            f()
    for f, match in [(lambda: P.attr_layer_norm(x, t(4, 8), eps=-1.0), "eps"), (lambda: P.attr_embed(t(5, 8), tok, x, scale=float("inf")), "scale"),
                     (lambda: P.attr_embed(x[:, :8], tok, x), "overlap")]:
        with pytest.raises(P.AttrError, match=match):
            f()


def test_autograd_sees_what_the_calls_write():
    for k in range(4):
        w = [torch.randn(4, 8, device="cuda", requires_grad=True) for _ in range(4)]
        z = sum((v * v).sum() for v in w)
        d = [v.detach() for v in w]
        tok, m = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
        if k == 0:
            P.attr_embed(torch.zeros(5, 8, device="cuda"), tok, d[0])
        elif k == 1:
            P.attr_embed_backward(torch.zeros(4, 8, device="cuda"), tok, d[1])
        elif k == 2:
            P.attr_layer_norm(torch.zeros(4, 8, device="cuda"), d[2])
        else:
            P.attr_layer_norm_backward(torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), m, m, dx=d[3])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()


def test_embed_backward_many_parts():
    """Parts of 32 neighbours, and of 64 in the longest batches, that begin, end and hold whole tokens; on both sides of
    the sort's sizes, and of the batches that need none."""
    for n, V in ((256, 40), (257, 40), (512, 9000), (513, 40), (2049, 600), (32768, 700), (262143, 700), (262144, 700),
                 (300001, 70000)):
        say(f"case: embed backward parts n={n} V={V}")
        B = Batch(1, n, False, n, ragged=False)
        token = np.where(B.r.random(B.rows) < 0.3, 1, B.r.integers(0, V, B.rows))
        back_case(V, 12, BF16, F32, B, token, False, 1.0)
    for n, V, d in ((400, 3, 700), (64, 1, 300), (65, 1, 300), (300, 100000, 2100)):   # tokens of many rows; a search too long
        B = Batch(n, 1, True, n)
        back_case(V, d, F16, F32, B, B.r.integers(0, V, B.rows), True, 0.7)


def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    """Refused: the current stream is not theirs."""
    x = torch.zeros(4, 8, device="cuda")
    tok, v = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    plan = P.MuonTensors([x], [x.clone()], [x.clone()])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: x.device.index + 1)
    for call in (lambda: P.attr_embed(x, tok, x.clone()), lambda: P.attr_embed_backward(x, tok, x.clone()),
                 lambda: P.attr_layer_norm(x, x.clone()), lambda: P.attr_layer_norm_backward(x, x, v, v, dx=x.clone()),
                 lambda: P.attr_muon_step(plan, 0.1)):
        with pytest.raises(ValueError, match="current GPU device"):
            call()


@pytest.mark.parametrize("d", [65, 769, 1025, 2100])
@pytest.mark.parametrize("dout,table", [(BF16, F32), (F16, F16), (F32, BF16)])
def test_embed_backward_sorted(d, dout, table):
    """Batches that are sorted, by one workgroup and by several: four and eight columns a lane, a token whose
    rows cross many parts, tables between aligned places and with gaps, written whole and added to."""
    for n, T, V, packed, accumulate, pad, shift in ((6, 500, 700, False, False, 3, 1), (6, 500, 700, True, True, 0, 1),
                                                    (9, 1000, 700, True, False, 0, 1), (9, 1000, 20011, False, True, 3, 0),
                                                    (9, 1000, 20011, True, False, 3, 1)):
        say(f"case: embed backward sorted d={d} {dout}->{table} n={n * T} V={V} packed={packed} accumulate={accumulate}")
        B = Batch(n, T, packed, d + V + pad)
        token = np.where(B.r.random(B.rows) < 0.3, V // 2, B.r.integers(-1, V + 1, B.rows))
        back_case(V, d, dout, table, B, token, accumulate, 0.7, pad, shift)


def forward_case(B, d, xt, yt, wt, pad, shift, eps=1e-5):
    """Layer norm of a batch against the oracle; y is x itself where pad and shift are 0 and the types are one."""
    x = B.put(B.r.standard_normal((B.rows, d)) * np.exp(B.r.standard_normal((B.rows, 1))) + 2 * B.r.standard_normal((B.rows, 1)),
              xt, pad, shift)
    xs = host(x.double())
    w, b = (torch.from_numpy(B.r.standard_normal(d)).cuda().to(wt) for _ in range(2))
    in_place = xt == yt and not pad and not shift
    y = (x, None) if in_place else B.empty(d, yt, pad, shift)
    mean, rstd = (torch.full((B.rows,), 77.0, device="cuda") for _ in range(2))
    P.attr_layer_norm(x, y[0], w, b, eps, mean, rstd, rows=B.c())
    inside, pads = ([row for _, row, ok in B.slots if ok == want] for want in (True, False))
    xs, wn, bn = xs[inside], host(w.double()), host(b.double())
    m = xs.mean(1)
    r = 1 / np.sqrt(np.square(xs - m[:, None]).mean(1) + eps)
    want = (xs - m[:, None]) * r[:, None] * wn + bn
    assert np.allclose(want[0], O.layer_norm(xs[0], wn, bn, eps)[0], rtol=1e-12, atol=1e-12)
    dm, dr = stat_tolerances(xs, eps)
    near(mean[inside], m, dm, F32)
    near(rstd[inside], r, dr * r, F32)
    unit = np.abs((xs - m[:, None]) * r[:, None])
    tol = np.abs(wn) * (r[:, None] * (dm[:, None] + U * np.abs(xs)) + unit * (dr[:, None] + 4 * U)) + 2 * U * (np.abs(want) + np.abs(bn))
    near(y[0][inside], want, tol, yt)
    assert (y[0][pads] == 0).all() and (mean[pads] == 0).all() and (rstd[pads] == 0).all()
    if not in_place:
        B.untouched(y, d, pad)


@pytest.mark.parametrize("n,T,d", [(10, 103, d) for d in (8, 512, 513, 769, 1023, 1024, 1025, 1500, 2048)]
                         + [(10, 26, d) for d in (2049, 3001, 4096, 4100, 5000, 8191, 8192, 8199)])
def test_layer_norm_of_many_rows(n, T, d):
    """Batches past the sizes at which a row takes more threads (1024 slots to 2048 columns, 256 beyond):
    packed, padded, with gaps and in place, widths that end inside a lane's vector."""
    for xt, yt, wt, packed, pad, shift in ((F32, BF16, F32, True, 3, 1), (BF16, BF16, BF16, False, 0, 0),
                                           (F32, F32, F16, True, 0, 0), (F16, F32, F32, False, 0, 1)):
        say(f"case: layer norm of many rows d={d} n={n * T} {xt}->{yt} w={wt} packed={packed}")
        forward_case(Batch(n, T, packed, d + 1), d, xt, yt, wt, pad, shift)


# ----------------------------------------------------------------------------
# the largest sizes, compared on the GPU in 64 bits
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("n,accumulate", [(40, True), (700, False)])
def test_embed_widest(n, accumulate):
    V, d = 30, 65536
    B = Batch(n, 1, True, n)
    say(f"case: embed d={d} n={n}")
    token = B.r.integers(-1, V + 1, B.rows)
    dt = back_case(V, d, BF16, F32, B, token, accumulate, 0.7)
    o = B.empty(d, BF16)
    P.attr_embed(dt, torch.from_numpy(token).cuda(), o[0], rows=B.c())
    inside = [row for _, row, ok in B.slots if ok]
    there = torch.from_numpy((token[inside] >= 0) & (token[inside] < V)).cuda()
    want = dt[torch.from_numpy(token[inside].clip(0, V - 1)).cuda()].to(BF16)
    assert torch.equal(o[0][inside], torch.where(there[:, None], want, 0))


def test_embed_of_the_largest_table():
    """2^28 rows: digits of four passes, zeros written beside them."""
    V, n = 2 ** 28, 5000
    say(f"case: embed backward V={V}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    token = torch.randint(0, V, (n,), generator=gen, device="cuda")
    token[::3], token[-1], token[7] = V - 1, V, 0
    g = torch.randint(-8, 9, (n, 1), generator=gen, device="cuda").to(F32)   # sums are whole numbers below 2^14: exact
    dt = torch.full((V, 1), 9.0, device="cuda")
    P.attr_embed_backward(g, token, dt)
    ok = token < V
    want = torch.zeros(V, device="cuda", dtype=torch.float64).index_add_(0, token[ok], g[ok, 0].double())
    assert torch.equal(dt[:, 0].double(), want)
    out = torch.full((n, 1), 9.0, device="cuda")
    P.attr_embed(dt, token, out)
    assert torch.equal(out[ok], dt[token[ok]]) and (out[~ok] == 0).all()


def test_more_rows_than_a_launch_has_waves():
    """2^21 workgroups of four rows each, and some more: they stride over what is left."""
    n, V = 2 ** 23 + 1001, 91
    say(f"case: embed and layer norm n={n}")
    gen = torch.Generator(device="cuda").manual_seed(2)
    token = torch.randint(0, V, (n,), generator=gen, device="cuda")
    table, out = torch.randn(V, 3, generator=gen, device="cuda"), torch.empty(n, 3, device="cuda")
    P.attr_embed(table, token, out)
    assert torch.equal(out, table[token])
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    y = torch.empty_like(out)
    P.attr_layer_norm(out, y, mean=mean, rstd=rstd)
    one, m1, r1 = torch.empty_like(table), torch.empty(V, device="cuda"), torch.empty(V, device="cuda")
    P.attr_layer_norm(table, one, mean=m1, rstd=r1)
    assert torch.equal(y, one[token]) and torch.equal(mean, m1[token]) and torch.equal(rstd, r1[token])


@pytest.mark.parametrize("n,T,d,per_example", [(520, 270, 40, True), (520, 90, 1030, True), (520, 70, 2100, True),
                                               (1, 300001, 40, False)])
def test_layer_norm_backward_long_shares(n, T, d, per_example):
    """Shares of more rows than a wave knows the places of at once (64).  dx as of few rows; sums: n u of the
    magnitudes' sum."""
    say(f"case: layer norm backward long shares n={n} T={T} d={d}")
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, dy = (torch.randn(n * T, d, generator=gen, device="cuda") for _ in range(2))
    w = 1 + 0.3 * torch.randn(d, generator=gen, device="cuda")
    length = torch.randint(0, T + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
    length[0] = T
    inside = (torch.arange(T, device="cuda") < length[:, None]).view(-1)
    mean, rstd = x.double().mean(1).float(), (1 / (x.double().var(1, correction=0) + 1e-5).sqrt()).float()
    x[~inside], dy[~inside] = float("nan"), float("nan")
    units = n if per_example else 1
    dx = torch.full_like(x, 77.0)
    dw, db = (torch.full((units, d), 0.5, device="cuda") for _ in range(2))
    P.attr_layer_norm_backward(dy, x, mean, rstd, w, dx, dw if per_example else dw[0], db if per_example else db[0],
                               per_example=per_example, accumulate=True, rows=P.ExampleRows(n, T, length=length))
    u = torch.where(inside[:, None], (x.double() - mean[:, None]) * rstd[:, None], 0.0)
    g = torch.where(inside[:, None], dy.double(), 0.0)
    e = g * w
    want = (e - e.mean(1, keepdim=True) - u * (e * u).mean(1, keepdim=True)) * rstd[:, None]
    r, a = rstd[:, None].double(), e.abs()
    tol = r * ((K + 4) * U * a.mean(1, keepdim=True) + 4 * U * a + u.abs() * ((K + 10) * U * (a * u.abs()).mean(1, keepdim=True)))
    assert ((dx.double() - want).abs() <= tol + 2.0 ** -149).all()
    terms = (T if per_example else n * T) + 6
    for got, term in ((dw, g * u), (db, g)):
        total, size = term.view(units, -1, d).sum(1), term.abs().view(units, -1, d).sum(1)
        assert ((got.double() - total - 0.5).abs() <= terms * U * size + U).all()


def test_layer_norm_past_fp32s_range():
    """A row whose sum passes fp32's range is NaN, one whose squares do has 1/std 0; their neighbours are their own."""
    x = torch.ones(4, 600, device="cuda")
    x[0], x[1, ::2], x[1, 1::2], x[2, 0] = 3e38, 3e38, -3e38, 2.0
    y, rstd = torch.empty_like(x), torch.empty(4, device="cuda")
    P.attr_layer_norm(x, y, rstd=rstd)
    assert torch.isnan(y[0]).all() and (y[1] == 0).all() and rstd[1] == 0
    assert torch.isfinite(y[2:]).all() and (y[3] == 0).all()
