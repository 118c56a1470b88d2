"""Embedding, layer norm and Muon on the CPU: the oracle's gradients against differences and
its orthogonalisation against singular values, and the refusals of the C entry points and the binding."""
import numpy as np
import pytest
import torch

import paper_2606_11660_amd as P
from oracle import training as O

INVALID, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4
FAKE, OUT, MORE, WS = 0x100000, 0x900000, 0xb00000, 0xa00000


def test_oracle_layer_norm_against_differences():
    r = np.random.default_rng(0)
    x, w, b, c = (r.standard_normal(13) for _ in range(4))
    y, mean, rstd = O.layer_norm(x, w, b)
    dx, dw, db = O.layer_norm_backward(c, x, mean, rstd, w)
    h = 1e-6
    for j in range(13):
        d = np.zeros(13)
        d[j] = h
        f = lambda x, w, b: O.layer_norm(x, w, b)[0] @ c  # noqa: E731
        for grad, lo, hi in ((dx, f(x - d, w, b), f(x + d, w, b)), (dw, f(x, w - d, b), f(x, w + d, b)),
                             (db, f(x, w, b - d), f(x, w, b + d))):
            assert abs(grad[j] - (hi - lo) / (2 * h)) < 1e-7


def test_oracle_embedding_gradient_against_differences():
    r = np.random.default_rng(1)
    table, token, c = r.standard_normal((5, 3)), np.array([4, 0, 7, 4, -1, 2]), r.standard_normal((6, 3))
    slots = O.row_slots(2, 3, 6, length=[3, 2])
    f = lambda t: sum((row @ c[i]) for i, row in O.embed(t, token, 1.5, slots).items())  # noqa: E731
    grad = O.embed_backward(c, token, 5, 1.5, slots)[0]
    for i in range(5):
        for j in range(3):
            d = np.zeros((5, 3))
            d[i, j] = 1e-6
            assert abs(grad[i, j] - (f(table + d) - f(table - d)) / 2e-6) < 1e-8


def test_oracle_orthogonalisation():
    """Singular values go through the polynomial, singular vectors stay."""
    r = np.random.default_rng(2)
    a, b, c = O.NS
    for shape in ((9, 14), (14, 9), (7, 7)):
        x = r.standard_normal(shape)
        u, s, vt = np.linalg.svd(x, full_matrices=False)
        s = s / np.linalg.norm(s)
        for _ in range(5):
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.abs(O.newton_schulz(x) - u * s @ vt).max() < 1e-12
        assert s.max() < 1.2025 and (s[:-1].min() > 0.6)
    assert (O.newton_schulz(np.zeros((3, 4))) == 0).all()


def _r(**kw):
    base = dict(n_rows=8, n_examples=4, T=2, row_offset=None, length=None)
    base.update(kw)
    return P._CRows(*base.values())


def _calls(rows):
    L = P.lib()
    return [L.attr_embed(rows, FAKE, FAKE, 0, 10, 8, 8, 1.0, OUT, 0, 8, None),
            L.attr_embed_backward(rows, FAKE, FAKE, 0, 8, 10, 8, 1.0, OUT, 0, 8, 0, None, 0, None),
            L.attr_layer_norm(rows, FAKE, 0, 8, 8, None, None, 0, 1e-5, OUT, 0, 8, None, None, None),
            L.attr_layer_norm_backward(rows, FAKE, 0, 8, FAKE, 0, 8, 8, FAKE, FAKE, None, 0, OUT, 8, None, 8, None, 8, 0, 0,
                                       None, 0, None)]


@pytest.mark.parametrize("bad,status", [
    (dict(n_rows=-1), INVALID), (dict(n_rows=7), INVALID), (dict(n_examples=-2), INVALID), (dict(T=0), INVALID),
    (dict(n_examples=2 ** 20, T=2 ** 11, n_rows=2 ** 31), UNSUPPORTED), (dict(n_examples=2 ** 62, T=4), UNSUPPORTED),
    (dict(T=2 ** 62), UNSUPPORTED), (dict(row_offset=FAKE + 4), ALIGN), (dict(length=FAKE + 2), ALIGN)])
def test_rows_refusals(bad, status):
    assert _calls(_r(**bad)) == [status] * 4, P.lib().attr_last_error()


def test_embed_refusals():
    L = P.lib()

    def call(rows=None, tok=FAKE, tab=MORE, tt=0, V=10, d=8, ldt=8, s=1.0, out=OUT, ot=0, ldo=8):
        return L.attr_embed(rows or _r(), tok, tab, tt, V, d, ldt, s, out, ot, ldo, None)
    for kw in (dict(tok=None), dict(tab=None), dict(out=None), dict(V=0), dict(V=2 ** 28 + 1), dict(d=0), dict(d=65537),
               dict(ldt=7), dict(ldo=7), dict(ldt=2 ** 41), dict(s=float("nan")), dict(s=float("inf")), dict(out=MORE + 32),
               dict(out=FAKE), dict(rows=_r(n_rows=2 ** 61))):
        assert call(**kw) == INVALID, (kw, L.attr_last_error())
    for kw in (dict(tt=3), dict(ot=7)):
        assert call(**kw) == UNSUPPORTED, kw
    for kw in (dict(tok=FAKE + 4), dict(tab=MORE + 2), dict(out=OUT + 1), dict(out=OUT + 1, ot=1)):
        assert call(**kw) == ALIGN, kw
    assert call(_r(n_examples=0, n_rows=0), tok=None, tab=None, out=None) == 0


def test_embed_backward_refusals():
    L = P.lib()
    big = _r(n_rows=8000, n_examples=4, T=2000)
    need = L.attr_embed_backward_workspace_size(big, 10, 8)
    assert need >= 4 * 4 * 8000 and L.attr_embed_backward_workspace_size(_r(T=0), 10, 8) == 0

    def call(rows=None, tok=FAKE, g=MORE, gt=0, ldd=8, V=10, d=8, s=1.0, out=OUT, ot=0, ldt=8, acc=0, ws=WS, n=need):
        return L.attr_embed_backward(rows or _r(), tok, g, gt, ldd, V, d, s, out, ot, ldt, acc, ws, n, None)
    for kw in (dict(tok=None), dict(g=None), dict(out=None), dict(V=0), dict(d=0), dict(ldt=7), dict(ldd=7), dict(acc=2),
               dict(s=float("nan")), dict(out=MORE), dict(out=FAKE)):
        assert call(**kw) == INVALID, (kw, L.attr_last_error())
    assert call(gt=3) == UNSUPPORTED and call(ot=3) == UNSUPPORTED
    assert call(_r(n_rows=2 ** 32)) == UNSUPPORTED
    assert call(tok=FAKE + 4) == ALIGN and call(g=MORE + 2) == ALIGN and call(out=OUT + 2) == ALIGN and call(big, g=0x1000000, ws=WS + 16) == ALIGN
    assert call(big, g=0x1000000, ws=None) == WORKSPACE and call(big, g=0x1000000, n=need - 1) == WORKSPACE
    assert call(_r(n_examples=0, n_rows=0), acc=1, tok=None, g=None, out=None, ws=None) == 0


def test_norm_refusals():
    L = P.lib()

    def call(rows=None, x=FAKE, xt=0, d=8, ldx=8, w=None, b=None, wt=0, eps=1e-5, y=OUT, yt=0, ldy=8, m=None, r=None):
        return L.attr_layer_norm(rows or _r(), x, xt, d, ldx, w, b, wt, eps, y, yt, ldy, m, r, None)
    for kw in (dict(x=None), dict(y=None), dict(d=0), dict(d=32769, ldx=32769, ldy=32769), dict(ldx=7), dict(ldy=7),
               dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(y=FAKE + 32), dict(y=FAKE, ldy=9),
               dict(y=FAKE, yt=1), dict(m=OUT), dict(m=MORE, r=MORE), dict(r=FAKE), dict(w=OUT), dict(b=OUT)):
        assert call(**kw) == INVALID, (kw, L.attr_last_error())
    assert call(xt=3) == UNSUPPORTED and call(yt=3) == UNSUPPORTED and call(w=MORE, wt=3) == UNSUPPORTED
    for kw in (dict(x=FAKE + 2), dict(y=OUT + 2), dict(w=MORE + 2), dict(b=MORE + 1, wt=1), dict(m=MORE + 2), dict(r=MORE + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(_r(n_examples=0, n_rows=0), x=None, y=None) == 0


def test_norm_backward_refusals():
    L = P.lib()
    big = _r(n_rows=4000, n_examples=4, T=1000)
    need = L.attr_layer_norm_backward_workspace_size(big, 8, 0)
    assert need > 0 and L.attr_layer_norm_backward_workspace_size(_r(), 8, 1) == 0
    assert L.attr_layer_norm_backward_workspace_size(big, 8, 2) == 0

    def call(rows=None, dy=MORE, yt=0, lddy=8, x=FAKE, xt=0, d=8, ldx=8, m=0xc00000, r=0xd00000, w=None, wt=0, dx=OUT, lddx=8,
             dw=0xe00000, ldw=8, db=0xf00000, ldb=8, per=0, acc=0, ws=WS, n=1 << 16):
        return L.attr_layer_norm_backward(rows or _r(), dy, yt, lddy, x, xt, d, ldx, m, r, w, wt, dx, lddx, dw, ldw, db, ldb,
                                          per, acc, ws, n, None)
    for kw in (dict(dy=None), dict(x=None), dict(m=None), dict(r=None), dict(d=0), dict(ldx=7), dict(lddy=7), dict(lddx=7),
               dict(per=2), dict(acc=2), dict(per=1, ldw=7), dict(per=1, ldb=7), dict(dx=FAKE + 32), dict(dx=MORE + 32),
               dict(dx=MORE, yt=1), dict(dx=FAKE, lddx=9), dict(dw=OUT), dict(db=0xe00000), dict(dw=0xc00000),
               dict(per=1, dw=OUT + 0x1000, db=OUT + 0x1000 + 28, ldw=16, ldb=16),     # columns that touch
               dict(per=1, dw=OUT + 0x1000, db=OUT + 0x1000 + 32, ldw=15, ldb=15),
               dict(per=1, dw=OUT + 0x1000, db=OUT + 0x1000 + 32, ldw=16, ldb=17)):
        assert call(**kw) == INVALID, (kw, L.attr_last_error())
    assert call(xt=3) == UNSUPPORTED and call(yt=3) == UNSUPPORTED and call(w=WS, wt=3) == UNSUPPORTED
    for kw in (dict(dy=MORE + 2), dict(x=FAKE + 2), dict(dx=OUT + 2), dict(dw=0xe00002), dict(db=0xf00001), dict(m=0xc00001),
               dict(r=0xd00002), dict(w=0x800002), dict(rows=big, ws=WS + 16)):
        assert call(**kw) == ALIGN, kw
    assert call(big, ws=None) == WORKSPACE and call(big, n=need - 1) == WORKSPACE
    assert call(_r(n_examples=0, n_rows=0), per=1, dy=None, x=None, m=None, r=None) == 0
    assert call(dx=None, dw=None, db=None) == 0


def _m(**kw):
    base = dict(p=FAKE, g=OUT, m=MORE, master=None, rows=4, cols=8, lr_scale=1.0, weight_decay=0.0)
    base.update(kw)
    return P._CMuonMatrix(*base.values())


def test_muon_refusals():
    L = P.lib()

    def call(mats=None, p=0, g=0, lr=0.1, mu=0.9, nest=1, steps=5, pairs=0, gs=None, ws=WS, n=1 << 30, count=None):
        mats = [_m()] if mats is None else mats
        arr = (P._CMuonMatrix * max(1, len(mats)))(*mats)
        return L.attr_muon_step(arr, len(mats) if count is None else count, p, g, lr, mu, nest, steps, pairs, gs, ws, n, None)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(count=-1), dict(lr=nan), dict(lr=inf), dict(mu=-0.1), dict(mu=1.0), dict(mu=nan), dict(nest=2), dict(steps=0),
               dict(steps=17), dict(pairs=2), dict(mats=[_m(p=None)]), dict(mats=[_m(g=None)]), dict(mats=[_m(m=None)]),
               dict(mats=[_m(rows=-1)]), dict(mats=[_m(lr_scale=nan)]), dict(mats=[_m(weight_decay=inf)]),
               dict(mats=[_m(), _m(master=0xd00000)])):
        assert call(**kw) == INVALID, (kw, L.attr_last_error())
    for kw in (dict(p=3), dict(g=3), dict(mats=[_m(rows=2 ** 20 + 1, cols=1)]), dict(mats=[_m(rows=2 ** 15, cols=2 ** 15)]),
               dict(mats=[_m(rows=2 ** 40, cols=2 ** 40)])):
        assert call(**kw) == UNSUPPORTED, (kw, L.attr_last_error())
    for kw in (dict(mats=[_m(p=FAKE + 2)]), dict(mats=[_m(g=OUT + 2)]), dict(mats=[_m(m=MORE + 2)]), dict(gs=FAKE + 2),
               dict(mats=[_m(master=0xd00002)], p=1), dict(ws=WS + 16)):
        assert call(**kw) == ALIGN, (kw, L.attr_last_error())
    wide = _m(rows=100, cols=80)
    arr = (P._CMuonMatrix * 1)(wide)
    need = L.attr_muon_step_workspace_size(arr, 1, 0)
    assert need > 0 and L.attr_muon_step_workspace_size(arr, 1, 1) > need and L.attr_muon_step_workspace_size(arr, 1, 2) == 0
    assert call(mats=[wide], n=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE
    assert call(mats=[]) == 0 and call(mats=[_m(rows=0, p=None, g=None, m=None)], ws=None) == 0


def test_muon_workspace_is_bounded():
    """Many matrices take turns: the workspace stays near what a round of them needs."""
    L = P.lib()
    sizes = []
    for n in (1, 8, 200):
        arr = (P._CMuonMatrix * n)(*[_m(rows=2048, cols=8192) for _ in range(n)])
        sizes.append(L.attr_muon_step_workspace_size(arr, n, 0))
    one = 2 * 2048 * 8192 + 2 * 2048 * 2048   # Y twice, A and B
    one *= 2   # bytes
    parts = 256 * 256 * 256 * 4   # few tiles: sums of parts, at most one tile for each CU
    assert one <= sizes[0] < one + parts + (1 << 16) and sizes[1] <= sizes[2] <= (1 << 30) + (1 << 20)


def test_binding_refusals():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU"):
        P.attr_layer_norm(x, x.clone())
    with pytest.raises(ValueError, match="rows"):
        P.attr_layer_norm(x, torch.zeros(3, 8))
    with pytest.raises(ValueError, match="contiguous last"):
        P.attr_layer_norm(x.t(), x.t())
    with pytest.raises(ValueError, match="one type"):
        P.attr_layer_norm(x, x.clone(), torch.ones(8), torch.ones(8, dtype=torch.float16))
    with pytest.raises(ValueError, match="8 elements"):
        P.attr_layer_norm(x, x.clone(), torch.ones(7))
    with pytest.raises(ValueError, match="mean"):
        P.attr_layer_norm(x, x.clone(), mean=torch.zeros(3))
    with pytest.raises(ValueError, match="need"):
        P.attr_layer_norm(x, x.clone(), rows=P.ExampleRows(3, 2))
    with pytest.raises(ValueError, match="length"):
        P.attr_layer_norm(x, x.clone(), rows=P.ExampleRows(2, 2, length=torch.zeros(2)))
    with pytest.raises(ValueError, match="token"):
        P.attr_embed(torch.zeros(5, 8), torch.zeros(4), x)
    with pytest.raises(ValueError, match="table"):
        P.attr_embed(torch.zeros(5, 9), torch.zeros(4, dtype=torch.int64), x)
    with pytest.raises(ValueError, match="dtable"):
        P.attr_embed_backward(x, torch.zeros(4, dtype=torch.int64), torch.zeros(5, 9))
    with pytest.raises(ValueError, match="forward"):
        P.attr_layer_norm_backward(x, x, None, None)
    m = torch.zeros(4)
    with pytest.raises(ValueError, match="x's type"):
        P.attr_layer_norm_backward(x, x, m, m, dx=x.to(torch.float16))
    with pytest.raises(ValueError, match="dweight"):
        P.attr_layer_norm_backward(x, x, m, m, dweight=torch.zeros(1, 8))
    with pytest.raises(ValueError, match="dbias must have 2 rows"):
        P.attr_layer_norm_backward(x, x, m, m, dbias=torch.zeros(3, 8), per_example=True, rows=P.ExampleRows(2, 2))
