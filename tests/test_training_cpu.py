"""The post-training steps on the CPU: the oracle's gradients against differences, its
8-bit format against torch's, and every refusal of the C entry points and the binding."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_11660_amd as P
from oracle import training as O

INVALID, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4
FAKE = 0x100000


def test_oracle_gradients_against_differences():
    r = np.random.default_rng(1)
    z, y = r.standard_normal((12, 17)) * 2, r.integers(0, 17, 12)
    y[3] = -100
    w = r.uniform(0.2, 1.0, 12).astype(np.float32)
    w[7] = 0
    length = np.array([3, 0, 2, 3])
    where = dict(weight=w, length=length)
    old, ref = r.normal(-2, 0.5, 12).astype(np.float32), r.normal(-2, 0.5, 12).astype(np.float32)
    adv = r.standard_normal(4).astype(np.float32)

    def policy(x):
        return O.policy_loss(x, y, 4, 3, adv, 1.25, logp_old=old, logp_ref=ref, beta=0.3, **where)

    def pref(x):
        loss, _, logp, grad = O.preference_loss(x, y, 4, 3, 1.25, logp_ref=ref, pair_weight=[0.5, 2.0], beta=0.4,
                                                margin=0.2, label_smoothing=0.1, **where)
        return loss, logp, grad
    for f in (policy, pref):
        grad, h = f(z)[2], 1e-6
        assert sorted(grad) == list(range(12))
        for row in range(12):
            for j in range(17):
                d = np.zeros_like(z)
                d[row, j] = h
                want = (f(z + d)[0].sum() - f(z - d)[0].sum()) / (2 * h)
                assert abs(grad[row][j] - want) < 1e-8, (f.__name__, row, j)


def test_oracle_e4m3_against_torch():
    x = np.concatenate([np.random.default_rng(2).uniform(-448, 448, 20000), O.E4M3, -O.E4M3,
                        (O.E4M3[1:] + O.E4M3[:-1]) / 2, 2.0 ** np.linspace(-14, 8.8, 999)]).astype(np.float32)
    x = np.clip(x, -448, 448)
    assert np.array_equal(O.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def _rows(**kw):
    base = dict(logits=FAKE, dtype=P.ATTR_F32, n_rows=8, V=100, ldl=100, logit_scale=1.0, target=FAKE, weight=None,
                n_examples=4, T=2, row_offset=None, length=None)
    base.update(kw)
    return P._CTokenRows(*base.values())


def _calls(rows):
    """Each entry point on these rows, with valid further arguments and no workspace."""
    L = P.lib()
    out = 0x900000
    return [L.attr_token_logp(rows, out, None, 0, None),
            L.attr_policy_loss(rows, FAKE, 0, None, None, 0.2, 0.2, 0.0, out, None, None, 0, None, 0, None),
            L.attr_preference_loss(rows, None, None, 0.1, 0.0, 0.0, out, None, None, None, 0, None, 0, None)]


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=P.ATTR_E4M3), UNSUPPORTED), (dict(V=0), INVALID), (dict(V=2 ** 28 + 1, ldl=2 ** 29), INVALID),
    (dict(ldl=99), INVALID), (dict(ldl=2 ** 41), INVALID), (dict(n_rows=-1), INVALID), (dict(n_rows=7), INVALID),
    (dict(n_rows=2 ** 62), INVALID), (dict(n_examples=-2), INVALID), (dict(T=0), INVALID),
    (dict(n_examples=2 ** 20, T=2 ** 11, n_rows=2 ** 31), UNSUPPORTED), (dict(n_examples=2 ** 62, T=4), UNSUPPORTED),
    (dict(T=2 ** 62), UNSUPPORTED),
    (dict(logit_scale=0.0), INVALID), (dict(logit_scale=-1.0), INVALID), (dict(logit_scale=float("nan")), INVALID),
    (dict(logit_scale=float("inf")), INVALID), (dict(logits=None), INVALID), (dict(target=None), INVALID),
    (dict(logits=FAKE + 2), ALIGN), (dict(target=FAKE + 4), ALIGN), (dict(weight=FAKE + 2), ALIGN),
    (dict(row_offset=FAKE + 4), ALIGN), (dict(length=FAKE + 2), ALIGN)])
def test_token_rows_refusals(bad, status):
    assert _calls(_rows(**bad)) == [status] * 3, P.lib().attr_last_error()


def test_token_calls_without_work():
    """No examples: nothing is enqueued, nothing is needed."""
    assert _calls(_rows(n_examples=0, n_rows=0, logits=None, target=None)) == [0, 0, 0]


def test_policy_refusals():
    L, rows = P.lib(), _rows()
    ws = L.attr_policy_loss_workspace_size(rows)
    assert ws >= 4 * 8

    def call(adv=FAKE, per=0, old=None, ref=None, lo=0.2, hi=0.2, beta=0.0, loss=0x900000, logp=None, d=None, ldd=100,
             w=0xa00000, wn=ws):
        return L.attr_policy_loss(rows, adv, per, old, ref, lo, hi, beta, loss, logp, d, ldd, w, wn, None)
    nan = float("nan")
    assert call(adv=None) == INVALID and call(loss=None) == INVALID and call(per=2) == INVALID
    assert call(lo=-0.1) == INVALID and call(lo=nan) == INVALID and call(hi=-1.0) == INVALID and call(hi=nan) == INVALID
    assert call(beta=-0.1) == INVALID and call(beta=nan) == INVALID and call(beta=float("inf")) == INVALID
    assert call(beta=0.1) == INVALID and b"logp_ref" in L.attr_last_error()
    assert call(adv=FAKE + 2) == ALIGN and call(loss=0x900002) == ALIGN and call(old=FAKE + 1) == ALIGN
    assert call(ref=FAKE + 2) == ALIGN and call(logp=FAKE + 2) == ALIGN
    assert call(d=0x800000, ldd=99) == INVALID and call(d=0x800002) == ALIGN
    assert call(d=FAKE + 400) == INVALID and b"overlap" in L.attr_last_error()
    assert call(d=FAKE, ldd=101) == INVALID
    assert call(w=None) == WORKSPACE and call(wn=ws - 1) == WORKSPACE and call(w=0xa00010) == ALIGN


def test_preference_refusals():
    L = P.lib()

    def call(rows=None, ref=None, pw=None, beta=0.1, margin=0.0, e=0.0, loss=0x900000, ratio=None, logp=None, d=None,
             ldd=100, w=0xa00000, wn=1 << 20):
        return L.attr_preference_loss(rows or _rows(), ref, pw, beta, margin, e, loss, ratio, logp, d, ldd, w, wn, None)
    nan, inf = float("nan"), float("inf")
    assert call(_rows(n_examples=3)) == INVALID and b"even" in L.attr_last_error()
    for kw in (dict(beta=nan), dict(beta=inf), dict(margin=nan), dict(margin=-inf), dict(e=-0.1), dict(e=1.1), dict(e=nan),
               dict(loss=None), dict(d=0x800000, ldd=10), dict(d=FAKE + 400)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(ref=FAKE + 2), dict(pw=FAKE + 2), dict(loss=0x900001), dict(ratio=FAKE + 2), dict(logp=FAKE + 2),
               dict(d=0x800001), dict(w=0xa00004)):
        assert call(**kw) == ALIGN, kw
    need = L.attr_preference_loss_workspace_size(_rows())
    assert call(wn=need - 1) == WORKSPACE and call(w=None) == WORKSPACE


def test_workspace_queries_of_odd_batches():
    L = P.lib()
    for name in ("attr_token_logp", "attr_policy_loss", "attr_preference_loss"):
        query = getattr(L, name + "_workspace_size")
        assert query(None) == 0
        assert query(_rows(n_examples=-1)) == 0 and query(_rows(T=0)) == 0 and query(_rows(n_examples=2 ** 40)) == 0
        assert query(_rows(n_examples=2 ** 20, T=2 ** 10, n_rows=2 ** 30)) % 256 == 0


def test_adamw_refusals():
    L = P.lib()

    def tensor(**kw):
        base = dict(p=0x100000, g=0x200000, m=0x300000, v=0x400000, master=None, m_scale=None, v_scale=None, n=100,
                    lr_scale=1.0, weight_decay=0.0)
        base.update(kw)
        return (P._CAdamTensor * 1)(P._CAdamTensor(*base.values()))

    def call(t=None, n=1, p=P.ATTR_F32, g=P.ATTR_F32, s=P.ATTR_F32, step=1, lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, root=0.0,
             gs=None):
        return L.attr_adamw_step(tensor() if t is None else t, n, p, g, s, step, lr, b1, b2, eps, root, gs, None)
    nan, inf = float("nan"), float("inf")
    assert call(n=0) == 0 and L.attr_adamw_step(None, 0, 0, 0, 0, 1, 0.1, 0.9, 0.9, 0.0, 0.0, None, None) == 0
    assert call(tensor(n=0, p=None, g=None, m=None, v=None)) == 0
    for kw in (dict(n=-1), dict(step=0), dict(b1=1.0), dict(b2=-0.1), dict(b1=nan), dict(eps=-1.0), dict(eps=nan),
               dict(root=inf), dict(lr=nan), dict(lr=inf)):
        assert call(**kw) == INVALID, kw
    assert L.attr_adamw_step(None, 1, 0, 0, 0, 1, 0.1, 0.9, 0.9, 0.0, 0.0, None, None) == INVALID
    for kw in (dict(p=P.ATTR_E4M3), dict(g=P.ATTR_E4M3), dict(s=P.ATTR_BF16), dict(s=7), dict(p=9)):
        assert call(**kw) == UNSUPPORTED, kw
    for kw in (dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(n=-5), dict(n=2 ** 40), dict(lr_scale=nan),
               dict(weight_decay=inf), dict(m_scale=FAKE), dict(v_scale=FAKE)):
        assert call(tensor(**kw)) == INVALID, kw
    assert call(tensor(m_scale=FAKE), s=P.ATTR_E4M3) == INVALID and call(s=P.ATTR_E4M3) == INVALID
    for kw in (dict(p=0x100002), dict(g=0x200002), dict(m=0x300001), dict(v=0x400002), dict(master=0x500002)):
        assert call(tensor(**kw)) == ALIGN, kw
    assert call(tensor(m_scale=0x500002, v_scale=0x600000), s=P.ATTR_E4M3) == ALIGN
    assert call(gs=0x700002) == ALIGN


def test_binding_refusals():
    """The binding checks shapes, types and devices before it calls the library."""
    z, y = torch.zeros((8, 100)), torch.zeros(8, dtype=torch.int64)
    for kw, text in ((dict(n_examples=5, T=2), "hold 8 rows"), (dict(n_examples=4, T=0), "T >= 1"),
                     (dict(n_examples=4, T=2, weight=torch.zeros(7)), "weight"),
                     (dict(n_examples=4, T=2, length=torch.zeros(4)), "length"),
                     (dict(n_examples=4, T=2, row_offset=torch.zeros(3, dtype=torch.int64)), "row_offset"),
                     (dict(n_examples=4, T=2), "same GPU")):
        with pytest.raises(ValueError, match=text):
            P.TokenRows(z, y, **kw).c()
    with pytest.raises(ValueError, match="contiguous last"):
        P.TokenRows(z.t(), y, 4, 2).c()
    with pytest.raises(ValueError, match="target"):
        P.TokenRows(z, y.int(), 4, 2).c()
    with pytest.raises(ValueError, match="at least one"):
        P.AdamTensors([], [], [], [])
    x = torch.zeros(10)
    with pytest.raises(ValueError, match="same GPU"):
        P.AdamTensors([x], [x], [x], [x])
    assert ctypes.sizeof(P._CTokenRows) == 96 and ctypes.sizeof(P._CAdamTensor) == 72


def test_token_calls_refuse_host_tensors():
    """Before anything of the GPU is touched."""
    rows = P.TokenRows(torch.zeros((8, 100)), torch.zeros(8, dtype=torch.int64), 4, 2)
    x = torch.zeros(8)
    for call in (lambda: P.attr_token_logp(rows, x), lambda: P.attr_policy_loss(rows, x, x),
                 lambda: P.attr_preference_loss(rows, x)):
        with pytest.raises(ValueError, match="same GPU"):
            call()


def test_native_calls_are_optional(monkeypatch):
    """Without the native part the binding warns once and checks in Python."""
    import sys
    monkeypatch.setattr(P, "_native_call", None)
    monkeypatch.setitem(sys.modules, "paper_2606_11660_amd._marshal", None)  # the import fails
    with pytest.warns(RuntimeWarning, match="check their tensors in Python"):
        assert P._native_token_call()(1, 2, 3) is None


def test_native_call_refuses_what_it_does_not_know():
    """Anything but the exact kinds of arguments goes to the Python checks: None, and no error."""
    from paper_2606_11660_amd import _marshal
    rows = P.TokenRows(torch.zeros((8, 100)), torch.zeros(8, dtype=torch.int64), 4, 2)
    x = torch.zeros(8)
    for args in ((0, 1, rows, P.TokenRows, (x,), (), (), None, (), 0, 0, 0), (9, 1, rows, P.TokenRows, (x,), (), (), None, (), 0, 0, 0),
                 ("a", 1, rows, P.TokenRows, (x,), (), (), None, (), 0, 0, 0), (0, 0, rows, P.TokenRows, (x,), (), (), None, (), 0, 0, 0),
                 (0, 1, object(), P.TokenRows, (x,), (), (), None, (), 0, 0, 0), (1, 1, rows, P.TokenRows, [x], (), (), x, ("a",) * 3, 0, 0, 0)):
        assert _marshal.token_call(*args) is None
    with pytest.raises(TypeError, match="12 arguments"):
        _marshal.token_call(1)


@pytest.mark.parametrize("scale,status", [(2.5e38, INVALID), (2.0e38, 0)])
def test_logit_scale_stays_finite(scale, status):
    """The scale times log2 e is what multiplies a logit: past 2e38 it is infinite."""
    assert _calls(_rows(logit_scale=scale, n_examples=0)) == [status] * 3


def test_outputs_stay_apart():
    """Outputs over inputs or each other are refused: rows are taken by several workgroups."""
    L, z = P.lib(), 0x100000   # 8 rows of 100 fp32 logits: 3200 bytes
    apart = dict(target=0x110000, weight=0x120000, row_offset=0x130000, length=0x140000)
    rows = _rows(**apart)
    old, ref, adv, loss, logp, ratio, d = (0x200000 + 0x10000 * i for i in range(7))
    no_ws = (None, 0, None)

    def logp_call(out):
        return L.attr_token_logp(rows, out, *no_ws)

    def policy(per=0, old=old, ref=ref, adv=adv, loss=loss, logp=logp, d=d):
        return L.attr_policy_loss(rows, adv, per, old, ref, 0.2, 0.2, 0.1, loss, logp, d, 100, *no_ws)

    def pref(ref=ref, pw=adv, loss=loss, ratio=ratio, logp=logp, d=d):
        return L.attr_preference_loss(rows, ref, pw, 0.1, 0.0, 0.0, loss, ratio, logp, d, 100, *no_ws)
    assert policy() == policy(per=1) == pref() == WORKSPACE   # apart: only the workspace is missing
    assert policy(d=z) == pref(d=z) == WORKSPACE              # dlogits over the logits
    assert policy(logp=adv + 16) == WORKSPACE                 # after the last example's advantage
    ends = (z, z + 3196, 0x110000, 0x110000 + 60, 0x120000 + 28, 0x130000 + 28, 0x140000 + 12)
    for at in ends:
        assert logp_call(at) == policy(logp=at) == policy(loss=at) == pref(logp=at) == pref(loss=at) == INVALID, hex(at)
        assert pref(ratio=at) == INVALID and b"overlap" in L.attr_last_error()
    for at in ends[2:]:
        assert policy(d=at) == pref(d=at) == INVALID, hex(at)
    for kw in (dict(logp=old), dict(logp=ref + 28), dict(logp=adv), dict(per=1, logp=adv + 16), dict(loss=adv),
               dict(loss=logp), dict(logp=d + 3196), dict(d=old), dict(d=loss)):
        assert policy(**kw) == INVALID, kw
    for kw in (dict(logp=ref), dict(loss=adv), dict(loss=ratio + 12), dict(ratio=logp), dict(ratio=d), dict(d=ref)):
        assert pref(**kw) == INVALID, kw


def test_default_workspaces_are_a_threads_own():
    """Calls of several launches that two threads make on one stream may interleave: no scratch is shared."""
    import threading
    device, seen = torch.device("cuda", 0), {}
    together = threading.Barrier(2)

    def look(k):
        first = P._ws(None, device, 0)
        together.wait()
        seen[k] = (first, P._ws(None, device, 0), P._ws(None, device, 64))
        together.wait()
    threads = [threading.Thread(target=look, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    (a, b, c), (d, e, f) = seen[0], seen[1]
    assert a is b and d is e and len({id(x) for x in (a, c, d, f)}) == 4
    own = P.Workspace("cuda")
    assert P._ws(own, device, 0) is own


def test_oracle_pairs_of_weight_zero():
    """Loss and gradients of 0 in 64 bits too, beside infinities and NaN."""
    z = np.random.default_rng(4).standard_normal((4, 9))
    z[0, 2], z[3] = -np.inf, np.nan
    loss, _, _, grad = O.preference_loss(z, [2, 1, 3, 4], 4, 1, pair_weight=[0.0, 0.0])
    assert (loss == 0).all() and all((g == 0).all() for g in grad.values())


def test_adamw_refuses_what_fp32_does_not_divide_by():
    """An eps that the reciprocal of fp32 does not take would turn weights that no gradient touched into NaN."""
    L, none = P.lib(), (P._CAdamTensor * 1)(P._CAdamTensor(n=0))

    def call(eps, root):
        return L.attr_adamw_step(none, 1, 0, 0, 0, 1, 1e-3, 0.9, 0.95, eps, root, None, None)
    least = 2.0 ** -126
    for eps, root in ((1e-40, 0.0), (least * 0.999, 1e-6), (5e-324, 0.0), (0.0, 1e-46), (1e-8, 5e-324)):
        assert call(eps, root) == INVALID and b"at least 2^-126" in L.attr_last_error(), (eps, root)
    for eps, root in ((0.0, 0.0), (least, 0.0), (1e-30, 0.0), (0.0, 2.0 ** -149), (0.0, 1e-40)):
        assert call(eps, root) == 0, (eps, root)


def test_overlaps_of_an_adamw_plan():
    """A buffer that the step writes overlaps nothing, also where gradients that overlap each other lie between."""
    long, short = (0, 1000, "g", 0), (10, 100, "g", 1)
    for spans in ([long, short, (2000, 2100, "p", 0), (2100, 2200, "m", 0)], [(0, 10, "p", 0), (10, 20, "p", 1)],
                  [(5, 9, "g", 0), (5, 9, "g", 1), (9, 12, "v", 0)], []):
        P._refuse_overlaps(spans)
    for spans, text in (([long, short, (500, 600, "p", 1)], "tensor 0's g and tensor 1's p overlap"),
                        ([(500, 600, "p", 1), short, long], "tensor 0's g and tensor 1's p"),
                        ([(0, 50, "p", 0), (49, 60, "g", 3)], "tensor 0's p and tensor 3's g"),
                        ([(0, 50, "p", 0), (10, 20, "p", 1)], "tensor 0's p and tensor 1's p"),
                        ([(0, 50, "m", 0), (0, 50, "v", 0)], "tensor 0's m and tensor 0's v"),
                        ([long, (990, 1200, "g", 1), (1199, 1300, "master", 0)], "tensor 1's g and tensor 0's master")):
        with pytest.raises(ValueError, match=text):
            P._refuse_overlaps(spans)


def test_written_counts_versions():
    """Of every tensor, with and without the native part; tensors of inference mode count none."""
    from paper_2606_11660_amd import _marshal
    x, w = torch.zeros(3), torch.nn.Parameter(torch.zeros(2))
    with torch.inference_mode():
        y = torch.zeros(3)
    for seq in ([x, w, y], (x, y, w)):
        before = x._version, w._version
        assert _marshal.written(seq) is True
        assert (x._version, w._version) == (before[0] + 1, before[1] + 1)
    assert _marshal.written(x) is None and _marshal.written([3, None]) is True
    before = x._version
    P._written([x, y])
    assert x._version == before + 1
