"""The operators of a training step together: the example runs, and its gradients are autograd's."""
import importlib.util
import os

import pytest
import torch

import paper_2606_11660_amd as P
from tests._util import say

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("training_step", os.path.join(ROOT, "examples", "training_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(ex, m, b):
    """The batch's loss and gradients in 64 bits on the CPU, and the norm's for each example."""
    w = {k: getattr(m, k).double().cpu().requires_grad_() for k in m.names}
    token, target = b.token.cpu(), b.target.cpu()
    x = torch.nn.functional.embedding(token, w["table"]) * ex.D ** 0.5
    y = torch.nn.functional.layer_norm(x, (ex.D,), w["weight"], w["bias"], 1e-5)
    each = torch.nn.functional.cross_entropy(y @ w["head"].t(), target, reduction="none") / len(token)
    grads = dict(zip(m.names, torch.autograd.grad(each.sum(), [w[k] for k in m.names], retain_graph=True)))
    per = []
    for i in range(ex.N):
        at = slice(int(b.offset[i]), int(b.offset[i] + b.length[i]))
        per.append(torch.cat(torch.autograd.grad(each[at].sum(), [w["weight"], w["bias"]], retain_graph=True)))
    return float(each.detach().sum()), grads, torch.stack(per)


def test_gradients(ex):
    """fp32 sums of up to 320 terms (logits, rows) through five stages one after another: 5 * 320 * 2^-24 =
    1e-4 of the terms' magnitudes, whose norm is some ten times their sums' at most (random signs)."""
    m, b = ex.Model(3, "cuda"), ex.Batch(3, "cuda")
    say("case: training step, gradients")
    got = ex.forward_backward(m, b)
    loss, grads, per = reference(ex, m, b)
    assert abs(float(got["loss"]) - loss) < 1e-5 * abs(loss)
    for k in m.names:
        off = float((m.grad[k].double().cpu() - grads[k]).norm() / grads[k].norm())
        say(k, off)
        assert off < 1e-3, k
    store = got["store"][:, ex.K * ex.K:].double().cpu()
    assert float((store - per).norm() / per.norm()) < 1e-3
    assert float((store.sum(0) - torch.cat([grads["weight"], grads["bias"]])).norm()) < 1e-3 * float(per.norm())


def test_gradient_against_differences(ex):
    """The loss's own difference along a direction, in the library's fp32: a step of 1e-2 of the norm of each
    weight moves it by the gradients' products with the direction."""
    m, b = ex.Model(5, "cuda"), ex.Batch(5, "cuda")
    ex.forward_backward(m, b)
    gen = torch.Generator(device="cuda").manual_seed(1)
    way = {k: torch.randn(m.grad[k].shape, generator=gen, device="cuda") * getattr(m, k).std() for k in m.names}
    want = sum(float((m.grad[k].double() * way[k]).sum()) for k in m.names)
    keep = {k: getattr(m, k).clone() for k in m.names}

    def f(t):
        for k in m.names:
            getattr(m, k).copy_(keep[k] + t * way[k])
        return float(ex.forward_backward(m, b)["loss"])
    h = 1e-2
    got = (8 * (f(h) - f(-h)) - (f(2 * h) - f(-2 * h))) / (12 * h)
    # the loss (about 6) in fp32 over h: 6 * 2^-22 / 1e-2 = 1.4e-4; fourth-order differences: h^4 times a fifth derivative
    assert abs(got - want) < 2e-3 * max(1.0, abs(want)), (got, want)


def test_example_runs(ex):
    out = ex.main(steps=4)
    assert all(torch.isfinite(out[k]).all() for k in ("head", "table", "score"))
    assert (out["index"][:, 0] == torch.arange(ex.N)).all() and (out["score"][:, 0] - 1).abs().max() < 1e-4
    again = ex.main(steps=4)
    assert torch.equal(out["head"], again["head"]) and torch.equal(out["table"], again["table"]) and out["loss"] == again["loss"]


def test_a_captured_step(ex):
    """A whole step as a graph, replayed with eager steps of a twin between: the same bits."""
    m, w, b = ex.Model(7, "cuda"), ex.Model(7, "cuda"), ex.Batch(7, "cuda")

    def step(t, k):
        ex.forward_backward(t, b)
        P.attr_muon_step(t.muon, lr=0.02)
        P.attr_adamw_step(t.adam, k, lr=0.01)
    P = ex.P
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(m, 1)
    side.synchronize()
    step(w, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(m, 2)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        step(w, 2)
        torch.cuda.synchronize()
        for name in m.names:
            assert torch.equal(getattr(m, name), getattr(w, name)), (k, name)


def test_captured_calls_of_every_plan():
    """The embedding's gradient without a sort, sorted by one workgroup and by several, the norm's with
    shares, Muon on thin, long and square matrices: one graph, replayed over new values beside eager work."""
    n_slots, V, d = (300, 3000, 9000), 5000, 72
    dout = [torch.empty(n, d, device="cuda") for n in n_slots]
    token = [torch.empty(n, dtype=torch.int64, device="cuda") for n in n_slots]
    table = [torch.empty(V, d, device="cuda") for _ in n_slots]
    x = torch.empty(3000, d, device="cuda")
    mean, rstd, dw = (torch.empty(n, device="cuda") for n in (3000, 3000, d))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    shapes = [(9000, 16), (2500, 70), (200, 200)]
    w, g, m = ([torch.zeros(s, device="cuda") for s in shapes] for _ in range(3))
    plan = P.MuonTensors(w, g, m)
    ws = P.Workspace()

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for t in dout + [x] + w + g + m:
            t.normal_(generator=gen)
        for t in token:
            t.random_(0, V, generator=gen)
            t[::3] = seed

    def calls():
        for a, b, c in zip(dout, token, table):
            P.attr_embed_backward(a, b, c, ws=ws)
        P.attr_layer_norm(x, y, mean=mean, rstd=rstd)
        P.attr_layer_norm_backward(y, x, mean, rstd, dx=dx, dweight=dw, ws=ws)
        P.attr_muon_step(plan, 0.02, ws=ws)

    outs = table + [y, mean, rstd, dx, dw] + w + m
    side = torch.cuda.Stream()
    fill(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for k in range(1, 4):
        fill(k)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        fill(k)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            calls()
        side.synchronize()
        for j, (a, b) in enumerate(zip(got, outs)):
            assert torch.equal(a, b) and torch.isfinite(a).all(), (k, j)
