"""The operators of a training step around the attributed modules, as timed cases: where the token rows
come from, what normalises them into the modules' inputs, and the optimizer step of the modules' matrices.

A case is a dict with an ``op``:

embed       attr_embed: rows of a table by token, scaled
embed_back  attr_embed_backward: the table's gradient, each token's rows summed in their order
norm        attr_layer_norm: layer norm of token rows, with the statistics that its backward pass takes
norm_back   attr_layer_norm_backward: the rows' gradient and the weight's and bias's, summed over all
            tokens or over each example's
muon        attr_muon_step: momentum, its orthogonalisation by Newton-Schulz products and the weights' step,
            over a model's matrices

``run`` computes the plain form from elementary torch operations in 32 bits, or, where ``own`` is
true, calls the library.  ``exact`` states the same definitions in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

F32, F16, BF16, F64 = torch.float32, torch.float16, torch.bfloat16, torch.float64
DT = {"f32": F32, "f16": F16, "bf16": BF16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}

EPS = 1e-5
COMMON = 10.0  # tokens below it are about equally likely, those above the less the higher
LR, MOMENTUM, DECAY, STEPS = 0.02, 0.95, 0.1, 5
A, B, C = 3.4445, -4.7750, 2.0315  # the Newton-Schulz polynomial a x + b x^3 + c x^5
GRAD_SCALE = 0.37  # what clipping the gradient's norm leaves


# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------
def listed():
    return [
        # one decoded token of each of four sequences: nothing but latency
        {"name": "embed_step", "op": "embed", "n": 4, "T": 1, "V": 50257, "d": 2048, "table": "bf16", "out": "bf16",
         "packed": False, "scaled": False},
        # a packed batch's rows from a 32-bit table, scaled by the root of the width
        {"name": "embed_batch", "op": "embed", "n": 16, "T": 2048, "V": 65536, "d": 2048, "table": "f32", "out": "bf16",
         "packed": True, "scaled": True},
        # a toy model's gradient
        {"name": "embed_back_small", "op": "embed_back", "n": 8, "T": 32, "V": 1000, "d": 64, "table": "f32", "out": "f32",
         "packed": False, "scaled": False, "accumulate": False},
        # padded slots of an odd vocabulary and width, a 16-bit gradient
        {"name": "embed_back_slots", "op": "embed_back", "n": 16, "T": 512, "V": 50257, "d": 769, "table": "f16", "out": "f16",
         "packed": False, "scaled": True, "accumulate": False},
        # a packed batch's gradient added to the 32-bit gradients of the batches before it
        {"name": "embed_back_batch", "op": "embed_back", "n": 16, "T": 2048, "V": 65536, "d": 2048, "table": "f32",
         "out": "bf16", "packed": True, "scaled": True, "accumulate": True},
        # a decoding step of 64 sequences
        {"name": "norm_step", "op": "norm", "n": 64, "T": 1, "d": 2048, "x": "bf16", "y": "bf16", "w": "bf16",
         "packed": False},
        # a packed batch: a 32-bit residual stream to 16-bit rows for the modules
        {"name": "norm_batch", "op": "norm", "n": 16, "T": 2048, "d": 2048, "x": "f32", "y": "bf16", "w": "f32",
         "packed": True},
        # padded slots of an odd width, every example's gradient of the weights on its own
        {"name": "norm_back_examples", "op": "norm_back", "n": 64, "T": 512, "d": 769, "x": "f32", "y": "f32", "w": "f32",
         "packed": False, "examples": True},
        # a packed batch of wide 16-bit rows
        {"name": "norm_back_batch", "op": "norm_back", "n": 16, "T": 1024, "d": 8192, "x": "bf16", "y": "bf16", "w": "bf16",
         "packed": True, "examples": False},
        # adapters of rank 16 on every module of a small model: many thin matrices
        {"name": "muon_adapters", "op": "muon", "layers": 12, "width": 768, "mlp": 2304, "rank": 16, "p": "f32", "g": "f32",
         "master": False},
        # a layer of a small model of odd sizes: bf16 weights with 32-bit masters
        {"name": "muon_masters", "op": "muon", "layers": 2, "width": 769, "mlp": 2310, "rank": 0, "p": "bf16", "g": "bf16",
         "master": True},
        # two layers with the widths of the 1B-shaped decoder, 16-bit weights
        {"name": "muon_large", "op": "muon", "layers": 2, "width": 2048, "mlp": 8192, "rank": 0, "p": "bf16", "g": "bf16",
         "master": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_back", "embed_back", "norm", "norm_back", "norm_back", "muon", "muon", "muon"])
    if op == "muon":
        rank = rng.choice([0, 0, 0, rng.randint(1, 64)])
        p = rng.choice(["f32", "bf16", "bf16", "f16"])
        master = p != "f32" and rng.random() < 0.5
        few = p != "f32" and not master  # weights of 16 bits
        width = _log(rng, 33, 2048 if few else 1400)
        mlp = width * rng.randint(1, 4) + rng.randint(0, 7)
        case = {"op": op, "layers": 1, "width": width, "mlp": mlp, "rank": rank, "p": p, "g": rng.choice(["f32", p]),
                "master": master}
        most = work(listed()[-1])["flops"] / (1 if few else 3)
        case["layers"] = _log(rng, 1, max(1, min(12, int(most / work(case)["flops"]))))
        return case
    d = _log(rng, 17, 8192)
    rows = _log(rng, 1, min(32768, int(6.7e7 / d)))
    n = _log(rng, 1, min(rows, 64))
    kinds = ["bf16", "bf16", "f16", "f32"]
    case = {"op": op, "n": n, "T": max(1, rows // n), "d": d, "packed": rng.random() < 0.5}
    if op in ("embed", "embed_back"):
        case.update(V=_log(rng, 100, max(101, min(262144, int(1.3e8 / d)))), table=rng.choice(kinds), out=rng.choice(kinds),
                    scaled=rng.random() < 0.5)
        if op == "embed_back":
            case["accumulate"] = case["table"] == "f32" and rng.random() < 0.4
        return case
    x = rng.choice(kinds)
    case.update(x=x, y=rng.choice([x, rng.choice(kinds)]), w=rng.choice(["f32", x]))
    if op == "norm_back":
        case["examples"] = rng.random() < 0.4
    return case


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _lengths(case):
    """Token counts of the examples, the same for every seed: one in full, the others spread down to a quarter."""
    n, T = case["n"], case["T"]
    return [max(1, T - (3 * T * ((7 * i) % n)) // (4 * n)) for i in range(n)]


def _randn(gen, *shape, dtype=F32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _where(case):
    """The batch's rows: how many, and where each example's are."""
    n, T, lens = case["n"], case["T"], _lengths(case)
    starts = [sum(lens[:i]) for i in range(n)]
    return {"case": case, "rows": sum(lens) if case["packed"] else n * T,
            "offset": torch.tensor(starts, dtype=torch.int64, device="cuda") if case["packed"] else None,
            "length": torch.tensor(lens, dtype=torch.int32, device="cuda")}


def _embedding(case, gen):
    st = _where(case)
    rows, V, d = st["rows"], case["V"], case["d"]
    u = torch.rand(rows, generator=gen, device="cuda", dtype=F64)
    st["token"] = (COMMON * (((V + COMMON) / COMMON) ** u - 1)).long().clamp_(0, V - 1)
    st["scale"] = math.sqrt(d) if case["scaled"] else 1.0
    if case["op"] == "embed":
        st["table"] = _randn(gen, V, d).mul_(1.0 / math.sqrt(d)).to(DT[case["table"]])
        st["out"] = torch.empty(rows, d, dtype=DT[case["out"]], device="cuda")
    else:
        st["dout"] = _randn(gen, rows, d).mul_(1e-2).to(DT[case["out"]])
        st["dtable"] = torch.empty(V, d, dtype=DT[case["table"]], device="cuda")
        if case["accumulate"]:
            st["dtable"].copy_(_randn(gen, V, d).mul_(1e-2))
    return st


def _norm(case, gen):
    st = _where(case)
    rows, d = st["rows"], case["d"]
    loud = torch.exp(0.5 * _randn(gen, rows, 1))
    x = (_randn(gen, rows, d) + 0.3 * _randn(gen, d)) * loud + 0.2 * _randn(gen, rows, 1)
    st["x"] = x.to(DT[case["x"]])
    st["weight"] = (1 + 0.1 * _randn(gen, d)).to(DT[case["w"]])
    st["bias"] = (0.1 * _randn(gen, d)).to(DT[case["w"]])
    if case["op"] == "norm":
        st["y"] = torch.empty(rows, d, dtype=DT[case["y"]], device="cuda")
        st["mean"], st["rstd"] = (torch.empty(rows, device="cuda") for _ in range(2))
        return st
    # what the forward pass has left
    st["mean"], st["rstd"] = (torch.empty(rows, device="cuda") for _ in range(2))
    for r in range(0, rows, 4096):
        x = st["x"][r:r + 4096].double()
        st["mean"][r:r + 4096] = x.mean(1)
        st["rstd"][r:r + 4096] = torch.rsqrt(x.var(1, correction=0) + EPS)
    st["dy"] = (1e-2 * _randn(gen, rows, d) * torch.exp(0.5 * _randn(gen, rows, 1))).to(DT[case["y"]])
    st["dx"] = torch.empty_like(st["x"])
    shape = (case["n"], d) if case["examples"] else (d,)
    st["dweight"], st["dbias"] = (torch.empty(shape, device="cuda") for _ in range(2))
    return st


def _shapes(case):
    """{(rows, columns): how many} of a model's matrices: a layer's seven modules, or their adapters."""
    w, m, r, n, got = case["width"], case["mlp"], case["rank"], case["layers"], {}
    for d_out, d_in in ((w, w),) * 4 + ((m, w),) * 2 + ((w, m),):
        for shape in ((r, d_in), (d_out, r)) if r else ((d_out, d_in),):
            got[shape] = got.get(shape, 0) + n
    return got


def _matrices(case, gen):
    """A model's weights, gradients and momenta, those of one shape in one buffer: gradients of a few large
    directions beside many small ones, and momenta of the same."""
    st = {"case": case, "p": [], "g": [], "m": [], "master": [], "grad_scale": torch.full((1,), GRAD_SCALE, device="cuda")}
    for (rows, cols), n in _shapes(case).items():
        k = max(1, min(rows, cols) // 16)
        left, right = _randn(gen, n, rows, k), _randn(gen, n, k, cols)
        m = torch.bmm(left, right).mul_(4e-3 / math.sqrt(k)) + _randn(gen, n, rows, cols).mul_(2e-3)
        g = (m + _randn(gen, n, rows, cols).mul_(3e-3)) / GRAD_SCALE
        p = _randn(gen, n, rows, cols).mul_(0.02)
        st["p"].append(p.to(DT[case["p"]]))
        st["g"].append(g.to(DT[case["g"]]))
        st["m"].append(m)
        if case["master"]:
            st["master"].append(p)
    if own:  # the plan that a training program keeps: the matrices' places
        import paper_2606_11660_amd as P
        each = {k: [x for group in st[k] for x in group] for k in ("p", "g", "m", "master")}
        st["plan"] = P.MuonTensors(each["p"], each["g"], each["m"], master=each["master"] or None, weight_decay=DECAY,
                                   lr_scale=[_lr_scale(x) for x in each["p"]])
    return st


def _lr_scale(p):
    return math.sqrt(max(1.0, p.shape[-2] / p.shape[-1]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    make = {"embed": _embedding, "embed_back": _embedding, "norm": _norm, "norm_back": _norm, "muon": _matrices}
    return make[case["op"]](case, gen)


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    import paper_2606_11660_amd as P
    case = st["case"]
    if case["op"] == "muon":
        P.attr_muon_step(st["plan"], LR, momentum=MOMENTUM, nesterov=True, steps=STEPS, grad_scale=st["grad_scale"])
        return _muon_outputs(st)
    where = P.ExampleRows(case["n"], case["T"], row_offset=st["offset"], length=st["length"])
    if case["op"] == "embed":
        return {"out": P.attr_embed(st["table"], st["token"], st["out"], scale=st["scale"], rows=where)}
    if case["op"] == "embed_back":
        return {"dtable": P.attr_embed_backward(st["dout"], st["token"], st["dtable"], scale=st["scale"],
                                                accumulate=case["accumulate"], rows=where)}
    if case["op"] == "norm":
        P.attr_layer_norm(st["x"], st["y"], weight=st["weight"], bias=st["bias"], eps=EPS, mean=st["mean"], rstd=st["rstd"],
                          rows=where)
        return {k: st[k] for k in ("y", "mean", "rstd")}
    P.attr_layer_norm_backward(st["dy"], st["x"], st["mean"], st["rstd"], weight=st["weight"], dx=st["dx"],
                               dweight=st["dweight"], dbias=st["dbias"], per_example=case["examples"], rows=where)
    return {k: st[k] for k in ("dx", "dweight", "dbias")}


def _muon_outputs(st):
    return {k: st[k] for k in ("p", "m", "master") if st[k]}


def _example_of_rows(st):
    """Each row's example, and whether the row is one of its tokens."""
    case, n, T = st["case"], st["case"]["n"], st["case"]["T"]
    examples = torch.arange(n, device="cuda")
    if case["packed"]:
        return (examples.repeat_interleave(st["length"].long(), output_size=st["rows"]),
                torch.ones(st["rows"], dtype=torch.bool, device="cuda"))
    inside = (torch.arange(T, device="cuda") < st["length"][:, None]).view(-1)
    return examples.repeat_interleave(T, output_size=n * T), inside


def _run_plain(st):
    case = st["case"]
    if case["op"] == "muon":
        return _plain_muon(st)
    example, inside = _example_of_rows(st)
    inside = inside[:, None]
    zero = torch.zeros((), device="cuda")
    if case["op"] == "embed":
        x = st["table"][st["token"]].float() * st["scale"]
        st["out"].copy_(torch.where(inside, x, zero))
        return {"out": st["out"]}
    if case["op"] == "embed_back":
        x = torch.where(inside, st["dout"].float() * st["scale"], zero)
        got = st["dtable"].float() if case["accumulate"] else torch.zeros(st["dtable"].shape, device="cuda")
        st["dtable"].copy_(got.index_add(0, st["token"], x))
        return {"dtable": st["dtable"]}
    x, w = st["x"].float(), st["weight"].float()
    if case["op"] == "norm":
        mean = x.mean(1, keepdim=True)
        rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        y = (x - mean) * rstd * w + st["bias"].float()
        st["y"].copy_(torch.where(inside, y, zero))
        st["mean"].copy_(torch.where(inside, mean, zero)[:, 0])
        st["rstd"].copy_(torch.where(inside, rstd, zero)[:, 0])
        return {k: st[k] for k in ("y", "mean", "rstd")}
    dy = torch.where(inside, st["dy"].float(), zero)
    rstd = st["rstd"][:, None]
    unit = torch.where(inside, (x - st["mean"][:, None]) * rstd, zero)
    e = dy * w
    dx = (e - e.mean(1, keepdim=True) - unit * (e * unit).mean(1, keepdim=True)) * rstd
    st["dx"].copy_(torch.where(inside, dx, zero))
    for name, each in (("dweight", dy * unit), ("dbias", dy)):
        if case["examples"]:
            st[name].copy_(torch.zeros(st[name].shape, device="cuda").index_add(0, example, each))
        else:
            st[name].copy_(each.sum(0))
    return {k: st[k] for k in ("dx", "dweight", "dbias")}


def _plain_muon(st):
    masters = st["master"] or st["p"]
    for p, w, g, m in zip(st["p"], masters, st["g"], st["m"]):
        g = g.float() * st["grad_scale"]
        m.copy_(m * MOMENTUM + g * (1 - MOMENTUM))
        u = m * MOMENTUM + g * (1 - MOMENTUM)
        wide = p.shape[1] <= p.shape[2]
        x = (u if wide else u.mT).contiguous()
        x = x / x.square().sum((1, 2), keepdim=True).sqrt()
        for _ in range(STEPS):
            gram = torch.bmm(x, x.mT)
            x = A * x + torch.bmm(B * gram + C * torch.bmm(gram, gram), x)
        o = x if wide else x.mT
        w.copy_(w.float() * (1 - LR * _lr_scale(p) * DECAY) - o * (LR * _lr_scale(p)))
        if st["master"]:
            p.copy_(w)
    return _muon_outputs(st)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def _distinct(case, rows):
    """How many tokens of the vocabulary a batch of so many rows is expected to hold."""
    V = case["V"]
    edges = np.log((np.arange(V + 1) + COMMON) / COMMON) / math.log((V + COMMON) / COMMON)
    return float(np.sum(1 - (1 - np.diff(edges)) ** rows))


def work(case):
    if case["op"] == "muon":
        flops, n = 0.0, 0
        for (rows, cols), count in _shapes(case).items():
            s, t = min(rows, cols), max(rows, cols)
            flops += count * STEPS * (s * s * t + s ** 3 + 2.0 * s * s * t)  # two of three products are symmetric
            n += count * rows * cols
        return {"bytes": n * (2 * BYTES[case["p"]] + BYTES[case["g"]] + 8 + (8 - BYTES[case["p"]]) * case["master"]), "flops": flops}
    d, lens = case["d"], _lengths(case)
    tokens = sum(lens)
    rows = tokens if case["packed"] else case["n"] * case["T"]
    if case["op"] == "embed":
        return {"bytes": 8 * tokens + d * (_distinct(case, tokens) * BYTES[case["table"]] + rows * BYTES[case["out"]]),
                "flops": tokens * d}
    if case["op"] == "embed_back":
        table = 2 * _distinct(case, tokens) if case["accumulate"] else case["V"]
        return {"bytes": 8 * tokens + d * (tokens * BYTES[case["out"]] + table * BYTES[case["table"]]), "flops": 2 * tokens * d}
    x, y = BYTES[case["x"]], BYTES[case["y"]]
    if case["op"] == "norm":
        return {"bytes": d * (tokens * x + rows * y + 2 * BYTES[case["w"]]) + 8 * rows, "flops": 8 * tokens * d}
    return {"bytes": d * (tokens * (x + y) + rows * x + BYTES[case["w"]] + 8 * (case["n"] if case["examples"] else 1))
            + 8 * tokens, "flops": 14 * tokens * d}


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "muon":
        return _exact_muon(st)
    lens, n, T = _lengths(case), case["n"], case["T"]
    starts = [sum(lens[:i]) if case["packed"] else i * T for i in range(n)]
    spans = [slice(a, a + k) for a, k in zip(starts, lens)]
    return {"embed": _exact_embed, "embed_back": _exact_embed_back, "norm": _exact_norm, "norm_back": _exact_norm_back}[
        case["op"]](st, spans)


def _exact_embed(st, spans):
    out = torch.zeros(st["out"].shape, dtype=F64, device="cuda")
    for at in spans:
        out[at] = st["scale"] * torch.nn.functional.embedding(st["token"][at], st["table"]).double()
    return {"out": out}


def _exact_embed_back(st, spans):
    """Token by token in groups: the rows of one token are neighbours in the sorted order, and its sum is
    the difference of the running sum at its ends."""
    case = st["case"]
    at = torch.cat([torch.arange(s.start, s.stop, device="cuda") for s in spans])
    token, order = torch.sort(st["token"][at], stable=True)
    got = st["dtable"].double() if case["accumulate"] else torch.zeros(st["dtable"].shape, dtype=F64, device="cuda")
    ids, count = torch.unique_consecutive(token, return_counts=True)
    end = count.cumsum(0)
    for c in range(0, case["d"], 512):
        x = st["dout"][at[order], c:c + 512].double()
        run = torch.cat([torch.zeros_like(x[:1]), x.cumsum(0)])
        got[ids, c:c + 512] += st["scale"] * (run[end] - run[end - count])
    return {"dtable": got}


def _exact_norm(st, spans):
    d = st["case"]["d"]
    y = torch.zeros(st["y"].shape, dtype=F64, device="cuda")
    mean, rstd = (torch.zeros(st["rows"], dtype=F64, device="cuda") for _ in range(2))
    for at in spans:
        x = st["x"][at].double()
        y[at] = torch.nn.functional.layer_norm(x, (d,), st["weight"].double(), st["bias"].double(), EPS)
        mean[at], rstd[at] = x.mean(1), 1 / (x.var(1, correction=0) + EPS).sqrt()
    return {"y": y, "mean": mean, "rstd": rstd}


def _exact_norm_back(st, spans):
    """autograd's gradients of the 64-bit layer norm, example by example."""
    case, d = st["case"], st["case"]["d"]
    w = st["weight"].double().requires_grad_()
    b = torch.zeros(d, dtype=F64, device="cuda", requires_grad=True)
    dx = torch.zeros(st["dx"].shape, dtype=F64, device="cuda")
    dw, db = [], []
    for at in spans:
        x = st["x"][at].double().requires_grad_()
        y = torch.nn.functional.layer_norm(x, (d,), w, b, EPS)
        dx[at], dwi, dbi = torch.autograd.grad(y, (x, w, b), st["dy"][at].double())
        dw.append(dwi)
        db.append(dbi)
    dw, db = torch.stack(dw), torch.stack(db)
    return {"dx": dx, "dweight": dw if case["examples"] else dw.sum(0), "dbias": db if case["examples"] else db.sum(0)}


def _exact_muon(st):
    """Matrix by matrix, the polynomial by powers: x^3 = (x x') x, x^5 = (x x') x^3."""
    got = {k: [] for k in ("p", "m", "master") if st[k]}
    for p, w, g, m in zip(st["p"], st["master"] or st["p"], st["g"], st["m"]):
        new_m = MOMENTUM * m.double() + (1 - MOMENTUM) * (g.double() * float(st["grad_scale"]))
        new_p = torch.empty(p.shape, dtype=F64, device="cuda")
        for i in range(p.shape[0]):
            x = MOMENTUM * new_m[i] + (1 - MOMENTUM) * g[i].double() * float(st["grad_scale"])
            x = x if x.shape[0] <= x.shape[1] else x.t().contiguous()
            x = x / torch.linalg.vector_norm(x)
            for _ in range(STEPS):
                gram = x @ x.t().contiguous()
                cube = gram @ x
                x = A * x + B * cube + C * (gram @ cube)
            rate = LR * _lr_scale(p)
            o = x if p.shape[1] <= p.shape[2] else x.t()
            new_p[i] = w[i].double() - rate * DECAY * w[i].double() - rate * o
        got["p"].append(new_p)
        got["m"].append(new_m)
        if st["master"]:
            got["master"].append(new_p)
    return got
