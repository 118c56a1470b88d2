"""The post-training operators as timed cases: the losses whose gradients are attributed, and the
optimizer step whose second moments normalise them.

A case is a dict with an ``op``:

logp    attr_token_logp: log-probabilities of given tokens from the model's logits, what a rollout
        records while it decodes, and what a reference model gives for whole sequences
policy  attr_policy_loss: the clipped policy loss with a KL term, per example, and its gradient with
        respect to the logits
pref    attr_preference_loss: the paired log-ratio loss of chosen and rejected sequences, and its
        gradient with respect to the logits
adamw   attr_adamw_step: one AdamW step over a model's tensors, states in 32 or in 8 bits

``run`` computes the plain form from elementary torch operations in 32 bits, or, where ``own`` is
true, calls the library.  ``exact`` states the same definitions in 64 bits.
"""
import math
import random

import torch

own = False

F32, F16, BF16, F8 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
DT = {"f32": F32, "f16": F16, "bf16": BF16, "f8": F8}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "f8": 1}

CLIP_LOW, CLIP_HIGH, BETA_KL = 0.2, 0.28, 0.04
BETA_PREF, SMOOTHING = 0.1, 0.05
LR, BETA1, BETA2, EPS, EPS_ROOT, DECAY = 3e-4, 0.9, 0.95, 1e-8, 1e-6, 0.1
GRAD_SCALE = 0.37      # what clipping the gradient's norm leaves
F8_MAX, F8_LEAST, BLOCK, AMAX_LEAST = 448.0, 2.0 ** -9, 256, 2.0 ** -100


# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------
def listed():
    return [
        # one decoded token of one sequence: nothing but latency
        {"name": "logp_token", "op": "logp", "n": 1, "T": 1, "V": 50257, "dtype": "bf16",
         "packed": False, "prompt": 0.0, "masked": 0, "scale": 1.0},
        # a decoding step of 256 sequences with 32-bit logits and a large vocabulary, at a temperature
        {"name": "logp_step", "op": "logp", "n": 256, "T": 1, "V": 262144, "dtype": "f32",
         "packed": False, "prompt": 0.0, "masked": 0, "scale": 1.25},
        # the reference model's log-probabilities of a batch; the vocabulary's padding is masked
        {"name": "logp_batch", "op": "logp", "n": 16, "T": 512, "V": 65536, "dtype": "bf16",
         "packed": True, "prompt": 0.25, "masked": 43, "scale": 1.0},
        # a toy model's rollouts
        {"name": "policy_small", "op": "policy", "n": 8, "T": 32, "V": 1000, "dtype": "f32",
         "packed": False, "prompt": 0.0, "masked": 0, "scale": 1.0, "kl": True, "per_token": False},
        # a batch of rollouts in padded slots, prompts masked, an odd vocabulary
        {"name": "policy_rollouts", "op": "policy", "n": 16, "T": 512, "V": 50257, "dtype": "bf16",
         "packed": False, "prompt": 0.25, "masked": 0, "scale": 1.0, "kl": True, "per_token": False},
        # the largest batch: long packed rollouts of a model with a large vocabulary
        {"name": "policy_large", "op": "policy", "n": 8, "T": 2048, "V": 131072, "dtype": "bf16",
         "packed": True, "prompt": 0.125, "masked": 0, "scale": 1.0, "kl": True, "per_token": False},
        # 32-bit logits, advantages for each token, no reference model, sampled at a temperature
        {"name": "policy_f32", "op": "policy", "n": 7, "T": 333, "V": 32003, "dtype": "f32",
         "packed": True, "prompt": 0.0, "masked": 3, "scale": 1.25, "kl": False, "per_token": True},
        # two short pairs
        {"name": "pref_small", "op": "pref", "n": 4, "T": 48, "V": 8192, "dtype": "f32",
         "packed": False, "prompt": 0.25, "masked": 0, "scale": 1.0},
        # a batch of pairs, fp16 logits with a loss scale
        {"name": "pref_batch", "op": "pref", "n": 16, "T": 512, "V": 50257, "dtype": "f16",
         "packed": True, "prompt": 0.25, "masked": 0, "scale": 1.0},
        # adapters of rank 16 on every module of a small model: many small tensors
        {"name": "adamw_adapters", "op": "adamw", "layers": 12, "width": 768, "mlp": 2304, "rank": 16,
         "p": "f32", "g": "f32", "master": False, "state": "f32", "pad": 1, "step": 7},
        # four layers with the widths of the 1B-shaped decoder: bf16 weights, 32-bit masters and states
        {"name": "adamw_masters", "op": "adamw", "layers": 4, "width": 2048, "mlp": 8192, "rank": 0,
         "p": "bf16", "g": "bf16", "master": True, "state": "f32", "pad": 256, "step": 1000},
        # two of them with states in 8 bits
        {"name": "adamw_8bit", "op": "adamw", "layers": 2, "width": 2048, "mlp": 8192, "rank": 0,
         "p": "f32", "g": "bf16", "master": False, "state": "f8", "pad": 256, "step": 100},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logp", "policy", "policy", "pref", "adamw", "adamw"])
    if op == "adamw":
        rank = rng.choice([0, 0, rng.randint(2, 64)])
        state = rng.choice(["f32", "f8"])
        p = rng.choice(["f32", "bf16"])
        width = _log(rng, 33, 2048)
        mlp = width * rng.randint(2, 4) + rng.randint(0, 7)
        per_layer = 7 * rank * (width + mlp) if rank else 4 * width * width + 3 * width * mlp
        return {"op": op, "layers": _log(rng, 1, max(1, min(12, int(2.6e8 / per_layer)))), "width": width,
                "mlp": mlp, "rank": rank, "p": p, "g": rng.choice(["f32", "bf16", "f16"]),
                "master": p == "bf16", "state": state, "pad": 256 if state == "f8" else rng.choice([1, 256]),
                "step": _log(rng, 1, 10000)}
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    V = _log(rng, 200, 262144 if op == "logp" else 131072)
    rows = _log(rng, 1, min(16384, int(1.9e9 / V / (BYTES[dtype] // 2))))
    n = _log(rng, 1, min(rows, 64))
    if op == "pref":
        n += n % 2
    case = {"op": op, "n": n, "T": max(1, rows // n), "V": V, "dtype": dtype, "packed": rng.random() < 0.5,
            "prompt": rng.choice([0.0, 0.25]), "masked": rng.choice([0, 0, min(V // 8, 43)]),
            "scale": rng.choice([1.0, 1.0, 1.25])}
    if op == "policy":
        case["kl"] = rng.random() < 0.6
        case["per_token"] = rng.random() < 0.3
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


def _tokens(case, gen):
    """A model's logits over a batch's token rows, the tokens whose log-probabilities count, and what
    the rollout and the reference model said of them."""
    n, T, V, lens = case["n"], case["T"], case["V"], _lengths(case)
    rows = sum(lens) if case["packed"] else n * T
    starts = [sum(lens[:i]) for i in range(n)] if case["packed"] else [i * T for i in range(n)]
    logits = _randn(gen, rows, V, dtype=DT[case["dtype"]]).mul_(2.5)
    if case["masked"]:
        logits[:, V - case["masked"]:] = -math.inf
    target = torch.randint(0, V - case["masked"], (rows,), generator=gen, device="cuda")
    at = torch.arange(rows, device="cuda")
    logits[at, target] += _randn(gen, rows).mul_(3.0).add_(math.log(V)).to(logits.dtype)  # mostly likely tokens
    weight = torch.zeros(rows)
    for i in range(n):
        first = int(lens[i] * case["prompt"])
        weight[starts[i] + first:starts[i] + lens[i]] = 1.0 / (lens[i] - first) if case["op"] == "policy" else 1.0
    if case["dtype"] == "f16":
        weight *= 64.0 if case["op"] == "policy" else 1.0  # a loss scale
    st = {"case": case, "rows": rows, "logits": logits, "target": target, "weight": weight.cuda(),
          "offset": torch.tensor(starts, dtype=torch.int64, device="cuda") if case["packed"] else None,
          "length": torch.tensor(lens, dtype=torch.int32, device="cuda"),
          "logp": torch.empty(rows, dtype=F32, device="cuda")}
    if case["op"] == "logp":
        return st
    said = torch.empty(rows, dtype=F32, device="cuda")
    for r in range(0, rows, 1024):
        z = logits[r:r + 1024].float() * case["scale"]
        said[r:r + 1024] = z.gather(1, target[r:r + 1024, None])[:, 0] - z.logsumexp(1)
    st["old"] = said + 0.15 * _randn(gen, rows)
    st["ref"] = said + 0.3 * _randn(gen, rows)
    st["advantage"] = _randn(gen, rows if case.get("per_token") else n)
    st["pair_weight"] = torch.full((n // 2,), (64.0 if case["dtype"] == "f16" else 1.0) / max(1, n // 2), device="cuda")
    st["loss"] = torch.empty(n if case["op"] == "policy" else n // 2, dtype=F32, device="cuda")
    st["log_ratio"] = torch.empty(n, dtype=F32, device="cuda")
    st["dlogits"] = torch.empty_like(logits)
    return st


def _shapes(case):
    """(elements, weight decay) of a model's tensors: a layer's seven modules, or their adapters, and two vectors."""
    w, m, got = case["width"], case["mlp"], []
    for _ in range(case["layers"]):
        for d_in, d_out in ((w, w),) * 4 + ((w, m),) * 2 + ((m, w),):
            got += [(case["rank"] * d_in, DECAY), (d_out * case["rank"], DECAY)] if case["rank"] else [(d_in * d_out, DECAY)]
        if not case["rank"]:
            got += [(w, 0.0), (w + 1, 0.0)]
    return got


def _blocks(x):
    """The 8-bit form of x in blocks of 256: values of the 8-bit format, and what each block's are multiplied by."""
    x = x.view(-1, BLOCK)
    amax = x.abs().amax(1, keepdim=True).clamp(min=AMAX_LEAST)
    q = x * (F8_MAX / amax)
    return q, (amax / F8_MAX)[:, 0]


def _tensors(case, gen):
    """A model's weights, gradients and states, each kind in one buffer, its tensors one after the other."""
    shapes, pad = _shapes(case), case["pad"]
    sizes = [-(-n // pad) * pad for n, _ in shapes]
    total = sum(sizes)
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    place, at = [], 0
    for (n, _), size in zip(shapes, sizes):
        used[at:at + n] = True
        place.append((at, n))
        at += size
    p = _randn(gen, total).mul_(0.02).mul_(used)
    loud = torch.exp(_randn(gen, -(-total // 64))).repeat_interleave(64)[:total]  # gradients' sizes differ by the row
    g = (_randn(gen, total).mul_(1e-2).mul_(loud).mul_(used)).to(DT[case["g"]])
    m = _randn(gen, total).mul_(3e-3).mul_(loud).mul_(used)
    v = _randn(gen, total).square_().add_(0.05).mul_(1e-5).mul_(loud.square_()).mul_(used)
    st = {"case": case, "place": place, "total": total, "g": g, "m": m, "v": v, "p": p, "master": None,
          "m_scale": None, "v_scale": None, "grad_scale": torch.full((1,), GRAD_SCALE, device="cuda"),
          "decay": torch.zeros(total, dtype=F32, device="cuda")}
    for (_, d), (at, n) in zip(shapes, place):
        st["decay"][at:at + n] = d
    if case["master"]:
        st["master"], st["p"] = p, p.to(DT[case["p"]])
    if case["state"] == "f8":
        (m, st["m_scale"]), (v, st["v_scale"]) = _blocks(m), _blocks(v.sqrt_())
        st["m"], st["v"] = m.view(-1).to(F8), v.clamp_(min=F8_LEAST).mul_(used.view_as(v)).view(-1).to(F8)
    if own:  # the plan that a training program keeps: the tensors' places
        import paper_2606_11660_amd as P

        def cut(x, each=1):
            return None if x is None else [x[a // each:a // each + -(-n // each)] for a, n in place]

        st["plan"] = P.AdamTensors(p=cut(st["p"]), g=cut(st["g"]), m=cut(st["m"]), v=cut(st["v"]),
                                   master=cut(st["master"]), m_scale=cut(st["m_scale"], BLOCK),
                                   v_scale=cut(st["v_scale"], BLOCK), weight_decay=[d for _, d in shapes])
    return st


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return _tensors(case, gen) if case["op"] == "adamw" else _tokens(case, gen)


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    import paper_2606_11660_amd as P
    case = st["case"]
    if case["op"] == "adamw":
        P.attr_adamw_step(st["plan"], case["step"], LR, BETA1, BETA2, EPS, eps_root=EPS_ROOT, grad_scale=st["grad_scale"])
        return _adamw_outputs(st)
    rows = P.TokenRows(st["logits"], st["target"], case["n"], case["T"], row_offset=st["offset"],
                       length=st["length"], weight=st["weight"], logit_scale=case["scale"])
    if case["op"] == "logp":
        return {"logp": P.attr_token_logp(rows, st["logp"])}
    if case["op"] == "policy":
        P.attr_policy_loss(rows, st["advantage"], st["loss"], logp=st["logp"], dlogits=st["dlogits"], logp_old=st["old"],
                           logp_ref=st["ref"] if case["kl"] else None, per_token=case["per_token"],
                           clip_low=CLIP_LOW, clip_high=CLIP_HIGH, beta=BETA_KL if case["kl"] else 0.0)
        return {"loss": st["loss"], "logp": st["logp"], "dlogits": st["dlogits"]}
    P.attr_preference_loss(rows, st["loss"], log_ratio=st["log_ratio"], logp=st["logp"], dlogits=st["dlogits"],
                           logp_ref=st["ref"], pair_weight=st["pair_weight"], beta=BETA_PREF, label_smoothing=SMOOTHING)
    return {"loss": st["loss"], "log_ratio": st["log_ratio"], "logp": st["logp"], "dlogits": st["dlogits"]}


def _adamw_outputs(st):
    return {k: st[k] for k in ("p", "master", "m", "v", "m_scale", "v_scale") if st[k] is not None}


def _example_of_rows(st):
    """Each row's example, and whether the row counts."""
    case = st["case"]
    n, T = case["n"], case["T"]
    examples = torch.arange(n, device="cuda")
    if case["packed"]:
        return examples.repeat_interleave(st["length"].long(), output_size=st["rows"]), st["weight"] != 0
    inside = (torch.arange(T, device="cuda") < st["length"][:, None]).view(-1)
    return examples.repeat_interleave(T, output_size=n * T), inside & (st["weight"] != 0)


def _plain_logp(st):
    """exp(s (z - max)), its row sums and the targets' log-probabilities."""
    z = st["logits"].float()
    z = (z - z.amax(1, keepdim=True)) * st["case"]["scale"]
    zy = z.gather(1, st["target"][:, None])[:, 0]
    e = torch.exp(z)
    total = e.sum(1)
    return e, total, zy - torch.log(total)


def _plain_dlogits(st, e, total, c):
    """s c (1[j = target] - p_j), c the loss's derivative by the row's log-probability."""
    c = c * st["case"]["scale"]
    d = e * (-c / total)[:, None]
    return d.scatter_add(1, st["target"][:, None], c[:, None]).to(st["logits"].dtype)


def _sum_examples(x, example, n):
    return torch.zeros(n, dtype=F32, device="cuda").index_add(0, example, x)


def _run_plain(st):
    case = st["case"]
    if case["op"] == "adamw":
        return _plain_adamw(st)
    example, counts = _example_of_rows(st)
    zero = torch.zeros((), device="cuda")
    e, total, logp = _plain_logp(st)
    logp = torch.where(counts, logp, zero)
    if case["op"] == "logp":
        return {"logp": logp}
    w = torch.where(counts, st["weight"], zero)
    if case["op"] == "policy":
        a = st["advantage"] if case["per_token"] else st["advantage"][example]
        ratio = torch.exp(logp - st["old"])
        free, held = -a * ratio, -a * ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
        loss, c = torch.maximum(free, held), torch.where(free >= held, free, zero)
        if case["kl"]:
            less = torch.expm1(st["ref"] - logp)
            loss = loss + BETA_KL * (less - (st["ref"] - logp))
            c = c - BETA_KL * less
        loss = _sum_examples(torch.where(counts, w * loss, zero), example, case["n"])
        c = torch.where(counts, w * c, zero)
        return {"loss": loss, "logp": logp, "dlogits": _plain_dlogits(st, e, total, c)}
    n_pairs = case["n"] // 2
    log_ratio = _sum_examples(torch.where(counts, w * (logp - st["ref"]), zero), example, case["n"])
    h = BETA_PREF * (log_ratio[:n_pairs] - log_ratio[n_pairs:])

    def softplus(x):
        return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))

    pw = st["pair_weight"]
    loss = pw * ((1 - SMOOTHING) * softplus(-h) + SMOOTHING * softplus(h))
    dh = pw * BETA_PREF * (SMOOTHING / (1 + torch.exp(-h)) - (1 - SMOOTHING) / (1 + torch.exp(h)))
    c = torch.cat([dh, -dh])[example] * w
    return {"loss": loss, "log_ratio": log_ratio, "logp": logp, "dlogits": _plain_dlogits(st, e, total, c)}


def _plain_adamw(st):
    case, eight = st["case"], st["case"]["state"] == "f8"
    w = st["p"] if st["master"] is None else st["master"]
    g = st["g"].float() * st["grad_scale"]
    m, v = st["m"].float(), st["v"].float()
    if eight:
        m = (m.view(-1, BLOCK) * st["m_scale"][:, None]).view(-1)
        v = (v.view(-1, BLOCK) * st["v_scale"][:, None]).view(-1).square()
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    root = torch.sqrt(v * (1 / (1 - BETA2 ** case["step"])) + EPS_ROOT) + EPS
    x = w.float()
    x = x - x * (LR * st["decay"]) - (m * (1 / (1 - BETA1 ** case["step"]))) / root * LR
    w.copy_(x)
    if st["master"] is not None:
        st["p"].copy_(x)
    if eight:
        q, scale = _blocks(m)
        st["m"].copy_(q.view(-1).to(F8))
        st["m_scale"].copy_(scale)
        q, scale = _blocks(torch.sqrt(v))
        st["v"].copy_(torch.where(q > 0, q.clamp(min=F8_LEAST), q).view(-1).to(F8))  # never zero for what is not
        st["v_scale"].copy_(scale)
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
    return _adamw_outputs(st)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    if case["op"] == "adamw":
        n = sum(k for k, _ in _shapes(case))
        states = 2 * BYTES[case["state"]] + (8.0 / BLOCK if case["state"] == "f8" else 0)
        weights = 2 * 4 + BYTES[case["p"]] if case["master"] else 2 * BYTES[case["p"]]
        return {"bytes": n * (weights + 2 * states + BYTES[case["g"]]), "flops": 16 * n}
    lens = _lengths(case)
    rows = sum(lens) if case["packed"] else case["n"] * case["T"]
    counted = sum(x - int(x * case["prompt"]) for x in lens)
    row = case["V"] * BYTES[case["dtype"]]
    if case["op"] == "logp":
        return {"bytes": counted * row + 16 * rows, "flops": 4 * counted * case["V"]}
    return {"bytes": (counted + rows) * row + 24 * rows, "flops": 8 * counted * case["V"]}


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return _exact_adamw(st) if case["op"] == "adamw" else _exact_tokens(st)


def _exact_tokens(st):
    """Row by row through log_softmax and the examples one by one; the gradient is autograd's."""
    case = st["case"]
    n, T, lens = case["n"], case["T"], _lengths(case)
    starts = st["offset"].tolist() if case["packed"] else [i * T for i in range(n)]
    logp = torch.zeros(st["rows"], dtype=torch.float64, device="cuda")
    dlogits = None if case["op"] == "logp" else torch.zeros(st["rows"], case["V"], dtype=F32, device="cuda")

    def rows_of(i):
        at = torch.arange(starts[i], starts[i] + lens[i], device="cuda")
        return at[st["weight"][at] != 0]

    def log_p(at):
        z = (st["logits"][at].double() * case["scale"]).requires_grad_(dlogits is not None)
        return z, torch.log_softmax(z, 1)[torch.arange(len(at), device="cuda"), st["target"][at]]

    def keep(at, lp, z, value):
        logp[at] = lp.detach()
        if dlogits is not None:
            dlogits[at] = (torch.autograd.grad(value, z)[0] * case["scale"]).float()

    if case["op"] == "logp":
        for i in range(n):
            at = rows_of(i)
            keep(at, log_p(at)[1], None, None)
        return {"logp": logp}
    if case["op"] == "policy":
        losses = []
        for i in range(n):
            at = rows_of(i)
            z, lp = log_p(at)
            a = (st["advantage"][at] if case["per_token"] else st["advantage"][i]).double()
            ratio = (lp - st["old"][at].double()).exp()
            value = -torch.minimum(ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a)
            if case["kl"]:
                d = st["ref"][at].double() - lp
                value = value + BETA_KL * (d.exp() - d - 1)
            value = (value * st["weight"][at].double()).sum()
            keep(at, lp, z, value)
            losses.append(value.detach())
        return {"loss": torch.stack(losses), "logp": logp, "dlogits": dlogits}
    losses, ratios = [], [None] * n
    for i in range(n // 2):
        (a, b), sums, kept = (rows_of(i), rows_of(n // 2 + i)), [], []
        for at in (a, b):
            z, lp = log_p(at)
            sums.append((st["weight"][at].double() * (lp - st["ref"][at].double())).sum())
            kept.append((at, lp, z))
        h = BETA_PREF * (sums[0] - sums[1])
        f = torch.nn.functional.logsigmoid
        value = -st["pair_weight"][i].double() * ((1 - SMOOTHING) * f(h) + SMOOTHING * f(-h))
        grads = torch.autograd.grad(value, [kept[0][2], kept[1][2]])
        for (at, lp, _), g in zip(kept, grads):
            logp[at] = lp.detach()
            dlogits[at] = (g * case["scale"]).float()
        losses.append(value.detach())
        ratios[i], ratios[n // 2 + i] = sums[0].detach(), sums[1].detach()
    return {"loss": torch.stack(losses), "log_ratio": torch.stack(ratios), "logp": logp, "dlogits": dlogits}


def _exact_adamw(st):
    case, got = st["case"], {}
    t, eight = case["step"], case["state"] == "f8"
    per = torch.arange(st["total"], device="cuda") // BLOCK
    was_m = st["m"].double() * (st["m_scale"].double()[per] if eight else 1.0)
    was_v = (st["v"].double() * st["v_scale"].double()[per]) ** 2 if eight else st["v"].double()
    g = st["g"].double() * float(st["grad_scale"])
    m = BETA1 * was_m + (1 - BETA1) * g
    v = BETA2 * was_v + (1 - BETA2) * g ** 2
    x = (st["p"] if st["master"] is None else st["master"]).double()
    new = x - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t) + EPS_ROOT).sqrt() + EPS)
    for (a, n), (_, decay) in zip(st["place"], _shapes(case)):
        new[a:a + n] -= LR * decay * x[a:a + n]
    got["p"] = new
    if st["master"] is not None:
        got["master"] = new
    if not eight:
        return {**got, "m": m, "v": v}
    for name, y in (("m", m), ("v", v.sqrt())):
        amax = y.view(-1, BLOCK).abs().amax(1).clamp(min=AMAX_LEAST)
        q = y * (F8_MAX / amax)[per]
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)  # the 8-bit format's, three bits below the leading one
        code = torch.round(q / step) * step
        got[name] = torch.where(q > 0, code.clamp(min=F8_LEAST), code) if name == "v" else code
        got[name + "_scale"] = amax / F8_MAX
    return got
