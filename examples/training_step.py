"""Training steps of a small model with the library's own ends, and whose examples taught it.

    python examples/training_step.py

An embedding, a layer norm and a linear head, trained on packed sequences of different lengths;
the products with the head's weights are the user's own (torch).  The library does the rest, in
the order in which a training program would call it:

1. attr_embed           the tokens' rows of the table, scaled by the root of the width
2. attr_layer_norm      the head's input rows, which are the activations that attribution reads
3. attr_policy_loss     with advantage 1 and no clipping: the log-likelihood's gradient, over the logits
4. attr_layer_norm_backward   the rows' gradient, the weights' over the batch and for each example
5. attr_embed_backward  the table's gradient, added up in the order of the rows
6. attr_muon_step       on the head; attr_adamw_step on the table and the norm's vectors
7. attr_project         each example's compressed gradient of the head, beside its gradient of the
                        norm's weights in one row of the store; unit rows, scored against each other
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_11660_amd as P  # noqa: E402

N, T, D, V, K = 12, 20, 64, 320, 16   # examples, tokens at most, width, vocabulary, projection


class Model:
    def __init__(self, seed: int, device: str):
        gen = torch.Generator(device=device).manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=gen, device=device)  # noqa: E731
        self.table, self.head = randn(V, D) / D ** 0.5, randn(V, D) / D ** 0.5
        self.weight, self.bias = 1 + 0.1 * randn(D), 0.1 * randn(D)
        self.names = ("table", "head", "weight", "bias")
        self.grad = {k: torch.zeros_like(getattr(self, k)) for k in self.names}
        vectors = ("table", "weight", "bias")
        zeros = lambda ks: [torch.zeros_like(getattr(self, k)) for k in ks]  # noqa: E731
        self.adam = P.AdamTensors([getattr(self, k) for k in vectors], [self.grad[k] for k in vectors], zeros(vectors),
                                  zeros(vectors))
        self.muon = P.MuonTensors([self.head], [self.grad["head"]], zeros(["head"]), weight_decay=0.01,
                                  update_scale=max(1.0, V / D) ** 0.5)


class Batch:
    """Packed sequences, each token predicting the next one."""

    def __init__(self, seed: int, device: str):
        gen = torch.Generator(device=device).manual_seed(seed + 1000)
        length = torch.randint(3, T + 1, (N,), generator=gen, device=device)
        self.length, self.offset = length.to(torch.int32), length.cumsum(0) - length
        n = int(length.sum())
        first = torch.randint(0, V, (N,), generator=gen, device=device).repeat_interleave(length)
        place = torch.arange(n, device=device) - self.offset.repeat_interleave(length)
        self.token, self.target = (first + 7 * place) % V, (first + 7 * place + 7) % V    # a rule to learn
        self.rows = P.ExampleRows(N, T, self.offset, self.length)
        self.mean_of_tokens = torch.full((n,), 1.0 / n, device=device)


def forward_backward(m: Model, b: Batch) -> dict:
    """The batch's loss and its gradients, and what attribution takes."""
    n, dev = len(b.token), m.head.device
    new = lambda *s: torch.empty(s, device=dev)  # noqa: E731
    x, y, mean, rstd = new(n, D), new(n, D), new(n), new(n)
    P.attr_embed(m.table, b.token, x, scale=D ** 0.5, rows=b.rows)
    P.attr_layer_norm(x, y, m.weight, m.bias, mean=mean, rstd=rstd, rows=b.rows)
    logits, logp, loss = y @ m.head.t(), new(n), new(N)
    rows = P.TokenRows(logits, b.target, N, T, row_offset=b.offset, length=b.length, weight=b.mean_of_tokens)
    # at ratio 1 the policy loss's gradient with advantage 1 is that of -logp
    P.attr_policy_loss(rows, torch.ones(N, device=dev), loss, logp=logp, dlogits=logits)
    torch.mm(logits.t(), y, out=m.grad["head"])
    dy = logits @ m.head
    each = torch.zeros((N, K * K + 2 * D), device=dev)       # a store row: the head's block, the norm's gradients
    P.attr_layer_norm_backward(dy, x, mean, rstd, m.weight, dweight=each[:, K * K:K * K + D], dbias=each[:, K * K + D:],
                               per_example=True, rows=b.rows)
    P.attr_layer_norm_backward(dy, x, mean, rstd, m.weight, dx=dy, dweight=m.grad["weight"], dbias=m.grad["bias"],
                               rows=b.rows)
    P.attr_embed_backward(dy, b.token, m.grad["table"], scale=D ** 0.5, rows=b.rows)
    return {"loss": -(logp * b.mean_of_tokens).sum(), "y": y, "dlogits": logits, "store": each}


def main(steps: int = 30, seed: int = 0, device: str = "cuda") -> dict:
    m, b = Model(seed, device), Batch(seed, device)
    losses = []
    for step in range(1, steps + 1):
        losses.append(forward_backward(m, b)["loss"])
        P.attr_muon_step(m.muon, lr=0.02)
        P.attr_adamw_step(m.adam, step, lr=0.01, beta1=0.9, beta2=0.95)
    r = forward_backward(m, b)
    gen = torch.Generator(device=device).manual_seed(seed)
    R, S = (torch.randn(k, K, generator=gen, device=device) / K ** 0.5 for k in (V, D))
    P.attr_project([P.Module(r["y"], r["dlogits"], R, S, 0)], K, N, T, r["store"], row_offset=b.offset, length=b.length)
    unit = torch.empty_like(r["store"])
    P.attr_precond_apply(r["store"], P.PRECOND_NONE, None, True, unit)
    score, index = torch.empty((N, 3), device=device), torch.empty((N, 3), dtype=torch.int64, device=device)
    P.attr_score_topk(unit, unit, 3, score, index)
    return {"loss": torch.stack(losses).tolist(), "score": score.cpu(), "index": index.cpu(),
            "head": m.head.cpu(), "table": m.table.cpu()}


if __name__ == "__main__":
    out = main()
    print("loss %.4f -> %.4f" % (out["loss"][0], out["loss"][-1]))
    for q in range(4):
        print("example %d: most alike %s" % (q, ", ".join("%d (%.2f)" % (i, s) for i, s in zip(out["index"][q], out["score"][q]))))
