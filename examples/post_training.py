"""A round of post-training on a toy model, and what its rollouts taught it.

    python examples/post_training.py

A linear head over fixed features stands for the language model; the products with its
weights are the user's own (torch).  The library does the rest, in the order in which a
training program would call it:

1. attr_token_logp    log-probabilities of the rollouts' tokens under the policy that
                      sampled them and under the reference model
2. attr_policy_loss   the clipped policy loss with a KL term, its gradient written over
                      the logits; then attr_adamw_step on the head, with 8-bit states
3. attr_preference_loss on pairs of rollouts, again with a step
4. attr_project       each rollout's compressed gradient, normalised by the optimizer's
                      second moment (its row and column means), attr_precond_apply to
                      unit rows, attr_score_topk for the rollouts most like each query
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_11660_amd as P  # noqa: E402

N, T, D, V, K = 16, 24, 64, 256, 16   # rollouts, tokens, features, vocabulary, projection


def main(steps: int = 12, seed: int = 0, device: str = "cuda") -> dict:
    gen = torch.Generator(device=device).manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=gen, device=device)  # noqa: E731
    features = randn(N * T, D) / D ** 0.5
    head = randn(V, D) * 2.0
    reference = head + 0.1 * randn(V, D)
    tokens = torch.randint(0, V, (N * T,), generator=gen, device=device)
    length = torch.randint(T // 2, T + 1, (N,), generator=gen, device=device).to(torch.int32)
    weight = (1.0 / length.float()).repeat_interleave(T)      # means over each rollout's tokens
    reward = randn(N)
    advantage = (reward - reward.mean()) / reward.std()

    def rows(w):
        return P.TokenRows(features @ w.t(), tokens, N, T, length=length, weight=weight)

    logp_old, logp_ref = (torch.empty(N * T, device=device) for _ in range(2))
    P.attr_token_logp(rows(head), logp_old)
    P.attr_token_logp(rows(reference), logp_ref)

    grad = torch.zeros_like(head)
    blocks = head.numel() // 256
    states = dict(m=[torch.zeros(head.shape, dtype=torch.float8_e4m3fn, device=device)],
                  v=[torch.zeros(head.shape, dtype=torch.float8_e4m3fn, device=device)],
                  m_scale=[torch.zeros(blocks, device=device)], v_scale=[torch.zeros(blocks, device=device)])
    plan = P.AdamTensors([head], [grad], weight_decay=0.01, **states)
    step = 0

    def update(dlogits):
        nonlocal step
        torch.mm(dlogits.t(), features, out=grad)
        clip = (1.0 / grad.norm()).clamp(max=1.0).reshape(1)      # stays on the device
        step += 1
        P.attr_adamw_step(plan, step, lr=0.02, beta1=0.9, beta2=0.95, eps_root=1e-12, grad_scale=clip)

    policy, preference = [], []
    loss, pair_loss = torch.empty(N, device=device), torch.empty(N // 2, device=device)
    for _ in range(steps):
        r = rows(head)
        P.attr_policy_loss(r, advantage, loss, dlogits=r.logits, logp_old=logp_old, logp_ref=logp_ref, beta=0.02)
        policy.append(float(loss.sum()))
        update(r.logits)
    for _ in range(steps):   # the first half of the rollouts was preferred to the second
        r = rows(head)
        P.attr_preference_loss(r, pair_loss, dlogits=r.logits, logp_ref=logp_ref, beta=0.5)
        preference.append(float(pair_loss.sum()))
        update(r.logits)

    # every rollout's gradient of the policy loss at the trained weights, compressed
    r = rows(head)
    dlogits = torch.empty_like(r.logits)
    P.attr_policy_loss(r, advantage, loss, dlogits=dlogits, logp_old=logp_old, logp_ref=logp_ref, beta=0.02)
    scale = states["v_scale"][0].repeat_interleave(256).view(V, D)
    second = (states["v"][0].float() * scale).square()
    module = P.Module(features, dlogits, randn(V, K) / K ** 0.5, randn(D, K) / K ** 0.5, 0,
                      v_out=second.mean(1).contiguous(), v_in=second.mean(0).contiguous())
    raw, store = torch.empty((N, K * K), device=device), torch.empty((N, K * K), device=device)
    P.attr_project([module], K, N, T, raw, length=length)
    P.attr_precond_apply(raw, P.PRECOND_NONE, None, True, store)
    score = torch.empty((N, 3), device=device)
    index = torch.empty((N, 3), dtype=torch.int64, device=device)
    P.attr_score_topk(store, store, 3, score, index)
    return {"policy": policy, "preference": preference, "score": score.cpu(), "index": index.cpu(), "head": head.cpu()}


if __name__ == "__main__":
    out = main()
    print("policy loss      %.4f -> %.4f" % (out["policy"][0], out["policy"][-1]))
    print("preference loss  %.4f -> %.4f" % (out["preference"][0], out["preference"][-1]))
    for q in range(4):
        print("rollout %d: most alike %s" % (q, ", ".join("%d (%.2f)" % (i, s) for i, s in zip(out["index"][q], out["score"][q]))))
