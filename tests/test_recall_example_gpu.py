"""GPU: the recall example runs the LSTM loop, the delta rule, the log
probabilities and AdamW together: it learns, its gradient is that of the same model
written in plain torch on the CPU in float64, and token by token it answers what
the loops over whole sequences say.

Tolerances: float32 loops of 12 steps keep 1e-5 of a gradient's largest entry per
operator (two recurrences and two products in a row here: 1e-4), and 2e-5 of log
probabilities of the size of 1 to 10.
"""
import os
import sys

import pytest
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import recall_lm as ex  # noqa: E402
from paper_1805_01772_amd import lstmloop as ll  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def plain_loss(p, model, tokens, targets, length):
    """Minus the mean log probability of the targets, step by step."""
    T, B = tokens.shape
    H, n, D = model.H, model.heads, model.D
    h = c = torch.zeros(B, H, dtype=torch.float64)
    S = torch.zeros(B, n, D, D, dtype=torch.float64)
    total = 0.0
    for t in range(T):
        on = (t < length).double().view(B, 1)
        z = torch.cat([p["embed"][tokens[t]], h], 1) @ p["W"] + p["bias"]
        i, f, g, o = z.split(H, 1)
        c2 = torch.sigmoid(f) * c + torch.sigmoid(i) * torch.tanh(g)
        h2 = torch.sigmoid(o) * torch.tanh(c2)
        h, c = on * h2 + (1 - on) * h, on * c2 + (1 - on) * c
        q, k, v = (x.view(B, n, D) for x in (h @ p["qkv"]).split(n * D, 1))
        a, b = (h @ p["gates"]).split(n, 1)
        q, k = (F.normalize(F.silu(x), dim=-1) for x in (q, k))
        S2 = torch.exp(-F.softplus(a - 4.0)).view(B, n, 1, 1) * S
        u = torch.sigmoid(b).view(B, n, 1) * (v - torch.einsum("bnk,bnkv->bnv", k, S2))
        S2 = S2 + k.unsqueeze(-1) * u.unsqueeze(-2)
        S = on.view(B, 1, 1, 1) * S2 + (1 - on.view(B, 1, 1, 1)) * S
        y = torch.einsum("bnk,bnkv->bnv", q, S) * D ** -0.5
        logp = torch.log_softmax(y.flatten(1) @ p["out"], 1)
        want = targets[t].long()
        total = total - (logp.gather(1, want.clamp(min=0).view(B, 1)).view(B) * (want >= 0)).sum()
    return total / (targets >= 0).sum()


def test_gradient_of_the_whole_model():
    tokens, targets, length = ex.make_batch(5, 3, 4, 9, 7, torch.Generator().manual_seed(3))
    model = ex.RecallModel(16, seed=4)
    T, B = tokens.shape
    plain = {n: p.detach().double().cpu().requires_grad_() for n, p in model.params.items()}
    loss = plain_loss(plain, model, tokens, targets, length)
    loss.backward()
    lstm = ll.Plan(T, B, model.I, model.H)
    delta = ll.DeltaPlan(T, B, model.heads, model.heads, model.D, model.D)
    logits = model.logits(tokens.to(DEV), length.to(DEV), lstm, delta).flatten(0, 1)
    t = targets.flatten().to(DEV)
    weight = -(t >= 0).float() / (t >= 0).sum()
    logp, d = torch.empty(T * B, device=DEV), torch.empty_like(logits)
    with ll.LogprobPlan(T * B, model.vocab) as plan:
        plan.fwd_bwd(logits.detach(), t, weight, None, logp, None, None, d)
    grads = torch.autograd.grad(logits, list(model.params.values()), d)
    assert abs((weight * logp).sum().item() - loss.item()) <= 2e-5 * max(1, abs(loss.item()))
    for n, g in zip(model.params, grads):
        want = plain[n].grad
        err = (g.double().cpu() - want).abs().max().item() / want.abs().max().item()
        print(f"    {n}: {err:.1e}", flush=True)
        assert err <= 1e-4, (n, err)
    for p in (lstm, delta):
        p.close()


def test_learns_and_answers_token_by_token():
    model, losses = ex.train(steps=120, say=None)
    first, last = sum(losses[:10]) / 10, sum(losses[-10:]) / 10
    print(f"    loss {first:.3f} -> {last:.3f}", flush=True)
    assert last < 0.8 * first
    tokens, _, _ = ex.make_batch(8, 4, 4, 16, 16, torch.Generator().manual_seed(7))
    tokens = tokens.to(DEV)
    T, B = tokens.shape
    ids, logp = ex.answer(model, tokens, top=4)
    full = torch.full((B,), T, dtype=torch.int32, device=DEV)
    with torch.no_grad(), ll.Plan(T, B, model.I, model.H) as lstm, \
            ll.DeltaPlan(T, B, model.heads, model.heads, model.D, model.D) as delta:
        want = torch.log_softmax(model.logits(tokens, full, lstm, delta).double(), -1)
        torch.cuda.synchronize()
    assert (logp.double() - want.gather(-1, ids.long())).abs().max().item() <= 2e-5 * 10
    assert (logp[..., :-1] >= logp[..., 1:]).all()
