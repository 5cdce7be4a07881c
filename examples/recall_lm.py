"""A small recurrent language model that learns to recall, on the library's loops.

A sequence states pairs "key value" and then asks for some of the keys; the model
answers each with the value that was paired with it.  The LSTM loop (I -> H) tells
keys from values, the gated delta rule holds the pairs in its state matrix, the log
probabilities make the loss and its gradient, AdamW takes the step.  Answering runs
one token at a time: a plan of one step for the LSTM, delta_loop_step for the state
matrix, and the most likely tokens with their log probabilities.

    python examples/recall_lm.py --steps 2000

torch makes the data, the plain matrix products and the graph that joins the
operators; the recurrences, the loss and the optimizer run in the library.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1805_01772_amd import lstmloop as ll  # noqa: E402


class LstmLoop(torch.autograd.Function):
    """lstm_loop_fwd / lstm_loop_bwd of one layer from a zero state."""

    @staticmethod
    def forward(ctx, plan, x, seq_len, W, bias):
        T, B, _ = x.shape
        H = bias.numel() // 4
        zero = torch.zeros(1, B, H, device=x.device)
        y, hT, cT = torch.empty(T, B, H, device=x.device), torch.empty_like(zero), torch.empty_like(zero)
        plan.fwd(x, seq_len, [W], [bias], zero, zero, y, hT, cT)
        ctx.plan, ctx.zero = plan, zero        # the plan reads the state again in its backward
        ctx.save_for_backward(x, seq_len, W, bias)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, seq_len, W, bias = ctx.saved_tensors
        dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(bias)
        ctx.plan.bwd(x, seq_len, [W], dy.contiguous(), None, None, dx, [dW], [db], None, None)
        return None, dx, None, dW, db


class DeltaLoop(torch.autograd.Function):
    """delta_loop_fwd / delta_loop_bwd from a zero state."""

    @staticmethod
    def forward(ctx, plan, q, k, v, g, beta, seq_len):
        y = torch.empty_like(v)
        plan.fwd(q, k, v, g, beta, seq_len, None, y, None)
        ctx.plan = plan
        ctx.save_for_backward(q, k, v, g, beta, seq_len)
        return y

    @staticmethod
    def backward(ctx, dy):
        ins = ctx.saved_tensors
        grads = [torch.empty_like(t) for t in ins[:5]]
        ctx.plan.bwd(*ins, dy.contiguous(), None, *grads)
        return (None, *grads, None)


class RecallModel:
    """Parameters, the layers around the loops, and both ways to run them."""

    def __init__(self, vocab, I=32, H=64, heads=2, D=32, device="cuda:0", seed=0):
        gen = torch.Generator().manual_seed(seed)

        def new(*shape, scale):
            return (scale * torch.randn(*shape, generator=gen)).to(device).requires_grad_()

        self.vocab, self.I, self.H, self.heads, self.D = vocab, I, H, heads, D
        n = heads * D
        self.params = dict(
            embed=new(vocab, I, scale=1.0), W=new(I + H, 4 * H, scale=(I + H) ** -0.5),
            bias=new(4 * H, scale=0.0), qkv=new(H, 3 * n, scale=H ** -0.5),
            gates=new(H, 2 * heads, scale=H ** -0.5), out=new(n, vocab, scale=n ** -0.5))

    def inputs(self, h):
        """q, k (unit length), v, the log of the decay and the writing strength of
        h [.., H]; the decay starts near 1."""
        p, shape = self.params, h.shape[:-1] + (self.heads, self.D)
        q, k, v = (h @ p["qkv"]).split(self.heads * self.D, dim=-1)
        a, b = (h @ p["gates"]).split(self.heads, dim=-1)
        unit = lambda t: F.normalize(F.silu(t).view(shape), dim=-1)
        return (unit(q), unit(k), v.reshape(shape).contiguous(), -F.softplus(a - 4.0).contiguous(),
                torch.sigmoid(b).contiguous())

    def logits(self, tokens, seq_len, lstm, delta):
        """[T, B, vocab] over whole sequences (plans for their shape)."""
        p = self.params
        h = LstmLoop.apply(lstm, F.embedding(tokens, p["embed"]), seq_len, p["W"], p["bias"])
        y = DeltaLoop.apply(delta, *self.inputs(h), seq_len)
        return y.flatten(2) @ p["out"]

    @torch.no_grad()
    def start(self, B):
        """The state of B sequences before their first token."""
        d = self.params["W"].device
        return dict(h=torch.zeros(1, B, self.H, device=d), c=torch.zeros(1, B, self.H, device=d),
                    S=torch.zeros(B, self.heads, self.D, self.D, device=d),
                    one=torch.ones(B, dtype=torch.int32, device=d), lstm=ll.Plan(1, B, self.I, self.H))

    @torch.no_grad()
    def step(self, state, tokens):
        """One token for each sequence; its logits [B, vocab]."""
        p, B = self.params, tokens.numel()
        x = F.embedding(tokens, p["embed"]).view(1, B, self.I)
        h, c = torch.empty_like(state["h"]), torch.empty_like(state["c"])
        out = torch.empty(1, B, self.H, device=x.device)
        state["lstm"].fwd(x, state["one"], [p["W"]], [p["bias"]], state["h"], state["c"], out, h, c,
                          save_for_backward=False)
        state["h"], state["c"] = h, c
        q, k, v, g, beta = self.inputs(out[0])
        y = torch.empty_like(v)
        ll.delta_loop_step(q, k, v, g, beta, state["S"], y)
        return y.flatten(1) @ p["out"]


def make_batch(B, pairs, asks, keys, values, gen):
    """tokens [T, B], targets [T, B] int32 (-1: nothing to predict), lengths [B]:
    each row states `pairs` pairs of distinct keys and asks for 1 to `asks`."""
    T = 2 * pairs + asks
    tokens = torch.zeros(T, B, dtype=torch.int64)
    targets = torch.full((T, B), -1, dtype=torch.int32)
    length = torch.randint(2 * pairs + 1, T + 1, (B,), generator=gen)
    for b in range(B):
        ks = torch.randperm(keys, generator=gen)[:pairs]
        vs = keys + torch.randint(0, values, (pairs,), generator=gen)
        tokens[0:2 * pairs:2, b], tokens[1:2 * pairs:2, b] = ks, vs
        ask = torch.randint(0, pairs, (asks,), generator=gen)
        tokens[2 * pairs:, b] = ks[ask]
        targets[2 * pairs:, b] = vs[ask].int()
        targets[length[b]:, b] = -1
    return tokens, targets, length.int()


def train(steps=2000, B=32, pairs=4, asks=4, keys=16, values=16, lr=4e-3, clip=1.0, seed=0,
          device="cuda:0", say=print):
    """Returns the model and the loss of every step."""
    gen = torch.Generator().manual_seed(seed)
    model = RecallModel(keys + values, device=device, seed=seed)
    T, params = 2 * pairs + asks, list(model.params.values())
    lstm = ll.Plan(T, B, model.I, model.H)
    delta = ll.DeltaPlan(T, B, model.heads, model.heads, model.D, model.D)
    logprob = ll.LogprobPlan(T * B, model.vocab)
    data = [p.detach() for p in params]
    adamw = ll.AdamWPlan(data, [torch.zeros_like(p) for p in data], [torch.zeros_like(p) for p in data],
                         weight_decay=[0.01 if p.dim() > 1 else 0.0 for p in data])
    logp = torch.empty(T * B, device=device)
    losses = []
    for n in range(1, steps + 1):
        tokens, targets, length = (t.to(device) for t in make_batch(B, pairs, asks, keys, values, gen))
        logits = model.logits(tokens, length, lstm, delta).flatten(0, 1)
        targets = targets.flatten()
        wanted = targets >= 0
        weight = -wanted.float() / wanted.sum()              # the loss is minus the mean of logp
        dlogits = torch.empty_like(logits)
        logprob.fwd_bwd(logits.detach(), targets, weight, None, logp, None, None, dlogits)
        grads = torch.autograd.grad(logits, params, dlogits)
        norm = torch.stack([g.square().sum() for g in grads]).sum().sqrt()
        adamw.step([g.contiguous() for g in grads], lr=lr, step=n, eps=1e-8,
                   grad_scale=(clip / norm.clamp(min=clip)).view(1))
        losses.append((weight * logp).sum())
        if say and (n % 50 == 0 or n == 1):
            say(f"step {n}: loss {losses[-1].item():.4f}", flush=True)
    for what, plan in (("lstm", lstm), ("delta", delta), ("logprob", logprob)):
        error = plan.status_sync()
        if error:
            raise RuntimeError(f"{what}: device error {error}")
    for plan in (lstm, delta, logprob, adamw):
        plan.close()
    return model, [x.item() for x in losses]


@torch.no_grad()
def answer(model, tokens, top=3):
    """Feed tokens [T, B] one at a time; the `top` most likely next tokens after
    each and their log probabilities, [T, B, top]."""
    T, B = tokens.shape
    state = model.start(B)
    ids = torch.empty(T, B, top, dtype=torch.int32, device=tokens.device)
    logp = torch.empty(T, B, top, device=tokens.device)
    with ll.LogprobPlan(B, model.vocab, top_k=top) as plan:
        for t in range(T):
            plan.fwd(model.step(state, tokens[t]), None, None, None, None, ids[t], logp[t])
        torch.cuda.synchronize()
    state["lstm"].close()
    return ids, logp


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=2000)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()
    model, _ = train(args.steps, seed=args.seed)
    tokens, targets, _ = make_batch(64, 4, 4, 16, 16, torch.Generator().manual_seed(args.seed + 1))
    ids, logp = answer(model, tokens.to("cuda:0"))
    asked = targets >= 0
    right = (ids[..., 0].cpu() == targets)[asked].float().mean().item()
    print(f"answers right: {100 * right:.1f}% of {int(asked.sum())}", flush=True)
    t = int(asked[:, 0].nonzero()[0])
    print(f"first row, token {t}: wanted {int(targets[t, 0])}, most likely "
          + ", ".join(f"{i} ({p:.2f})" for i, p in zip(ids[t, 0].tolist(), logp[t, 0].tolist())), flush=True)


if __name__ == "__main__":
    main()
