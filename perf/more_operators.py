"""Performance cases of three more operators of a recurrent language model: the
embedding lookup that makes the loops' inputs with the gradient of its table,
linear attention with a decay for each head (a loop whose state is a matrix,
with its one-token step), and beam search's selection with the reordering of
the beams' states.

``listed`` names the cases, ``draw`` gives more of the same ranges,
``prepare`` makes what a program holds before the call, ``run`` is one pass,
``work`` the bytes and operations the call cannot do without and ``exact``
the same outputs in 64 bits.  With ``own`` false ``run`` computes the
operators from elementary torch operations in 32 bits (64 for the long sums
of a table's gradient, and for the scores of beams that lie close together).

Keys of a case: ``op`` (linattn / linattn_step / embed / beam) and

- linattn: ``mode`` (train / infer), ``dtype``, sizes ``T``, ``B``, ``Hk``,
  ``Hv``, ``Dk``, ``Dv``, lengths drawn from ``lo`` .. ``T``, ``state``
  (random initial state instead of none), ``fused`` (q, k and v are slices of
  one projection's rows);
- linattn_step: ``slots`` states in the pool, ``B`` of them advanced;
- embed: ``mode`` (lookup / train / tied, whose table's gradient is added to
  one that is there), ``N`` tokens, ``V`` rows of ``D``, the types ``table``,
  ``x``, ``dx`` and ``grad``, ``skip`` (share of places without a token),
  ``scale``;
- beam: ``B`` searches of ``K`` beams over ``V`` tokens, ``dtype``, ``eos``
  (an end token, finished beams and lengths), ``penalty`` (of lengths),
  ``masked`` columns, ``hist`` tokens of history a beam, and a pool of
  ``slots`` states of ``H`` heads of ``D`` x ``D``.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
C = 64                 # tokens per chunk of the plain form


def _lin(name, mode, dtype, T, B, Hk, Hv, Dk, Dv, lo, state=False, fused=False):
    return dict(name=name, op="linattn", mode=mode, dtype=dtype, T=T, B=B, Hk=Hk, Hv=Hv, Dk=Dk,
                Dv=Dv, lo=lo, state=state, fused=fused)


def _step(name, dtype, slots, B, Hk, Hv, Dk, Dv):
    return dict(name=name, op="linattn_step", dtype=dtype, slots=slots, B=B, Hk=Hk, Hv=Hv, Dk=Dk,
                Dv=Dv)


def _embed(name, mode, N, V, D, table, x, dx, grad, skip, scale):
    return dict(name=name, op="embed", mode=mode, N=N, V=V, D=D, table=table, x=x, dx=dx,
                grad=grad, skip=skip, scale=scale)


def _beam(name, B, K, V, dtype, eos, penalty, masked, hist, slots, H, D):
    return dict(name=name, op="beam", B=B, K=K, V=V, dtype=dtype, eos=eos, penalty=penalty,
                masked=masked, hist=hist, slots=slots, H=H, D=D)


def listed():
    return [
        # one token for a few sequences: the latency of a serving step
        _step("linattn_step_b4_f32", "f32", 4, 4, 2, 4, 32, 32),
        # one token for a full serving batch out of a larger pool of states
        _step("linattn_step_b256_bf16", "bf16", 320, 256, 32, 32, 128, 128),
        # prompts of unequal length read into fresh states
        _lin("linattn_infer_ragged_bf16", "infer", "bf16", 1000, 4, 8, 16, 128, 128, 100),
        # a float32 training step, short odd lengths (none among them), sizes of a head
        # that are no power of two, shared key heads
        _lin("linattn_train_t100_f32", "train", "f32", 100, 64, 4, 8, 64, 72, 0, state=True),
        # an ordinary training step: q, k and v from one projection
        _lin("linattn_train_t2048_bf16", "train", "bf16", 2048, 8, 16, 16, 128, 128, 256,
             fused=True),
        # one long sequence: few rows, many steps
        _lin("linattn_train_long_bf16", "train", "bf16", 16384, 1, 16, 16, 128, 128, 16384,
             state=True),
        # the inputs of a serving step, one token a sequence
        _embed("embed_lookup_n128_bf16", "lookup", 128, 32000, 1024, "bf16", "bf16", "bf16", "f32",
               0.0, 1.0),
        # the batch of the 1024-unit loops, 128 rows of 200 tokens: bfloat16 inputs, the loops'
        # float gradients, float masters
        _embed("embed_train_t200_b128", "train", 25600, 32000, 1024, "f32", "bf16", "f32", "f32",
               0.25, 32.0),
        # a long batch and a large vocabulary, whose table also makes the logits
        _embed("embed_tied_n131072_bf16", "tied", 131072, 131072, 1024, "bf16", "bf16", "bf16",
               "f32", 0.02, 1.0),
        # one search of a few beams: the latency of a step
        _beam("beam_b1_k4_f32", 1, 4, 32000, "f32", 2, 0.0, 0, 128, 4, 4, 64),
        # many searches, rows of an odd width, hypotheses ranked by length
        _beam("beam_b48_k5_v50001_f32", 48, 5, 50001, "f32", 2, 0.6, 100, 255, 256, 4, 64),
        # a full serving batch, a large vocabulary and large states in a pool
        _beam("beam_b32_k8_v131072_bf16", 32, 8, 131072, "bf16", 1, 1.0, 72, 1024, 288, 16, 128),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, min(hi // step * step, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["train", "train", "infer", "step", "lookup", "embed", "embed", "beam", "beam"])
    dtype = rng.choice(["f32", "bf16"])
    for _ in range(10000):
        if kind in ("train", "infer", "step"):
            Hk = rng.choice([1, 2, 3, 4, 8, 16])
            Hv = Hk * rng.choice([1, 1, 2, 3])
            Dk, Dv = _log_int(rng, 32, 128, 8), _log_int(rng, 32, 128, 8)
            if kind == "step":
                B = _log_int(rng, 1, 256)
                c = _step("", dtype, B + rng.randint(0, 64), B, Hk, Hv, Dk, Dv)
                fits = B * Hv <= 8192
            else:
                T, B = _log_int(rng, 60, 16384), _log_int(rng, 1, 64)
                c = _lin("", kind, dtype, T, B, Hk, Hv, Dk, Dv, rng.choice([T, T // 8, 0]),
                         state=rng.random() < 0.5, fused=rng.random() < 0.5)
                # no dearer than the largest listed cases, whose heads are widest
                fits = T * B * Hv <= 262144
        elif kind in ("lookup", "embed"):
            N, V, D = _log_int(rng, 1, 131072), _log_int(rng, 100, 200000), _log_int(rng, 32, 2048)
            pick = lambda: rng.choice(["f32", "bf16"])
            c = _embed("", "lookup" if kind == "lookup" else rng.choice(["train", "tied"]), N, V, D,
                       pick(), pick(), pick(), pick(), rng.choice([0.0, 0.02, 0.25]),
                       rng.choice([1.0, round(math.sqrt(D), 3)]))
            fits = N * D <= 1 << 27 and V * D <= 1 << 27
        else:
            B, K, V = _log_int(rng, 1, 64), rng.choice([2, 3, 4, 5, 6, 8, 12, 16]), _log_int(rng, 1000, 200000)
            H, D = rng.choice([1, 2, 4, 8, 16]), _log_int(rng, 32, 128, 4)
            eos = rng.choice([-1, rng.randint(0, 99)])
            c = _beam("", B, K, V, dtype, eos, rng.choice([0.0, 0.6, 1.0]) if eos >= 0 else 0.0,
                      rng.choice([0, rng.randint(1, V // 4)]), _log_int(rng, 8, 1024),
                      B * K + rng.randint(0, 32), H, D)
            fits = (B * K * V * (2 if dtype == "bf16" else 4) <= 67108864
                    and c["slots"] * H * D * D <= 288 * 16 * 128 * 128)
        if fits:
            del c["name"]
            return c
    raise RuntimeError("no case drawn")


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _lengths(c, seed):
    r = random.Random(seed * 7919 + 17)
    s = [r.randint(c["lo"], c["T"]) for _ in range(c["B"])]
    if c["lo"] < c["T"]:
        s[r.randrange(c["B"])] = c["T"]      # some sequence fills the batch's padded length
        if c["lo"] == 0 and c["B"] > 1 and min(s) > 0:
            s[s.index(min(s))] = 0           # and one has no token at all
    return s


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 54321)
    return g


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _slices(c, row):
    """q, k and v (or their gradients) as slices of one projection's rows."""
    Hk, Hv, Dk, Dv = c["Hk"], c["Hv"], c["Dk"], c["Dv"]
    cut = row.split([Hk * Dk, Hk * Dk, Hv * Dv], dim=2)
    return [a.unflatten(2, n) for a, n in zip(cut, ((Hk, Dk), (Hk, Dk), (Hv, Dv)))]


def _decays(Hv):
    """Logarithms of the heads' decays: half-lives from one token to a thousand."""
    return -(0.7 * torch.exp2(-10.0 * torch.arange(Hv, device=DEV) / max(1, Hv - 1)))


def _lin_inputs(c, seed):
    g = _generator(seed)
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)
    T, B, Hk, Hv, Dk, Dv = (c[n] for n in ("T", "B", "Hk", "Hv", "Dk", "Dv"))
    op = _type(c["dtype"])
    # a feature map has gone over q and k: mostly positive, so that sums grow
    parts = [torch.nn.functional.silu(normal(T, B, Hk, Dk)).to(op),
             torch.nn.functional.silu(normal(T, B, Hk, Dk)).to(op), normal(T, B, Hv, Dv).to(op)]
    d = {}
    if c["fused"]:
        parts = _slices(c, torch.cat([p.reshape(T, B, -1) for p in parts], dim=2))
    d["q"], d["k"], d["v"] = parts
    d["g"] = _decays(Hv)
    d["S0"] = normal(B, Hv, Dk, Dv) if c["state"] else None
    d["seq_len"] = torch.tensor(_lengths(c, seed), dtype=torch.int32, device=DEV)
    if c["mode"] == "train":
        d["dy"] = normal(T, B, Hv, Dv).to(op)
        d["dST"] = normal(B, Hv, Dk, Dv) * 0.1 if c["state"] else None
    return d


def _step_inputs(c, seed):
    g = _generator(seed)
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)
    B, Hk, Hv, Dk, Dv, op = c["B"], c["Hk"], c["Hv"], c["Dk"], c["Dv"], _type(c["dtype"])
    d = dict(q=torch.nn.functional.silu(normal(B, Hk, Dk)).to(op),
             k=torch.nn.functional.silu(normal(B, Hk, Dk)).to(op), v=normal(B, Hv, Dv).to(op))
    d["g"] = _decays(Hv)
    d["S"] = normal(c["slots"], Hv, Dk, Dv)
    at = torch.randperm(c["slots"], device=DEV, generator=g)[:B].to(torch.int32)
    if B > 2:
        at[B // 2] = -1                      # a place of the batch that no sequence holds
    d["slots"] = at
    return d


def _embed_inputs(c, seed):
    """Tokens as text has them: the r-th most frequent about 1 / r of the time,
    frequent ones anywhere in the vocabulary, the padding at the end."""
    g = _generator(seed)
    N, V, D = c["N"], c["V"], c["D"]
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)
    rank = torch.exp(torch.rand(N, device=DEV, generator=g) * math.log(V)).long().clamp(1, V) - 1
    t = torch.randperm(V, device=DEV, generator=g)[rank].to(torch.int32)
    if c["skip"]:
        t[N - int(N * c["skip"]):] = -1
    d = dict(tokens=t, table=(normal(V, D) * 0.5).to(_type(c["table"])))
    if c["mode"] != "lookup":
        d["dx"] = normal(N, D).to(_type(c["dx"]))
        # what the gradient of the tied logits has left there
        d["dtable"] = ((normal(V, D) if c["mode"] == "tied" else torch.zeros(V, D, device=DEV))
                       .to(_type(c["grad"])))
    return d


def _beam_inputs(c, seed):
    """Beams some steps into their search: unequal scores, some finished, one
    search at its first step (a single beam that counts)."""
    g = _generator(seed)
    B, K, V, op = c["B"], c["K"], c["V"], _type(c["dtype"])
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)
    x = (normal(B * K, V) * 2.5).to(op)
    if c["masked"]:                          # the vocabulary's padding, and words not allowed
        half = c["masked"] // 2
        x[:, V - c["masked"]:] = torch.finfo(op).min
        x[:, V - c["masked"]:V - half] = -math.inf
    scores = -(20 + 2 * torch.rand(B, K, device=DEV, generator=g)).sort(1).values
    lengths = torch.randint(5, 200, (B, 1), device=DEV, generator=g).expand(B, K).contiguous()
    done = torch.zeros(B, K, dtype=torch.int32, device=DEV)
    if c["eos"] >= 0:
        done = (torch.rand(B, K, device=DEV, generator=g) < 0.15).to(torch.int32)
        lengths = lengths - done * torch.randint(0, 5, (B, K), device=DEV, generator=g)
    if B > 2:
        scores[1, 0], scores[1, 1:], done[1], lengths[1] = 0.0, -math.inf, 0, 0
    d = dict(logits=x, scores=scores, finished=done, lengths=lengths.to(torch.int32))
    d["history"] = torch.randint(0, V, (B * K, c["hist"]), device=DEV, generator=g).to(torch.int32)
    d["S"] = normal(c["slots"], c["H"], c["D"], c["D"])
    d["slots"] = torch.randperm(c["slots"], device=DEV, generator=g)[:B * K].view(B, K).to(torch.int32)
    return d


# --------------------------------------------------------------------------
# what a program keeps between calls
# --------------------------------------------------------------------------
def prepare(case, seed):
    c = case
    make = {"linattn": _lin_inputs, "linattn_step": _step_inputs, "embed": _embed_inputs,
            "beam": _beam_inputs}[c["op"]]
    s = dict(make(c, seed), case=c)
    new = lambda *n, t=torch.float32: torch.empty(*n, dtype=t, device=DEV)
    if c["op"] == "linattn":
        T, B, Hv, Dk, Dv, op = c["T"], c["B"], c["Hv"], c["Dk"], c["Dv"], _type(c["dtype"])
        s["y"], s["ST"] = new(T, B, Hv, Dv, t=op), new(B, Hv, Dk, Dv)
        if c["mode"] == "train":
            if c["fused"]:
                width = 2 * c["Hk"] * Dk + Hv * Dv
                s["dq"], s["dk"], s["dv"] = _slices(c, new(T, B, width, t=op))
            else:
                s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in ("q", "k", "v"))
            s["dS0"] = new(B, Hv, Dk, Dv)
    elif c["op"] == "linattn_step":
        s["y"] = new(c["B"], c["Hv"], c["Dv"], t=_type(c["dtype"]))
    elif c["op"] == "embed":
        s["x"] = new(c["N"], c["D"], t=_type(c["x"]))
    else:
        B, K = c["B"], c["K"]
        for n in ("parents", "tokens", "finished_out", "lengths_out", "slots_out"):
            s[n] = new(B, K, t=torch.int32)
        s["scores_out"] = new(B, K)
    if own:
        _plan(c, s)
    return s


def _plan(c, s):
    from paper_1805_01772_amd import lstmloop as ll
    if c["op"] == "linattn":
        tokens = ("q", "k", "v") + (("dq", "dk", "dv") if c["mode"] == "train" else ())
        ld = {n + "_ld": s[n].stride(1) for n in tokens}
        s["plan"] = ll.LinattnPlan(c["T"], c["B"], c["Hk"], c["Hv"], c["Dk"], c["Dv"],
                                   dtype=c["dtype"], inference=c["mode"] == "infer", **ld)
    elif c["op"] == "embed":
        s["plan"] = ll.EmbedPlan(c["N"], c["V"], c["D"], table_dtype=c["table"], x_dtype=c["x"],
                                 dx_dtype=c["dx"], grad_dtype=c["grad"], scale=c["scale"],
                                 inference=c["mode"] == "lookup")
    elif c["op"] == "beam":
        s["plan"] = ll.BeamPlan(c["B"], c["K"], c["V"], dtype=c["dtype"], eos=c["eos"],
                                length_penalty=c["penalty"])


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state["case"], state)


def _run_own(c, s):
    from paper_1805_01772_amd import lstmloop as ll
    if c["op"] == "linattn":
        train = c["mode"] == "train"
        ins = (s["q"], s["k"], s["v"], s["g"], s["seq_len"])
        s["plan"].fwd(*ins, s["S0"], s["y"], s["ST"], save_for_backward=train)
        res = dict(y=s["y"], ST=s["ST"])
        if train:
            s["plan"].bwd(*ins, s["dy"], s["dST"], s["dq"], s["dk"], s["dv"], s["dS0"])
            res.update({n: s[n] for n in ("dq", "dk", "dv", "dS0")})
        return res
    if c["op"] == "linattn_step":
        ll.linattn_loop_step(s["q"], s["k"], s["v"], s["g"], s["S"], s["y"], slots=s["slots"])
        return dict(y=s["y"], S=s["S"])
    if c["op"] == "embed":
        s["plan"].fwd(s["table"], s["tokens"], s["x"])
        res = dict(x=s["x"])
        if c["mode"] != "lookup":
            s["plan"].bwd(s["tokens"], s["dx"], s["dtable"], accumulate=c["mode"] == "tied")
            res["dtable"] = s["dtable"]
        return res
    s["plan"].select(s["logits"], s["scores"], s["finished"], s["lengths"], s["parents"],
                     s["tokens"], s["scores_out"], s["finished_out"], s["lengths_out"])
    ll.ll_beam_reorder(s["parents"], [s["history"]])
    ll.ll_beam_reorder(s["parents"], [s["S"]], slots=s["slots"], slots_out=s["slots_out"])
    return _beam_result(s)


def _beam_result(s):
    return {n: s[n] for n in ("parents", "tokens", "scores_out", "finished_out", "lengths_out",
                              "history", "S", "slots_out")}


def _run_plain(c, s):
    return {"linattn": _plain_lin_pass, "linattn_step": _plain_step, "embed": _plain_embed,
            "beam": _plain_beam}[c["op"]](c, s)


# ------------------------------------------- linear attention with decays
def _plain_lin(q, k, v, g, S, seq_len):
    """S_t = e^g S_{t-1} + k_t v_t^T, y_t = S_t^T q_t / sqrt(Dk), by chunks of C
    tokens: everything inside the chunks at once, then the state from chunk to
    chunk (a loop that a recurrence in this form cannot do without)."""
    T, B, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    n = -(-T // C)
    dead = torch.arange(n * C, device=q.device)[:, None] >= seq_len[None, :]

    def lay(a):                              # [T, B, H, D] -> [B, Hv, n, C, D], 0 past the end
        a = torch.cat([a, a.new_zeros(n * C - T, *a.shape[1:])])
        a = torch.where(dead[..., None, None], 0.0, a)
        a = a.repeat_interleave(Hv // a.shape[2], dim=2)
        return a.unflatten(0, (n, C)).permute(2, 3, 0, 1, 4).contiguous()

    q, k, v = lay(q / math.sqrt(Dk)), lay(k), lay(v)
    i = torch.arange(C, device=q.device)
    far = i[:, None] - i[None, :]
    # weights by distance; how many tokens of the chunk a row has decides the state's
    decay = torch.where(far >= 0, (g[:, None, None] * far.clamp(min=0)).exp(), 0.0)[:, None]
    live = (seq_len[:, None] - C * torch.arange(n, device=q.device)).clamp(0, C)   # [B, n]
    left = (live[..., None] - 1 - i).clamp(min=0)                                  # [B, n, C]
    inside = (decay * (q @ k.transpose(-1, -2).contiguous())) @ v
    qd = q * (g[:, None, None] * (i + 1)[:, None]).exp()[:, None]
    kd = k * (g[:, None, None, None] * left[:, None, :, :, None]).exp()
    KV = kd.transpose(-1, -2).contiguous() @ v
    end = (g[:, None] * live[:, None, :]).exp()[..., None, None]                   # [B, Hv, n, 1, 1]
    ys = []
    for j in range(n):
        ys.append(qd[:, :, j] @ S)
        S = end[:, :, j] * S + KV[:, :, j]
    y = (torch.stack(ys, 2) + inside).permute(2, 3, 0, 1, 4).reshape(n * C, B, Hv, Dv)[:T]
    return torch.where(dead[:T, :, None, None], 0.0, y), S


def _plain_lin_pass(c, s):
    train = c["mode"] == "train"
    f = lambda a: a.detach().float().requires_grad_(train)
    S0 = s["S0"] if c["state"] else torch.zeros_like(s["ST"])
    ins = [f(a) for a in (s["q"], s["k"], s["v"], S0)]
    op = _type(c["dtype"])
    with torch.set_grad_enabled(train):
        y, ST = _plain_lin(*ins[:3], s["g"], ins[3], s["seq_len"])
    res = dict(y=y.detach().to(op), ST=ST.detach())
    if train:
        outs, grads = [y], [s["dy"].float()]
        if c["state"]:
            outs, grads = outs + [ST], grads + [s["dST"]]
        got = torch.autograd.grad(outs, ins, grads)
        res.update({n: a.to(t) for n, a, t in zip(("dq", "dk", "dv", "dS0"), got,
                                                  (op, op, op, torch.float32))})
    return res


def _plain_step(c, s):
    r = c["Hv"] // c["Hk"]
    q = s["q"].float().repeat_interleave(r, 1) / math.sqrt(c["Dk"])
    k, v = s["k"].float().repeat_interleave(r, 1), s["v"].float()
    held = s["slots"] >= 0
    at = s["slots"].clamp(min=0).long()
    S = s["S"][at] * s["g"].exp()[None, :, None, None] + k[..., None] * v[..., None, :]
    y = torch.where(held[:, None, None], (S * q[..., None]).sum(-2), 0.0)
    # a place without a sequence writes to no state: the others' slots only
    s["S"].index_copy_(0, at[held], S[held])
    return dict(y=y.to(_type(c["dtype"])), S=s["S"])


# -------------------------------------------------------------- embedding
def _plain_embed(c, s):
    t = s["tokens"].long()
    held = t >= 0
    x = torch.where(held[:, None], s["table"][t.clamp(min=0)].float() * c["scale"], 0.0)
    res = dict(x=x.to(_type(c["x"])))
    if c["mode"] != "lookup":
        # a frequent token's row is a sum of thousands: 64 bits
        d = torch.zeros(c["V"], c["D"], dtype=torch.float64, device=DEV)
        # places without a token add zeros, to rows apart from each other
        at = torch.where(held, t, torch.arange(c["N"], device=DEV) % c["V"])
        d.index_add_(0, at, torch.where(held[:, None], s["dx"].double(), 0.0))
        d = d * c["scale"]
        if c["mode"] == "tied":
            d = d + s["dtable"]
        s["dtable"].copy_(d)
        res["dtable"] = s["dtable"]
    return res


# ------------------------------------------------------------ beam search
def _penalty(lengths, alpha):
    """What a score is divided by to rank hypotheses of unequal length."""
    return ((5.0 + lengths.double()) / 6.0) ** alpha


def _plain_beam(c, s):
    B, K, V, eos = c["B"], c["K"], c["V"], c["eos"]
    x = s["logits"].float()
    m = x.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    # scores of different beams are compared: 64 bits from the sum on
    ls = (x - m).exp().sum(1, dtype=torch.float64).log()
    # the K most likely of every beam, equal ones by index
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    keys = (order << 32) + (0x7FFFFFFF - torch.arange(V, device=DEV))
    ids = 0x7FFFFFFF - (keys.topk(K, dim=1).values & 0xFFFFFFFF)
    logp = ((x.gather(1, ids).double() - m.double()) - ls[:, None]).view(B, K, K)
    ids = ids.view(B, K, K)
    score = s["scores"].double()[..., None] + logp
    length = (s["lengths"] + 1)[..., None].expand(B, K, K)
    done = s["finished"].bool()[..., None]
    # a finished beam goes on as it is, in one place
    first = torch.arange(K, device=DEV) == 0
    score = torch.where(done, torch.where(first, s["scores"].double()[..., None], -math.inf), score)
    length = torch.where(done, s["lengths"][..., None], length)
    ids = torch.where(done, max(eos, 0), ids)
    rank = (score / _penalty(length, c["penalty"])).view(B, K * K)
    at = (torch.arange(K, device=DEV)[:, None] * V + ids).view(B, K * K)
    # by rank, equal ones by beam and token
    by = at.sort(1).indices
    by = by.gather(1, rank.gather(1, by).sort(dim=1, descending=True, stable=True).indices)[:, :K]
    pick = lambda a: a.expand(B, K, K).reshape(B, K * K).gather(1, by)
    some = pick(score) > -math.inf           # a place for which there is no candidate
    own_place = torch.arange(K, device=DEV).expand(B, K)
    i32 = lambda a: a.to(torch.int32)
    s["parents"].copy_(torch.where(some, by // K, own_place))
    s["tokens"].copy_(torch.where(some, pick(ids), -1))
    s["scores_out"].copy_(torch.where(some, pick(score), -math.inf))
    s["finished_out"].copy_(some & (pick(done) | (pick(ids) == eos)))
    s["lengths_out"].copy_(torch.where(some, pick(length), s["lengths"].gather(1, own_place)))
    _plain_reorder(c, s)
    return _beam_result(s)


def _plain_reorder(c, s):
    B, K = c["B"], c["K"]
    p = s["parents"].long()
    row = torch.arange(B, device=DEV)[:, None] * K
    s["history"].copy_(s["history"][(row + p).view(-1)])
    # in the pool a beam's first successor keeps its state, the others copy it into the
    # states of beams that have none
    k = torch.arange(K, device=DEV)
    child = p[:, :, None] == k                                   # [B, place, beam]
    first = ~((p[:, :, None] == p[:, None, :]) & (k[:, None] > k[None, :])).any(2)
    free = ~child.any(1)
    nth_free = torch.where(free, k, K).sort(1).values            # free beams in order
    nth = (~first).cumsum(1) - 1                                 # number of this copy
    old = s["slots"].long()
    dst = old.gather(1, nth_free.gather(1, nth.clamp(min=0)).clamp(max=K - 1))
    src = old.gather(1, p)
    s["slots_out"].copy_(torch.where(first, src, dst))
    s["S"][dst[~first]] = s["S"][src[~first]]


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    c = case
    size = lambda name: 2 if name == "bf16" else 4
    if c["op"] == "embed":
        N, V, D = c["N"] * (1 - c["skip"]), c["V"], c["D"]
        # rows of the table that occur, by the tokens' distribution
        seen = V * (1 - math.exp(-N / V)) if N < 64 else sum(
            (1 - math.exp(-N * p)) * w for p, w in _shares(V))
        by = seen * D * size(c["table"]) + c["N"] * (D * size(c["x"]) + 4)
        fl = c["N"] * D
        if c["mode"] != "lookup":
            by += N * D * size(c["dx"]) + c["N"] * 4
            by += (V if c["mode"] == "train" else 2 * seen) * D * size(c["grad"])
            fl += N * D
        return {"bytes": by, "flops": float(fl)}
    es = size(c["dtype"])
    if c["op"] == "beam":
        rows = c["B"] * c["K"]
        live = rows * (0.85 if c["eos"] >= 0 else 1.0)
        # beams that take another's state: about half of them here
        moved = 0.5 * rows * (1 - 1 / c["K"])
        return {"bytes": live * c["V"] * es + 2 * moved * (4 * c["hist"] + 4 * c["H"] * c["D"] ** 2)
                + rows * 40, "flops": 4.0 * live * c["V"]}
    Hk, Hv, Dk, Dv = c["Hk"], c["Hv"], c["Dk"], c["Dv"]
    tok = 2 * Hk * Dk * es + 2 * Hv * Dv * es
    if c["op"] == "linattn_step":
        n = c["B"]
        return {"bytes": n * (tok + 8 * Hv * Dk * Dv + 4), "flops": 5.0 * n * Hv * Dk * Dv}
    # the recurrence's own operations: the outer product and S q; in the gradient S dy, and
    # for the other state the outer product and a product for each of dk and dv
    n = c["B"] * (c["lo"] + c["T"]) / 2.0
    state = 4 * c["B"] * Hv * Dk * Dv * (2 if c["state"] else 1)
    by, fl = n * tok + state, 4.0 * n * Hv * Dk * Dv
    if c["mode"] == "train":
        by += n * (tok + Hv * Dv * es) + state
        fl *= 3
    return {"bytes": by, "flops": fl}


def _shares(V):
    """(probability of a token, how many such) of _embed_inputs' distribution:
    rank r has log(1 + 1 / r) / log V."""
    r, out = 1, []
    while r < V:
        w = max(1, r // 8)
        out.append((math.log1p(1 / (r + w / 2.0 - 0.5)) / math.log(V), min(w, V - r)))
        r += w
    return out


# --------------------------------------------------------------------------
# the same outputs in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    return {"linattn": _exact_lin, "linattn_step": _exact_step, "embed": _exact_embed,
            "beam": _exact_beam}[case["op"]](case, seed)


def _exact_lin(c, seed):
    """Every pair of tokens: y_t = sum_{i <= t} e^{g (t - i)} (q_t.k_i) v_i / sqrt(Dk) + the
    state's part, row by row of the batch, R tokens against all at a time."""
    d = _lin_inputs(c, seed)
    T, B, Hk, Hv, Dk, Dv = (c[n] for n in ("T", "B", "Hk", "Hv", "Dk", "Dv"))
    r, scale, R = Hv // Hk, 1.0 / math.sqrt(Dk), 512
    new = lambda *n: torch.zeros(*n, dtype=torch.float64, device=DEV)
    train = c["mode"] == "train"
    heads = lambda a: a.double().transpose(0, 1).contiguous()    # [L, H, D] -> [H, L, D]
    back = lambda a: a.transpose(0, 1)
    t_ = lambda a: a.transpose(-1, -2).contiguous()
    g = d["g"].double()[:, None, None]
    y, ST = new(T, B, Hv, Dv), new(B, Hv, Dk, Dv)
    dq, dk, dv, dS0 = new(T, B, Hv, Dk), new(T, B, Hv, Dk), new(T, B, Hv, Dv), new(B, Hv, Dk, Dv)
    for b, L in enumerate(_lengths(c, seed)):
        S0 = d["S0"][b].double() if c["state"] else new(Hv, Dk, Dv)
        dST = d["dST"][b].double() if train and c["state"] else new(Hv, Dk, Dv)
        q = heads(d["q"][:L, b]).repeat_interleave(r, 0) * scale
        k = heads(d["k"][:L, b]).repeat_interleave(r, 0)
        v = heads(d["v"][:L, b])
        pos = torch.arange(L, dtype=torch.float64, device=DEV)[:, None]
        to_end = (g * (L - 1 - pos)).exp()
        from_start = (g * (pos + 1)).exp()
        ST[b] = (g * L).exp() * S0 + t_(k * to_end) @ v
        if train:
            dy = heads(d["dy"][:L, b])
            dq[:L, b] = back(from_start * (dy @ t_(S0)))
            dk[:L, b] = back(to_end * (v @ t_(dST)))
            dv[:L, b] = back(to_end * (k @ dST))
            dS0[b] = (g * L).exp() * dST + t_(q * from_start) @ dy
        for i in range(0, L, R):
            n = min(R, L - i)
            far = pos[i:i + n] - pos[:i + n].T
            w = torch.where(far >= 0, (g * far.clamp(min=0)).exp(), 0.0)
            P = w * (q[:, i:i + n] @ t_(k[:, :i + n]))
            y[i:i + n, b] = back(P @ v[:, :i + n] + from_start[:, i:i + n] * (q[:, i:i + n] @ S0))
            if train:
                F = w * (dy[:, i:i + n] @ t_(v[:, :i + n]))
                dq[i:i + n, b] += back(F @ k[:, :i + n])
                dk[:i + n, b] += back(t_(F) @ q[:, i:i + n])
                dv[:i + n, b] += back(t_(P) @ dy[:, i:i + n])
    res = dict(y=y, ST=ST)
    if train:
        shared = lambda a: a.unflatten(2, (Hk, r)).sum(3)        # a key head serves r value heads
        res.update(dq=shared(dq) * scale, dk=shared(dk), dv=dv, dS0=dS0)
    return res


def _exact_step(c, seed):
    d = _step_inputs(c, seed)
    f = lambda a: a.double()
    r = c["Hv"] // c["Hk"]
    S, y = f(d["S"]), torch.zeros(c["B"], c["Hv"], c["Dv"], dtype=torch.float64, device=DEV)
    rows = torch.nonzero(d["slots"] >= 0)[:, 0]
    at = d["slots"][rows].long()
    k, q = (f(d[n][rows]).repeat_interleave(r, 1) for n in ("k", "q"))
    S[at] = (S[at] * f(d["g"]).exp()[:, None, None]
             + torch.einsum("bhk,bhv->bhkv", k, f(d["v"][rows])))
    y[rows] = torch.einsum("bhkv,bhk->bhv", S[at], q) / math.sqrt(c["Dk"])
    return dict(y=y, S=S)


def _exact_embed(c, seed):
    """Sums over sorted tokens: differences of the running sum at the borders
    of each token's run, some columns at a time."""
    d = _embed_inputs(c, seed)
    t = d["tokens"].long()
    x = d["table"].double()[t.clamp(min=0)] * c["scale"]
    x[t < 0] = 0.0
    res = dict(x=x)
    if c["mode"] != "lookup":
        order = t.argsort(stable=True)
        order = order[(t < 0).sum():]
        ends = torch.bincount(t[order], minlength=c["V"]).cumsum(0)
        cols = []
        for j in range(0, c["D"], 256):
            run = d["dx"][:, j:j + 256][order].double().cumsum(0)
            run = torch.cat([run.new_zeros(1, run.shape[1]), run])
            at = run[ends]
            cols.append(torch.cat([at[:1], at[1:] - at[:-1]]) * c["scale"])
        res["dtable"] = torch.cat(cols, 1)
        if c["mode"] == "tied":
            res["dtable"] += d["dtable"]
    return res


def _exact_beam(c, seed):
    """Scores from the definition, over every candidate of a search at once;
    choices are whole numbers and held to the plain form's."""
    d = _beam_inputs(c, seed)
    B, K, V = c["B"], c["K"], c["V"]
    out = torch.empty(B, K, dtype=torch.float64, device=DEV)
    for b in range(B):
        lp = torch.log_softmax(d["logits"][b * K:(b + 1) * K].double(), 1)
        score = d["scores"][b].double()[:, None] + lp
        length = (d["lengths"][b] + 1).double()[:, None].expand(K, V).clone()
        over = d["finished"][b].bool()
        score[over] = -math.inf
        score[over, max(c["eos"], 0)] = d["scores"][b].double()[over]
        length[over] = d["lengths"][b].double()[over][:, None]
        rank = (score / ((5.0 + length) / 6.0) ** c["penalty"]).flatten()
        out[b] = score.flatten()[rank.topk(K).indices]
    res = {n: None for n in ("parents", "tokens", "scores_out", "finished_out", "lengths_out",
                             "history", "S", "slots_out")}
    res["scores_out"] = out
    return res
