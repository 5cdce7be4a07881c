"""Performance cases of the operators around the loops: the gated delta rule
(a recurrence whose state is a matrix per head), the log probabilities a
sequence model is trained and scored by, and the AdamW step over its tensors.

``listed`` names the cases, ``draw`` gives more of the same ranges,
``prepare`` makes what a program holds before the call, ``run`` is one pass,
``work`` the bytes and operations the call cannot do without and ``exact``
the same outputs in 64 bits.  With ``own`` false ``run`` computes the
operators from elementary torch operations in 32 bits.

Keys of a case: ``op`` (delta / delta_step / logprob / adamw) and

- delta: ``mode`` (train / infer), ``dtype``, sizes ``T``, ``B``, ``Hk``,
  ``Hv``, ``Dk``, ``Dv``, lengths drawn from ``lo`` .. ``hi``, ``state``
  (random initial state instead of none), ``fused`` (q, k and v are slices of
  one projection's rows);
- delta_step: ``slots`` states in the pool, ``B`` of them advanced;
- logprob: ``mode`` (train / policy, which has its gradient in a call of its
  own, / score), ``dtype``, ``N`` rows, ``V`` columns,
  ``top`` alternatives, ``masked`` columns at the lowest value of the type
  or minus infinity;
- adamw: ``tensors`` of ``lo`` .. ``hi`` elements, ``bits`` of the states,
  ``grad`` type, ``copy`` (a bfloat16 copy of the parameters is written).
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
C = 64                 # tokens per chunk of the plain form
QB = 256               # elements per scale of an 8-bit state
B1, B2, EPS = 0.9, 0.95, 1e-8


def _delta(name, mode, dtype, T, B, Hk, Hv, Dk, Dv, lo, state=False, fused=False):
    return dict(name=name, op="delta", mode=mode, dtype=dtype, T=T, B=B, Hk=Hk, Hv=Hv, Dk=Dk,
                Dv=Dv, lo=lo, hi=T, state=state, fused=fused)


def _step(name, dtype, slots, B, Hk, Hv, Dk, Dv):
    return dict(name=name, op="delta_step", dtype=dtype, slots=slots, B=B, Hk=Hk, Hv=Hv, Dk=Dk,
                Dv=Dv)


def _logprob(name, mode, dtype, N, V, top, masked):
    return dict(name=name, op="logprob", mode=mode, dtype=dtype, N=N, V=V, top=top, masked=masked)


def _adamw(name, tensors, lo, hi, bits, grad, copy, sizes):
    return dict(name=name, op="adamw", tensors=tensors, lo=lo, hi=hi, bits=bits, grad=grad,
                copy=copy, sizes=sizes)


def listed():
    return [
        # one token for a few sequences: the latency of a serving step
        _step("delta_step_b4_f32", "f32", 4, 4, 2, 4, 32, 32),
        # one token for a full serving batch out of a larger pool of states
        _step("delta_step_b256_bf16", "bf16", 320, 256, 16, 32, 128, 128),
        # prompts of unequal length read into fresh states
        _delta("delta_infer_ragged_bf16", "infer", "bf16", 1000, 4, 8, 16, 128, 128, 100),
        # a float32 training step at the width of the 512-unit models, short odd lengths
        # (none among them), sizes of a head that are no power of two
        _delta("delta_train_t100_f32", "train", "f32", 100, 64, 4, 8, 64, 72, 0, state=True),
        # an ordinary training step: q, k and v from one projection, shared key heads
        _delta("delta_train_t2048_bf16", "train", "bf16", 2048, 8, 8, 16, 128, 128, 256,
               fused=True),
        # one long sequence: few rows, many steps
        _delta("delta_train_long_bf16", "train", "bf16", 16384, 1, 16, 16, 128, 128, 16384,
               state=True),
        # scoring a few rows with the most likely alternatives: latency, a long axis
        _logprob("logprob_score_n8_bf16", "score", "bf16", 8, 32000, 8, 100),
        # scoring prompts, rows of an odd width
        _logprob("logprob_score_n2047_f32", "score", "f32", 2047, 50001, 16, 0),
        # the loss of a training step with its gradient, a large vocabulary
        _logprob("logprob_train_n4096_bf16", "train", "bf16", 4096, 131072, 0, 72),
        # a small model: many small tensors, where launches count
        _adamw("adamw_small_f32", 48, 33, 65536, 32, "f32", False, 1),
        # a large model, states in 32 bits, bfloat16 operands written beside the masters
        _adamw("adamw_large_f32", 40, 1 << 20, 1 << 24, 32, "f32", True, 2),
        # the same with states in 8 bits and bfloat16 gradients
        _adamw("adamw_large_q8", 40, 1 << 20, 1 << 24, 8, "bf16", True, 2),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, min(hi // step * step, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["delta", "delta", "infer", "step", "score", "train", "policy", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    for _ in range(10000):
        if kind in ("delta", "infer", "step"):
            Hk = rng.choice([1, 2, 3, 4, 8, 16])
            Hv = Hk * rng.choice([1, 1, 2, 3])
            Dk, Dv = _log_int(rng, 32, 128, 8), _log_int(rng, 32, 128, 8)
            if kind == "step":
                B = _log_int(rng, 1, 256)
                c = _step("", dtype, B + rng.randint(0, 64), B, Hk, Hv, Dk, Dv)
            else:
                T, B = _log_int(rng, 60, 16384), _log_int(rng, 1, 64)
                c = _delta("", "train" if kind == "delta" else "infer", dtype, T, B, Hk, Hv, Dk, Dv,
                           rng.choice([T, T // 8, 0]), state=rng.random() < 0.5,
                           fused=rng.random() < 0.5)
            # no dearer than the largest listed cases of its kind, whose heads are widest
            fits = {"delta": c.get("T", 0) * c["B"] * Hv <= 262144,
                    "infer": c.get("T", 0) * c["B"] * Hv <= 262144,
                    "step": c["B"] * Hv <= 8192}[kind]
        elif kind == "adamw":
            lo = _log_int(rng, 33, 1 << 20)
            hi = _log_int(rng, lo, 1 << 24)
            c = _adamw("", _log_int(rng, 1, 200), lo, hi, rng.choice([32, 8]),
                       rng.choice(["f32", "bf16"]), rng.random() < 0.5, rng.randint(3, 1 << 20))
            fits = sum(_sizes(c)) <= 230 << 20
        else:
            N, V = _log_int(rng, 1, 8192), _log_int(rng, 1000, 200000)
            top = rng.choice([1, 4, 8, 16]) if kind != "train" else 0
            c = _logprob("", kind, dtype, N, V, top, rng.choice([0, rng.randint(1, V // 4)]))
            fits = N * V * (2 if dtype == "bf16" else 4) <= (1 << 30) // (2 if top else 1)
        if fits:
            del c["name"]
            return c
    raise RuntimeError("no case drawn")


def _op_type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _sizes(c):
    r = random.Random(c["sizes"])
    return [_log_int(r, c["lo"], c["hi"]) for _ in range(c["tensors"])]


def _lengths(c, seed):
    r = random.Random(seed * 7919 + 17)
    s = [r.randint(c["lo"], c["hi"]) for _ in range(c["B"])]
    if c["lo"] < c["hi"]:
        s[r.randrange(c["B"])] = c["hi"]     # some sequence fills the batch's padded length
        if c["lo"] == 0 and c["B"] > 1 and min(s) > 0:
            s[s.index(min(s))] = 0           # and one has no token at all
    return s


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 12345)
    return g


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _slices(c, row):
    """q, k and v (or their gradients) as slices of one projection's rows."""
    Hk, Hv, Dk, Dv = c["Hk"], c["Hv"], c["Dk"], c["Dv"]
    cut = row.split([Hk * Dk, Hk * Dk, Hv * Dv], dim=2)
    return [a.unflatten(2, n) for a, n in zip(cut, ((Hk, Dk), (Hk, Dk), (Hv, Dv)))]


def _delta_inputs(c, seed):
    """Keys and queries of unit length, a write strength in (0, 1), decays whose
    half-life runs from a few to a few thousand tokens over the heads."""
    g = _generator(seed)
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)
    rand = lambda *s: torch.rand(*s, device=DEV, generator=g)
    unit = lambda a: a / a.norm(dim=-1, keepdim=True)
    T, B, Hk, Hv, Dk, Dv = (c[n] for n in ("T", "B", "Hk", "Hv", "Dk", "Dv"))
    op = _op_type(c)
    parts = [unit(normal(T, B, Hk, Dk)).to(op), unit(normal(T, B, Hk, Dk)).to(op),
             normal(T, B, Hv, Dv).to(op)]
    d = {}
    if c["fused"]:
        parts = _slices(c, torch.cat([p.reshape(T, B, -1) for p in parts], dim=2))
    d["q"], d["k"], d["v"] = parts
    rate = torch.exp(math.log(0.3) + (math.log(3e-4) - math.log(0.3)) *
                     torch.arange(Hv, device=DEV) / max(1, Hv - 1))
    d["g"] = -rate * (0.5 + rand(T, B, Hv))
    d["beta"] = torch.sigmoid(normal(T, B, Hv))
    d["S0"] = normal(B, Hv, Dk, Dv) * 0.3 if c["state"] else None
    d["seq_len"] = torch.tensor(_lengths(c, seed), dtype=torch.int32, device=DEV)
    if c["mode"] == "train":
        d["dy"] = normal(T, B, Hv, Dv).to(op)
        d["dST"] = normal(B, Hv, Dk, Dv) * 0.1 if c["state"] else None
    return d


def _step_inputs(c, seed):
    g = _generator(seed)
    normal = lambda *s: torch.randn(*s, device=DEV, generator=g)
    unit = lambda a: a / a.norm(dim=-1, keepdim=True)
    B, Hk, Hv, Dk, Dv, op = c["B"], c["Hk"], c["Hv"], c["Dk"], c["Dv"], _op_type(c)
    d = dict(q=unit(normal(B, Hk, Dk)).to(op), k=unit(normal(B, Hk, Dk)).to(op),
             v=normal(B, Hv, Dv).to(op))
    d["g"] = -0.2 * torch.rand(B, Hv, device=DEV, generator=g)
    d["beta"] = torch.sigmoid(normal(B, Hv))
    d["S"] = normal(c["slots"], Hv, Dk, Dv) * 0.3
    at = torch.randperm(c["slots"], device=DEV, generator=g)[:B].to(torch.int32)
    if B > 2:
        at[B // 2] = -1                      # a place of the batch that no sequence holds
    d["slots"] = at
    return d


def _logprob_inputs(c, seed):
    g = _generator(seed)
    N, V, op = c["N"], c["V"], _op_type(c)
    x = (torch.randn(N, V, device=DEV, generator=g) * 2.5).to(op)
    if c["masked"]:                          # the vocabulary's padding, and words not allowed
        half = c["masked"] // 2
        x[:, V - c["masked"]:] = torch.finfo(op).min
        x[:, V - c["masked"]:V - half] = -math.inf
    t = torch.randint(0, V - c["masked"], (N,), device=DEV, generator=g).to(torch.int32)
    if N > 4:
        t[1::7] = -1                         # tokens outside the loss
        x[3] = -math.inf                     # a row in which nothing is allowed
    d = dict(logits=x, targets=t)
    if c["mode"] != "score":
        scale = 1.0 / N
        d["dlogp"] = -scale * (0.5 + torch.rand(N, device=DEV, generator=g))
        d["dentropy"] = -0.01 * scale * torch.rand(N, device=DEV, generator=g)
        d["dtop"] = None
    if c["mode"] == "policy" and c["top"]:   # the alternatives drawn towards a teacher's
        d["dtop"] = scale * torch.randn(N, c["top"], device=DEV, generator=g)
    return d


def _adamw_inputs(c, seed):
    """All tensors in one arena per kind, each on a fresh run of QB elements, so
    that a program may also walk the arena as rows of QB."""
    g = _generator(seed)
    sizes = _sizes(c)
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // QB) * QB
    normal = lambda: torch.randn(at, device=DEV, generator=g)
    ends = torch.tensor([a + n for a, n in zip(starts, sizes)], device=DEV)
    owner = torch.repeat_interleave(torch.arange(len(sizes), device=DEV),
                                    torch.tensor([-(-n // QB) for n in sizes], device=DEV))
    live = torch.arange(at, device=DEV).view(-1, QB) < ends[owner][:, None]
    d = dict(p=normal() * 0.05, grad=normal() * 1e-3)
    for k in ("p", "grad"):
        d[k].view(-1, QB).mul_(live)
    d["grad"] = d["grad"].to(torch.bfloat16 if c["grad"] == "bf16" else torch.float32)
    if c["bits"] == 32:
        d["m"] = normal().mul_(3e-4)
        d["v"] = normal().mul_(1e-3).square_()
        for k in ("m", "v"):
            d[k].view(-1, QB).mul_(live)
    else:
        d["m"] = torch.randint(-127, 128, (at,), device=DEV, generator=g, dtype=torch.int8)
        d["v"] = torch.randint(1, 256, (at,), device=DEV, generator=g, dtype=torch.uint8)
        for k in ("m", "v"):
            d[k].view(-1, QB).mul_(live)
        d["m_scale"] = torch.rand(at // QB, device=DEV, generator=g) * 1e-3
        d["v_scale"] = torch.rand(at // QB, device=DEV, generator=g) * 1e-5
    d["copy"] = torch.zeros(at, dtype=torch.bfloat16, device=DEV) if c["copy"] else None
    d["grad_scale"] = torch.full((1,), 0.75, device=DEV)
    decay = torch.tensor([0.1 if i % 3 else 0.0 for i in range(len(sizes))], device=DEV)
    d["decay"] = decay[owner][:, None]
    d["sizes"], d["starts"] = sizes, starts
    d["hyper"] = dict(lr=1e-3, beta1=B1, beta2=B2, eps=EPS, step=100, seed=seed & 0xFFFF)
    return d


# --------------------------------------------------------------------------
# what a program keeps between calls
# --------------------------------------------------------------------------
def prepare(case, seed):
    c = case
    make = {"delta": _delta_inputs, "delta_step": _step_inputs, "logprob": _logprob_inputs,
            "adamw": _adamw_inputs}[c["op"]]
    s = dict(make(c, seed), case=c)
    new = lambda *n, t=torch.float32: torch.empty(*n, dtype=t, device=DEV)
    if c["op"] == "delta":
        T, B, Hv, Dk, Dv = c["T"], c["B"], c["Hv"], c["Dk"], c["Dv"]
        s["y"], s["ST"] = new(T, B, Hv, Dv, t=_op_type(c)), new(B, Hv, Dk, Dv)
        if c["mode"] == "train":
            if c["fused"]:
                width = 2 * c["Hk"] * Dk + Hv * Dv
                s["dq"], s["dk"], s["dv"] = _slices(c, new(T, B, width, t=_op_type(c)))
            else:
                s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in ("q", "k", "v"))
            s["dg"], s["dbeta"], s["dS0"] = new(T, B, Hv), new(T, B, Hv), new(B, Hv, Dk, Dv)
    elif c["op"] == "delta_step":
        s["y"] = new(c["B"], c["Hv"], c["Dv"], t=_op_type(c))
    elif c["op"] == "logprob":
        N, top = c["N"], c["top"]
        s["logp"], s["entropy"], s["lse"] = new(N), new(N), new(N)
        s["top_ids"] = new(N, top, t=torch.int32) if top else None
        s["top_logp"] = new(N, top) if top else None
        if c["mode"] != "score":
            s["dlogits"] = torch.empty_like(s["logits"])
    if own:
        _plan(c, s)
    return s


def _plan(c, s):
    from paper_1805_01772_amd import lstmloop as ll
    if c["op"] == "delta":
        tokens = ("q", "k", "v") + (("dq", "dk", "dv") if c["mode"] == "train" else ())
        ld = {n + "_ld": s[n].stride(1) for n in tokens}
        s["plan"] = ll.DeltaPlan(c["T"], c["B"], c["Hk"], c["Hv"], c["Dk"], c["Dv"],
                                 dtype=c["dtype"], inference=c["mode"] == "infer", **ld)
    elif c["op"] == "logprob":
        s["plan"] = ll.LogprobPlan(c["N"], c["V"], dtype=c["dtype"], top_k=c["top"])
    elif c["op"] == "adamw":
        cut = lambda a: [a[i:i + n] for i, n in zip(s["starts"], s["sizes"])]
        rows = lambda a: [a[i // QB:i // QB + -(-n // QB)] for i, n in zip(s["starts"], s["sizes"])]
        q8 = c["bits"] == 8
        s["grads"] = cut(s["grad"])
        s["plan"] = ll.AdamWPlan(cut(s["p"]), cut(s["m"]), cut(s["v"]),
                                 m_scale=rows(s["m_scale"]) if q8 else None,
                                 v_scale=rows(s["v_scale"]) if q8 else None,
                                 copies=cut(s["copy"]) if c["copy"] else None,
                                 weight_decay=[0.1 if i % 3 else 0.0 for i in range(c["tensors"])],
                                 grad_dtype=c["grad"])


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state["case"], state)


def _run_own(c, s):
    from paper_1805_01772_amd import lstmloop as ll
    if c["op"] == "delta":
        train = c["mode"] == "train"
        ins = (s["q"], s["k"], s["v"], s["g"], s["beta"], s["seq_len"])
        s["plan"].fwd(*ins, s["S0"], s["y"], s["ST"], save_for_backward=train)
        res = dict(y=s["y"], ST=s["ST"])
        if train:
            s["plan"].bwd(*ins, s["dy"], s["dST"], s["dq"], s["dk"], s["dv"], s["dg"], s["dbeta"],
                          s["dS0"])
            res.update({n: s[n] for n in ("dq", "dk", "dv", "dg", "dbeta", "dS0")})
        return res
    if c["op"] == "delta_step":
        ll.delta_loop_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["S"], s["y"],
                           slots=s["slots"])
        return dict(y=s["y"], S=s["S"])
    if c["op"] == "logprob":
        res = dict(logp=s["logp"], entropy=s["entropy"], lse=s["lse"])
        if c["mode"] == "train":             # the loss's weights are known beforehand
            s["plan"].fwd_bwd(s["logits"], s["targets"], s["dlogp"], s["dentropy"], s["logp"],
                              s["entropy"], s["lse"], s["dlogits"])
        else:
            s["plan"].fwd(s["logits"], s["targets"], s["logp"], s["entropy"], s["lse"],
                          s["top_ids"], s["top_logp"])
        if c["mode"] == "policy":            # the gradient comes after, from values of its own
            s["plan"].bwd(s["logits"], s["targets"], s["lse"], s["entropy"], s["top_ids"],
                          s["dlogp"], s["dentropy"], s["dtop"], s["dlogits"])
        if c["top"]:
            res.update(top_ids=s["top_ids"], top_logp=s["top_logp"])
        if c["mode"] != "score":
            res["dlogits"] = s["dlogits"]
        return res
    s["plan"].step(s["grads"], grad_scale=s["grad_scale"], **s["hyper"])
    return _adamw_result(c, s)


def _adamw_result(c, s):
    res = dict(p=s["p"])
    if c["copy"]:
        res["copy"] = s["copy"]
    if c["bits"] == 32:
        res.update(m=s["m"], v=s["v"])
    else:                                    # the values that the codes stand for
        res["m"], res["v"] = _dequant(s["m"], s["v"], s["m_scale"], s["v_scale"])
    return res


def _run_plain(c, s):
    if c["op"] == "delta":
        return _plain_delta_pass(c, s)
    if c["op"] == "delta_step":
        return _plain_step(c, s)
    if c["op"] == "logprob":
        return _plain_logprob(c, s)
    return _plain_adamw(c, s)


# ---------------------------------------------------- the gated delta rule
def _plain_delta(q, k, v, g, beta, S, seq_len):
    """S_t = e^g_t S_{t-1} + k_t u_t^T, u_t = beta_t (v_t - e^g_t S_{t-1}^T k_t),
    y_t = S_t^T q_t / sqrt(Dk), by chunks of C tokens: everything inside the
    chunks at once, then the state from chunk to chunk (a loop that a
    recurrence in this form cannot do without)."""
    T, B, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    n = -(-T // C)
    dead = torch.arange(n * C, device=q.device)[:, None] >= seq_len[None, :]

    def lay(a):                              # [T, B, H, ..] -> [B, Hv, n, C, ..], 0 past the end
        a = torch.cat([a, a.new_zeros(n * C - T, *a.shape[1:])])
        a = torch.where(dead.view(n * C, B, *([1] * (a.dim() - 2))), 0.0, a)
        a = a.repeat_interleave(Hv // a.shape[2], dim=2)
        return a.unflatten(0, (n, C)).permute(2, 3, 0, 1, *range(4, a.dim() + 1)).contiguous()

    q, k, v, g, beta = lay(q / math.sqrt(Dk)), lay(k), lay(v), lay(g), lay(beta)
    G = g.cumsum(-1)
    low = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
    decay = torch.where(low, G[..., :, None] - G[..., None, :], -math.inf).exp()
    kt = k.transpose(-1, -2).contiguous()
    A = torch.where(low.tril(-1), beta[..., None] * decay * (k @ kt), 0.0)
    P = decay * (q @ kt)
    eye = torch.eye(C, device=q.device)
    A2 = A @ A
    A4 = A2 @ A2
    A8 = A4 @ A4
    A16 = A8 @ A8
    inv = (eye - A) @ (eye + A2) @ (eye + A4) @ (eye + A8) @ (eye + A16) @ (eye + A16 @ A16)
    eG = G.exp()[..., None]
    U = inv @ (beta[..., None] * v)
    W = inv @ (beta[..., None] * eG * k)
    qd = q * eG
    kd = (k * (G[..., -1:] - G).exp()[..., None]).transpose(-1, -2).contiguous()
    end = G[..., -1].exp()[..., None, None]
    ys = []
    for i in range(n):
        u = U[:, :, i] - W[:, :, i] @ S
        ys.append(qd[:, :, i] @ S + P[:, :, i] @ u)
        S = end[:, :, i] * S + kd[:, :, i] @ u
    y = torch.stack(ys, 2).permute(2, 3, 0, 1, 4).reshape(n * C, B, Hv, Dv)[:T]
    return torch.where(dead[:T, :, None, None], 0.0, y), S


def _plain_delta_pass(c, s):
    train = c["mode"] == "train"
    f = lambda a: a.float().requires_grad_(train)
    S0 = s["S0"] if c["state"] else torch.zeros_like(s["ST"])
    ins = [f(a.detach()) for a in (s["q"], s["k"], s["v"], s["g"], s["beta"], S0)]
    op = _op_type(c)
    with torch.set_grad_enabled(train):
        y, ST = _plain_delta(*ins, s["seq_len"])
    res = dict(y=y.detach().to(op), ST=ST.detach())
    if train:
        outs, grads = [y], [s["dy"].float()]
        if c["state"]:
            outs, grads = outs + [ST], grads + [s["dST"]]
        got = torch.autograd.grad(outs, ins, grads)
        types = (op, op, op, torch.float32, torch.float32, torch.float32)
        res.update({n: a.to(t) for n, a, t in zip(("dq", "dk", "dv", "dg", "dbeta", "dS0"), got,
                                                  types)})
    return res


def _plain_step(c, s):
    r = c["Hv"] // c["Hk"]
    q = s["q"].float().repeat_interleave(r, 1) / math.sqrt(c["Dk"])
    k, v = s["k"].float().repeat_interleave(r, 1), s["v"].float()
    held = (s["slots"] >= 0)[:, None, None]
    at = s["slots"].clamp(min=0).long()
    old = s["S"][at]
    S = old * s["g"].exp()[..., None, None]
    u = s["beta"][..., None] * (v - (S * k[..., None]).sum(-2))
    S = S + k[..., None] * u[..., None, :]
    y = torch.where(held, (S * q[..., None]).sum(-2), 0.0)
    # a place without a sequence writes to no state: the others' slots only
    s["S"].index_copy_(0, at[s["slots"] >= 0], S[s["slots"] >= 0])
    return dict(y=y.to(_op_type(c)), S=s["S"])


# ------------------------------------------------------ log probabilities
def _plain_logprob(c, s):
    x = s["logits"].float()
    t = s["targets"].long()
    m = x.amax(1, keepdim=True)
    none = m == -math.inf                    # rows in which nothing is allowed
    e = (x - torch.where(none, 0.0, m)).exp()
    z = e.sum(1, keepdim=True)
    lse = torch.where(none, -math.inf, m + z.log())
    p = torch.where(none, 0.0, e / z)
    lp = torch.where(x == -math.inf, 0.0, x - lse)
    ent = -(p * lp).sum(1)
    at = x.gather(1, t.clamp(min=0)[:, None])
    # a word that is not allowed has log probability minus infinity
    logp = torch.where(at == -math.inf, -math.inf, at - lse)[:, 0]
    res = dict(logp=torch.where(t < 0, 0.0, logp), entropy=ent, lse=lse[:, 0])
    if c["top"]:                             # largest first, equal ones by index
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        keys = (order << 32) + (0x7FFFFFFF - torch.arange(x.shape[1], device=x.device))
        ids = 0x7FFFFFFF - (keys.topk(c["top"], dim=1).values & 0xFFFFFFFF)
        top = x.gather(1, ids)
        res["top_ids"] = ids.to(torch.int32)
        res["top_logp"] = torch.where(top == -math.inf, -math.inf, top - lse)
    if c["mode"] != "score":
        dl = torch.where(t < 0, 0.0, s["dlogp"])[:, None]
        every = dl + s["dtop"].sum(1, keepdim=True) if s["dtop"] is not None else dl
        d = -p * (every + s["dentropy"][:, None] * (lp + ent[:, None]))
        d.scatter_add_(1, t.clamp(min=0)[:, None], dl)
        if s["dtop"] is not None:
            d.scatter_add_(1, ids, s["dtop"])
        res["dlogits"] = torch.where(none, 0.0, d).to(_op_type(c))
    return res


# ------------------------------------------------------------------ AdamW
def _dequant(m, v, ms, vs):
    """m = sign (c / 127)^2 scale, v = (c / 255)^4 scale."""
    cm = m.view(-1, QB).float()
    cv = v.view(-1, QB).float()
    cv2 = cv * cv
    return ((cm * cm.abs()) * (ms * (1.0 / 16129.0))[:, None]).view(-1), \
        ((cv2 * cv2) * (vs * (1.0 / 4228250625.0))[:, None]).view(-1)


def _quant(x, power, top, rnd):
    """Codes of x by rows of QB: |x| / max = (code / top)^power, rounded up or
    down at random so that the mean is x; a positive v never becomes 0."""
    a = x.abs()
    scale = a.amax(1, keepdim=True)
    w = torch.where(scale >= 2.0 ** -126, a * (1.0 / scale), 0.0)
    if power == 2:
        y = (w.sqrt() * top).floor().clamp(max=top - 1)
        lo, hi = y * y, (y + 1) * (y + 1)
        full = float(top * top)
    else:
        y = (w.sqrt().sqrt() * top).floor().clamp(max=top - 1)
        lo, hi = (y * y) * (y * y), ((y + 1) * (y + 1)) * ((y + 1) * (y + 1))
        full = float(top ** 4)
    code = y + ((w * full - lo) > rnd * (hi - lo)).float()
    return code, scale[:, 0]


def _plain_adamw(c, s):
    h = s["hyper"]
    q8 = c["bits"] == 8
    m, v = (_dequant(s["m"], s["v"], s["m_scale"], s["v_scale"]) if q8 else (s["m"], s["v"]))
    g = s["grad"].float() * s["grad_scale"]
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1 - h["beta2"])
    den = v.sqrt() * (1 / math.sqrt(1 - h["beta2"] ** h["step"])) + h["eps"]
    step = (m * (1 / (1 - h["beta1"] ** h["step"]))) / den
    keep = 1.0 - h["lr"] * s["decay"]
    p = (s["p"].view(-1, QB) * keep - step.view(-1, QB) * h["lr"]).view(-1)
    s["p"].copy_(p)
    if c["copy"]:
        s["copy"].copy_(p)
    if q8:
        # an element's place counts within its own tensor
        place = torch.arange(m.numel(), device=m.device).view(-1, QB)
        bits = _hash_places(c, s, place, h["seed"])
        m, v = m.view(-1, QB), v.view(-1, QB)
        cm, s["m_scale"][:] = _quant(m, 2, 127, (bits & 0xFFFF).float() * (1 / 65536))
        cv, s["v_scale"][:] = _quant(v, 4, 255, (bits >> 16).float() * (1 / 65536))
        s["m"].copy_((torch.where(m < 0, -cm, cm)).view(-1))
        s["v"].copy_(torch.where(v > 0, cv.clamp(min=1), cv).view(-1))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _adamw_result(c, s)


def _hash_places(c, s, place, seed):
    """32 random bits for each element: a mix of its place in its tensor, the
    tensor's number and the step's seed."""
    if "first" not in s:                     # the arena row at which each row's tensor starts
        starts = torch.tensor(s["starts"], device=DEV)
        rows = torch.tensor([-(-n // QB) for n in s["sizes"]], device=DEV)
        index = torch.repeat_interleave(torch.arange(c["tensors"], device=DEV), rows)
        s["first"], s["index"] = starts[index][:, None], index[:, None]
    h = (place - s["first"] + (s["index"] + 1) * 0xBB67AE85 + seed * 0x9E3779B9) & 0xFFFFFFFF
    h = ((h ^ (h >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    h = ((h ^ (h >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0x9E3779B9) & 0xFFFFFFFF
    return h ^ (h >> 16)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "adamw":
        n, state = sum(_sizes(c)), 4 if c["bits"] == 32 else 1 + 4 / QB
        by = n * (8 + (2 if c["grad"] == "bf16" else 4) + 4 * state + (2 if c["copy"] else 0))
        return {"bytes": by, "flops": 14.0 * n}
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "logprob":
        n = c["N"] * c["V"]
        # in training the gradient needs each row's sum first, but a row may
        # stay on the chip between: read once, written once
        passes = {"score": 1, "train": 2, "policy": 3}[c["mode"]]
        return {"bytes": n * es * passes + c["N"] * (4 * 6 + 8 * c["top"]),
                "flops": (5.0 if passes == 1 else 12.0) * n}
    Hk, Hv, Dk, Dv = c["Hk"], c["Hv"], c["Dk"], c["Dv"]
    tok = 2 * Hk * Dk * es + 2 * Hv * Dv * es + 8 * Hv
    if c["op"] == "delta_step":
        n = c["B"]
        return {"bytes": n * (tok + 8 * Hv * Dk * Dv + 4), "flops": 7.0 * n * Hv * Dk * Dv}
    # the recurrence's own operations: S k, the outer product, S q; in the
    # gradient those again for S (rebuilt or kept) and twice as many for dS
    n = c["B"] * (c["lo"] + c["hi"]) / 2.0
    by = n * tok + 4 * c["B"] * Hv * Dk * Dv * (2 if c["state"] else 1)
    fl = 6.0 * n * Hv * Dk * Dv
    if c["mode"] == "train":
        by += n * (tok + Hv * Dv * es) + 4 * c["B"] * Hv * Dk * Dv * (2 if c["state"] else 1)
        fl *= 3
    return {"bytes": by, "flops": fl}


# --------------------------------------------------------------------------
# the same outputs in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    return {"delta": _exact_delta, "delta_step": _exact_step, "logprob": _exact_logprob,
            "adamw": _exact_adamw}[case["op"]](case, seed)


def _exact_delta(c, seed):
    """Token by token; the gradient by the reverse recurrence over dS, with the
    states rebuilt from kept ones."""
    d = _delta_inputs(c, seed)
    T, B, Hv, Dk, Dv = c["T"], c["B"], c["Hv"], c["Dk"], c["Dv"]
    r = Hv // c["Hk"]
    f = lambda a: a.double()
    wide = lambda a: f(a).repeat_interleave(r, 1)
    scale = 1.0 / math.sqrt(Dk)
    zero = torch.zeros(B, Hv, Dk, Dv, dtype=torch.float64, device=DEV)
    live = torch.arange(T, device=DEV)[:, None] < d["seq_len"][None, :]
    # past its end a row neither decays nor writes
    g = torch.where(live[..., None], f(d["g"]), 0.0).exp()
    beta = torch.where(live[..., None], f(d["beta"]), 0.0)

    def advance(S, t):
        k = wide(d["k"][t])
        S = S * g[t][..., None, None]
        e = f(d["v"][t]) - torch.einsum("bhkv,bhk->bhv", S, k)
        return S + k[..., None] * (beta[t][..., None] * e)[..., None, :], e

    every = max(1, int(math.sqrt(T)))
    S, kept = f(d["S0"]) if c["state"] else zero, []
    y = torch.zeros(T, B, Hv, Dv, dtype=torch.float64, device=DEV)
    for t in range(T):
        if t % every == 0:
            kept.append(S)
        S, _ = advance(S, t)
        y[t] = torch.einsum("bhkv,bhk->bhv", S, wide(d["q"][t])) * scale * live[t][:, None, None]
    res = dict(y=y, ST=S)
    if c["mode"] != "train":
        return res
    dS = f(d["dST"]) if c["state"] else zero
    new = lambda *n: torch.zeros(*n, dtype=torch.float64, device=DEV)
    out = dict(dq=new(T, B, Hv, Dk), dk=new(T, B, Hv, Dk), dv=new(T, B, Hv, Dv),
               dg=new(T, B, Hv), dbeta=new(T, B, Hv))
    for at in reversed(range(len(kept))):
        t0, states, errs = at * every, [kept[at]], []
        for t in range(t0, min(T, t0 + every)):
            S, e = advance(states[-1], t)
            states.append(S)
            errs.append(e)
        for t in reversed(range(t0, t0 + len(errs))):
            Sp, S, e = states[t - t0], states[t - t0 + 1], errs[t - t0]
            m = live[t][:, None, None]
            q, k = wide(d["q"][t]) * scale, wide(d["k"][t])
            dy, b = f(d["dy"][t]) * m, beta[t][..., None]
            out["dq"][t] = torch.einsum("bhkv,bhv->bhk", S, dy) * scale
            dS = dS + q[..., None] * dy[..., None, :]
            dk_write = torch.einsum("bhkv,bhv->bhk", dS, b * e) * m
            du = torch.einsum("bhkv,bhk->bhv", dS, k)
            out["dbeta"][t] = (du * e).sum(-1) * live[t][:, None]
            de = b * du
            out["dv"][t] = de
            Sd = Sp * g[t][..., None, None]
            out["dk"][t] = dk_write - torch.einsum("bhkv,bhv->bhk", Sd, de)
            dSd = dS - k[..., None] * de[..., None, :]
            out["dg"][t] = (dSd * Sd).sum((-1, -2)) * live[t][:, None]
            dS = dSd * g[t][..., None, None]
    for n in ("dq", "dk"):                   # a key head serves r value heads
        out[n] = out[n].unflatten(2, (c["Hk"], r)).sum(3)
    return dict(res, **out, dS0=dS)


def _exact_step(c, seed):
    d = _step_inputs(c, seed)
    f = lambda a: a.double()
    r = c["Hv"] // c["Hk"]
    S, y = f(d["S"]), torch.zeros(c["B"], c["Hv"], c["Dv"], dtype=torch.float64, device=DEV)
    rows = torch.nonzero(d["slots"] >= 0)[:, 0]
    at = d["slots"][rows].long()
    k, q = (f(d[n][rows]).repeat_interleave(r, 1) for n in ("k", "q"))
    Sd = S[at] * f(d["g"][rows]).exp()[..., None, None]
    e = f(d["v"][rows]) - torch.einsum("bhkv,bhk->bhv", Sd, k)
    Sn = Sd + torch.einsum("bhk,bhv->bhkv", k, f(d["beta"][rows])[..., None] * e)
    S[at] = Sn
    y[rows] = torch.einsum("bhkv,bhk->bhv", Sn, q) / math.sqrt(c["Dk"])
    return dict(y=y, S=S)


def _exact_logprob(c, seed):
    """Row blocks in 64 bits: log-softmax from its definition, the gradient by
    differentiating sum(dlogp logp + dentropy entropy) through it."""
    d = _logprob_inputs(c, seed)
    N = c["N"]
    outs = []
    for i in range(0, N, 256):
        x = d["logits"][i:i + 256].double()
        t = d["targets"][i:i + 256].long()
        dead = (x == -math.inf).all(1)
        lse = torch.logsumexp(x, 1)
        lp = x - torch.where(dead, 0.0, lse)[:, None]
        p = lp.exp()
        plp = torch.where(p > 0, p * lp, 0.0)
        one = dict(lse=lse, entropy=-plp.sum(1))
        has = t >= 0
        row = torch.arange(len(t), device=DEV)
        one["logp"] = torch.where(has, lp[row, t.clamp(min=0)], 0.0)
        if c["top"]:                         # stable: equal ones by index
            order = lp.sort(dim=1, descending=True, stable=True).indices[:, :c["top"]]
            one["top_logp"] = lp.gather(1, order)
        if c["mode"] != "score":
            dl = torch.where(has, d["dlogp"][i:i + 256].double(), 0.0)
            de = d["dentropy"][i:i + 256].double()
            w = -(plp + p * one["entropy"][:, None]) * de[:, None] - p * dl[:, None]
            w[row, t.clamp(min=0)] += dl
            if d["dtop"] is not None:
                dt = d["dtop"][i:i + 256].double()
                w = w - p * dt.sum(1, keepdim=True)
                w.scatter_add_(1, order, dt)
            one["dlogits"] = torch.where(dead[:, None], 0.0, w).to(
                torch.float32 if c["dtype"] == "bf16" else torch.float64)
        outs.append(one)
    res = {n: torch.cat([o[n] for o in outs]) for n in outs[0]}
    if c["top"]:
        res["top_ids"] = None
    return res


def _exact_adamw(c, seed):
    d = _adamw_inputs(c, seed)
    h = d["hyper"]
    f = lambda a: a.double()
    if c["bits"] == 32:
        m, v = f(d["m"]), f(d["v"])
    else:
        m = (f(d["m"]) / 127).view(-1, QB)
        m = (m * m.abs() * f(d["m_scale"])[:, None]).view(-1)
        v = ((f(d["v"]) / 255).view(-1, QB) ** 4 * f(d["v_scale"])[:, None]).view(-1)
    g = f(d["grad"]) * f(d["grad_scale"])
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    up = (m / (1 - h["beta1"] ** h["step"])) / (torch.sqrt(v / (1 - h["beta2"] ** h["step"]))
                                               + h["eps"])
    p = f(d["p"]).view(-1, QB)
    p = (p - h["lr"] * (f(d["decay"]) * p + up.view(-1, QB))).view(-1)
    res = dict(p=p)
    if c["copy"]:
        res["copy"] = p
    # the codes of an 8-bit state are a rounding of the 32-bit result, not a value of their own
    res["m"], res["v"] = (m, v) if c["bits"] == 32 else (None, None)
    return res
