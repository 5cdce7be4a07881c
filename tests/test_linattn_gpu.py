"""GPU: linear attention with a decay for each head against the float64 oracle, and
what the loop fixes exactly.

Tolerances.  float32: a product of two 24-bit operands and sums of up to 128 terms,
chained over the tokens; 2^-24 a rounding, a few dozen of them on the way to an output,
with random signs: relative 2-norm 5e-6 leaves a factor of ten.  bfloat16 outputs are one
rounding of that, at most 2^-8 of the value: 2-norm 2^-8.  Float outputs of a bfloat16
call (states) are float32's.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import linattn as oa
from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
OP = {"f32": torch.float32, "bf16": torch.bfloat16}
INS = ("q", "k", "v", "g", "seq_len")


def make(T, B, Hk, Hv, Dk, Dv, dtype, lens=None, state=True, seed=0, fused=False, decay=0.3):
    rng = np.random.default_rng(seed)
    n = rng.standard_normal
    op = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV).to(OP[dtype])
    f32 = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV)
    c = dict(q=op(n((T, B, Hk, Dk))), k=op(n((T, B, Hk, Dk))), v=op(n((T, B, Hv, Dv))),
             g=f32(-decay * rng.random(Hv) ** 3))
    if fused:
        row = torch.cat([c[x].reshape(T, B, -1) for x in "qkv"], 2)
        parts = row.split([Hk * Dk, Hk * Dk, Hv * Dv], 2)
        for x, a, s in zip("qkv", parts, ((Hk, Dk), (Hk, Dk), (Hv, Dv))):
            c[x] = a.unflatten(2, s)
    c["seq_len"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    c["S0"] = f32(n((B, Hv, Dk, Dv))) if state else None
    c["dy"] = op(n((T, B, Hv, Dv)))
    c["dST"] = f32(n((B, Hv, Dk, Dv))) if state else None
    return c


def new_outputs(c, dtype, fused=False):
    T, B, Hk, Dk = c["q"].shape
    Hv, Dv = c["v"].shape[2:]
    new = lambda *s, t=torch.float32: torch.full(s, math.nan, dtype=t, device=DEV)
    r = dict(y=new(T, B, Hv, Dv, t=OP[dtype]), ST=new(B, Hv, Dk, Dv), dS0=new(B, Hv, Dk, Dv))
    if fused:
        parts = new(T, B, 2 * Hk * Dk + Hv * Dv, t=OP[dtype]).split([Hk * Dk, Hk * Dk, Hv * Dv], 2)
        r.update({"d" + x: a.unflatten(2, s) for x, a, s in zip("qkv", parts, ((Hk, Dk), (Hk, Dk), (Hv, Dv)))})
    else:
        r.update({"d" + x: new(*c[x].shape, t=OP[dtype]) for x in "qkv"})
    return r


def run(c, dtype, backward=True, fused=False, plan=None, scale=0.0, stream=None):
    T, B, Hk, Dk = c["q"].shape
    Hv, Dv = c["v"].shape[2:]
    ld = {x + "_ld": c[x].stride(1) for x in "qkv"} if fused else {}
    ld.update({"d" + n: v for n, v in ld.items()})
    p = plan or ll.LinattnPlan(T, B, Hk, Hv, Dk, Dv, dtype=dtype, scale=scale, **ld)
    r = new_outputs(c, dtype, fused)
    ins = [c[n] for n in INS]
    p.fwd(*ins, c["S0"], r["y"], r["ST"], save_for_backward=backward, stream=stream)
    if backward:
        p.bwd(*ins, c["dy"], c["dST"], r["dq"], r["dk"], r["dv"], r["dS0"], stream=stream)
    else:
        r = {n: r[n] for n in ("y", "ST")}
    err = p.status_sync()
    if plan is None:
        p.close()
    return r, err


def reference(c, backward=True, scale=None):
    f = lambda a: None if a is None else a.double().cpu().numpy()
    lens = None if c["seq_len"] is None else c["seq_len"].cpu().numpy()
    y, S, tape = oa.linattn_forward(*[f(c[n]) for n in ("q", "k", "v", "g")], lens, f(c["S0"]), scale)
    r = dict(y=y, ST=S)
    if backward:
        r.update(oa.linattn_backward(tape, f(c["dy"]), f(c["dST"])))
    return r


def check(got, ref, dtype):
    for n, want in ref.items():
        a = got[n].double().cpu().numpy()
        assert np.isfinite(a).all(), n
        tol = 2.0 ** -8 if dtype == "bf16" and n in ("y", "dq", "dk", "dv") else 5e-6
        norm = np.linalg.norm(want)
        err = np.linalg.norm(a - want)
        print(f"    {n}: {err / norm if norm else err:.2e}", flush=True)
        assert err <= tol * norm if norm else err == 0, (n, err / norm if norm else err)


def by_pairs(c, scale=None):
    """The gradient through float64 torch from the sum over pairs, for long rows."""
    T, B, Hk, Dk = c["q"].shape
    Hv, Dv = c["v"].shape[2:]
    r = Hv // Hk
    scale = 1 / math.sqrt(Dk) if scale is None else scale
    f = lambda a: a.double().cpu()
    out = {n: torch.zeros(s, dtype=torch.float64) for n, s in
           (("y", (T, B, Hv, Dv)), ("ST", (B, Hv, Dk, Dv)), ("dS0", (B, Hv, Dk, Dv)), ("dq", (T, B, Hk, Dk)),
            ("dk", (T, B, Hk, Dk)), ("dv", (T, B, Hv, Dv)))}
    for b in range(B):
        L = T if c["seq_len"] is None else int(c["seq_len"][b])
        t = torch.arange(L, dtype=torch.float64)
        for h in range(Hv):
            g = f(c["g"][h])
            q, k = f(c["q"][:L, b, h // r]), f(c["k"][:L, b, h // r])
            v, dy = f(c["v"][:L, b, h]), f(c["dy"][:L, b, h])
            zero = torch.zeros(Dk, Dv, dtype=torch.float64)
            S0, dST = (f(c[n][b, h]) if c[n] is not None else zero for n in ("S0", "dST"))
            far = t[:, None] - t
            w = torch.where(far >= 0, (g * far.clamp(min=0)).exp(), 0.0) * scale
            start, end = (g * (t + 1)).exp()[:, None] * scale, (g * (L - 1 - t)).exp()[:, None]
            P, F = w * (q @ k.T), w * (dy @ v.T)
            out["y"][:L, b, h] = P @ v + start * (q @ S0)
            out["ST"][b, h] = (g * L).exp() * S0 + (end * k).T @ v
            out["dq"][:L, b, h // r] += F @ k + start * (dy @ S0.T)
            out["dk"][:L, b, h // r] += F.T @ q + end * (v @ dST.T)
            out["dv"][:L, b, h] = P.T @ dy + end * (k @ dST)
            out["dS0"][b, h] = (g * L).exp() * dST + (start * q).T @ dy
    return {n: a.numpy() for n, a in out.items()}


CASES = [
    # T, B, Hk, Hv, Dk, Dv, lengths
    (1, 1, 1, 1, 8, 8, None),
    (1, 3, 2, 4, 32, 40, [1, 0, 1]),
    (5, 2, 1, 3, 16, 24, [5, 2]),
    (31, 2, 2, 2, 72, 56, [31, 1]),
    (32, 2, 2, 2, 96, 128, [32, 16]),
    (33, 1, 1, 1, 128, 64, None),
    (63, 2, 2, 2, 72, 56, [63, 1]),
    (64, 2, 1, 2, 64, 64, None),
    (65, 3, 2, 2, 128, 128, [65, 64, 0]),
    (129, 2, 1, 2, 120, 104, [129, 66]),
    (200, 3, 2, 4, 24, 96, [200, 0, 130]),
    (300, 1, 1, 1, 128, 8, None),
    (130, 2, 1, 1, 8, 128, [70, 130]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:6])))
def test_against_oracle(case, dtype):
    *sizes, lens = case
    c = make(*sizes, dtype, lens, seed=sum(sizes))
    got, err = run(c, dtype)
    assert err == 0
    check(got, reference(c), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("sizes", [(1500, 2, 1, 2, 40, 64, [1500, 777]), (2111, 1, 2, 2, 64, 72, None),
                                   (1100, 3, 1, 1, 128, 128, [0, 1100, 65])], ids=lambda c: "x".join(map(str, c[:6])))
def test_rows_in_parts(sizes, state, dtype):
    """Few rows of many tokens, cut into parts whose states are joined."""
    *n, lens = sizes
    c = make(*n, dtype, lens, seed=n[0], state=state)
    got, err = run(c, dtype)
    assert err == 0
    check(got, by_pairs(c), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_against_differences(dtype):
    """Central differences of the kernel's own forward in direction d; the loss is linear in
    each input alone, so that its difference is exact but for roundings."""
    c = make(70, 2, 1, 2, 32, 24, dtype, [70, 40], seed=31)
    got, _ = run(c, dtype)
    gen = torch.Generator(device=DEV).manual_seed(3)
    weigh = lambda r: ((r["y"].double() * c["dy"].double()).sum() + (r["ST"].double() * c["dST"].double()).sum()).item()
    size = lambda r: ((r["y"].double() * c["dy"].double()).norm() + (r["ST"].double() * c["dST"].double()).norm()).item()
    for n in ("q", "k", "v", "S0"):
        d = torch.randn(c[n].shape, device=DEV, generator=gen).to(c[n].dtype)
        if n != "S0":
            for b, L in enumerate((70, 40)):
                d[L:, b] = 0
        ends = [run({**c, n: x}, dtype, backward=False)[0] for x in (d, torch.zeros_like(d))]
        slope = weigh(ends[0]) - weigh(ends[1])
        want = (got["d" + n].double() * d.double()).sum().item()
        # roundings of y (random signs: the norm of its terms) and of the gradient's
        eps = 2.0 ** -8 if dtype == "bf16" else 5e-6
        tol = 4 * eps * (size(ends[0]) + size(ends[1]) + (got["d" + n].double() * d.double()).norm().item())
        assert abs(slope - want) <= tol, (n, slope, want, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_slices_of_one_projection(dtype):
    c = make(100, 3, 2, 4, 32, 48, dtype, [100, 64, 7], seed=5, fused=True)
    a, _ = run(c, dtype, fused=True)
    check(a, reference(c), dtype)
    b, _ = run({n: t if t is None else t.contiguous() for n, t in c.items()}, dtype)
    for n in b:
        assert torch.equal(a[n], b[n]), n


def test_no_state_given_and_scale():
    c = make(70, 2, 2, 2, 40, 32, "f32", state=False, seed=6)
    got, _ = run(c, "f32", scale=0.5)
    check(got, reference(c, scale=0.5), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [80, 1400])
def test_padding_may_hold_nan_and_is_not_read_into_results(T, dtype):
    lens = [T - 10, 0, T // 2 - 7]
    c = make(T, 3, 1, 2, 32, 32, dtype, lens, seed=7)
    a, _ = run(c, dtype)
    for b, n in enumerate(lens):
        for x in ("q", "k", "v", "dy"):
            c[x][n:, b] = math.nan
    d, _ = run(c, dtype)
    for n in a:
        assert torch.equal(a[n], d[n]), n
    for b, n in enumerate(lens):
        for x in ("y", "dq", "dk", "dv"):
            assert not d[x][n:, b].any(), x
    assert torch.equal(d["ST"][1], c["S0"][1]) and torch.equal(d["dS0"][1], c["dST"][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_do_not_depend_on_each_other(dtype):
    c = make(90, 3, 1, 2, 32, 64, dtype, [90, 10, 77], seed=8)
    a, _ = run(c, dtype)
    one = {n: t if t is None or n == "g" else (t[2:3] if n in ("seq_len", "S0", "dST") else t[:, 2:3]).clone(
        memory_format=torch.contiguous_format) for n, t in c.items()}
    b, _ = run(one, dtype)
    for n in b:
        assert torch.equal(b[n], a[n][2:3] if n in ("ST", "dS0") else a[n][:, 2:3]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [150, 1300])
def test_extreme_decays(T, dtype):
    """Nothing is kept (g = -inf, -1e4), all is kept (0, -0, the smallest), strong decays."""
    c = make(T, 1, 2, 8, 32, 32, dtype, seed=9)
    c["g"].copy_(torch.tensor([-math.inf, -1e4, -200.0, -60.0, 0.0, -0.0, -1e-45, -1e-6]))
    got, _ = run(c, dtype)
    check(got, by_pairs({**c, "g": c["g"].double().clamp(min=-1e5)}), dtype)
    one = T - 1                              # alone: y_t = scale (q_t.k_t) v_t
    want = (c["q"][one, 0, 0].double() @ c["k"][one, 0, 0].double()) / math.sqrt(32) * c["v"][one, 0, 0].double()
    assert (got["y"][one, 0, 0].double() - want).norm() <= (2.0 ** -8 if dtype == "bf16" else 5e-6) * want.norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_slow_decay_does_not_drift(dtype):
    """A decay whose float differs from 1 by a few units, over 128 chunks: a rounded power
    of it, taken again in every chunk, would be off by up to 128 times 2^-24 and more."""
    c = make(8192, 1, 1, 1, 8, 8, dtype, seed=12)
    c["g"].fill_(-3.3e-7)
    got, _ = run(c, dtype)
    check(got, by_pairs(c), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_state_carries_over_pieces_exactly_where_chunks_meet(dtype):
    """128 tokens at once, or 64 and 64 with the state handed over: the same chunks, the same bits."""
    c = make(128, 2, 1, 2, 64, 32, dtype, seed=10)
    whole, _ = run(c, dtype, backward=False)
    cut = lambda a, b: {n: t if t is None or n in ("g", "seq_len", "S0", "dST") else t[a:b].contiguous()
                        for n, t in c.items()}
    first, _ = run(cut(0, 64), dtype, backward=False)
    second = cut(64, 128)
    second["S0"] = first["ST"]
    last, _ = run(second, dtype, backward=False)
    assert torch.equal(torch.cat([first["y"], last["y"]]), whole["y"])
    assert torch.equal(last["ST"], whole["ST"])


@pytest.mark.parametrize("T", [100, 1200])
def test_state_in_place_and_repeatable(T):
    c = make(T, 2, 2, 4, 32, 32, "bf16", [T, T // 2 + 1], seed=11)
    a, _ = run(c, "bf16")
    b, _ = run(c, "bf16")
    for n in a:
        assert torch.equal(a[n], b[n]), n
    # the saved forward keeps the state that it began with, also where ST is S0
    S, r = c["S0"].clone(), new_outputs(c, "bf16")
    with ll.LinattnPlan(T, 2, 2, 4, 32, 32, dtype="bf16") as p:
        ins = [c[n] for n in INS]
        p.fwd(*ins, S, r["y"], S)
        p.bwd(*ins, c["dy"], c["dST"], r["dq"], r["dk"], r["dv"], r["dS0"])
        assert p.status_sync() == 0
    assert torch.equal(S, a["ST"])
    for n in ("y", "dq", "dk", "dv", "dS0"):
        assert torch.equal(r[n], a[n]), n
    S = c["S0"].clone()
    with ll.LinattnPlan(T, 2, 2, 4, 32, 32, dtype="bf16", inference=True) as p:
        y = torch.empty_like(a["y"])
        p.fwd(*ins, S, y, S, save_for_backward=False)
        assert p.status_sync() == 0
    assert torch.equal(S, a["ST"]) and torch.equal(y, a["y"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["q", "k", "v", "S0"])
@pytest.mark.parametrize("T", [40, 1100])
def test_infinity_stays_in_its_row_and_head(T, name, dtype):
    """NaN or infinity comes out of the head that held it, and nothing in the others."""
    c = make(T, 3, 2, 2, 24, 16, dtype, lens=[T, T - 5, T // 2])
    clean, _ = run(c, dtype)
    if name == "S0":
        c[name][1, 1, 3, 5] = math.inf
    else:
        c[name][T // 3, 1, 1, 4] = math.inf
    r, err = run(c, dtype)
    assert err == 0
    assert not torch.isfinite(r["y"][:, 1, 1]).all()
    for n, want in clean.items():
        got = r[n].clone()
        got.select(1 if n in ("y", "dq", "dk", "dv") else 0, 1).select(-3 if n in ("ST", "dS0") else -2, 1).zero_()
        want.select(1 if n in ("y", "dq", "dk", "dv") else 0, 1).select(-3 if n in ("ST", "dS0") else -2, 1).zero_()
        assert torch.equal(got, want), n


def test_bad_length_counts_as_zero_and_is_reported():
    c = make(20, 3, 1, 1, 16, 16, "f32", [20, 21, -1], seed=12)
    got, err = run(c, "f32")
    assert err == ll.LL_DEVERR_SEQ_LEN
    c["seq_len"] = torch.tensor([20, 0, 0], dtype=torch.int32, device=DEV)
    want, err = run(c, "f32")
    assert err == 0
    for n in want:
        assert torch.equal(got[n], want[n]), n


def test_other_stream():
    c = make(1300, 2, 1, 2, 32, 32, "bf16", seed=13)
    want, _ = run(c, "bf16")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, _ = run(c, "bf16", stream=s)
    s.synchronize()
    for n in want:
        assert torch.equal(got[n], want[n]), n


def test_single_row_as_it_lies():
    """Slices of a single row's projection: the binding takes the distances from the tensors."""
    c = make(50, 1, 2, 2, 16, 16, "f32", seed=14, fused=True)
    dense = {n: t if t is None else t.contiguous() for n, t in c.items()}
    with ll.LinattnPlan(50, 1, 2, 2, 16, 16) as p:
        a, _ = run(c, "f32", plan=p)
        b, _ = run(dense, "f32", plan=p)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_refusals():
    c = make(10, 2, 1, 2, 16, 16, "f32", seed=15)
    p = ll.LinattnPlan(10, 2, 1, 2, 16, 16)
    ins = [c[n] for n in INS]
    y, ST = torch.empty_like(c["v"]), torch.empty_like(c["S0"])
    outs = [torch.empty_like(c[n]) for n in "qkv"]
    with pytest.raises(ll.LoopError) as e:
        p.bwd(*ins, c["dy"], c["dST"], *outs)
    assert e.value.status == ll.LL_ESTATE
    p.fwd(*ins, c["S0"], y, ST)
    with pytest.raises(ll.LoopError) as e:
        p.bwd(c["q"].clone(), *ins[1:], c["dy"], c["dST"], *outs)
    assert e.value.status == ll.LL_EINVAL
    with pytest.raises(ll.LoopError) as e:
        p.bwd(*ins, c["dy"], c["dST"], *outs, c["dST"])
    assert e.value.status == ll.LL_EINVAL and "dST" in str(e.value)
    p.bwd(*ins, c["dy"], c["dST"], *outs)          # the saved forward was kept
    for bad in (c["q"].to(torch.bfloat16), c["q"][:5], c["q"].transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises(ValueError):
            p.fwd(bad, *ins[1:], c["S0"], y, ST)
    with pytest.raises(ValueError):
        p.fwd(*ins[:3], c["g"][:1], c["seq_len"], c["S0"], y, ST)
    odd = torch.empty(c["q"].numel() + 1, device=DEV)[1:].view_as(c["q"])
    with pytest.raises(ll.LoopError) as e:
        p.fwd(odd, *ins[1:], c["S0"], y, ST)
    assert e.value.status == ll.LL_EINVAL and "16-byte" in str(e.value)
    p.close()
    with ll.LinattnPlan(10, 2, 1, 2, 16, 16, inference=True) as p:
        with pytest.raises(ll.LoopError) as e:
            p.fwd(*ins, c["S0"], y, ST)
        assert e.value.status == ll.LL_EINVAL


def test_distances_of_the_saved_forward():
    """A gradient with other distances than its forward's is refused, and the forward kept."""
    c = make(40, 1, 2, 2, 16, 16, "f32", seed=16)
    lib, n = ll.load_library(), 32
    with ll.LinattnPlan(40, 1, 2, 2, 16, 16) as p:
        ins = [c[x] for x in INS]
        r = new_outputs(c, "f32")
        p.fwd(*ins, None, r["y"], None)
        set_ld = lambda *ld: lib.ll_linattn_plan_set_ld(p._h, (ctypes.c_int64 * 6)(*ld))
        assert set_ld(3 * n, n, n, n, n, n) == ll.LL_OK
        at = lambda t: None if t is None else t.data_ptr()
        bwd = lambda: lib.linattn_loop_bwd(p._h, None, *map(at, ins), at(c["dy"]), None, at(r["dq"]), at(r["dk"]),
                                           at(r["dv"]), None)
        assert bwd() == ll.LL_ESTATE and "distances" in ll.ll_last_error()
        assert set_ld(n, n, n, n, n, n) == ll.LL_OK
        p.bwd(*ins, c["dy"], None, r["dq"], r["dk"], r["dv"])
        check({x: r[x] for x in ("dq", "dk", "dv")},
              {x: v for x, v in reference({**c, "S0": None, "dST": None}).items() if x in ("dq", "dk", "dv")}, "f32")


# ------------------------------------------------------------ one token
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [(1, 1, 1, 8, 8), (3, 2, 4, 32, 32), (5, 1, 3, 128, 104), (4, 4, 4, 72, 40),
                                   (9, 2, 2, 128, 128)], ids=str)
def test_step_against_oracle(sizes, dtype):
    B, Hk, Hv, Dk, Dv = sizes
    c = make(1, B, Hk, Hv, Dk, Dv, dtype, seed=B)
    S, y = c["S0"].clone(), torch.full((B, Hv, Dv), math.nan, dtype=OP[dtype], device=DEV)
    ll.linattn_loop_step(c["q"][0], c["k"][0], c["v"][0], c["g"], S, y)
    ref = reference(c, backward=False)
    check(dict(y=y, ST=S), dict(y=ref["y"][0], ST=ref["ST"]), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_follow_the_loop(dtype):
    """37 steps against one loop over 37 tokens (other orders of the sums)."""
    c = make(37, 2, 2, 4, 64, 64, dtype, seed=3)
    want, _ = run(c, dtype, backward=False)
    S, ys = c["S0"].clone(), []
    for t in range(37):
        ys.append(torch.empty_like(c["v"][0]))
        ll.linattn_loop_step(c["q"][t], c["k"][t], c["v"][t], c["g"], S, ys[-1])
    ref = reference(c, backward=False)
    check(dict(y=torch.stack(ys), ST=S), ref, dtype)
    check(want, ref, dtype)


def test_step_extreme_decays():
    c = make(1, 2, 4, 4, 16, 16, "f32", seed=17)
    c["g"].copy_(torch.tensor([-math.inf, 0.0, -300.0, -1e-7]))
    S, y = c["S0"].clone(), torch.empty_like(c["v"][0])
    ll.linattn_loop_step(c["q"][0], c["k"][0], c["v"][0], c["g"], S, y)
    ref = reference({**c, "g": c["g"].double().clamp(min=-700)}, backward=False)
    check(dict(y=y, ST=S), dict(y=ref["y"][0], ST=ref["ST"]), "f32")


def test_step_slots_and_slices():
    c = make(1, 5, 1, 2, 32, 32, "bf16", seed=4, fused=True)
    pool = torch.randn(9, 2, 32, 32, device=DEV)
    slots = torch.tensor([7, -1, 0, 9, -5], dtype=torch.int32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    S, y = pool.clone(), torch.full((5, 2, 32), math.nan, dtype=torch.bfloat16, device=DEV)
    one = [c[n][0] for n in "qkv"]
    ll.linattn_loop_step(*one, c["g"], S, y, slots=slots, device_error=err)
    assert err.item() == ll.LL_DEVERR_SLOT
    for b, s in enumerate([7, None, 0, None, None]):
        if s is None:
            assert not y[b].any()
            continue
        S1, y1 = pool[s:s + 1].clone(), torch.empty(1, 2, 32, dtype=torch.bfloat16, device=DEV)
        ll.linattn_loop_step(*[a[b:b + 1].contiguous() for a in one], c["g"], S1, y1)
        assert torch.equal(S[s], S1[0]) and torch.equal(y[b], y1[0])
    rest = [i for i in range(9) if i not in (0, 7)]
    assert torch.equal(S[rest], pool[rest])


def test_step_state_past_32_bit_offsets():
    """A pool of more than 2^31 elements: its last slot."""
    n = 131500
    pool = torch.empty(n, 1, 128, 128, device=DEV)
    pool[-1] = 0.25
    c = make(1, 1, 1, 1, 128, 128, "f32", seed=6)
    c["S0"] = pool[-1:].clone()
    y = torch.empty(1, 1, 128, device=DEV)
    ll.linattn_loop_step(c["q"][0], c["k"][0], c["v"][0], c["g"], pool, y,
                         slots=torch.tensor([n - 1], dtype=torch.int32, device=DEV))
    ref = reference(c, backward=False)
    check(dict(y=y, ST=pool[-1:]), dict(y=ref["y"][0], ST=ref["ST"]), "f32")


def test_step_refuses_rows_that_overlap():
    c = make(1, 4, 1, 1, 16, 16, "f32", seed=18)
    S, y = c["S0"].clone(), torch.empty_like(c["v"][0])
    with pytest.raises(ValueError, match="overlap"):
        ll.linattn_loop_step(c["q"][0][:1].expand(4, 1, 16), c["k"][0], c["v"][0], c["g"], S, y)


# ------------------------------------------------------------ what a decay leaves of a state
def units(g, T, times):
    """Roundings (2^-24 each) of a state that e^g has been applied to for T tokens, by `times`
    products: the exponent's (|g| T in all), and for each product its exponential's last
    place (two), another of the exponent's product and its own."""
    return (abs(g) * T + 4 * times) * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("g,T", [(-0.25, 64), (-0.25, 100), (-1.0, 33), (-0.05, 64), (-0.011, 128), (-0.02, 70), (-5.0, 5),
                                 (-0.05, 1100), (-0.01, 2111)])
def test_what_is_left_of_a_state_keeps_its_bits(g, T, dtype):
    """Tokens that add nothing: each element of the last state is e^{g T} of the first one's,
    whatever that factor is, and so is the state's gradient (l S as S + (l - 1) S would leave
    roundings of S itself, which are anything of a small l S)."""
    c = make(T, 2, 1, 2, 24, 40, dtype, [T, T - 3], seed=T)
    c["g"].copy_(torch.tensor([g, g / 2]))
    c["k"].zero_()
    c["dy"].zero_()
    r, err = run(c, dtype)
    assert err == 0
    for b, L in enumerate((T, T - 3)):
        for h, x in enumerate(c["g"].double().tolist()):
            for got, first in (("ST", "S0"), ("dS0", "dST")):
                want = math.exp(x * L) * c[first][b, h].double()
                off = ((r[got][b, h].double() - want).abs() / want.abs()).max().item()
                assert off <= units(x, L, -(-L // 32) + 1), (got, b, h, off)


def test_step_keeps_what_is_left_of_a_state():
    c = make(1, 2, 1, 6, 16, 24, "f32", seed=20)
    c["g"].copy_(torch.tensor([-0.1, -0.69, -0.7, -3.0, -9.0, -17.0]))
    c["k"].zero_()
    S, y = c["S0"].clone(), torch.empty_like(c["v"][0])
    for _ in range(3):
        ll.linattn_loop_step(c["q"][0], c["k"][0], c["v"][0], c["g"], S, y)
    for h, x in enumerate(c["g"].double().tolist()):
        want = math.exp(3 * x) * c["S0"][:, h].double()
        assert ((S[:, h].double() - want).abs() / want.abs()).max() <= units(x, 3, 3), x


def test_many_heads():
    """3.5 million rows of one head: more work-groups than 2^23 in the gradient."""
    B, D = 3_500_000, 8
    gen = torch.Generator(device=DEV).manual_seed(21)
    n = lambda *s: torch.randn(*s, device=DEV, generator=gen)
    c = dict(q=n(1, B, 1, D), k=n(1, B, 1, D), v=n(1, B, 1, D), g=torch.tensor([-0.3], device=DEV), seq_len=None,
             S0=n(B, 1, D, D), dy=n(1, B, 1, D), dST=n(B, 1, D, D))
    r, err = run(c, "f32", scale=1.0)
    assert err == 0
    q, k, v, dy = (c[x][0, :, 0].double() for x in ("q", "k", "v", "dy"))
    left = math.exp(c["g"].double().item())
    S = left * c["S0"][:, 0].double() + k[:, :, None] * v[:, None, :]
    dS = c["dST"][:, 0].double() + q[:, :, None] * dy[:, None, :]
    want = dict(y=(q[:, :, None] * S).sum(1), ST=S, dq=(S * dy[:, None, :]).sum(2), dk=(dS * v[:, None, :]).sum(2),
                dv=(dS * k[:, :, None]).sum(1), dS0=left * dS)
    for x, w in want.items():
        a = r[x].double().view_as(w)
        off = (a - w).flatten(1).norm(dim=1) / w.flatten(1).norm(dim=1)
        for rows in (off[:1000], off[-1000:]):
            assert rows.max() < 1e-4, x          # (a row's own norm may be small next to its terms')
        assert ((a - w).norm() / w.norm()).item() <= 5e-6, x


# ------------------------------------------------------------ bfloat16 results, element by element
def check_rounded_once(got, want, name):
    """Each element is the float result, rounded once: half a step of bfloat16 at that value
    (2^-8 of the power of two below it), and what the float result may be off by itself: 5e-6 of
    a row's norm as above, times four for the largest of its elements.  (A product that kept
    one bfloat16 piece of a state or of another product would be off by about a step more.)"""
    a = got.double().cpu().numpy()
    step = np.where(want == 0, 0.0, 2.0 ** (np.floor(np.log2(np.abs(want) + (want == 0))) - 8))
    rms = np.sqrt((want ** 2).mean(-1, keepdims=True))
    over = np.abs(a - want) - step - 2e-5 * rms
    print(f"    {name}: {over.max():.2e}", flush=True)
    assert (over <= 0).all(), (name, over.max(), (over > 0).mean())


@pytest.mark.parametrize("case", [c for c in CASES if c[0] in (31, 64, 65, 129, 200)] +
                         [(1500, 2, 1, 2, 40, 64, [1500, 777]), (1100, 2, 1, 1, 128, 128, [65, 1100])],
                         ids=lambda c: "x".join(map(str, c[:6])))
def test_bfloat16_results_are_rounded_once(case):
    *sizes, lens = case
    c = make(*sizes, "bf16", lens, seed=sum(sizes) + 1)
    got, err = run(c, "bf16")
    assert err == 0
    want = by_pairs(c)
    for n in ("y", "dq", "dk", "dv"):
        check_rounded_once(got[n], want[n], n)


def test_bfloat16_step_is_rounded_once():
    c = make(1, 40, 2, 4, 128, 104, "bf16", seed=23)
    S, y = c["S0"].clone(), torch.empty_like(c["v"][0])
    ll.linattn_loop_step(c["q"][0], c["k"][0], c["v"][0], c["g"], S, y)
    check_rounded_once(y, reference(c, backward=False)["y"][0], "y")


@pytest.mark.parametrize("power,tol", [(-105, 5e-6), (-118, 5e-6 + 2.0 ** -12)])
@pytest.mark.parametrize("name", ["k", "v"])
def test_small_numbers(name, power, tol):
    """Operands near 1 times 2^power: all their bits down to 2^-109; below, a bfloat16 piece is
    a multiple of 2^-133, so an operand is off by at most 2^-134, here 2^-16 of one near 1; the
    sums' norm by sixteen times that at most."""
    c = make(70, 1, 1, 2, 32, 40, "f32", seed=22)
    c[name] *= 2.0 ** power
    c["S0"] *= 2.0 ** power
    got, err = run(c, "f32")
    assert err == 0
    for n, want in by_pairs(c).items():
        off = np.linalg.norm(got[n].double().cpu().numpy() - want) / np.linalg.norm(want)
        assert off <= tol, (n, off)
