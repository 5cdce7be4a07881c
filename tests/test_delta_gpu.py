"""GPU: the gated delta rule against the float64 oracle, and what the loop
fixes exactly.

Tolerances.  float32: products keep 24 bits and sums of up to 128 terms are
chained over the tokens; 2^-24 a rounding, a few hundred of them with random
signs: relative 2-norm 5e-6.  bfloat16 outputs are one rounding of that (8
significant bits), at most 2^-8 of the value: 2-norm 2^-8.  Float outputs of a bfloat16 call (states,
dg, dbeta) are float32's.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import delta as od
from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
OP = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(T, B, Hk, Hv, Dk, Dv, dtype, lens=None, state=True, seed=0, fused=False, decay=0.3):
    rng = np.random.default_rng(seed)
    n = rng.standard_normal
    unit = lambda a: a / np.linalg.norm(a, axis=-1, keepdims=True)
    op = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV).to(OP[dtype])
    f32 = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV)
    c = dict(q=op(unit(n((T, B, Hk, Dk)))), k=op(unit(n((T, B, Hk, Dk)))), v=op(n((T, B, Hv, Dv))),
             g=f32(-decay * rng.random((T, B, Hv))), beta=f32(rng.random((T, B, Hv))))
    if fused:
        row = torch.cat([c[x].reshape(T, B, -1) for x in "qkv"], 2)
        parts = row.split([Hk * Dk, Hk * Dk, Hv * Dv], 2)
        for x, a, s in zip("qkv", parts, ((Hk, Dk), (Hk, Dk), (Hv, Dv))):
            c[x] = a.unflatten(2, s)
    c["seq_len"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    c["S0"] = f32(0.5 * n((B, Hv, Dk, Dv))) if state else None
    c["dy"] = op(n((T, B, Hv, Dv)))
    c["dST"] = f32(n((B, Hv, Dk, Dv))) if state else None
    return c


def run(c, dtype, backward=True, fused=False, plan=None, scale=0.0, stream=None):
    T, B, Hk, Dk = c["q"].shape
    Hv, Dv = c["v"].shape[2:]
    ld = {x + "_ld": c[x].stride(1) for x in "qkv"} if fused else {}
    if fused:
        ld.update({"d" + n: v for n, v in ld.items()})
    p = plan or ll.DeltaPlan(T, B, Hk, Hv, Dk, Dv, dtype=dtype, scale=scale, **ld)
    new = lambda *s, t=torch.float32: torch.full(s, math.nan, dtype=t, device=DEV)
    r = dict(y=new(T, B, Hv, Dv, t=OP[dtype]), ST=new(B, Hv, Dk, Dv))
    ins = [c[n] for n in ("q", "k", "v", "g", "beta", "seq_len")]
    p.fwd(*ins, c["S0"], r["y"], r["ST"], save_for_backward=backward, stream=stream)
    if backward:
        if fused:
            row = new(T, B, 2 * Hk * Dk + Hv * Dv, t=OP[dtype])
            parts = row.split([Hk * Dk, Hk * Dk, Hv * Dv], 2)
            r.update({"d" + x: a.unflatten(2, s) for x, a, s in
                      zip("qkv", parts, ((Hk, Dk), (Hk, Dk), (Hv, Dv)))})
        else:
            r.update({"d" + x: new(*c[x].shape, t=OP[dtype]) for x in "qkv"})
        r.update(dg=new(T, B, Hv), dbeta=new(T, B, Hv), dS0=new(B, Hv, Dk, Dv))
        p.bwd(*ins, c["dy"], c["dST"], r["dq"], r["dk"], r["dv"], r["dg"], r["dbeta"], r["dS0"],
              stream=stream)
    err = p.status_sync()
    if plan is None:
        p.close()
    return r, err


def reference(c, backward=True, scale=None):
    f = lambda a: None if a is None else a.double().cpu().numpy()
    lens = None if c["seq_len"] is None else c["seq_len"].cpu().numpy()
    y, S, tape = od.delta_forward(*[f(c[n]) for n in ("q", "k", "v", "g", "beta")], lens, f(c["S0"]), scale)
    r = dict(y=y, ST=S)
    if backward:
        r.update(od.delta_backward(tape, f(c["dy"]), f(c["dST"])))
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


CASES = [
    # T, B, Hk, Hv, Dk, Dv, lengths
    (1, 1, 1, 1, 8, 8, None),
    (1, 3, 2, 4, 32, 40, [1, 0, 1]),
    (5, 2, 1, 3, 16, 24, [5, 2]),
    (63, 2, 2, 2, 72, 56, [63, 1]),
    (64, 2, 1, 2, 64, 64, None),
    (65, 3, 2, 2, 128, 128, [65, 64, 0]),
    (129, 2, 1, 2, 120, 136, [129, 66]),
    (200, 3, 2, 4, 24, 96, [200, 0, 130]),
    (300, 1, 1, 1, 128, 8, None),
    (130, 2, 1, 1, 8, 200, [70, 130]),
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
def test_padding_may_hold_nan_and_is_not_read_into_results(dtype):
    lens = [70, 0, 33]
    c = make(80, 3, 1, 2, 32, 32, dtype, lens, seed=7)
    a, _ = run(c, dtype)
    for b, n in enumerate(lens):
        for x in ("q", "k", "v", "g", "beta", "dy"):
            c[x][n:, b] = math.nan
    d, _ = run(c, dtype)
    for n in a:
        assert torch.equal(a[n], d[n]), n
    for b, n in enumerate(lens):
        for x in ("y", "dq", "dk", "dv", "dg", "dbeta"):
            assert not d[x][n:, b].any(), x
    assert torch.equal(d["ST"][1], c["S0"][1]) and torch.equal(d["dS0"][1], c["dST"][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_do_not_depend_on_each_other(dtype):
    c = make(90, 3, 1, 2, 32, 64, dtype, [90, 10, 77], seed=8)
    a, _ = run(c, dtype)
    one = {n: t if t is None else (t[2:3] if n in ("seq_len", "S0", "dST") else t[:, 2:3]).clone(memory_format=torch.contiguous_format)
           for n, t in c.items()}
    b, _ = run(one, dtype)
    for n in b:
        assert torch.equal(b[n], a[n][2:3] if n in ("ST", "dS0") else a[n][:, 2:3]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_extreme_gates(dtype):
    """Full resets (g = -inf), strong decays, beta 0 and tiny, large keys' state."""
    c = make(150, 2, 1, 2, 32, 32, dtype, seed=9)
    c["g"][40, :, 0] = -math.inf
    c["g"][64, :, 1] = -math.inf
    c["g"][100:110] = -60.0
    c["beta"][10:20] = 0.0
    c["beta"][30:35, 0] = 1e-30
    c["beta"][70:80] = 1.0
    got, _ = run(c, dtype)
    ref = reference({**c, "g": c["g"].clamp(min=-700)})
    check(got, ref, dtype)


def test_state_carries_over_pieces_exactly_where_chunks_meet():
    """128 tokens at once, or 64 and 64 with the state handed over: the same chunks, the same bits."""
    c = make(128, 2, 1, 2, 64, 32, "bf16", seed=10)
    whole, _ = run(c, "bf16", backward=False)
    cut = lambda a, b: {n: t if t is None or n in ("seq_len", "S0", "dST") else t[a:b].contiguous() for n, t in c.items()}
    first, _ = run(cut(0, 64), "bf16", backward=False)
    second = cut(64, 128)
    second["S0"] = first["ST"]
    last, _ = run(second, "bf16", backward=False)
    assert torch.equal(torch.cat([first["y"], last["y"]]), whole["y"])
    assert torch.equal(last["ST"], whole["ST"])


def test_state_in_place_and_repeatable():
    c = make(100, 2, 2, 4, 32, 32, "bf16", [100, 51], seed=11)
    a, _ = run(c, "bf16")
    b, _ = run(c, "bf16")
    for n in a:
        assert torch.equal(a[n], b[n]), n
    S = c["S0"].clone()
    with ll.DeltaPlan(100, 2, 2, 4, 32, 32, dtype="bf16", inference=True) as p:
        y = torch.empty_like(a["y"])
        p.fwd(c["q"], c["k"], c["v"], c["g"], c["beta"], c["seq_len"], S, y, S, save_for_backward=False)
        assert p.status_sync() == 0
    assert torch.equal(S, a["ST"]) and torch.equal(y, a["y"])


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
    c = make(130, 2, 1, 2, 32, 32, "bf16", seed=13)
    want, _ = run(c, "bf16")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, _ = run(c, "bf16", stream=s)
    s.synchronize()
    for n in want:
        assert torch.equal(got[n], want[n]), n


def test_captured_into_a_graph():
    c = make(70, 2, 1, 2, 32, 32, "bf16", seed=14)
    T, B, Hk, Dk = c["q"].shape
    p = ll.DeltaPlan(T, B, Hk, 2, Dk, 32, dtype="bf16")
    ins = [c[n] for n in ("q", "k", "v", "g", "beta", "seq_len")]
    out = dict(y=torch.empty_like(c["v"]), ST=torch.empty_like(c["S0"]), dq=torch.empty_like(c["q"]),
               dk=torch.empty_like(c["k"]), dv=torch.empty_like(c["v"]), dg=torch.empty_like(c["g"]),
               dbeta=torch.empty_like(c["beta"]), dS0=torch.empty_like(c["S0"]))

    def step():
        p.fwd(*ins, c["S0"], out["y"], out["ST"])
        p.bwd(*ins, c["dy"], c["dST"], out["dq"], out["dk"], out["dv"], out["dg"], out["dbeta"], out["dS0"])

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in (20, 21, 22):
        new = make(70, 2, 1, 2, 32, 32, "bf16", seed=seed)
        for n, t in new.items():
            if t is not None:
                c[n].copy_(t)
        want, _ = run(new, "bf16")
        g.replay()
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], want[n]), (seed, n)
    p.close()


def test_refusals():
    c = make(10, 2, 1, 2, 16, 16, "f32", seed=15)
    p = ll.DeltaPlan(10, 2, 1, 2, 16, 16)
    ins = [c[n] for n in ("q", "k", "v", "g", "beta", "seq_len")]
    y, ST = torch.empty_like(c["v"]), torch.empty_like(c["S0"])
    outs = [torch.empty_like(c[n]) for n in ("q", "k", "v", "g", "beta")]
    with pytest.raises(ll.LoopError) as e:
        p.bwd(*ins, c["dy"], c["dST"], *outs)
    assert e.value.status == ll.LL_ESTATE
    p.fwd(*ins, c["S0"], y, ST)
    with pytest.raises(ll.LoopError) as e:
        p.bwd(c["q"].clone(), *ins[1:], c["dy"], c["dST"], *outs)
    assert e.value.status == ll.LL_EINVAL
    p.bwd(*ins, c["dy"], c["dST"], *outs)          # the saved forward was kept
    for bad in (c["q"].to(torch.bfloat16), c["q"][:5], c["q"].transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises(ValueError):
            p.fwd(bad, *ins[1:], c["S0"], y, ST)
    odd = torch.empty(c["q"].numel() + 1, device=DEV)[1:].view_as(c["q"])
    with pytest.raises(ll.LoopError) as e:
        p.fwd(odd, *ins[1:], c["S0"], y, ST)
    assert e.value.status == ll.LL_EINVAL and "16-byte" in str(e.value)
    p.close()
    with ll.DeltaPlan(10, 2, 1, 2, 16, 16, inference=True) as p:
        with pytest.raises(ll.LoopError) as e:
            p.fwd(*ins, c["S0"], y, ST)
        assert e.value.status == ll.LL_EINVAL


# ------------------------------------------------------------ one token
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [(1, 1, 1, 8, 8), (3, 2, 4, 32, 32), (5, 1, 3, 128, 136), (4, 4, 4, 72, 40),
                                   (9, 2, 2, 128, 512)], ids=str)
def test_step_against_oracle(sizes, dtype):
    B, Hk, Hv, Dk, Dv = sizes
    c = make(1, B, Hk, Hv, Dk, Dv, dtype, seed=B)
    S, y = c["S0"].clone(), torch.full((B, Hv, Dv), math.nan, dtype=OP[dtype], device=DEV)
    ll.delta_loop_step(c["q"][0], c["k"][0], c["v"][0], c["g"][0], c["beta"][0], S, y)
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
        ll.delta_loop_step(*[c[n][t] for n in ("q", "k", "v", "g", "beta")], S, ys[-1])
    ref = reference(c, backward=False)
    check(dict(y=torch.stack(ys), ST=S), ref, dtype)
    check(want, ref, dtype)


def test_step_slots_and_slices():
    c = make(1, 5, 1, 2, 32, 32, "bf16", seed=4, fused=True)
    pool = torch.randn(9, 2, 32, 32, device=DEV)
    slots = torch.tensor([7, -1, 0, 9, -5], dtype=torch.int32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    S, y = pool.clone(), torch.full((5, 2, 32), math.nan, dtype=torch.bfloat16, device=DEV)
    one = [c[n][0] for n in ("q", "k", "v", "g", "beta")]
    ll.delta_loop_step(*one, S, y, slots=slots, device_error=err)
    assert err.item() == ll.LL_DEVERR_SLOT
    for b, s in enumerate([7, None, 0, None, None]):
        if s is None:
            assert not y[b].any()
            continue
        S1, y1 = pool[s:s + 1].clone(), torch.empty(1, 2, 32, dtype=torch.bfloat16, device=DEV)
        ll.delta_loop_step(*[a[b:b + 1].contiguous() for a in one], S1, y1)
        assert torch.equal(S[s], S1[0]) and torch.equal(y[b], y1[0])
    rest = [i for i in range(9) if i not in (0, 7)]
    assert torch.equal(S[rest], pool[rest])


def test_step_state_past_32_bit_offsets():
    """A pool of more than 2^31 elements: its last slot."""
    n = 33000
    pool = torch.empty(n, 1, 256 // 2, 512, device=DEV)
    pool[-1] = 0.25
    c = make(1, 1, 1, 1, 128, 512, "f32", seed=6)
    c["S0"] = pool[-1:].clone()
    y = torch.empty(1, 1, 512, device=DEV)
    ll.delta_loop_step(*[c[x][0] for x in ("q", "k", "v", "g", "beta")], pool, y,
                       slots=torch.tensor([n - 1], dtype=torch.int32, device=DEV))
    ref = reference(c, backward=False)
    check(dict(y=y, ST=pool[-1:]), dict(y=ref["y"][0], ST=ref["ST"]), "f32")
