"""GPU: arrays that start anywhere an element may: logits shifted by a token, targets and
weights from the second on, gates of a later time step.  Tolerances as in the other
tests of the operators; where only the output lies elsewhere, the same bits."""
import ctypes
import math

import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll
from test_delta_gpu import make, run
from test_logprob_gpu import DEV, OP, check_fwd, check_gradient, logits, targets, weights

pytestmark = pytest.mark.gpu


def moved(t, by):
    """The same values, `by` elements past an allocation's start, with guards around."""
    buf = torch.full((t.numel() + by + 8,), 7, dtype=t.dtype, device=DEV)
    view = buf[by:by + t.numel()].view(t.shape)
    view.copy_(t)
    return view, buf


def guards_stand(buf, by, n):
    assert (buf[:by] == 7).all() and (buf[by + n:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5, 1001, 6), (600, 515, 4), (3, 280001, 8), (4, 40003, 0)], ids=str)
@pytest.mark.parametrize("by", [1, 3])
def test_logits_and_the_rest_shifted(shape, by, dtype):
    N, V, top = shape
    (x, _), (t, _) = moved(logits(N, V, dtype, seed=V), by), moved(targets(N, V), by)
    x[N // 2] = -math.inf
    f = lambda *s, d=torch.float32: moved(torch.zeros(*s, dtype=d, device=DEV), by)[0]
    out = dict(logp=f(N), entropy=f(N), lse=f(N))
    if top:
        out.update(top_ids=f(N, top, d=torch.int32), top_logp=f(N, top))
    dl, dh, dt = (None if w is None else moved(w, by)[0] for w in weights(N, top))
    with ll.LogprobPlan(N, V, dtype=dtype, top_k=top) as p:
        p.fwd(x, t, **out)
        check_fwd(x, t, out, top)
        want = None
        for at in (by, 0, 2, 5):             # as the logits, then otherwise
            d, buf = moved(torch.zeros_like(x), at)
            p.bwd(x, t, out["lse"], out["entropy"], out.get("top_ids"), dl, dh, dt, d)
            check_gradient(d, x, t, dl, dh, dt, dtype, top)
            guards_stand(buf, at, N * V)
            want = d.clone() if want is None else want
            assert torch.equal(d, want), at
        want = None
        for at in (by, 0, 2, 5):
            d, buf = moved(torch.zeros_like(x), at)
            p.fwd_bwd(x, t, dl, dh, out["logp"], out["entropy"], out["lse"], d)
            check_fwd(x, t, {n: out[n] for n in ("logp", "entropy", "lse")}, 0)
            check_gradient(d, x, t, dl, dh, None, dtype, 0)
            guards_stand(buf, at, N * V)
            want = d.clone() if want is None else want
            assert torch.equal(d, want), at
        p.fwd_bwd(x, t, dl, dh, out["logp"], out["entropy"], out["lse"], x)     # in place
        assert torch.equal(x, want)


def test_the_next_token_s_loss():
    """logits[:-1] against targets[1:] of one sequence, and the other way round, of an odd width."""
    x, t = logits(20, 1001, "bf16", seed=3), targets(20, 1001)
    for a, b in ((x[:-1], t[1:]), (x[1:], t[:-1])):
        out = dict(logp=torch.zeros(19, device=DEV), entropy=torch.zeros(19, device=DEV),
                   lse=torch.zeros(19, device=DEV))
        d, (dl, dh, _) = torch.empty(19, 1001, dtype=torch.bfloat16, device=DEV), weights(19, 0)
        with ll.LogprobPlan(19, 1001, dtype="bf16") as p:
            p.fwd_bwd(a, b, dl, dh, out["logp"], out["entropy"], out["lse"], d)
        check_fwd(a, b, out, 0)
        check_gradient(d, a, b, dl, dh, None, "bf16", 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_and_lengths_shifted(dtype):
    c = make(90, 3, 1, 3, 16, 24, dtype, [90, 10, 0], seed=4)
    want, _ = run(c, dtype)
    for n in ("g", "beta", "seq_len"):
        c[n] = moved(c[n], 3)[0]
    got, err = run(c, dtype)
    assert err == 0
    for n in want:
        assert torch.equal(got[n], want[n]), n
    (dg, b1), (db, b2) = (moved(torch.zeros_like(want[n]), 1) for n in ("dg", "dbeta"))
    ins = [c[n] for n in ("q", "k", "v", "g", "beta", "seq_len")]
    with ll.DeltaPlan(90, 3, 1, 3, 16, 24, dtype=dtype) as p:
        p.fwd(*ins, c["S0"], torch.empty_like(c["v"]), None)
        p.bwd(*ins, c["dy"], c["dST"], *(torch.empty_like(c[n]) for n in "qkv"), dg, db)
    assert torch.equal(dg, want["dg"]) and torch.equal(db, want["dbeta"])
    guards_stand(b1, 1, dg.numel())
    guards_stand(b2, 1, db.numel())


def test_steps_through_the_gates_of_a_sequence():
    """g[t] and beta[t] of a single row with one head: every fourth one is 16-byte aligned."""
    c = make(9, 1, 1, 1, 16, 16, "f32", seed=5)
    want, _ = run(c, "f32", backward=False)
    S, y = c["S0"].clone(), torch.empty_like(c["v"][0])
    slots, err = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    for t in range(9):
        ll.delta_loop_step(*(c[n][t] for n in ("q", "k", "v", "g", "beta")), S, y, slots=slots[1:2],
                           device_error=err[2:])
        assert (y - want["y"][t]).norm() <= 1e-5 * want["y"][t].norm()
    assert not err.any()


def test_what_is_still_refused():
    lib = ll.load_library()
    x, t = logits(4, 64, "f32"), targets(4, 64)
    v = torch.zeros(64, device=DEV)
    with ll.LogprobPlan(4, 64) as p:
        at = lambda a, by=0: ctypes.c_void_p(a.data_ptr() + by)
        fwd = lambda a, b, c: lib.ll_logprob_fwd(p._h, None, 3, a, b, c, None, None, None, None)
        for bad in ((at(x, 2), at(t), at(v)), (at(x), at(t, 2), at(v)), (at(x), at(t), at(v, 1))):
            assert fwd(*bad) == ll.LL_EINVAL and "4-byte aligned" in ll.ll_last_error()
        assert lib.ll_logprob_bwd(p._h, None, 3, at(x), None, at(v), *[None] * 5, at(x, 2)) == ll.LL_EINVAL
        assert lib.ll_logprob_fwd_bwd(p._h, None, 3, at(x), *[None] * 6, at(x, 2)) == ll.LL_EINVAL
    q = torch.zeros(256, device=DEV)
    d = ll.make_delta_desc(1, 1, 1, 1, 8, 8)
    step = lambda *o: lib.delta_loop_step(ctypes.byref(d), None, *(ctypes.c_void_p(q.data_ptr() + i) for i in o),
                                          None, 1, at(q), None)
    for bad in ((4, 0, 0, 0, 0, 0), (0, 8, 0, 0, 0, 0), (0, 0, 4, 0, 0, 0), (0, 0, 0, 2, 0, 0), (0, 0, 0, 0, 1, 0),
                (0, 0, 0, 0, 0, 4)):
        assert step(*bad) == ll.LL_EINVAL and "aligned" in ll.ll_last_error()
