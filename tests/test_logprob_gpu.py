"""GPU: log probabilities, entropy, alternatives and their gradient against the
float64 oracle.

Tolerances.  lse, logp and entropy are sums of V positive float terms of a few
roundings each (2^-23 of the value or of lse, whichever is larger): 2e-6 of the
row's |lse| + 1, entropy times the logits' spread (log s - t / s: both terms of
the size of the spread).  Gradients: p has the relative error of lse's absolute
one, 1e-5 of the largest entry of a row; bfloat16 (8 significant bits) adds half a
unit, 2^-8.  Ids are equal.
"""
import math

import numpy as np
import pytest
import torch

from oracle import logprob as ol
from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
OP = {"f32": torch.float32, "bf16": torch.bfloat16}


def logits(N, V, dtype, seed=0, ld=None, scale=2.5, kind="normal"):
    rng = np.random.default_rng(seed)
    x = scale * rng.standard_normal((N, V))
    if kind == "ties":
        x = np.round(x)
    elif kind == "equal":
        x[:] = -1.5
    elif kind == "rising":
        x = np.tile(np.linspace(-4, 4, V), (N, 1))
    elif kind == "spiky":
        x[:, ::2048] += 20          # the largest ones of many rows' threads together
    elif kind == "large":
        x = 1e30 * np.sign(x) * (np.abs(x) > 3) + x
    ld = ld or V
    buf = torch.full((N, ld), math.nan, dtype=OP[dtype], device=DEV)
    buf[:, :V] = torch.from_numpy(x.astype(np.float32)).to(DEV).to(OP[dtype])
    return buf[:, :V]


def fwd(x, t, top, dtype, N=None):
    n, V = x.shape
    out = dict(logp=torch.full((n,), math.nan, device=DEV), entropy=torch.full((n,), math.nan, device=DEV),
               lse=torch.full((n,), math.nan, device=DEV))
    ids = torch.full((n, top), -7, dtype=torch.int32, device=DEV) if top else None
    tl = torch.full((n, top), math.nan, device=DEV) if top else None
    p = ll.LogprobPlan(N or n, V, dtype=dtype, top_k=top, ld=x.stride(0) if n > 1 else 0)
    p.fwd(x, t, out["logp"], out["entropy"], out["lse"], ids, tl)
    if top:
        out.update(top_ids=ids, top_logp=tl)
    return p, out


def near(got, want, tol, what):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], what)
    assert np.isfinite(got[fine]).all(), what
    err = np.abs(got - np.where(fine, want, 0))[fine] / np.broadcast_to(tol, want.shape)[fine]
    if err.size:
        print(f"    {what}: {err.max():.2f} of the tolerance", flush=True)
        assert err.max() <= 1, (what, err.max())


def check_fwd(x, t, out, top):
    ref = ol.logprob_forward(x.double().cpu().numpy(), None if t is None else t.cpu().numpy(), top)
    size = np.where(np.isfinite(ref["lse"]), np.abs(ref["lse"]), 0) + 1
    near(out["lse"], ref["lse"], 2e-6 * size, "lse")
    xs = x.double().cpu().numpy()
    ok = np.isfinite(xs) & (ref["p"] > 1e-12)
    spread = np.array([np.ptp(r[o]) if o.any() else 0 for r, o in zip(xs, ok)]) + 1
    near(out["entropy"], ref["entropy"], 2e-6 * (size + spread), "entropy")
    if t is not None:
        big = np.where(np.isfinite(ref["logp"]), np.abs(ref["logp"]), 0)
        near(out["logp"], ref["logp"], 2e-6 * (size + big), "logp")
    if top:
        np.testing.assert_array_equal(out["top_ids"].cpu().numpy(), ref["top_ids"])
        big = np.where(np.isfinite(ref["top_logp"]), np.abs(ref["top_logp"]), 0)
        near(out["top_logp"], ref["top_logp"], 2e-6 * (size[:, None] + big), "top_logp")
    return ref


def targets(N, V, seed=1):
    rng = np.random.default_rng(seed)
    t = rng.integers(0, V, N)
    t[::3] = -1
    if N > 1:
        t[1] = V - 1
    return torch.from_numpy(t.astype(np.int32)).to(DEV)


SHAPES = [(1, 1, 1), (2, 3, 2), (3, 7, 4), (5, 40, 32), (4, 257, 8), (3, 1000, 16), (2, 4099, 32), (300, 2000, 8),
          (600, 515, 4), (1, 70001, 16), (7, 33000, 32), (40, 9000, 0), (2, 131072, 5), (700, 4096, 20)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype):
    N, V, top = shape
    x, t = logits(N, V, dtype, seed=V), targets(N, V)
    p, out = fwd(x, t, top, dtype)
    check_fwd(x, t, out, top)
    assert p.status_sync() == 0
    p.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["ties", "equal", "rising", "spiky", "large"])
@pytest.mark.parametrize("shape", [(4, 3001, 16), (2, 100003, 32), (600, 2048, 32)], ids=str)
def test_hard_orders(kind, shape, dtype):
    N, V, top = shape
    x, t = logits(N, V, dtype, seed=3, kind=kind), targets(N, V)
    p, out = fwd(x, t, top, dtype)
    check_fwd(x, t, out, top)
    p.close()


@pytest.mark.parametrize("N", [6, 800])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks(dtype, N):
    """Minus infinity and the type's lowest value: some, all but one, all; and
    their gradients."""
    V, top = 5000, 8
    x, t = logits(N, V, dtype, seed=4), targets(N, V)
    low = torch.finfo(OP[dtype]).min
    x[0, 1000:] = -math.inf
    x[1] = -math.inf
    x[2] = low
    x[3] = -math.inf
    x[3, 77] = 3.0
    x[4, :4999] = low
    x[5, ::2] = -math.inf
    x[5, 1::2] = low
    t[0], t[1], t[4], t[5] = 2000, 3, 4999, 8
    p, out = fwd(x, t, top, dtype)
    check_fwd(x, t, out, top)
    run_gradient(p, x, t, out, dtype, top)
    p.close()


def weights(N, top, seed=9):
    rng = np.random.default_rng(seed)
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV)
    return f(N), f(N), (f(N, top) if top else None)


def check_gradient(d, x, t, dl, dh, dt, dtype, top):
    ref = ol.logprob_forward(x.double().cpu().numpy(), None if t is None else t.cpu().numpy(), top)
    f = lambda a: None if a is None else a.double().cpu().numpy()
    want = ol.logprob_backward(ref, f(dl), f(dh), f(dt))
    top_of = np.abs(want).max(1, keepdims=True)
    lse = np.where(np.isfinite(ref["lse"]), np.abs(ref["lse"]), 0)[:, None]
    tol = 1e-5 * top_of * (1 + lse) + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) + 1e-37
    near(d, want, tol, "dlogits")


def run_gradient(p, x, t, out, dtype, top):
    N = x.shape[0]
    dl, dh, dt = weights(N, top)
    d = torch.full((N, x.stride(0)), math.nan, dtype=OP[dtype], device=DEV)[:, :x.shape[1]]
    p.bwd(x, t, out["lse"], out["entropy"], out.get("top_ids"), dl, dh, dt, d)
    check_gradient(d, x, t, dl, dh, dt, dtype, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradient(shape, dtype):
    N, V, top = shape
    x, t = logits(N, V, dtype, seed=V + 1), targets(N, V)
    p, out = fwd(x, t, top, dtype)
    if top:
        t[0] = out["top_ids"][0, 0]            # a token that is target and alternative
    run_gradient(p, x, t, out, dtype, top)
    dl, dh, dt = weights(N, top)
    d = torch.empty_like(x)
    for a, b, c in ((dl, None, None), (None, dh, None), (None, None, dt), (None, None, None)):
        p.bwd(x, t, out["lse"], out["entropy"] if b is not None else None,
              out.get("top_ids") if c is not None else None, a, b, c, d)
        check_gradient(d, x, t, a, b, c, dtype, top)
    p.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES + [(3, 200001, 0), (2, 66000, 0)], ids=str)
def test_both_in_one_call(shape, dtype):
    N, V, _ = shape
    x, t = logits(N, V, dtype, seed=V + 2), targets(N, V)
    if N > 2:
        x[2] = -math.inf
    dl, dh, _ = weights(N, 0)
    p = ll.LogprobPlan(N, V, dtype=dtype)
    out = {n: torch.full((N,), math.nan, device=DEV) for n in ("logp", "entropy", "lse")}
    d = torch.full_like(x, math.nan)
    p.fwd_bwd(x, t, dl, dh, out["logp"], out["entropy"], out["lse"], d)
    check_fwd(x, t, out, 0)
    check_gradient(d, x, t, dl, dh, None, dtype, 0)
    keep = x.clone()
    p.fwd_bwd(x, t, dl, dh, out["logp"], out["entropy"], out["lse"], x)     # in place
    assert torch.equal(x, d)
    p.fwd_bwd(keep, None, None, dh, None, None, None, d)                    # entropy alone, no outputs
    check_gradient(d, keep, None, None, dh, None, dtype, 0)
    p.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows_in_place_and_fewer_rows(dtype):
    """Rows 1003 apart (no alignment but an element's), the gradient over the
    logits, a plan made for more rows; what lies between the rows stays."""
    N, V, top = 9, 1001, 6
    x, t = logits(N, V, dtype, seed=8, ld=1003), targets(N, V)
    p, out = fwd(x, t, top, dtype, N=50)
    check_fwd(x, t, out, top)
    dl, dh, dt = weights(N, top)
    want = torch.empty(N, 1003, dtype=OP[dtype], device=DEV)[:, :V]
    p.bwd(x, t, out["lse"], out["entropy"], out["top_ids"], dl, dh, dt, want)
    p.bwd(x, t, out["lse"], out["entropy"], out["top_ids"], dl, dh, dt, x)
    assert torch.equal(x, want)
    assert torch.isnan(torch.as_strided(x, (N, 2), (1003, 1), V)).all()
    p.fwd(x[:0], t[:0], out["logp"][:0], None, None, out["top_ids"][:0], out["top_logp"][:0])
    p.close()


@pytest.mark.parametrize("N", [3, 400])
def test_nan_and_infinity_stay_in_their_rows(N):
    x, t = logits(N, 6000, "f32", seed=10), targets(N, 6000)
    _, clean = fwd(x, t, 8, "f32")
    x[1, 5] = math.nan
    x[2, 5999] = math.inf
    _, out = fwd(x, t, 8, "f32")
    keep = [0] + list(range(3, N))
    for n in out:
        assert torch.equal(out[n][keep], clean[n][keep]), n
    assert torch.isnan(out["lse"][1:3]).all() and torch.isnan(out["entropy"][1:3]).all()
    assert ((out["top_ids"] >= 0) & (out["top_ids"] < 6000)).all()
    x[0] = math.nan
    _, out = fwd(x, t, 8, "f32")
    assert ((out["top_ids"] >= 0) & (out["top_ids"] < 6000)).all()


def test_bad_targets_are_reported():
    x = logits(4, 100, "f32", seed=11)
    t = torch.tensor([5, 100, -2, -1], dtype=torch.int32, device=DEV)
    p, out = fwd(x, t, 0, "f32")
    assert p.status_sync() == ll.LL_DEVERR_TARGET and p.status_sync() == 0
    check_fwd(x, t, out, 0)
    run_gradient(p, x, t, out, "f32", 0)
    p.close()


def test_repeatable_and_split_rows_again():
    """Rows split over work-groups: the second call finds the arrivals cleared."""
    x, t = logits(2, 90000, "bf16", seed=12), targets(2, 90000)
    p, a = fwd(x, t, 16, "bf16")
    for _ in range(3):
        b = {n: torch.zeros_like(v) for n, v in a.items()}
        p.fwd(x, t, b["logp"], b["entropy"], b["lse"], b["top_ids"], b["top_logp"])
        for n in a:
            assert torch.equal(a[n], b[n]), n
    p.close()


def test_offsets_past_32_bits():
    """The last rows of a bfloat16 batch of more than 2^31 elements."""
    N, V = 17000, 131072
    x = torch.zeros(N, V, dtype=torch.bfloat16, device=DEV)
    tail = logits(3, V, "bf16", seed=13)
    x[-3:] = tail
    t = targets(N, V)
    p, out = fwd(x, t, 4, "bf16")
    small = {n: v[-3:] for n, v in out.items()}
    check_fwd(tail, t[-3:], small, 4)
    dl, dh, dt = weights(N, 4)
    p.bwd(x, t, out["lse"], out["entropy"], out["top_ids"], dl, dh, dt, x)
    check_gradient(x[-3:], tail, t[-3:], dl[-3:], dh[-3:], dt[-3:], "bf16", 4)
    p.close()


def test_refusals():
    x, t = logits(4, 64, "f32", seed=14), targets(4, 64)
    v = torch.empty(4, device=DEV)
    d = torch.empty_like(x)
    with ll.LogprobPlan(4, 64, top_k=2) as p:
        for call in (lambda: p.fwd(x, t, v, v, v), lambda: p.fwd(x, None, v, v, v, v, v),
                     lambda: p.fwd(x.bfloat16(), t, v), lambda: p.fwd(x[:, :32], t, v)):
            with pytest.raises((ll.LoopError, ValueError)):
                call()
        for call in (lambda: p.bwd(x, None, v, None, None, v, None, None, d),
                     lambda: p.bwd(x, t, v, None, None, None, v, None, d),
                     lambda: p.bwd(x, t, v, None, None, None, None, torch.empty(4, 2, device=DEV), d),
                     lambda: p.fwd_bwd(x, None, v, None, None, None, None, d)):
            with pytest.raises(ll.LoopError) as e:
                call()
            assert e.value.status == ll.LL_EINVAL
        big = logits(5, 64, "f32")
        with pytest.raises(ll.LoopError):
            p.fwd(big, targets(5, 64), torch.empty(5, device=DEV), None, None,
                  torch.empty(5, 2, dtype=torch.int32, device=DEV), torch.empty(5, 2, device=DEV))
