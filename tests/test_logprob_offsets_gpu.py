"""GPU: log probabilities and their gradient of rows whose logits share a large
offset (a mask of the type's lowest value over a whole row is one), every entry held
to its own size, against the float64 oracle.

Tolerances.  A row's sum of V positive terms: 2e-6 of it (products, exponentials and
their sum).  log p = (x - m) - log s: that, and 2^-24 of each difference, 2e-6
(1 + |log p|).  lse is stored as one float: 2^-23 of it more.  The entropy, log s -
t / s, has both terms of the size of the spread of the likely logits.  p has the
absolute error of log p and that of the exponent's float product (2^-23 of |log p|)
as its relative one: 4e-6 (1 + |log p|) of p, times the factor it is multiplied by;
that factor's own terms and the marked entries' sums 2e-6 each of what is summed.  A
row's lse that is saved as a float, below 32 in magnitude, adds 2^-20 of p at most.
bfloat16 (8 significant bits) adds 2^-8 of the value.
"""
import math

import numpy as np
import pytest
import torch

from oracle import logprob as ol
from paper_1805_01772_amd import lstmloop as ll
from test_logprob_gpu import DEV, OP, fwd, targets, weights

pytestmark = pytest.mark.gpu

KINDS = ["normal", "lowest", "lowest and not allowed", "one above lowest", 20.0, -45.0, 200.0, 1e4, -3e5, 1e6, 1e30]


def rows(N, V, dtype, kind, seed=0):
    rng = np.random.default_rng(seed)
    x = 2.5 * rng.standard_normal((N, V))
    low = float(torch.finfo(OP[dtype]).min)
    if kind == "lowest":
        x[:] = low
    elif kind == "lowest and not allowed":
        x[:] = low
        x[:, ::2] = -np.inf
    elif kind == "one above lowest":
        x[:] = low
        x[:, V // 3] = low * 0.5
    elif kind != "normal":
        x += kind
    return torch.from_numpy(x.astype(np.float32)).to(DEV).to(OP[dtype])


def held(got, want, tol, what):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], what)
    assert np.isfinite(got[fine]).all(), what
    off = np.abs(got - np.where(fine, want, 0))[fine] / np.broadcast_to(tol, want.shape)[fine]
    if off.size:
        print(f"    {what}: {off.max():.2f} of the tolerance", flush=True)
        assert off.max() <= 1, (what, off.max())


def check_outputs(x, t, out, top):
    f = ol.logprob_forward(x.double().cpu().numpy(), None if t is None else t.cpu().numpy(), top)
    lp = np.where(f["p"] > 1e-12, f["lp"], 0)
    spread = 1 + np.abs(lp).max(1)
    held(out["lse"], f["lse"], 2.0 ** -23 * np.abs(f["lse"]) + 2e-6, "lse")
    held(out["entropy"], f["entropy"], 2e-6 * spread, "entropy")
    held(out["logp"], f["logp"], 2e-6 * (1 + np.abs(f["logp"])), "logp")
    if top:
        np.testing.assert_array_equal(out["top_ids"].cpu().numpy(), f["top_ids"])
        held(out["top_logp"], f["top_logp"], 2e-6 * (1 + np.abs(f["top_logp"])), "top_logp")
    return f


def check_entries(d, f, dl, dh, dt, dtype, what):
    """Every entry by its own p, the marked ones by what is added there too."""
    g = lambda a: None if a is None else a.double().cpu().numpy()
    dl, dh, dt = g(dl), g(dh), g(dt)
    want = ol.logprob_backward(f, dl, dh, dt)
    p, N = f["p"], len(f["p"])
    lp = np.where(p > 0, np.abs(np.where(p > 0, f["lp"], 0)), 0)
    w = np.zeros(N) if dl is None else np.where(f["targets"] < 0, 0, dl)
    c = np.abs(w) + (0 if dt is None else np.abs(dt).sum(1))
    h = np.zeros(N) if dh is None else np.abs(dh)
    tol = p * (1 + lp) * 4e-6 * (c[:, None] + h[:, None] * (lp + f["entropy"][:, None] + 1))
    r = np.arange(N)
    if dl is not None:
        np.add.at(tol, (r, np.maximum(f["targets"], 0)), 2e-6 * np.abs(w))
    if dt is not None:
        for j in range(dt.shape[1]):
            np.add.at(tol, (r, f["top_ids"][:, j]), 2e-6 * np.abs(dt[:, j]))
    held(d, want, tol + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) + 1e-37, what)
    if dtype == "f32":                       # a row's gradient sums to 0
        total = d.double().sum(1).cpu().numpy()
        assert (np.abs(total) <= tol.sum(1) + 1e-30).all(), (what, np.abs(total).max())


SHAPES = [(5, 5000, 8), (700, 5000, 3), (3, 280001, 16), (300, 33000, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_its_gradient(shape, kind, dtype):
    N, V, top = shape
    x, t = rows(N, V, dtype, kind, seed=V), targets(N, V)
    p, out = fwd(x, t, top, dtype)
    f = check_outputs(x, t, out, top)
    dl, dh, dt = weights(N, top)
    d = torch.full_like(x, math.nan)
    for a, b, c, what in ((dl, dh, dt, "all"), (dl, None, None, "dlogp"), (None, dh, None, "dentropy"),
                          (None, None, dt, "dtop")):
        if what == "dtop" and not top:
            continue
        p.bwd(x, t, out["lse"], out["entropy"], out.get("top_ids"), a, b, c, d)
        check_entries(d, f, a, b, c, dtype, what)
    p.bwd(x, t, out["lse"], out["entropy"], out.get("top_ids"), dl, dh, dt, d)
    p.bwd(x, t, out["lse"], out["entropy"], out.get("top_ids"), dl, dh, dt, x)  # in place: the same bits
    assert torch.equal(x, d)
    p.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("shape", [(5, 5000), (300, 33000), (2, 140001)], ids=str)
def test_both_in_one_call(shape, kind, dtype):
    N, V = shape
    x, t = rows(N, V, dtype, kind, seed=V + 1), targets(N, V)
    dl, dh, _ = weights(N, 0)
    out = {n: torch.full((N,), math.nan, device=DEV) for n in ("logp", "entropy", "lse")}
    d = torch.full_like(x, math.nan)
    with ll.LogprobPlan(N, V, dtype=dtype) as p:
        p.fwd_bwd(x, t, dl, dh, out["logp"], out["entropy"], out["lse"], d)
        f = check_outputs(x, t, out, 0)
        check_entries(d, f, dl, dh, None, dtype, "both")
        p.fwd_bwd(x, t, dl, None, out["logp"], None, None, d)
        check_entries(d, f, dl, None, None, dtype, "dlogp")


@pytest.mark.parametrize("offset", [0.0, 60.0, -500.0])
def test_a_vocabulary_in_two_parts(offset):
    """Each part's logits with the lse and entropy of the whole: an lse that is not
    this row's own is taken as it is."""
    N, V = 6, 4000
    x = rows(N, 2 * V, "f32", offset or "normal", seed=5)
    f = ol.logprob_forward(x.double().cpu().numpy(), None)
    lse = torch.from_numpy(f["lse"]).float().to(DEV)
    _, dh, _ = weights(N, 0)
    ent = torch.from_numpy(f["entropy"]).float().to(DEV)
    # p from the stored float's own value
    p = np.exp(x.double().cpu().numpy() - lse.double().cpu().numpy()[:, None])
    lp = np.log(p)
    h, e = dh.double().cpu().numpy()[:, None], ent.double().cpu().numpy()[:, None]
    want, tol = -p * h * (lp + e), 4e-6 * p * np.abs(h) * (1 + np.abs(lp)) * (1 + np.abs(lp) + e) + 1e-37
    with ll.LogprobPlan(N, V) as plan:
        for part in (slice(0, V), slice(V, 2 * V)):
            y = x[:, part].contiguous()
            d = torch.empty_like(y)
            plan.bwd(y, None, lse, ent, None, None, dh, None, d)
            held(d, want[:, part], tol[:, part], "part")
