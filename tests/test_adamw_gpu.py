"""GPU: AdamW over many tensors against float64, and the 8-bit states' codes.

Tolerances.  m, v, p: at most five float roundings, 2^-24 each, of the terms
summed: 4e-7 of the largest term; the update has a root and a reciprocal of one
unit more: 1e-6 of it.  An 8-bit state's code is one of the two next to the
value; one unit further where the value lies within 1e-5 of a code.
"""
import math

import numpy as np
import pytest
import torch

from oracle import adamw as oa
from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=7)
SIZES = [1, 2, 3, 5, 255, 256, 257, 4095, 4096, 4097, 0, 10000, 65536 + 3]


def tensors(sizes, bits, grad, seed=0):
    rng = np.random.default_rng(seed)
    f = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(DEV)
    n = rng.standard_normal
    d = dict(p=[f(n(s)) for s in sizes], g=[f(0.1 * n(s)) for s in sizes])
    if grad == "bf16":
        d["g"] = [a.bfloat16() for a in d["g"]]
    if bits == 32:
        d["m"], d["v"] = [f(0.05 * n(s)) for s in sizes], [f((0.1 * n(s)) ** 2) for s in sizes]
    else:
        rows = [-(-s // 256) for s in sizes]
        d["m"] = [torch.from_numpy(rng.integers(-127, 128, s).astype(np.int8)).to(DEV) for s in sizes]
        d["v"] = [torch.from_numpy(rng.integers(0, 256, s).astype(np.uint8)).to(DEV) for s in sizes]
        d["ms"], d["vs"] = [f(0.1 * rng.random(r)) for r in rows], [f(0.01 * rng.random(r)) for r in rows]
    d["copy"] = [torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in sizes]
    d["wd"] = [0.1 if i % 2 else 0.0 for i in range(len(sizes))]
    return d


def clone(d):
    return {k: [a.clone() for a in v] if k != "wd" else v for k, v in d.items()}


def plan(d, bits, grad, copies=True):
    q = dict(m_scale=d["ms"], v_scale=d["vs"]) if bits == 8 else {}
    return ll.AdamWPlan(d["p"], d["m"], d["v"], copies=d["copy"] if copies else None,
                        weight_decay=d["wd"], grad_dtype=grad, **q)


def f64(a):
    return a.double().cpu().numpy()


def close(got, want, terms, tol, what):
    err = np.abs(f64(got) - want)
    assert (err <= tol * terms + 1e-38).all(), (what, (err / (terms + 1e-38)).max())


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_step(bits, grad):
    d = tensors(SIZES, bits, grad)
    old = clone(d)
    scale = torch.tensor([0.5], device=DEV)
    with plan(d, bits, grad) as p:
        p.step(d["g"], grad_scale=scale, seed=3, **HYPER)
    for i, s in enumerate(SIZES):
        if not s:
            continue
        if bits == 32:
            m0, v0 = f64(old["m"][i]), f64(old["v"][i])
        else:
            m0, v0 = oa.dequant(*(old[n][i].cpu().numpy() for n in ("m", "v", "ms", "vs")))
        p0, g0 = f64(old["p"][i]), f64(old["g"][i])
        p1, m1, v1 = oa.adamw(p0, g0, m0, v0, weight_decay=d["wd"][i], grad_scale=0.5, **HYPER)
        close(d["p"][i], p1, np.abs(p0) + 10 * np.abs(p1 - p0), 1e-6, "p")
        assert torch.equal(d["copy"][i], d["p"][i].bfloat16())
        if bits == 32:
            close(d["m"][i], m1, np.abs(m0) + np.abs(g0), 4e-7, "m")
            close(d["v"][i], v1, v0 + g0 * g0, 4e-7, "v")
            continue
        for x, name, power, top in ((m1, "m", 2, 127), (v1, "v", 4, 255)):
            sc = f64(d[name + "s"][i])
            np.testing.assert_allclose(sc, oa.row_max(x), rtol=2e-6)
            lo, chance = oa.neighbours(x, sc, power, top)
            c = d[name][i].cpu().numpy().astype(int)
            if name == "m":
                assert ((np.sign(c) == np.sign(x)) | (c == 0)).all()
                c = np.abs(c)
            else:
                assert (c[x > 0] >= 1).all()
                lo = np.maximum(lo, 1 - (chance > 0))       # never 0 for a positive value
            ok = (c == lo) | (c == lo + 1) | ((c == lo - 1) & (chance < 1e-4)) | ((c == 1) & (lo == 0))
            assert ok.all(), (name, i)


def test_random_rounding_keeps_the_mean():
    """The mean of the codes' values over 400 seeds against the value: 6 of its
    standard errors."""
    n = 256
    d = tensors([n], 8, "f32", seed=5)
    old = clone(d)
    got = np.zeros((2, 400, n))
    for seed in range(400):
        d = clone(old)
        with plan(d, 8, "f32") as p:
            p.step(d["g"], seed=seed, **HYPER)
        got[:, seed] = oa.dequant(*(d[k][0].cpu().numpy() for k in ("m", "v", "ms", "vs")))
    m0, v0 = oa.dequant(*(old[k][0].cpu().numpy() for k in ("m", "v", "ms", "vs")))
    _, m1, v1 = oa.adamw(f64(old["p"][0]), f64(old["g"][0]), m0, v0, weight_decay=0.0, **HYPER)
    for x, want, power, top in ((got[0], m1, 2, 127), (got[1], v1, 4, 255)):
        lo, chance = oa.neighbours(want, oa.row_max(want), power, top)
        gap = oa.row_max(want)[0] * (((lo + 1) / top) ** power - (lo / top) ** power)
        se = gap * np.sqrt(np.maximum(chance * (1 - chance), 1e-4) / 400)
        rare = np.abs(want) < oa.row_max(want)[0] * (1.0 / top) ** power if power == 4 else np.zeros(n, bool)
        assert (np.abs(x.mean(0) - want) < 6 * se + gap / 65536 + 1e-6 * np.abs(want))[~rare].all()
    assert len({got[0, s].tobytes() for s in range(400)}) > 390


def test_a_slow_average_moves_on():
    """v under a gradient a tenth of the old one's: 300 steps of 0.99 bring it
    down as float would, within the codes' width."""
    n = 1024
    d = tensors([n], 8, "f32", seed=6)
    d["v"][0].fill_(200)
    d["vs"][0].fill_(1e-2)
    d["g"][0].fill_(0.01)
    with plan(d, 8, "f32") as p:
        for s in range(300):
            p.step(d["g"], lr=0.0, beta1=0.9, beta2=0.99, step=s + 1, seed=s)
    _, v = oa.dequant(*(d[k][0].cpu().numpy() for k in ("m", "v", "ms", "vs")))
    v0 = (200 / 255) ** 4 * 1e-2
    want = v0 * 0.99 ** 300 + 1e-4 * (1 - 0.99 ** 300)
    assert abs(v.mean() / want - 1) < 0.05


def test_from_zero_states():
    """The first step from zeroed codes: sign(g) lr within eps, whatever the size."""
    n = 600
    d = tensors([n], 8, "f32", seed=7)
    for k in ("m", "v", "ms", "vs"):
        d[k][0].zero_()
    d["g"][0][:300] *= 1e-4
    d["g"][0][5] = 0.0
    old = clone(d)
    with plan(d, 8, "f32") as p:
        p.step(d["g"], lr=1e-3, step=1)
    up = f64(old["p"][0]) - f64(d["p"][0])
    want, _, _ = oa.adamw(f64(old["p"][0]), f64(old["g"][0]), np.zeros(n), np.zeros(n), 1e-3, 0.9, 0.999, 1e-8,
                          1, 0.0)
    np.testing.assert_allclose(up, f64(old["p"][0]) - want, atol=3e-7)


@pytest.mark.parametrize("bits", [32, 8])
def test_missing_gradients_and_skipped_steps(bits):
    d = tensors([300, 5000, 70], bits, "f32", seed=8)
    old = clone(d)
    with plan(d, bits, "f32") as p:
        p.step([d["g"][0], None, d["g"][2]], **HYPER)
        for k in d:
            if k not in ("wd", "g"):
                assert torch.equal(d[k][1], old[k][1]), k
        assert not torch.equal(d["p"][0], old["p"][0]) and not torch.equal(d["p"][2], old["p"][2])
        mid = clone(d)
        for bad in (math.inf, -math.inf, math.nan):
            p.step(d["g"], grad_scale=torch.tensor([bad], device=DEV), **HYPER)
        for k in d:
            if k != "wd":
                assert all(torch.equal(a, b) for a, b in zip(d[k], mid[k])), k


def test_nan_gradient_stays_visible():
    """8 bits: the row of a NaN is NaN afterwards, its neighbours are not."""
    d = tensors([1024], 8, "f32", seed=9)
    d["g"][0][300] = math.nan
    with plan(d, 8, "f32") as p:
        p.step(d["g"], **HYPER)
    assert torch.isnan(d["ms"][0]).tolist() == [False, True, False, False]
    assert torch.isnan(d["vs"][0]).tolist() == [False, True, False, False]


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(bits):
    """More tensors than one launch's gradients; each like it had been alone."""
    sizes = [17 + 13 * i for i in range(600)]
    d = tensors(sizes, bits, "f32", seed=10)
    old = clone(d)
    with plan(d, bits, "f32") as p:
        p.step(d["g"], **HYPER)
    for i in (0, 255, 256, 511, 512, 599):
        one = {k: [v[i]] for k, v in clone(old).items()}
        with plan(one, bits, "f32") as p:
            p.step(one["g"], **HYPER)
        assert torch.equal(one["p"][0], d["p"][i])
        if bits == 32:
            assert torch.equal(one["m"][0], d["m"][i]) and torch.equal(one["v"][0], d["v"][i])


def test_elements_past_32_bit_offsets():
    """A tensor of 2^30 + 9 floats: byte offsets past 2^32, its last elements."""
    n = (1 << 30) + 9
    p, g = torch.ones(n, device=DEV), torch.full((n,), 0.5, device=DEV)
    m, v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    with ll.AdamWPlan([p], [m], [v]) as plan_:
        plan_.step([g], lr=0.25, step=1)
    for x, want in ((p, 0.75), (m, 0.05), (v, 0.00025)):
        for part in (x[:100], x[-100:], x[1 << 29:(1 << 29) + 100]):
            np.testing.assert_allclose(f64(part), want, rtol=1e-6)


def test_repeatable_and_other_stream():
    a, b = tensors(SIZES, 8, "bf16", seed=11), tensors(SIZES, 8, "bf16", seed=11)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with plan(a, 8, "bf16") as p, plan(b, 8, "bf16") as q:
        for k in range(3):
            p.step(a["g"], seed=k, **HYPER)
            q.step(b["g"], seed=k, stream=s, **HYPER)
        torch.cuda.synchronize()
    for k in a:
        if k != "wd":
            assert all(torch.equal(x, y) for x, y in zip(a[k], b[k])), k


def test_refusals():
    d = tensors([100, 7], 32, "f32", seed=12)
    with plan(d, 32, "f32") as p:
        for kw in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(lr=-1.0),
                   dict(lr=math.nan)):
            with pytest.raises(ll.LoopError) as e:
                p.step(d["g"], **{**HYPER, **kw})
            assert e.value.status == ll.LL_EINVAL
        for bad in (d["g"][:1], [d["g"][0].bfloat16(), d["g"][1]], [d["g"][0][:50], d["g"][1]]):
            with pytest.raises(ValueError):
                p.step(bad, **HYPER)
        odd = torch.empty(101, device=DEV)[1:]
        with pytest.raises(ll.LoopError) as e:
            p.step([odd, d["g"][1]], **HYPER)
        assert "16-byte" in str(e.value)
    with pytest.raises(ValueError):
        ll.AdamWPlan(d["p"], d["m"][:1], d["v"])
    with pytest.raises(ValueError):
        ll.AdamWPlan(d["p"], d["m"], d["v"], m_scale=d["p"])
