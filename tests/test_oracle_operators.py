"""Pins for the oracles of the gated delta rule, the log probabilities and AdamW
(CPU): closed forms, torch.autograd in float64, central differences."""
import numpy as np
import pytest
import torch

from oracle import adamw as oa, delta as od, logprob as ol


def _delta_case(rng, T=5, B=3, Hk=2, Hv=4, Dk=3, Dv=2):
    n = rng.standard_normal
    return dict(q=n((T, B, Hk, Dk)), k=0.6 * n((T, B, Hk, Dk)), v=n((T, B, Hv, Dv)),
                g=-rng.random((T, B, Hv)), beta=rng.random((T, B, Hv)), S0=0.5 * n((B, Hv, Dk, Dv)))


def test_delta_step_writes_what_the_key_lacks():
    """With beta = 1 and a unit key S_t^T k_t = v_t; with beta = 0 and g = 0 nothing moves."""
    rng = np.random.default_rng(0)
    c = _delta_case(rng, T=1)
    c["k"] /= np.linalg.norm(c["k"], axis=-1, keepdims=True)
    c["beta"][:] = 1
    _, S, _ = od.delta_forward(**c)
    for b in range(3):
        for h in range(4):
            np.testing.assert_allclose(S[b, h].T @ c["k"][0, b, h // 2], c["v"][0, b, h], atol=1e-12)
    c["beta"][:] = 0
    c["g"][:] = 0
    np.testing.assert_array_equal(od.delta_forward(**c)[1], c["S0"])


@pytest.mark.parametrize("lens", [None, [5, 0, 3]])
def test_delta_gradient_against_differences(lens):
    rng = np.random.default_rng(1)
    c = _delta_case(rng)
    lens = None if lens is None else np.array(lens)
    dy, dS = rng.standard_normal((5, 3, 4, 2)), rng.standard_normal((3, 4, 3, 2))

    def loss(x):
        y, S, _ = od.delta_forward(**x, seq_len=lens)
        return (y * dy).sum() + (S * dS).sum()

    _, _, tape = od.delta_forward(**c, seq_len=lens)
    grads = od.delta_backward(tape, dy, dS)
    for name in ("q", "k", "v", "g", "beta", "S0"):
        got = grads["d" + name]
        assert got.shape == c[name].shape
        for _ in range(12):
            at = tuple(rng.integers(0, n) for n in c[name].shape)
            ends = []
            for s in (1e-5, -1e-5):
                x = {k: a.copy() for k, a in c.items()}
                x[name][at] += s
                ends.append(loss(x))
            assert abs((ends[0] - ends[1]) / 2e-5 - got[at]) < 1e-7, (name, at)


def test_logprob_against_torch():
    rng = np.random.default_rng(2)
    x = 2 * rng.standard_normal((6, 11))
    x[1, 3:] = -np.inf
    t = np.array([0, 1, -1, 10, 4, 99])
    f = ol.logprob_forward(x, t, 4)
    xt = torch.from_numpy(x).requires_grad_(True)
    lp = torch.log_softmax(xt, 1)
    np.testing.assert_allclose(f["lse"], torch.logsumexp(xt, 1).detach().numpy(), atol=1e-12)
    sel = [0, 1, 3, 4]
    np.testing.assert_allclose(f["logp"][sel], lp[sel, t[sel]].detach().numpy(), atol=1e-12)
    assert f["logp"][2] == 0 and f["logp"][5] == 0
    np.testing.assert_array_equal(f["top_ids"], torch.sort(xt, dim=1, descending=True, stable=True).indices[:, :4])
    dl, dh, dt = rng.standard_normal(6), rng.standard_normal(6), rng.standard_normal((6, 4))
    dt[1, 3] = 0          # an alternative with probability 0
    ent = -(lp.exp() * torch.where(torch.isinf(xt), torch.zeros(()).double(), lp)).sum(1)
    top = torch.gather(torch.where(torch.isinf(lp), torch.zeros(()).double(), lp), 1,
                       torch.from_numpy(f["top_ids"]))
    loss = (lp[sel, t[sel]] * torch.from_numpy(dl[sel])).sum() + (ent * torch.from_numpy(dh)).sum() \
        + (top * torch.from_numpy(dt)).sum()
    loss.backward()
    np.testing.assert_allclose(ol.logprob_backward(f, dl, dh, dt), xt.grad.numpy(), atol=1e-12)


def test_logprob_empty_row():
    f = ol.logprob_forward(np.full((1, 5), -np.inf), np.array([2]), 3)
    assert f["lse"][0] == -np.inf and f["logp"][0] == -np.inf and f["entropy"][0] == 0
    np.testing.assert_array_equal(f["top_ids"], [[0, 1, 2]])
    assert not ol.logprob_backward(f, np.ones(1), np.ones(1), np.ones((1, 3))).any()


def test_adamw_against_torch():
    rng = np.random.default_rng(3)
    p, m, v = rng.standard_normal(50), np.zeros(50), np.zeros(50)
    pt = torch.from_numpy(p.copy()).requires_grad_(True)
    opt = torch.optim.AdamW([pt], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    for step in range(1, 6):
        g = rng.standard_normal(50)
        pt.grad = torch.from_numpy(g)
        opt.step()
        p, m, v = oa.adamw(p, g, m, v, 1e-2, 0.9, 0.95, 1e-8, step, 0.1)
    np.testing.assert_allclose(p, pt.detach().numpy(), atol=1e-14)


def test_codes_stand_between_their_neighbours():
    rng = np.random.default_rng(4)
    x = rng.standard_normal(700)
    s = oa.row_max(x)
    for power, top in ((2, 127), (4, 255)):
        lo, chance = oa.neighbours(x, s, power, top)
        assert (lo >= 0).all() and (lo < top).all()
        assert (chance >= 0).all() and (chance <= 1 + 1e-12).all()
        r = s[np.arange(700) // 256]
        mean = r * ((1 - chance) * (lo / top) ** power + chance * ((lo + 1) / top) ** power)
        np.testing.assert_allclose(mean, np.abs(x), rtol=1e-10)
