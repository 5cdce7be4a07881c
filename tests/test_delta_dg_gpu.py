"""GPU: the gradient of g at tokens that forget much of the state.  dg_t = e^{g_t}
<D_t, S_{t-1}> for the gradient D_t of the decayed state, so it is small where the
decay is strong, and has to be right there beside neighbours that are 1e4 to 1e20
times larger.

Tolerance.  Of e^{g_t} |D_t| |S_{t-1}| (2-norms, the oracle's recurrence in float64),
which bounds dg_t: 5e-6, as for the other float results, and the exponent's rounding,
2^-23 |g| a decay."""
import numpy as np
import pytest
import torch

from test_delta_gpu import make, reference, run

pytestmark = pytest.mark.gpu


def bounds(c):
    """e^g |D| |S| of one row and head, token by token."""
    n = lambda a: a.double().cpu().numpy()
    q, k, v, g, beta, dy = (n(c[x])[:, 0, 0] for x in ("q", "k", "v", "g", "beta", "dy"))
    S, D = n(c["S0"])[0, 0], n(c["dST"])[0, 0]
    T, scale = len(q), q.shape[1] ** -0.5
    states = []
    for t in range(T):
        states.append(S)
        S = np.exp(g[t]) * S
        S = S + np.outer(k[t], beta[t] * (v[t] - S.T @ k[t]))
    out = np.zeros(T)
    for t in reversed(range(T)):
        D = D + scale * np.outer(q[t], dy[t])
        D = D - np.outer(k[t], beta[t] * (D.T @ k[t]))
        out[t] = np.exp(g[t]) * np.linalg.norm(D) * np.linalg.norm(states[t])
        D = np.exp(g[t]) * D
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-3.0, -10.0, -20.0, -45.0])
@pytest.mark.parametrize("size", [(32, 32), (64, 72), (128, 104)], ids=str)
def test_strong_decays(size, low, dtype):
    T = 170
    c = make(T, 1, 1, 1, *size, dtype, seed=int(-low))
    at = [3, 17, 31, 32, 47, 63, 80, 96, 110, 127, 128, 150, 169]
    c["g"][at] = low
    got, err = run(c, dtype)
    assert err == 0
    want = reference(c)["dg"][:, 0, 0]
    off = np.abs(got["dg"].double().cpu().numpy()[:, 0, 0] - want)
    g = c["g"].double().cpu().numpy()[:, 0, 0]
    tol = (5e-6 + 2.0 ** -23 * np.abs(g)) * bounds(c)
    print(f"    {(off / tol).max():.2f} of the tolerance, {(off / tol)[at].max():.2f} where it is strong", flush=True)
    assert (off <= tol).all(), (off / tol).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_token_forgets(dtype):
    """Decays of 0.15 to 0.45 a token all along (a half-life of two tokens)."""
    c = make(672, 1, 1, 1, 104, 104, dtype, seed=3)
    c["g"] = -0.3 * (0.5 + torch.rand_like(c["g"]))
    got, _ = run(c, dtype)
    want = reference(c)["dg"]
    off = np.linalg.norm(got["dg"].double().cpu().numpy() - want) / np.linalg.norm(want)
    print(f"    {off:.2e}", flush=True)
    # a token's own terms alone: eight roundings of 2^-24, not a chunk's sum of them
    assert off <= 8 * 2.0 ** -24
