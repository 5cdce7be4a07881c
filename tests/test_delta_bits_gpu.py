"""GPU: the products inside a bfloat16 call of the gated delta rule keep float's 24
bits.  Each case leaves a result of about 2^-16 where terms of size 1 cancel, on the
way of one operand; the inputs are exact in their types.

Tolerance.  At most eight float roundings of terms up to 2 (2^-23 each, one or two
pieces' dropped products 2^-24 each): 2^-20, and the result's own rounding, 2^-8 of
the value.  (Operands of 17 bits would be off by up to 2^-18 and more.)
"""
import numpy as np
import pytest
import torch

from test_delta_gpu import reference, run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, DK, DV = 32, 32, 32


def case(name):
    T = 3 if name in ("update", "decay", "F", "H") else 1
    rng = np.random.default_rng(7)
    # x: all of a float's bits; r: the small difference
    x = rng.uniform(1, 2, (B, DV)).astype(np.float32)
    r = (rng.choice([-1, 1], (B, DV)) * rng.uniform(1, 4, (B, DV)) * 2.0 ** -16).astype(np.float32)
    z = lambda *s: np.zeros(s, np.float32)
    c = dict(q=z(T, B, 1, DK), k=z(T, B, 1, DK), v=z(T, B, 1, DV), g=z(T, B, 1), beta=z(T, B, 1),
             S0=z(B, 1, DK, DV), dy=z(T, B, 1, DV), dST=z(B, 1, DK, DV))
    q, k, v, beta, S0 = (c[n] for n in ("q", "k", "v", "beta", "S0"))
    if name == "state":            # y = S0[0] + S0[1]
        S0[:, 0, 0], S0[:, 0, 1] = x, r - x
        q[0, :, 0, :2] = 1
        k[0, :, 0, 5] = 1
    elif name in ("update", "decay"):   # y_2 = P_20 U_0 + P_21 U_1
        k[0, :, 0, 0] = k[1, :, 0, 1] = k[2, :, 0, 5] = 1
        q[2, :, 0, :2] = 1
        v[0], v[1] = 1, -1
        beta[:2] = 1
        if name == "update":
            beta[0, :, 0], beta[1, :, 0] = x[:, 0], x[:, 0] - r[:, 0]
        else:
            c["g"][1, :, 0] = -np.abs(r[:, 0])
            c["g"][2, :, 0] = -0.3 * x[:, 1]
    elif name == "dR":             # dk = -S0 dR
        k[0, :, 0, 0] = 1
        beta[:] = 1
        c["dST"][:, 0, 0, 0], c["dST"][:, 0, 0, 1] = x[:, 0], r[:, 0] - x[:, 0]
        S0[:, 0, 1:, :2] = 1
    elif name == "F":              # dk_0 = F_10 q_1 + F_20 q_2
        k[0, :, 0, 0] = k[1, :, 0, 2] = k[2, :, 0, 3] = 1
        q[1:, :, 0, 5] = 1
        v[0], beta[0, :, 0] = 1, x[:, 0]
        S0[:, 0, 0, 0] = r[:, 0]
        c["dy"][1, :, 0, 0], c["dy"][2, :, 0, 1] = 1, -1
    elif name == "H":              # dk_2 = H_20 k_0 + H_21 k_1
        k[:2, :, 0, 0] = k[2, :, 0, 1] = 1
        v[0] = 1
        beta[0, :, 0], beta[1, :, 0], beta[2] = x[:, 0], 1 - r[:, 0], 1
        c["dST"][:, 0, 1, 0] = 0.5 * x[:, 1]
    bf = ("q", "k", "v", "dy")
    out = {n: torch.from_numpy(a).to(DEV) for n, a in c.items()}
    for n in bf:
        assert torch.equal(out[n].bfloat16().float(), out[n]), n
        out[n] = out[n].bfloat16()
    return dict(out, seq_len=None)


@pytest.mark.parametrize("name", ["state", "update", "decay", "dR", "F", "H"])
def test_small_differences_of_large_terms(name):
    c = case(name)
    got, err = run(c, "bf16", scale=1.0)
    assert err == 0
    ref = reference(c, scale=1.0)
    small = 0
    for n in ("y", "dq", "dk", "dv"):
        want, a = ref[n], got[n].double().cpu().numpy()
        off = np.abs(a - want) / (2.0 ** -20 + 2.0 ** -8 * np.abs(want))
        print(f"    {n}: {off.max():.2f} of the tolerance", flush=True)
        assert off.max() <= 1, (n, off.max())
        small += ((np.abs(want) > 2.0 ** -18) & (np.abs(want) < 2.0 ** -11)).sum()
    assert small >= B                        # the case holds such a difference in every row
