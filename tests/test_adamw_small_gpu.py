"""GPU: AdamW where gradients, their squares or eps are so small that float32 has them
as subnormal numbers or not at all, against float64 of the float32 inputs.

Tolerance.  The squares of g at 2^-70 and below lose bits or vanish in float32 (v is
stored so): the update is checked against the stored m and v, a root, a product, a
quotient: 1e-6 of it; where sqrt(v) r2 + eps is subnormal itself its absolute spacing
2^-149 counts too."""
import numpy as np
import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("eps", [1e-8, 1e-15, 1e-20, 1e-30, 1e-37, 2e-40, 1e-44])
@pytest.mark.parametrize("bits", [32, 8])
def test_update_of_small_gradients(eps, bits):
    n = 8192
    rng = np.random.default_rng(1)
    g = torch.from_numpy((rng.standard_normal(n) * 2.0 ** -rng.integers(0, 80, n)).astype(np.float32)).to(DEV)
    g[::97] = 0.0
    p, z = torch.zeros(n, device=DEV), lambda t: torch.zeros(n, dtype=t, device=DEV)
    if bits == 32:
        m, v, q = z(torch.float32), z(torch.float32), {}
    else:
        m, v = z(torch.int8), z(torch.uint8)
        q = dict(m_scale=[torch.zeros(n // 256, device=DEV)], v_scale=[torch.zeros(n // 256, device=DEV)])
    with ll.AdamWPlan([p], [m], [v], **q) as plan:
        plan.step([g], lr=1.0, beta1=0.5, beta2=0.75, eps=eps, step=1)
    a = g.cpu()
    m1, v1 = (a * 0.5).double(), (a * a * 0.25).double()   # as float32 has them
    if bits == 32:
        assert torch.equal(m.cpu().double(), m1) and torch.equal(v.cpu().double(), v1)
    e = float(np.float32(eps))
    den = torch.sqrt(v1) * 2 + e
    want = torch.where(m1 == 0, 0.0, 2 * m1 / den)
    off = (p.cpu().double() + want).abs()
    assert torch.isfinite(p).all()
    tol = want.abs() * (1e-6 + 2.0 ** -149 / den) + 1e-38
    assert (off <= tol).all(), (off / tol).max().item()
