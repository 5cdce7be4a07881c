"""GPU: rows so long that several work-groups share one (the last to arrive joins
their sums and their alternatives).  Tolerances as in the tests of shorter rows.
"""
import math

import numpy as np
import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll
from test_logprob_gpu import OP, DEV, check_fwd, check_gradient, fwd, logits, run_gradient, targets, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "rising", "spiky"])
@pytest.mark.parametrize("shape", [(1, 400001, 32), (3, 280000, 5), (2, 1000003, 0)], ids=str)
def test_split_rows(shape, kind, dtype):
    N, V, top = shape
    x, t = logits(N, V, dtype, seed=21, kind=kind), targets(N, V)
    p, out = fwd(x, t, top, dtype)
    check_fwd(x, t, out, top)
    if kind == "normal":
        run_gradient(p, x, t, out, dtype, top)
    for _ in range(3):                       # the next calls find the arrivals cleared
        b = {n: torch.zeros_like(v) for n, v in out.items()}
        p.fwd(x, t, b["logp"], b["entropy"], b["lse"], b.get("top_ids"), b.get("top_logp"))
        for n in out:
            assert torch.equal(out[n], b[n]), n
    p.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_without_a_token(dtype):
    """Work-groups whose whole part is masked: by minus infinity, by the type's
    lowest value, all but one token of the last part, and the whole row."""
    V, top = 600000, 16
    x = logits(5, V, dtype, seed=22)
    t = torch.tensor([7, 3, V - 1, 11, 450000], dtype=torch.int32, device=DEV)
    x[0, 20:] = -math.inf
    x[1, :500000] = torch.finfo(OP[dtype]).min
    x[2] = -math.inf
    x[2, -1] = 0.5
    x[3] = -math.inf
    x[4, :450000] = -math.inf
    p, out = fwd(x, t, top, dtype)
    check_fwd(x, t, out, top)
    run_gradient(p, x, t, out, dtype, top)
    p.close()


def test_alternatives_all_in_one_part_or_spread():
    """The most likely tokens side by side inside the last part, then one in
    every part, then at the borders of the parts; equal ones by their number."""
    V, top = 500009, 32
    x = logits(3, V, "f32", seed=23, scale=0.5)
    x[0, V - 40:] += 30
    x[1, ::15000] = 25.0
    x[2, 65535:65560] = 9.0
    x[2, 131070:131080] = 9.0
    t = targets(3, V)
    p, out = fwd(x, t, top, "f32")
    check_fwd(x, t, out, top)
    p.close()


def test_nan_in_one_part():
    V = 400000
    x, t = logits(2, V, "f32", seed=24), targets(2, V)
    _, clean = fwd(x, t, 8, "f32")
    x[1, V - 3] = math.nan
    p, out = fwd(x, t, 8, "f32")
    for n in out:
        assert torch.equal(out[n][:1], clean[n][:1]), n
    assert torch.isnan(out["lse"][1]) and torch.isnan(out["entropy"][1])
    assert ((out["top_ids"] >= 0) & (out["top_ids"] < V)).all()
    p.close()


def test_fewer_rows_than_planned_split_more():
    """One plan, calls of 1 to 5 rows: the number of work-groups to a row follows
    the call, the results do not."""
    V, top = 300000, 12
    x, t = logits(5, V, "bf16", seed=25), targets(5, V)
    p, all_rows = fwd(x, t, top, "bf16", N=700)
    check_fwd(x, t, all_rows, top)
    for n in (1, 2, 4):
        out = {k: torch.full_like(v[:n], 7) for k, v in all_rows.items()}
        p.fwd(x[:n], t[:n], out["logp"], out["entropy"], out["lse"], out["top_ids"], out["top_logp"])
        check_fwd(x[:n], t[:n], out, top)
    dl, dh, dt = weights(5, top)
    d = torch.empty_like(x)
    p.bwd(x, t, all_rows["lse"], all_rows["entropy"], all_rows["top_ids"], dl, dh, dt, d)
    check_gradient(d, x, t, dl, dh, dt, "bf16", top)
    assert p.status_sync() == 0
    p.close()
