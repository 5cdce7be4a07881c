"""GPU: a single row whose q, k and v are slices of one projection.  The stride of
a dimension of one says nothing (torch puts what it likes there), so the tokens'
distance is the first stride, whatever the plan was created with.  Tolerances as in
the other tests of the delta rule.
"""
import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll
from test_delta_gpu import DEV, check, make, reference, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 2, 70, 200])
def test_slices_of_one_projection_single_row(T, dtype):
    c = make(T, 1, 2, 4, 32, 48, dtype, [T], seed=T, fused=True)
    got, err = run(c, dtype, fused=True)
    assert err == 0
    check(got, reference(c), dtype)


def plan_and_tensors(T=40):
    buf = torch.randn(T, 1, 64, device=DEV) * 0.3
    q, k, v = (buf[..., 16 * i:16 * i + 16].view(T, 1, 1, 16) for i in range(3))
    g, beta = -torch.rand(T, 1, 1, device=DEV), torch.rand(T, 1, 1, device=DEV)
    return ll.DeltaPlan(T, 1, 1, 1, 16, 16), (q, k, v, g, beta, None)


def test_a_plan_serves_dense_and_sliced_tensors_in_turn():
    p, ins = plan_and_tensors()
    dense = tuple(t.contiguous() for t in ins[:3]) + ins[3:]
    ys = []
    for x in (ins, dense, ins):
        y = torch.empty_like(dense[2])
        p.fwd(*x, None, y, None)
        outs = [torch.empty_like(t) for t in dense[:5]]
        p.bwd(*x, dense[2], None, *outs)
        ys.append([y] + outs)
    for other in ys[1:]:
        for a, b in zip(ys[0], other):
            assert torch.equal(a, b)
    p.close()


def test_another_distance_drops_the_saved_forward_and_bad_ones_are_refused():
    p, ins = plan_and_tensors()
    dense = tuple(t.contiguous() for t in ins[:3]) + ins[3:]
    outs = [torch.empty_like(t) for t in dense[:5]]
    y = torch.empty_like(dense[2])
    p.fwd(*ins, None, y, None)
    with pytest.raises(ll.LoopError) as e:
        p.bwd(*dense, dense[2], None, *outs)
    assert e.value.status == ll.LL_ESTATE
    p.fwd(*dense, None, y, None)
    odd = torch.empty(40, 1, 18, device=DEV)[..., :16].view(40, 1, 1, 16)      # 72 bytes apart
    with pytest.raises(ll.LoopError) as e:
        p.fwd(odd, *dense[1:], None, y, None)
    assert e.value.status == ll.LL_EINVAL
    with pytest.raises((ValueError, ll.LoopError)):
        p.fwd(dense[0][:1].expand(40, 1, 1, 16), *dense[1:], None, y, None)    # all tokens one
    p.bwd(*dense, dense[2], None, *outs)                                       # still there
    p.close()
