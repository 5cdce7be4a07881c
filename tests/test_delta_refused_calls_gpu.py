"""GPU: a refused call leaves a plan as it was: its saved forward, its tokens'
distances.  Single rows, whose distances the binding takes from the tensors."""
import ctypes

import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, H, D = 40, 2, 16


def inputs(seed=0):
    """Slices of a projection's rows and the same values dense."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.randn(T, 1, 3 * H * D, device=DEV, generator=gen) * 0.3
    sliced = [a.unflatten(2, (H, D)) for a in buf.split(H * D, 2)]
    gates = [-torch.rand(T, 1, H, device=DEV, generator=gen), torch.rand(T, 1, H, device=DEV, generator=gen), None]
    return sliced + gates, [a.contiguous() for a in sliced] + gates


def outputs(ins):
    return [torch.full(t.shape, float("nan"), device=DEV) for t in ins[:5]]


def forward(p, ins):
    y = torch.empty(T, 1, H, D, device=DEV)
    p.fwd(*ins, None, y, None)
    return y


def gradient_is(p, ins, want):
    outs = outputs(ins)
    p.bwd(*ins, want[0], None, *outs)
    for a, b in zip(outs, want[1]):
        assert torch.equal(a, b)


@pytest.fixture
def plan():
    with ll.DeltaPlan(T, 1, H, H, D, D) as p:
        yield p


@pytest.mark.parametrize("first", ["sliced", "dense"])
@pytest.mark.parametrize("bad", ["other tensors", "type", "shape", "output", "alignment", "gradient's type"])
def test_the_saved_forward_is_kept(plan, first, bad):
    sliced, dense = inputs()
    ins, other = (sliced, dense) if first == "sliced" else (dense, sliced)
    dy = forward(plan, ins).clone()
    outs = outputs(ins)
    plan.bwd(*ins, dy, None, *outs)
    want = (dy, outs)
    forward(plan, ins)
    desc = [getattr(plan.desc, n + "_ld") for n in ("q", "k", "v", "dq", "dk", "dv")]
    y = torch.empty_like(dy)
    if bad == "other tensors":
        with pytest.raises(ll.LoopError) as e:
            plan.bwd(*other, dy, None, *outputs(ins))
        assert e.value.status == ll.LL_ESTATE
    elif bad == "type":
        with pytest.raises(ValueError):
            plan.fwd(other[0], other[1].double(), *other[2:], None, y, None)
    elif bad == "shape":
        with pytest.raises(ValueError):
            plan.fwd(*other[:3], other[3][:-1], *other[4:], None, y, None)
    elif bad == "output":
        with pytest.raises(ValueError):
            plan.fwd(*other, None, y.bfloat16(), None)
    elif bad == "alignment":
        odd = torch.empty(y.numel() + 1, device=DEV)[1:].view_as(y)
        with pytest.raises(ll.LoopError) as e:
            plan.fwd(*other, None, odd, None)
        assert e.value.status == ll.LL_EINVAL
    else:
        wide = torch.empty(T, 1, 3 * H * D, device=DEV)[..., :H * D].unflatten(2, (H, D))
        with pytest.raises(ValueError):
            plan.bwd(*ins, dy, None, wide, *outputs(ins)[1:4], outputs(ins)[4].double())
    assert desc == [getattr(plan.desc, n + "_ld") for n in ("q", "k", "v", "dq", "dk", "dv")]
    gradient_is(plan, ins, want)


def test_distances_set_and_set_back(plan):
    sliced, dense = inputs(1)
    dy = forward(plan, dense).clone()
    outs = outputs(dense)
    plan.bwd(*dense, dy, None, *outs)
    forward(plan, dense)
    lib, n = ll.load_library(), H * D
    set_ld = lambda *ld: lib.ll_delta_plan_set_ld(plan._h, (ctypes.c_int64 * 6)(*ld))
    at = lambda t: None if t is None else t.data_ptr()
    again = outputs(dense)
    bwd = lambda: lib.delta_loop_bwd(plan._h, torch.cuda.current_stream().cuda_stream, *map(at, dense), at(dy),
                                     None, *map(at, again), None)
    assert set_ld(3 * n, n, n, n, n, n) == ll.LL_OK
    assert bwd() == ll.LL_ESTATE and "distances" in ll.ll_last_error()
    assert set_ld(n, n, n, n, n, n) == ll.LL_OK
    assert bwd() == ll.LL_OK
    for a, b in zip(again, outs):
        assert torch.equal(a, b)


def test_desc_follows_the_tensors(plan):
    sliced, dense = inputs(2)
    forward(plan, sliced)
    assert (plan.desc.q_ld, plan.desc.v_ld) == (3 * H * D, 3 * H * D)
    forward(plan, dense)
    assert (plan.desc.q_ld, plan.desc.v_ld) == (H * D, H * D)
