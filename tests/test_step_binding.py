"""The one-token step's binding checks its operands before the library is called (no
GPU: a stub in the library's place, tensors of host memory that call themselves the
device's)."""
import ctypes
import types

import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll


class OnDevice(torch.Tensor):
    is_cuda = True


STREAM = types.SimpleNamespace(cuda_stream=0)
B, HK, HV, DK, DV = 4, 2, 4, 8, 16


def new(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def operands():
    return dict(q=new(B, HK, DK), k=new(B, HK, DK), v=new(B, HV, DV), g=new(B, HV), beta=new(B, HV),
                S=new(B, HV, DK, DV), y=new(B, HV, DV))


@pytest.fixture
def calls(monkeypatch):
    got = []

    class Stub:
        def delta_loop_step(self, desc, *args):
            got.append(ctypes.cast(desc, ctypes.POINTER(ll.ll_delta_desc)).contents)
            return ll.LL_OK
    monkeypatch.setattr(ll, "load_library", lambda *a: Stub())
    return got


def test_dense_and_sliced_rows_pass(calls):
    ll.delta_loop_step(**operands(), stream=STREAM)
    row = new(B, 2 * HK * DK + HV * DV)
    q, k, v = row.split([HK * DK, HK * DK, HV * DV], 1)
    ll.delta_loop_step(**{**operands(), "q": q.unflatten(1, (HK, DK)), "k": k.unflatten(1, (HK, DK)),
                          "v": v.unflatten(1, (HV, DV))}, stream=STREAM)
    assert [(d.q_ld, d.k_ld, d.v_ld) for d in calls] == [(16, 16, 64), (96, 96, 96)]


@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_expanded_rows_are_refused(calls, name):
    """One row for the whole batch: a distance of 0 would be the library's default, and
    it would read B rows of a buffer of one."""
    x = operands()
    x[name] = x[name][:1].expand(B, -1, -1)
    with pytest.raises(ValueError, match=name):
        ll.delta_loop_step(**x, stream=STREAM)
    x[name] = new(64 + B * 256).as_strided(operands()[name].shape, (8, x[name].shape[-1], 1))   # rows that overlap
    with pytest.raises(ValueError, match=name):
        ll.delta_loop_step(**x, stream=STREAM)
    assert not calls


def test_a_single_row_has_no_distance(calls):
    x = {n: t[:1] for n, t in operands().items()}
    x["q"] = new(HK, DK).expand(1, -1, -1)
    ll.delta_loop_step(**x, stream=STREAM)
    assert calls[0].q_ld == HK * DK
