"""The binding of beam search (no GPU: a stub in the library's place, tensors of host
memory that call themselves the device's)."""
import types

import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll


class OnDevice(torch.Tensor):
    is_cuda = True


STREAM = types.SimpleNamespace(cuda_stream=0)


def new(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


@pytest.fixture
def calls(monkeypatch):
    got = []

    class Stub:
        def ll_beam_reorder(self, stream, searches, K, parents, n, tensors, slots, n_slots, slots_out, err):
            got.append(([(t.data, t.row_bytes) for t in tensors[:n]], n_slots))
            return ll.LL_OK
    monkeypatch.setattr(ll, "load_library", lambda *a: Stub())
    return got


def test_rows_that_hold_no_bytes_need_no_move(calls):
    """A history of width 0, as a search's first step has it, beside a tensor that has rows."""
    parents, x = new(2, 3, dtype=torch.int32), new(6, 5)
    ll.ll_beam_reorder(parents, [new(2, 3, 0), x, new(6, 0, 7, dtype=torch.int32)], stream=STREAM)
    ll.ll_beam_reorder(parents, [new(6, 0)], stream=STREAM)
    slots, pool = new(2, 3, dtype=torch.int32), new(9, 4)
    ll.ll_beam_reorder(parents, [new(9, 0), pool], slots=slots, slots_out=slots.clone(), stream=STREAM)
    ll.ll_beam_reorder(parents, [new(9, 0)], slots=slots, slots_out=slots.clone(), stream=STREAM)
    assert calls == [([(x.data_ptr(), 20)], 0), ([], 0), ([(pool.data_ptr(), 16)], 9), ([], 9)]
    for bad in (new(5, 0), new(2, 4, 0)):
        with pytest.raises(ValueError, match="rows are wanted"):
            ll.ll_beam_reorder(parents, [bad], stream=STREAM)


def test_current_stream_with_and_without_torchs_short_way(monkeypatch):
    """The stream's handle alone is not in torch's public interface: where torch does not
    have it, the stream's object says the same."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 40 + device, raising=False)
    assert ll._stream(None) == 43
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert ll._stream(None) == 77
    assert ll._stream(STREAM) == 0


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-60, -1e-46])
def test_embed_scale_that_is_zero_in_float(scale):
    """The descriptor's 0 means 1: a factor of 0 is refused, also one that a float holds as 0."""
    with pytest.raises(ValueError, match="scale"):
        ll.EmbedPlan(4, 10, 16, scale=scale)
