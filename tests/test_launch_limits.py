"""Sizes whose launches would have 2^32 work-items or more are refused with a message
before anything is allocated or launched (no GPU)."""
import ctypes
import os

import pytest

from paper_1805_01772_amd import lstmloop as ll


def _lib():
    if not os.path.exists(ll.LIB_PATH):
        from paper_1805_01772_amd import build_lib
        build_lib.build()
    return ll.load_library()


NOWHERE = 1 << 20                            # no such device: sizes that fit are refused for that


@pytest.mark.parametrize("N,fits", [(1 << 24, False), ((1 << 24) - 1, True)])
def test_rows_of_log_probabilities(N, fits):
    lib, h = _lib(), ctypes.c_void_p()
    st = lib.ll_logprob_plan_create(ctypes.byref(ll.ll_logprob_desc(N, 10, 0, 0, 0)), NOWHERE, ctypes.byref(h))
    assert st != ll.LL_OK and h.value is None
    assert ("2^24" in ll.ll_last_error()) is not fits


@pytest.mark.parametrize("B,Hv,Dv,fits", [
    (1 << 20, 16, 32, False), ((1 << 20) - 1, 16, 32, True),      # one column tile: 2^24 work-groups
    (1 << 19, 8, 128, False), ((1 << 19) - 1, 8, 128, True), (1 << 20, 1, 512, False)])
def test_one_token(B, Hv, Dv, fits):
    lib = _lib()
    d = ll.make_delta_desc(1, B, 1, Hv, 8, Dv, "bf16")
    st = lib.delta_loop_step(ctypes.byref(d), *[None] * 8, B, None, None)
    # null operands are what the sizes that fit are refused for
    assert st == (ll.LL_EINVAL if fits else ll.LL_EUNSUPPORTED)
    assert fits or "work-groups" in ll.ll_last_error()


@pytest.mark.parametrize("T,B,fits", [(64 << 10, 1 << 10, False), (64 << 10, 1023, True)])
def test_chunks(T, B, fits):
    """8 heads: 2^23 chunks."""
    lib, h = _lib(), ctypes.c_void_p()
    d = ll.make_delta_desc(T, B, 8, 8, 8, 8, "bf16", inference=True)
    st = lib.ll_delta_plan_create(ctypes.byref(d), NOWHERE, ctypes.byref(h))
    assert (st == ll.LL_EUNSUPPORTED and "work-groups" in ll.ll_last_error()) is not fits
    assert h.value is None


@pytest.mark.parametrize("n,fits", [((1 << 36), False), ((1 << 36) - 4096, True)])
def test_elements_of_adamw(n, fits):
    lib, h = _lib(), ctypes.c_void_p()
    t = ll.ll_adamw_tensor(4096, None, 8192, 12288, None, None, n, 0.0, 0)
    st = lib.ll_adamw_plan_create(ctypes.byref(ll.ll_adamw_desc(1, 32, 0, 0)), ctypes.byref(t), NOWHERE,
                                  ctypes.byref(h))
    assert (st == ll.LL_EUNSUPPORTED and "chunks" in ll.ll_last_error()) is not fits
    assert h.value is None
