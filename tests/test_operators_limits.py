"""Limits of the operators' sizes that the descriptors alone decide (no GPU)."""
import ctypes
import os

import pytest

from paper_1805_01772_amd import lstmloop as ll


def _lib():
    if not os.path.exists(ll.LIB_PATH):
        from paper_1805_01772_amd import build_lib
        build_lib.build()
    return ll.load_library()


@pytest.mark.parametrize("kw,fits", [
    (dict(B=8192, dtype="f32"), True), (dict(B=8193, dtype="f32"), False),
    (dict(B=16384, dtype="bf16"), True), (dict(B=16385, dtype="bf16"), False),
    (dict(B=8, v_ld=1 << 21, dtype="f32"), True), (dict(B=8, v_ld=(1 << 21) + 8, dtype="f32"), False),
    (dict(B=8, dv_ld=(1 << 21) + 8, dtype="f32"), False),
    (dict(B=8, q_ld=1 << 24, dtype="f32"), True),
])
def test_a_time_step_spans_at_most_64_mib(kw, fits):
    """2048 values a token: 8 KiB in float32, 4 KiB in bfloat16."""
    d = ll.make_delta_desc(T_max=4, Hk=4, Hv=16, Dk=64, Dv=128, **kw)
    lib, h = _lib(), ctypes.c_void_p()
    # (no such device: sizes that fit are refused for that)
    status = lib.ll_delta_plan_create(ctypes.byref(d), 1 << 20, ctypes.byref(h))
    assert h.value is None
    if fits:
        assert status != ll.LL_EUNSUPPORTED or "2^26" not in ll.ll_last_error(), ll.ll_last_error()
    else:
        assert status == ll.LL_EUNSUPPORTED and "2^26" in ll.ll_last_error()


def test_one_token_has_no_such_limit():
    d = ll.make_delta_desc(T_max=1, B=8193, Hk=4, Hv=16, Dk=64, Dv=128, dtype="f32")
    lib = _lib()
    # null operands are what this call is refused for
    assert lib.delta_loop_step(ctypes.byref(d), *[None] * 8, 4, None, None) == ll.LL_EINVAL


def test_distances_need_a_plan_and_values():
    lib = _lib()
    assert lib.ll_delta_plan_set_ld(None, (ctypes.c_int64 * 6)()) == ll.LL_EINVAL
