"""Refusals of the operators' entry points that need no GPU: descriptors, null
and misaligned arguments; the binding's structures follow the header."""
import ctypes
import os
import re

import pytest

from paper_1805_01772_amd import lstmloop as ll

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lstmloop.h")


def _lib():
    if not os.path.exists(ll.LIB_PATH):
        from paper_1805_01772_amd import build_lib
        build_lib.build()
    return ll.load_library()


@pytest.mark.parametrize("kw,status", [
    (dict(T_max=0), ll.LL_EINVAL), (dict(B=0), ll.LL_EINVAL), (dict(Hk=0), ll.LL_EINVAL),
    (dict(Hk=3), ll.LL_EINVAL), (dict(dtype=7), ll.LL_EINVAL), (dict(Dk=12), ll.LL_EUNSUPPORTED),
    (dict(Dk=136), ll.LL_EUNSUPPORTED), (dict(Dv=520), ll.LL_EUNSUPPORTED), (dict(Dv=4), ll.LL_EUNSUPPORTED),
    (dict(q_ld=63), ll.LL_EINVAL), (dict(k_ld=32), ll.LL_EINVAL), (dict(v_ld=130), ll.LL_EINVAL),
    (dict(dq_ld=-64), ll.LL_EINVAL), (dict(scale=float("nan")), ll.LL_EINVAL),
    (dict(scale=float("inf")), ll.LL_EINVAL),
    (dict(B=1 << 23), ll.LL_EUNSUPPORTED), (dict(T_max=2 ** 31 - 1, B=16), ll.LL_EUNSUPPORTED),
])
def test_delta_descriptor(kw, status):
    lib = _lib()
    base = dict(T_max=8, B=4, Hk=2, Hv=4, Dk=32, Dv=32, dtype="bf16")
    base.update(kw)
    d = ll.make_delta_desc(**base)
    h = ctypes.c_void_p(5)
    assert lib.ll_delta_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == status
    assert h.value is None and ll.ll_last_error()
    d.T_max = 1
    if "T_max" not in kw and "dq_ld" not in kw and status == ll.LL_EINVAL:
        assert lib.delta_loop_step(ctypes.byref(d), *[None] * 8, 4, None, None) == status


def test_delta_reserved_and_null():
    lib = _lib()
    d = ll.make_delta_desc(1, 4, 2, 4, 32, 32)
    d.reserved = 1
    h = ctypes.c_void_p()
    assert lib.ll_delta_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_delta_plan_create(None, 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_delta_plan_create(ctypes.byref(d), 0, None) == ll.LL_EINVAL
    assert lib.ll_delta_plan_destroy(None) == ll.LL_OK
    assert lib.delta_loop_fwd(*[None] * 11, 1) == ll.LL_EINVAL
    assert lib.delta_loop_bwd(*[None] * 16) == ll.LL_EINVAL
    assert lib.ll_delta_status_sync(None, None) == ll.LL_EINVAL
    assert lib.ll_delta_plan_bytes(None, None) == ll.LL_EINVAL
    d = ll.make_delta_desc(1, 4, 2, 4, 32, 32)
    at = lambda n: ctypes.c_void_p(4096 * n)      # never followed: the call refuses first
    good = [at(i) for i in range(1, 7)]           # q k v g beta S
    step = lambda *a: lib.delta_loop_step(ctypes.byref(d), None, *a)
    assert step(None, *good[1:], None, 4, at(8), None) == ll.LL_EINVAL
    assert step(*good, None, 3, at(8), None) == ll.LL_EINVAL          # fewer states than rows
    assert step(*good, at(7), 0, at(8), None) == ll.LL_EINVAL
    assert step(ctypes.c_void_p(4098), *good[1:], None, 4, at(8), None) == ll.LL_EINVAL
    assert "16-byte" in ll.ll_last_error()
    d.T_max = 2
    assert step(*good, None, 4, at(8), None) == ll.LL_EINVAL


@pytest.mark.parametrize("kw", [dict(N=0), dict(V=0), dict(dtype=5), dict(top_k=-1), dict(top_k=33),
                                dict(top_k=8, V=7), dict(ld=9), dict(V=2 ** 28 + 1)])
def test_logprob_descriptor(kw):
    lib = _lib()
    base = dict(N=4, V=10, dtype=0, top_k=0, ld=0)
    base.update(kw)
    d = ll.ll_logprob_desc(**base)
    h = ctypes.c_void_p(5)
    assert lib.ll_logprob_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert h.value is None and ll.ll_last_error()


def test_logprob_null():
    lib = _lib()
    d = ll.ll_logprob_desc(4, 10, 0, 0, 0)
    d.reserved[1] = 1
    h = ctypes.c_void_p()
    assert lib.ll_logprob_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_logprob_plan_create(None, 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_logprob_plan_create(ctypes.byref(d), 0, None) == ll.LL_EINVAL
    assert lib.ll_logprob_fwd(None, None, 1, *[None] * 7) == ll.LL_EINVAL
    assert lib.ll_logprob_bwd(None, None, 1, *[None] * 9) == ll.LL_EINVAL
    assert lib.ll_logprob_fwd_bwd(None, None, 1, *[None] * 8) == ll.LL_EINVAL
    assert lib.ll_logprob_status_sync(None, None) == ll.LL_EINVAL
    assert lib.ll_logprob_plan_destroy(None) == ll.LL_OK


@pytest.mark.parametrize("desc,tensor", [
    (dict(n_tensors=0), {}), (dict(n_tensors=65537), {}), (dict(state_bits=16), {}),
    (dict(grad_dtype=3), {}), (dict(reserved=1), {}),
    ({}, dict(n=-1)), ({}, dict(reserved=2)), ({}, dict(weight_decay=-0.1)),
    ({}, dict(weight_decay=float("nan"))), ({}, dict(p=None)), ({}, dict(m=None)),
    ({}, dict(p=4100)), ({}, dict(copy=4098)), (dict(state_bits=8), {}),
    (dict(state_bits=8), dict(m_scale=4098, v_scale=4096)),
])
def test_adamw_descriptor(desc, tensor):
    lib = _lib()
    d = dict(n_tensors=1, state_bits=32, grad_dtype=0, reserved=0)
    d.update(desc)
    t = dict(p=4096, copy=None, m=8192, v=12288, m_scale=None, v_scale=None, n=7, weight_decay=0.0, reserved=0)
    t.update(tensor)
    h = ctypes.c_void_p(5)
    st = lib.ll_adamw_plan_create(ctypes.byref(ll.ll_adamw_desc(**d)),
                                  ctypes.byref(ll.ll_adamw_tensor(**t)), 0, ctypes.byref(h))
    assert st == ll.LL_EINVAL
    assert h.value is None and ll.ll_last_error()


def test_adamw_null():
    lib = _lib()
    assert lib.ll_adamw_plan_create(None, None, 0, None) == ll.LL_EINVAL
    assert lib.ll_adamw_step(None, None, None, None, None) == ll.LL_EINVAL
    assert lib.ll_adamw_plan_destroy(None) == ll.LL_OK


@pytest.mark.parametrize("name", ["ll_delta_desc", "ll_logprob_desc", "ll_adamw_tensor", "ll_adamw_desc",
                                  "ll_adamw_hyper"])
def test_structures_follow_the_header(name):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text).group(1)
    kinds = {"int32_t": 4, "uint32_t": 4, "float": 4, "int64_t": 8, "double": 8}
    fields = []
    for line in body.split(";"):
        m = re.match(r"\s*(\w+)\s*(\**)\s*(.*)", line.strip())
        if not m or not m.group(3):
            continue
        for f in m.group(3).split(","):
            f = f.strip()
            size = 8 if m.group(2) or f.startswith("*") else kinds[m.group(1)]
            n = re.search(r"\[(\d+)\]", f)
            fields.append((re.sub(r"\[\d+\]|\*", "", f).strip(), size * (int(n.group(1)) if n else 1)))
    got = [(f[0], ctypes.sizeof(f[1])) for f in getattr(ll, name)._fields_]
    assert got == fields
