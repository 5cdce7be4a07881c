"""Refusals of the embedding's, linear attention's and beam search's entry points that
need no GPU: descriptors, null and misaligned arguments, sizes that no launch holds; the
binding's structures follow the header."""
import ctypes

import pytest

from paper_1805_01772_amd import lstmloop as ll
from test_operators_abi import _lib, test_structures_follow_the_header as structure_follows_the_header

NOWHERE = 1 << 20                            # no such device: sizes that fit are refused for that


@pytest.mark.parametrize("kw,status", [
    (dict(T_max=0), ll.LL_EINVAL), (dict(B=0), ll.LL_EINVAL), (dict(Hk=0), ll.LL_EINVAL),
    (dict(Hk=3), ll.LL_EINVAL), (dict(dtype=7), ll.LL_EINVAL), (dict(Dk=12), ll.LL_EUNSUPPORTED),
    (dict(Dk=136), ll.LL_EUNSUPPORTED), (dict(Dv=136), ll.LL_EUNSUPPORTED), (dict(Dv=4), ll.LL_EUNSUPPORTED),
    (dict(q_ld=63), ll.LL_EINVAL), (dict(k_ld=32), ll.LL_EINVAL), (dict(v_ld=130), ll.LL_EINVAL),
    (dict(dq_ld=-64), ll.LL_EINVAL), (dict(scale=float("nan")), ll.LL_EINVAL),
    (dict(scale=float("inf")), ll.LL_EINVAL), (dict(B=1 << 20), ll.LL_EUNSUPPORTED),
    (dict(T_max=2 ** 31 - 1), ll.LL_EUNSUPPORTED), (dict(T_max=1 << 28, B=1 << 10), ll.LL_EUNSUPPORTED),
])
def test_linattn_descriptor(kw, status):
    lib = _lib()
    base = dict(T_max=8, B=4, Hk=2, Hv=4, Dk=32, Dv=32, dtype="bf16")
    base.update(kw)
    d = ll.make_linattn_desc(**base)
    h = ctypes.c_void_p(5)
    assert lib.ll_linattn_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == status
    assert h.value is None and ll.ll_last_error()
    d.T_max = 1
    if "T_max" not in kw and "dq_ld" not in kw and status == ll.LL_EINVAL:
        assert lib.linattn_loop_step(ctypes.byref(d), *[None] * 7, 4, None, None) == status


def test_linattn_null():
    lib = _lib()
    d = ll.make_linattn_desc(1, 4, 2, 4, 32, 32)
    d.reserved = 1
    h = ctypes.c_void_p()
    assert lib.ll_linattn_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_linattn_plan_create(None, 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_linattn_plan_create(ctypes.byref(d), 0, None) == ll.LL_EINVAL
    assert lib.ll_linattn_plan_destroy(None) == ll.LL_OK
    assert lib.linattn_loop_fwd(*[None] * 10, 1) == ll.LL_EINVAL
    assert lib.linattn_loop_bwd(*[None] * 13) == ll.LL_EINVAL
    assert lib.ll_linattn_status_sync(None, None) == ll.LL_EINVAL
    assert lib.ll_linattn_plan_bytes(None, None) == ll.LL_EINVAL
    assert lib.ll_linattn_plan_set_ld(None, (ctypes.c_int64 * 6)()) == ll.LL_EINVAL
    d = ll.make_linattn_desc(1, 4, 2, 4, 32, 32)
    at = lambda n: ctypes.c_void_p(4096 * n)      # never followed: the call refuses first
    good = [at(i) for i in range(1, 6)]           # q k v g S
    step = lambda *a: lib.linattn_loop_step(ctypes.byref(d), None, *a)
    assert step(None, *good[1:], None, 4, at(8), None) == ll.LL_EINVAL
    assert step(*good, None, 3, at(8), None) == ll.LL_EINVAL          # fewer states than rows
    assert step(*good, at(7), 0, at(8), None) == ll.LL_EINVAL
    assert step(ctypes.c_void_p(4098), *good[1:], None, 4, at(8), None) == ll.LL_EINVAL
    assert "16-byte" in ll.ll_last_error()
    d.T_max = 2
    assert step(*good, None, 4, at(8), None) == ll.LL_EINVAL


@pytest.mark.parametrize("B,Hv,Dv,fits", [
    (1 << 20, 16, 32, False), ((1 << 20) - 1, 16, 32, True),      # one column tile: 2^24 work-groups
    (1 << 18, 16, 128, False), ((1 << 18) - 1, 16, 128, True)])
def test_linattn_one_token(B, Hv, Dv, fits):
    lib = _lib()
    d = ll.make_linattn_desc(1, B, 1, Hv, 8, Dv, "bf16")
    st = lib.linattn_loop_step(ctypes.byref(d), *[None] * 7, B, None, None)
    assert st == (ll.LL_EINVAL if fits else ll.LL_EUNSUPPORTED)
    assert fits or "work-groups" in ll.ll_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(N=0), 1), (dict(V=0), 1), (dict(D=0), 1), (dict(N=(1 << 24) + 1), 1), (dict(V=1 << 30), 1),
    (dict(D=(1 << 16) + 1), 1), (dict(table_dtype=2), 1), (dict(x_dtype=-1), 1), (dict(dx_dtype=5), 1),
    (dict(grad_dtype=2), 1), (dict(table_ld=15), 1), (dict(x_ld=-16), 1), (dict(dx_ld=1), 1),
    (dict(grad_ld=1 << 32), 1), (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(reserved=1), 1),
    (dict(N=1 << 24, D=1 << 16), ll.LL_EUNSUPPORTED),
])
def test_embed_descriptor(kw, status):
    lib = _lib()
    d = ll.ll_embed_desc(N=4, V=10, D=16, scale=1.0)
    for n, v in kw.items():
        setattr(d, n, v)
    h = ctypes.c_void_p(5)
    assert lib.ll_embed_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == status
    assert h.value is None and ll.ll_last_error()


def test_embed_null():
    lib = _lib()
    h = ctypes.c_void_p()
    assert lib.ll_embed_plan_create(None, 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_embed_plan_create(ctypes.byref(ll.ll_embed_desc(4, 10, 16)), 0, None) == ll.LL_EINVAL
    assert lib.ll_embed_fwd(None, None, 1, None, None, None) == ll.LL_EINVAL
    assert lib.ll_embed_bwd(None, None, 1, None, None, None, 0) == ll.LL_EINVAL
    assert lib.ll_embed_plan_bytes(None, None) == ll.LL_EINVAL
    assert lib.ll_embed_status_sync(None, None) == ll.LL_EINVAL
    assert lib.ll_embed_plan_destroy(None) == ll.LL_OK
    with pytest.raises(ValueError):
        ll.EmbedPlan(4, 10, 16, x_dtype="f16")
    with pytest.raises(ValueError):
        ll.EmbedPlan(4, 10, 16, scale=0.0)


@pytest.mark.parametrize("kw", [
    dict(B=0), dict(K=0), dict(K=33), dict(V=0), dict(V=2 ** 28 + 1), dict(B=1 << 19), dict(dtype=2), dict(ld=9),
    dict(eos=-2), dict(eos=10), dict(length_penalty=16.5), dict(length_penalty=float("nan")),
    dict(length_penalty=float("-inf"))])
def test_beam_descriptor(kw):
    lib = _lib()
    d = ll.ll_beam_desc(B=2, K=4, V=10, eos=-1)
    for n, v in kw.items():
        setattr(d, n, v)
    h = ctypes.c_void_p(5)
    assert lib.ll_beam_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert h.value is None and ll.ll_last_error()


def test_beam_null():
    lib = _lib()
    d = ll.ll_beam_desc(B=2, K=4, V=10, eos=-1)
    d.reserved[1] = 1
    h = ctypes.c_void_p()
    assert lib.ll_beam_plan_create(ctypes.byref(d), 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_beam_plan_create(None, 0, ctypes.byref(h)) == ll.LL_EINVAL
    assert lib.ll_beam_plan_create(ctypes.byref(d), 0, None) == ll.LL_EINVAL
    assert lib.ll_beam_select(None, None, 1, *[None] * 9) == ll.LL_EINVAL
    assert lib.ll_beam_status_sync(None, None) == ll.LL_EINVAL
    assert lib.ll_beam_plan_destroy(None) == ll.LL_OK


@pytest.mark.parametrize("change,status", [
    (dict(searches=-1), 1), (dict(K=0), 1), (dict(K=33), 1), (dict(searches=1 << 19), 1), (dict(parents=None), 1),
    (dict(n=-1), 1), (dict(n=257), 1), (dict(tensors=None), 1), (dict(slots=4096), 1), (dict(slots_out=4096), 1),
    (dict(slots=4096, slots_out=4096), 1), (dict(slots=4096, slots_out=8192, n_slots=0), 1), (dict(parents=4098), 1),
    (dict(row=0), 1), (dict(row=(1 << 36) + 1), 1), (dict(data=None), 1), (dict(n=2), 1),
    (dict(row=1 << 36, K=32, searches=1000), ll.LL_EUNSUPPORTED),
    (dict(row=1 << 36, slots=4096, slots_out=8192, n_slots=1 << 20), ll.LL_EUNSUPPORTED),
])
def test_beam_reorder_arguments(change, status):
    """(n = 2: the same tensor twice.)"""
    lib = _lib()
    a = dict(searches=2, K=4, parents=4096, n=1, data=1 << 20, row=64, slots=None, n_slots=0, slots_out=None, tensors=1)
    a.update(change)
    t = (ll.ll_beam_tensor * 2)(*[ll.ll_beam_tensor(a["data"], a["row"])] * 2)
    st = lib.ll_beam_reorder(None, a["searches"], a["K"], a["parents"], a["n"], t if a["tensors"] else None, a["slots"],
                             a["n_slots"], a["slots_out"], None)
    assert st == status and ll.ll_last_error()


@pytest.mark.parametrize("name", ["ll_linattn_desc", "ll_embed_desc", "ll_beam_desc", "ll_beam_tensor"])
def test_structures(name):
    structure_follows_the_header(name)


@pytest.mark.parametrize("pool", [False, True])
@pytest.mark.parametrize("n", [33, 64, 65, 256])
def test_beam_reorder_refuses_before_it_moves(n, pool):
    """The last tensor of many is too large for a launch: nothing of the others moves (the
    first launch of them would fail here, where there is no device)."""
    lib = _lib()
    t = (ll.ll_beam_tensor * n)(*[ll.ll_beam_tensor((i + 1) << 20, 64) for i in range(n)])
    t[n - 1] = ll.ll_beam_tensor(1 << 40, 1 << 36)
    st = lib.ll_beam_reorder(None, 64, 4, 4096, n, t, *((4096, 256, 8192) if pool else (None, 0, None)), None)
    assert st == ll.LL_EUNSUPPORTED and f"tensors[{n - 1}]" in ll.ll_last_error()


@pytest.mark.parametrize("B,Hv,fits", [(1 << 22, 1, False), ((1 << 22) - 1, 1, True), (1 << 20, 4, False), (1 << 20, 3, True)])
def test_linattn_heads_of_a_plan(B, Hv, fits):
    """Three passes of each head in one launch: 3 * 2^22 work-groups."""
    lib, h = _lib(), ctypes.c_void_p()
    d = ll.make_linattn_desc(1, B, 1, Hv, 8, 8, "bf16")
    st = lib.ll_linattn_plan_create(ctypes.byref(d), NOWHERE, ctypes.byref(h))
    assert (st == ll.LL_EUNSUPPORTED and "work-groups" in ll.ll_last_error()) is not fits
    assert st != ll.LL_OK and h.value is None


@pytest.mark.parametrize("change,what", [
    (dict(slots_out=4096), "slots_out"), (dict(slots_out=4096 + 28), "slots_out"), (dict(slots_out=8192 - 28), "slots_out"),
    (dict(slots_out=8192 + 4), "slots_out"), (dict(data=4096), "parents"), (dict(data=4096 - 600), "parents"),
    (dict(data=8192), "slots"), (dict(data=12288 + 16), "slots_out"), (dict(data=12288 - 640 + 16), "slots_out"),
    (dict(slots=None, slots_out=None, data=4096 + 16), "parents"),
])
def test_beam_reorder_arrays_that_are_read_and_written(change, what):
    """Work-groups read parents and slots while others write: no array of theirs is a result."""
    lib = _lib()
    a = dict(slots=8192, slots_out=12288, data=1 << 20)
    a.update(change)
    t = (ll.ll_beam_tensor * 1)(ll.ll_beam_tensor(a["data"], 64))
    st = lib.ll_beam_reorder(None, 2, 4, 4096, 1, t, a["slots"], 10 if a["slots"] else 0, a["slots_out"], None)
    assert st == ll.LL_EINVAL and "overlap" in ll.ll_last_error() and what in ll.ll_last_error()


def test_beam_reorder_pools_that_overlap_far_apart():
    """Sizes whose product passes 63 bits."""
    lib = _lib()
    t = (ll.ll_beam_tensor * 2)(ll.ll_beam_tensor(1 << 20, 1 << 36), ll.ll_beam_tensor(1 << 40, 16))
    st = lib.ll_beam_reorder(None, 2, 4, 4096, 2, t, 8192, 2 ** 31 - 1, 12288, None)
    assert st == ll.LL_EINVAL and "overlap" in ll.ll_last_error()
