"""GPU: the embedding and the gradient of its table against the float64 oracle, and what
the calls fix exactly.

Tolerances.  A lookup is one product and one rounding to its type: 2^-24 of the value for
the product, and 2^-8 more in bfloat16.  A gradient's row is a sum of n terms, rounded
2^-24 at a time, added in pieces of at most 64 and then piece by piece: its error is at
most (64 + n / 64 + 2) 2^-24 of the sum of the terms' magnitudes, checked element by
element, and 2^-8 of the value more in bfloat16.
"""
import math

import numpy as np
import pytest
import torch

from oracle import embed as oe
from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
OP = {"f32": torch.float32, "bf16": torch.bfloat16}


def tokens(N, V, seed=0, kind="text", skip=0.1):
    rng = np.random.default_rng(seed)
    if kind == "text":                       # rank r about 1 / r of the time
        t = np.exp(rng.random(N) * math.log(V + 0.5)).astype(np.int64) - 1
    elif kind == "one":
        t = np.full(N, V // 2)
    elif kind == "all":
        t = np.arange(N) % V
    elif kind == "none":
        t = np.full(N, -1)
    else:
        t = rng.integers(0, V, N)
    if skip and kind in ("text", "even"):
        t[rng.random(N) < skip] = -1
    return torch.from_numpy(np.clip(t, -1, V - 1).astype(np.int32)).to(DEV)


def rows(N, D, dtype, ld=0, seed=0):
    """N rows of D, ld elements apart, NaN between them."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    a = torch.full((N, ld or D), math.nan, dtype=OP[dtype], device=DEV)
    a[:, :D] = torch.randn(N, D, device=DEV, generator=gen)
    return a[:, :D]


def check_x(got, table, t, scale, dtype):
    want = oe.embed_forward(table.double().cpu().numpy(), t.cpu().numpy(), scale)
    eps = 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0)
    assert (np.abs(got.double().cpu().numpy() - want) <= eps * np.abs(want)).all()


def check_grad(got, t, dx, V, scale, dtype, old=None):
    n = lambda a: None if a is None else a.double().cpu().numpy()
    tt = t.cpu().numpy().ravel()
    dx = n(dx).reshape(-1, got.shape[1]).copy()
    dx[tt < 0] = 0                           # (may hold anything)
    want = oe.embed_backward(tt, dx, V, scale, n(old))
    size = oe.embed_backward(tt, np.abs(dx), V, abs(scale), None if old is None else np.abs(n(old)))
    count = np.bincount(tt[tt >= 0], minlength=V)[:, None]
    tol = (64 + count / 64 + 2) * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    err = np.abs(n(got) - want)
    print(f"    worst of the tolerance: {(err / np.maximum(tol, 1e-300)).max():.2g}", flush=True)
    assert (err <= tol).all()


CASES = [
    # N, V, D, kind
    (1, 1, 1, "one"), (1, 5, 3, "even"), (7, 3, 8, "even"), (64, 100, 33, "text"), (65, 2, 17, "even"),
    (200, 1, 40, "one"), (1000, 1023, 64, "text"), (1000, 1024, 72, "text"), (4096, 50, 16, "text"),
    (4097, 3000, 24, "text"), (4096, 200000, 7, "even"), (9001, 700, 130, "text"), (20000, 5, 512, "even"),
    (20001, 40000, 40, "text"), (70001, 33000, 9, "text"), (70000, 64, 20, "one"), (66000, 66000, 5, "all"),
    (300, 20, 1000, "text"), (5000, 300, 2056, "text"), (500, 10, 8, "none"), (140000, 3, 12, "even"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_against_oracle(case):
    N, V, D, kind = case
    t = tokens(N, V, seed=N + D, kind=kind)
    types = [("f32", "bf16")[i >> (N + D) % 4 & 1] for i in (0, 3, 5, 9)]
    print("   ", types, flush=True)
    table, dx = rows(V, D, types[0], seed=1), rows(N, D, types[2], seed=2)
    x = torch.full((N, D), math.nan, dtype=OP[types[1]], device=DEV)
    with ll.EmbedPlan(N, V, D, *types, scale=1.25) as p:
        p.fwd(table, t, x)
        check_x(x, table, t, 1.25, types[1])
        d = torch.full((V, D), math.nan, dtype=OP[types[3]], device=DEV)
        p.bwd(t, dx, d)
        check_grad(d, t, dx, V, 1.25, types[3])
        old = rows(V, D, types[3], seed=3).clone()
        d = old.clone()
        p.bwd(t, dx, d, accumulate=True)
        check_grad(d, t, dx, V, 1.25, types[3], old)
        untouched = torch.ones(V, dtype=torch.bool, device=DEV)
        untouched[t[t >= 0].long()] = False
        assert torch.equal(d[untouched], old[untouched])
        assert p.status_sync() == 0


@pytest.mark.parametrize("types", [(a, b, c, d) for a in OP for b in OP for c in OP for d in OP], ids=" ".join)
def test_types_and_distances(types):
    """Every combination of types; rows apart, starting at any element, what lies between
    left as it is."""
    N, V, D = 300, 40, 21
    t = tokens(N, V, seed=5)
    ld = dict(table_ld=24, x_ld=29, dx_ld=22, grad_ld=35)
    table, dx = rows(V, D, types[0], 24, seed=1), rows(N, D, types[2], 22, seed=2)
    xs = torch.full((N * 29 + 1,), math.nan, dtype=OP[types[1]], device=DEV)
    ds = torch.full((V * 35 + 3,), math.nan, dtype=OP[types[3]], device=DEV)
    x, d = xs[1:].view(N, 29)[:, :D], ds[3:].view(V, 35)[:, :D]
    with ll.EmbedPlan(N, V, D, *types, **ld) as p:
        p.fwd(table, t, x)
        p.bwd(t, dx, d)
        assert p.status_sync() == 0
    check_x(x, table, t, 1.0, types[1])
    check_grad(d, t, dx, V, 1.0, types[3])
    assert xs[0].isnan() and xs[1:].view(N, 29)[:, D:].isnan().all()
    assert ds[:3].isnan().all() and ds[3:].view(V, 35)[:, D:].isnan().all()


def test_places_without_a_token_are_not_read():
    N, V, D = 5000, 90, 24
    t = tokens(N, V, seed=6, skip=0.4)
    dx = rows(N, D, "f32", seed=2).clone()
    with ll.EmbedPlan(N, V, D) as p:
        a, b = torch.empty(V, D, device=DEV), torch.empty(V, D, device=DEV)
        p.bwd(t, dx, a)
        dx[t < 0] = math.nan
        p.bwd(t, dx, b)
        assert p.status_sync() == 0
    assert torch.equal(a, b)


def test_tokens_out_of_range_count_as_none_and_are_reported():
    t = torch.tensor([3, -2, 1, 10, 2 ** 31 - 1, 3, -2 ** 31, 9], dtype=torch.int32, device=DEV)
    none = torch.where((t < 0) | (t >= 10), torch.full_like(t, -1), t)
    table, dx = rows(10, 16, "f32", seed=1), rows(8, 16, "f32", seed=2)
    got = {}
    with ll.EmbedPlan(8, 10, 16) as p:
        for name, tt in (("bad", t), ("none", none)):
            x, d = torch.empty(8, 16, device=DEV), torch.empty(10, 16, device=DEV)
            p.fwd(table, tt, x)
            e1 = p.status_sync()
            p.bwd(tt, dx, d)
            got[name] = (x, d)
            want = ll.LL_DEVERR_TOKEN if name == "bad" else 0
            assert (e1, p.status_sync()) == (want, want)
    assert torch.equal(got["bad"][0], got["none"][0]) and torch.equal(got["bad"][1], got["none"][1])


def test_fewer_tokens_than_the_plan_holds():
    """One plan, calls of every size class and of none."""
    V, D = 500, 48
    with ll.EmbedPlan(70000, V, D, grad_dtype="bf16") as p:
        for N in (70000, 3, 16384, 5000, 4096, 1, 65536, 0):
            t, dx = tokens(N, V, seed=N), rows(N, D, "f32", seed=N)
            d = torch.full((V, D), math.nan, dtype=torch.bfloat16, device=DEV)
            p.bwd(t, dx, d)
            check_grad(d, t, dx, V, 1.0, "bf16")
            x = torch.empty(N, D, device=DEV)
            p.fwd(rows(V, D, "f32", seed=9), t, x)
            check_x(x, rows(V, D, "f32", seed=9), t, 1.0, "f32")
        keep = d.clone()
        p.bwd(t, dx, d, accumulate=True)
        assert torch.equal(d, keep) and p.status_sync() == 0


def test_same_bits_again_and_on_another_stream():
    N, V, D = 30000, 2000, 64
    t, dx = tokens(N, V, seed=8), rows(N, D, "bf16", seed=2)
    with ll.EmbedPlan(N, V, D, dx_dtype="bf16") as p:
        a = torch.empty(V, D, device=DEV)
        p.bwd(t, dx, a)
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        for _ in range(3):
            b = torch.empty(V, D, device=DEV)
            torch.cuda.synchronize()
            p.bwd(t, dx, b, stream=s)
            s.synchronize()
            assert torch.equal(a, b)


def test_leading_dimensions():
    t = tokens(60, 30, seed=9).view(5, 12)
    table = rows(30, 16, "bf16", seed=1)
    with ll.EmbedPlan(60, 30, 16, "bf16", "bf16") as p:
        x = torch.empty(5, 12, 16, dtype=torch.bfloat16, device=DEV)
        p.fwd(table, t, x)
        dx = rows(60, 16, "f32", seed=2).view(5, 12, 16)
        d = torch.empty(30, 16, device=DEV)
        p.bwd(t, dx, d)
        assert p.status_sync() == 0
    check_x(x, table, t, 1.0, "bf16")
    check_grad(d, t, dx, 30, 1.0, "f32")


def test_table_past_32_bit_offsets():
    """A table and a gradient of more than 2^32 bytes and 2^31 elements: the last row."""
    V, D = 1 << 20, 2064
    table = torch.empty(V, D, dtype=torch.bfloat16, device=DEV)
    table[-1] = 2.5
    t = torch.tensor([V - 1, -1, V - 1], dtype=torch.int32, device=DEV)
    with ll.EmbedPlan(3, V, D, "bf16", "bf16", "bf16", "bf16") as p:
        x = torch.empty(3, D, dtype=torch.bfloat16, device=DEV)
        p.fwd(table, t, x)
        assert (x[[0, 2]] == 2.5).all() and not x[1].any()
        table[:-1] = 0
        p.bwd(t, x, table, accumulate=True)
        assert (table[-1] == 7.5).all() and not table[-2].any()
        table[V - 3:] = 1
        p.bwd(t, x, table)
        assert (table[-1] == 5.0).all() and not table[V - 3:V - 1].any() and not table[0].any()
        assert p.status_sync() == 0


def test_refusals():
    t, table, x = tokens(8, 10), rows(10, 16, "f32"), torch.empty(8, 16, device=DEV)
    d = torch.empty(10, 16, device=DEV)
    with ll.EmbedPlan(8, 10, 16, inference=True) as p:
        p.fwd(table, t, x)
        with pytest.raises(ll.LoopError) as e:
            p.bwd(t, x, d)
        assert e.value.status == ll.LL_EINVAL and "inference" in str(e.value)
    with ll.EmbedPlan(7, 10, 16) as p:
        with pytest.raises(ll.LoopError) as e:
            p.fwd(table, t, x)
        assert e.value.status == ll.LL_EINVAL
    with ll.EmbedPlan(8, 10, 16) as p:
        for bad in (t.long(), t.cpu(), torch.stack([t, t], 1)[:, 0]):
            with pytest.raises(ValueError):
                p.fwd(table, bad, x)
        for bad in (table.bfloat16(), table[:9], rows(10, 16, "f32", 24), table.t().contiguous().t(), table.cpu()):
            with pytest.raises(ValueError):
                p.fwd(bad, t, x)
        with pytest.raises(ValueError):
            p.fwd(table, t, x[:7])
        with pytest.raises(ValueError):
            p.bwd(t, x, d.double())


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "bf16")], ids=" ".join)
@pytest.mark.parametrize("case", [
    (300001, 3000, 9, "text"),               # tiles of more than 2048 places, 128 of them
    (262145, 70, 4, "even"),
    (20000, (1 << 20) + 5, 8, "even"),       # three digits, counted and placed by many work-groups
    (300001, (1 << 20) + 5, 3, "text"),
], ids=lambda c: "x".join(map(str, c)))
def test_long_batches_and_large_vocabularies(case, types):
    N, V, D, kind = case
    t = tokens(N, V, seed=N + D, kind=kind)
    t[:2], t[-2:] = V - 1, 0
    dx = rows(N, D, types[0], seed=2)
    with ll.EmbedPlan(N, V, D, dx_dtype=types[0], grad_dtype=types[1], scale=0.75) as p:
        d = torch.full((V, D), math.nan, dtype=OP[types[1]], device=DEV)
        p.bwd(t, dx, d)
        check_grad(d, t, dx, V, 0.75, types[1])
        again = torch.full_like(d, math.nan)
        p.bwd(t, dx, again)
        assert torch.equal(d, again)
        old = rows(V, D, types[1], seed=3).clone()
        d = old.clone()
        p.bwd(t, dx, d, accumulate=True)
        check_grad(d, t, dx, V, 0.75, types[1], old)
        assert p.status_sync() == 0
