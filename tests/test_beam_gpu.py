"""GPU: beam search's step against the float64 oracle, and the reordering of states.

Parents, tokens, ends and lengths are equal to the oracle's, where its candidates lie at
least 1e-5 apart (a row's log s is good to about a unit of 1e-6: V terms of 2^-22 each with
random signs, and their sum's roundings); places nearer than that may change among each
other.  Scores: 1e-6 for log s, and the rounding to a float, 2^-24 of the value."""
import math

import numpy as np
import pytest
import torch

from oracle import beam as ob
from paper_1805_01772_amd import lstmloop as ll

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
OP = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(B, K, V, dtype, seed=0, ld=0, done=0.2, masked=0, first=True, at=0):
    """Logits that start `at` elements into their memory, with rows ld apart."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ld = ld or V
    mem = torch.full((B * K * ld + at,), math.nan, device=DEV).to(OP[dtype])
    x = mem[at:].view(B * K, ld)[:, :V]
    x.copy_(2 * torch.randn(B * K, V, device=DEV, generator=gen))
    if masked:
        x[:, V - masked:] = -math.inf
    c = dict(logits=x, scores=-20 * torch.rand(B, K, device=DEV, generator=gen) - 1,
             finished=(torch.rand(B, K, device=DEV, generator=gen) < done).int(),
             lengths=torch.randint(0, 50, (B, K), device=DEV, generator=gen).int())
    if first:                                # one search at its first step
        c["scores"][0, 0], c["scores"][0, 1:], c["finished"][0], c["lengths"][0] = 0.0, -math.inf, 0, 0
    return c


def run(c, eos=-1, penalty=0.0, dtype="f32", plan=None, searches=None):
    n, K = c["scores"].shape
    i = lambda: torch.full((n, K), -7, dtype=torch.int32, device=DEV)
    out = dict(parents=i(), tokens=i(), scores=torch.full((n, K), math.nan, device=DEV), finished=i(), lengths=i())
    p = plan or ll.BeamPlan(n, K, c["logits"].shape[1], dtype=dtype, ld=c["logits"].stride(0) if n * K > 1 else 0,
                            eos=eos, length_penalty=penalty)
    p.select(c["logits"], c["scores"], c["finished"], c["lengths"], out["parents"], out["tokens"], out["scores"],
             out["finished"], out["lengths"])
    err = p.status_sync()
    if plan is None:
        p.close()
    return out, err


def check(c, out, eos=-1, penalty=0.0):
    n = lambda a: None if a is None else a.double().cpu().numpy() if a.is_floating_point() else a.cpu().numpy()
    want = ob.beam_select(n(c["logits"]), n(c["scores"]), n(c["finished"]), n(c["lengths"]), eos, penalty)
    B, K = c["scores"].shape
    got = {k: n(v) for k, v in out.items()}
    for b in range(B):
        gap = np.abs(np.diff(want["ranks"][b][:K + 1]))
        near = {i for j, g in enumerate(gap) if g < 1e-5 for i in (j, j + 1)}
        sure = [k for k in range(K) if k not in near]
        for name in ("parents", "tokens", "finished", "lengths"):
            assert (got[name][b, sure] == want[name][b, sure]).all(), (b, name, got[name][b], want[name][b])
        s, w = got["scores"][b], want["scores"][b]
        held = np.isfinite(w)
        assert (np.isfinite(s) == held).all()
        assert (np.abs(s[held] - w[held]) <= 1e-6 + 2.0 ** -24 * np.abs(w[held]) + (1e-5 if near else 0)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [
    # B, K, V, masked
    (1, 1, 1, 0), (1, 4, 3, 0), (3, 2, 17, 3), (2, 5, 1000, 10), (5, 8, 257, 100), (4, 3, 50001, 0), (2, 32, 4000, 0),
    (1, 4, 200001, 100), (40, 8, 2048, 5), (1, 32, 70000, 0), (2, 7, 6, 1), (70, 4, 333, 0), (2, 16, 40, 30),
], ids=str)
@pytest.mark.parametrize("rule", [(-1, 0.0), (2, 0.0), (0, 0.7), (1, -0.5)], ids=str)
def test_against_oracle(case, rule, dtype):
    B, K, V, masked = case
    eos, penalty = rule
    eos = min(eos, V - 1)
    c = make(B, K, V, dtype, seed=B + V, masked=masked)
    if eos < 0:
        c["finished"] = None
    out, err = run(c, eos, penalty, dtype)
    assert err == 0
    check(c, out, eos, penalty)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at", [0, 1, 3, 7])
def test_rows_apart_and_unaligned(at, dtype):
    c = make(3, 4, 1001, dtype, seed=at, ld=1017, at=at)
    out, err = run(c, 5, 0.5, dtype)
    assert err == 0
    check(c, out, 5, 0.5)


def test_equal_candidates_by_beam_and_token():
    """Beams with the same logits and scores: exactly equal ranks."""
    x = torch.randn(1, 3000, device=DEV).bfloat16()
    x[0, [5, 6, 2900]] = 9.0
    c = dict(logits=x.expand(4, 3000).contiguous(), scores=torch.full((1, 4), -3.0, device=DEV), finished=None,
             lengths=torch.zeros(1, 4, dtype=torch.int32, device=DEV))
    out, _ = run(c, dtype="bf16")
    assert out["parents"].tolist() == [[0, 0, 0, 1]] and out["tokens"].tolist() == [[5, 6, 2900, 5]]
    x.fill_(0.25)
    c["logits"] = x.expand(4, 3000).contiguous()
    out, _ = run(c, dtype="bf16")
    assert out["parents"].tolist() == [[0, 0, 0, 0]] and out["tokens"].tolist() == [[0, 1, 2, 3]]


def test_places_without_a_candidate():
    V = 500
    x = torch.full((4, V), -math.inf, device=DEV)
    x[0, 77] = 1.0
    c = dict(logits=x, scores=torch.tensor([[-2.0, -1.0], [-math.inf, -math.inf]], device=DEV), finished=None,
             lengths=torch.tensor([[4, 5], [6, 7]], dtype=torch.int32, device=DEV))
    out, err = run(c)
    assert err == 0
    assert out["parents"].tolist() == [[0, 1], [0, 1]] and out["tokens"].tolist() == [[77, -1], [-1, -1]]
    assert out["scores"].tolist() == [[-2.0, -math.inf], [-math.inf, -math.inf]]
    assert out["lengths"].tolist() == [[5, 5], [6, 7]] and not out["finished"].any()


def test_finished_beams_without_an_end_token():
    c = make(3, 4, 900, "f32", seed=8, done=0.5)
    out, err = run(c)
    assert err == 0
    check(c, out)
    assert (out["tokens"][out["finished"] != 0] == -1).all() and out["finished"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_of_the_lowest_value(dtype):
    """Rows at the type's lowest value but for a few tokens, and altogether."""
    c = make(2, 3, 2000, dtype, seed=3, done=0.0, first=False)
    low = torch.finfo(OP[dtype]).min
    c["logits"][:, 4:] = low
    c["logits"][5] = low
    c["finished"] = None
    out, err = run(c, dtype=dtype)
    assert err == 0
    check(c, out)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_beams_without_numbers_offer_nothing(bad):
    c = make(2, 3, 1200, "f32", seed=4, done=0.0, first=False)
    c["finished"] = None
    c["logits"][1, 700] = bad
    out, err = run(c)
    assert err == ll.LL_DEVERR_BEAM
    ok = {**c, "logits": c["logits"].clone()}
    ok["logits"][1] = -math.inf
    check(ok, out)
    c["logits"][1, 700] = 0.0
    c["scores"][1, 2] = math.nan
    out, err = run(c)
    assert err == ll.LL_DEVERR_BEAM
    check({**c, "scores": torch.where(c["scores"].isnan(), -math.inf, c["scores"])}, out)


def test_rows_that_do_not_count_are_not_read():
    c = make(4, 4, 3000, "f32", seed=5, done=0.4)
    a, _ = run(c, 7, 1.0)
    dead = ((c["finished"] != 0) | (c["scores"] == -math.inf)).flatten()
    assert dead.any()
    c["logits"][dead] = math.nan
    b, err = run(c, 7, 1.0)
    assert err == 0
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_outputs_in_place_fewer_searches_other_stream():
    c = make(6, 4, 2500, "bf16", seed=6)
    want, _ = run(c, 3, 0.6, "bf16")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with ll.BeamPlan(9, 4, 2500, dtype="bf16", eos=3, length_penalty=0.6) as p:
        i = lambda: torch.empty(6, 4, dtype=torch.int32, device=DEV)
        parents, tokens = i(), i()
        sc, fi, le = (c[n].clone() for n in ("scores", "finished", "lengths"))
        torch.cuda.synchronize()
        p.select(c["logits"], sc, fi, le, parents, tokens, sc, fi, le, stream=s)
        s.synchronize()
        assert p.status_sync() == 0
    for got, n in ((parents, "parents"), (tokens, "tokens"), (sc, "scores"), (fi, "finished"), (le, "lengths")):
        assert torch.equal(got, want[n]), n


def test_select_refusals():
    c = make(2, 3, 100, "f32")
    i = torch.empty(2, 3, dtype=torch.int32, device=DEV)
    f = torch.empty(2, 3, device=DEV)
    with ll.BeamPlan(2, 3, 100) as p:
        for bad in (c["logits"].bfloat16(), c["logits"][:5], c["logits"].t().contiguous().t(), c["logits"].cpu()):
            with pytest.raises(ValueError):
                p.select(bad, c["scores"], None, None, i, i.clone(), f)
        with pytest.raises(ValueError):
            p.select(c["logits"], c["scores"], None, None, i.long(), i.clone(), f)
    with ll.BeamPlan(2, 3, 100, length_penalty=1.0) as p:
        with pytest.raises(ll.LoopError) as e:
            p.select(c["logits"], c["scores"], None, None, i, i.clone(), f)
        assert e.value.status == ll.LL_EINVAL and "lengths" in str(e.value)
    with ll.BeamPlan(1, 3, 100) as p:
        with pytest.raises(ll.LoopError):
            p.select(c["logits"], c["scores"], None, None, i, i.clone(), f)


# ------------------------------------------------------------ the beams' states
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 8, 9, 16, 17, 32])
def test_rows_in_place(K):
    """Rows of many lengths and types, starting anywhere: a copy by bytes."""
    B = 3
    gen = torch.Generator(device=DEV).manual_seed(K)
    parents = torch.randint(0, K, (B, K), device=DEV, generator=gen).int()
    if K > 2:
        parents[1] = torch.arange(K, device=DEV).int().flip(0)          # a permutation with cycles
        parents[2] = torch.arange(K, device=DEV).int()                  # nothing moves
    tensors = []
    for row, at in ((1, 0), (3, 1), (4, 0), (16, 0), (18, 2), (100, 4), (4096, 0), (5000, 8), (40000, 16), (4111, 3)):
        mem = torch.randint(0, 256, (B * K * row + at + 32,), device=DEV, generator=gen, dtype=torch.int64).to(torch.uint8)
        tensors.append((mem, at, row))
    views = [m[at:at + B * K * row].view(B * K, row) for m, at, row in tensors]
    before = [m.clone() for m, _, _ in tensors]
    ll.ll_beam_reorder(parents, views)
    at_row = (torch.arange(B, device=DEV)[:, None] * K + parents.long()).flatten()
    for (m, at, row), old in zip(tensors, before):
        want = old.clone()
        want[at:at + B * K * row] = old[at:at + B * K * row].view(B * K, row)[at_row].flatten()
        assert torch.equal(m, want), (row, at)


def test_many_tensors_and_leading_dimensions():
    B, K = 2, 4
    parents = torch.tensor([[3, 0, 0, 1], [2, 2, 1, 0]], dtype=torch.int32, device=DEV)
    ts = [torch.randn(B, K, 7 + i, device=DEV) for i in range(70)]
    want = [t.gather(1, parents.long()[..., None].expand_as(t)) for t in ts]
    ll.ll_beam_reorder(parents, ts)
    for a, b in zip(ts, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("K", [1, 2, 5, 8, 32])
def test_pool_copies_only_what_it_needs(K):
    B, n_slots = 3, 100
    gen = torch.Generator(device=DEV).manual_seed(K)
    parents = torch.randint(0, K, (B, K), device=DEV, generator=gen).int()
    slots = torch.randperm(n_slots, device=DEV, generator=gen)[:B * K].view(B, K).int()
    pools = [torch.randn(n_slots, 3, 5, device=DEV, generator=gen), torch.randn(n_slots, 9000, device=DEV, generator=gen),
             torch.randn(n_slots, 4099, device=DEV, generator=gen).bfloat16(),
             torch.randint(0, 9, (n_slots, 7), device=DEV, generator=gen).to(torch.uint8)]
    old = [p.clone() for p in pools]
    out = torch.full((B, K), -5, dtype=torch.int32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    ll.ll_beam_reorder(parents, pools, slots=slots, slots_out=out, device_error=err)
    want, copies = ob.beam_slots(parents.cpu().numpy(), slots.cpu().numpy())
    assert out.cpu().numpy().tolist() == want.tolist() and err.item() == 0
    for p, o in zip(pools, old):
        w = o.clone()
        for src, dst in copies:
            w[dst] = o[src]
        assert torch.equal(p, w)
        for b in range(B):
            for k in range(K):
                assert torch.equal(p[out[b, k].item()], o[slots[b, parents[b, k].item()].item()])


def test_bad_parents_and_slots():
    parents = torch.tensor([[1, 7, -3, 0]], dtype=torch.int32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    x = torch.arange(4, device=DEV)
    ll.ll_beam_reorder(parents, [x], device_error=err)
    assert x.tolist() == [1, 1, 2, 0] and err.item() == ll.LL_DEVERR_BEAM
    err.zero_()
    parents = torch.tensor([[2, 2, 0, 1], [0, 0, 1, 1]], dtype=torch.int32, device=DEV)
    slots = torch.tensor([[5, -1, 2, 9], [1, 0, 77, -9]], dtype=torch.int32, device=DEV)
    out = torch.empty_like(slots)
    pool = torch.arange(6, device=DEV).float()
    ll.ll_beam_reorder(parents, [pool], slots=slots, slots_out=out, device_error=err)
    # search 0: beam 2 copies into beam 3's slot, out of range; search 1: beams 0 and 1 into 2's and 3's
    assert out.tolist() == [[2, 9, 5, -1], [1, 77, 0, -9]]
    assert err.item() == ll.LL_DEVERR_SLOT
    assert pool.tolist() == [0, 1, 2, 3, 4, 5]


def test_pool_past_32_bit_offsets():
    """A pool of more than 2^32 bytes: its last slots."""
    n, row = 4200, 1 << 18
    pool = torch.empty(n, row, device=DEV)
    pool[-1], pool[-2] = 1.5, 2.5
    slots = torch.tensor([[n - 1, n - 2]], dtype=torch.int32, device=DEV)
    out = torch.empty_like(slots)
    ll.ll_beam_reorder(torch.zeros(1, 2, dtype=torch.int32, device=DEV), [pool], slots=slots, slots_out=out)
    assert out.tolist() == [[n - 1, n - 2]] and (pool[-2:] == 1.5).all()


def test_reorder_refusals():
    p = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    x = torch.randn(6, 4, device=DEV)
    for kw in (dict(slots=p), dict(slots_out=p), dict(slots=p, slots_out=p)):
        with pytest.raises(ll.LoopError) as e:
            ll.ll_beam_reorder(p, [x], **kw)
        assert e.value.status == ll.LL_EINVAL
    with pytest.raises(ll.LoopError) as e:
        ll.ll_beam_reorder(p, [x, x])
    assert e.value.status == ll.LL_EINVAL and "overlap" in str(e.value)
    for bad in (x[:5], x.t(), x.cpu()):
        with pytest.raises(ValueError):
            ll.ll_beam_reorder(p, [bad])
    with pytest.raises(ValueError):
        ll.ll_beam_reorder(p.flatten(), [x])
    with pytest.raises(ValueError):
        ll.ll_beam_reorder(p.long(), [x])


def test_slots_alone_and_no_searches():
    """Slots without tensors may have any numbers; a call for no searches does nothing."""
    parents = torch.tensor([[1, 1, 0]], dtype=torch.int32, device=DEV)
    slots = torch.tensor([[70, 9, 500]], dtype=torch.int32, device=DEV)
    out, err = torch.zeros_like(slots), torch.zeros(1, dtype=torch.int32, device=DEV)
    ll.ll_beam_reorder(parents, [], slots=slots, slots_out=out, device_error=err)
    assert out.tolist() == [[9, 500, 70]] and err.item() == 0
    none = torch.zeros(0, 3, dtype=torch.int32, device=DEV)
    ll.ll_beam_reorder(none, [torch.zeros(0, 5, device=DEV)])
    pool = torch.ones(4, 5, device=DEV)
    ll.ll_beam_reorder(none, [pool], slots=none, slots_out=none.clone())
    c = {n: t[:0] for n, t in make(2, 3, 50, "f32").items()}
    with ll.BeamPlan(2, 3, 50) as p:
        assert run(c, plan=p)[1] == 0
    assert (pool == 1).all()


def test_lengths_at_the_types_ends():
    c = make(2, 3, 50, "f32", first=False, done=0)
    c["lengths"][:] = torch.tensor([2 ** 31 - 1, -5, 3], dtype=torch.int32, device=DEV)
    out, err = run(c, penalty=0.5)
    assert err == 0
    grown = torch.tensor([2 ** 31 - 1, 1, 4], dtype=torch.int32, device=DEV)
    for b in range(2):
        assert torch.equal(out["lengths"][b], grown[out["parents"][b].long()])
        assert torch.isfinite(out["scores"][b]).all()


# ------------------------------------------------------------ places without a state
def in_pool(parents, slots, n_slots):
    """ll_beam_reorder of a pool whose slot s holds s: new slots, the pool, the error word."""
    parents = torch.tensor(parents, dtype=torch.int32, device=DEV)
    slots = torch.tensor(slots, dtype=torch.int32, device=DEV)
    out, err = torch.full_like(slots, -5), torch.zeros(1, dtype=torch.int32, device=DEV)
    pool = torch.arange(n_slots, device=DEV, dtype=torch.float32)[:, None].repeat(1, 5)
    ll.ll_beam_reorder(parents, [pool], slots=slots, slots_out=out, device_error=err)
    return out.tolist(), pool[:, 0].tolist(), err.item()


def test_successors_of_a_beam_without_a_state_have_none():
    """Not the slot, and the old state, of a beam that ended."""
    out, pool, err = in_pool([[0, 0, 2, 2]], [[-1, 4, 1, 0]], 6)
    assert out == [[-1, -1, 1, 4]] and err == 0
    assert pool == [0, 1, 2, 3, 1, 5]
    # 4 is nobody's where no beam with a state needs it
    out, pool, err = in_pool([[0, 0, 2]], [[-1, 4, 1]], 6)
    assert out == [[-1, -1, 1]] and err == 0 and pool == [0, 1, 2, 3, 4, 5]


def test_a_state_takes_a_free_slot_behind_places_without_one():
    out, pool, err = in_pool([[3, 3, 3, 0]], [[2, -1, 5, 0]], 6)
    assert out == [[0, 5, -1, 2]] and err == ll.LL_DEVERR_SLOT      # two successors, one free slot
    assert pool == [0, 1, 2, 3, 4, 0]


def test_a_state_that_finds_no_slot_is_reported():
    """A search's first step whose single beam alone has a slot."""
    out, pool, err = in_pool([[0, 0, 0], [2, 1, 0]], [[3, -1, -1], [0, -1, 1]], 4)
    assert out == [[3, -1, -1], [1, -1, 0]] and err == ll.LL_DEVERR_SLOT
    assert pool == [0, 1, 2, 3]
    out, pool, err = in_pool([[2, 1, 0]], [[0, -1, 1]], 4)
    assert out == [[1, -1, 0]] and err == 0


@pytest.mark.parametrize("K", [2, 3, 5, 8, 32])
def test_pool_with_places_without_a_state(K):
    """Every place's state is its parent's, or there is none; nothing else is written."""
    B, n_slots = 40, 40 * K + 7
    gen = torch.Generator(device=DEV).manual_seed(K)
    parents = torch.randint(0, K, (B, K), device=DEV, generator=gen).int()
    slots = torch.randperm(n_slots, device=DEV, generator=gen)[:B * K].view(B, K).int()
    slots[torch.rand(B, K, device=DEV, generator=gen) < 0.3] = -1
    pool = torch.arange(n_slots, device=DEV).float()[:, None].repeat(1, 33)
    out, err = torch.full_like(slots, -5), torch.zeros(1, dtype=torch.int32, device=DEV)
    ll.ll_beam_reorder(parents, [pool], slots=slots, slots_out=out, device_error=err)
    want, copies = ob.beam_slots(parents.cpu().numpy(), slots.cpu().numpy())
    assert out.cpu().numpy().tolist() == want.tolist()
    old = slots.gather(1, parents.long())
    assert ((out >= 0) <= (old >= 0)).all()
    lost = ((old >= 0) & (out < 0)).any().item()
    assert err.item() == (ll.LL_DEVERR_SLOT if lost else 0)
    rows = torch.arange(n_slots, device=DEV).float()
    for src, dst in copies:
        rows[dst] = src
    assert torch.equal(pool, rows[:, None].expand_as(pool))
    held = out >= 0
    assert torch.equal(pool[out[held].long(), 0], old[held].float())
    assert out[held].unique().numel() == int(held.sum())


def test_tensors_of_more_than_one_launch():
    """Two tensors that a launch holds one of: 4.3 million work-groups each move bytes here,
    twice (K = 2 rows, 2 searches, of an odd number of bytes)."""
    row = 1_100_000_003
    parents = torch.tensor([[1, 1], [1, 0]], dtype=torch.int32, device=DEV)
    ts = [torch.zeros(4, row, dtype=torch.uint8, device=DEV) for _ in range(2)]
    small = torch.arange(4, device=DEV)
    for i, t in enumerate(ts):
        t[:, :100] = t[:, -100:] = torch.arange(4, device=DEV, dtype=torch.uint8)[:, None] + 10 * i
    ll.ll_beam_reorder(parents, [ts[0], ts[1], small])
    for i, t in enumerate(ts):
        for part in (t[:, :100], t[:, -100:]):
            assert (part == torch.tensor([1, 1, 3, 2], device=DEV, dtype=torch.uint8)[:, None] + 10 * i).all()
        assert not t[:, 100:-100].any()
    assert small.tolist() == [1, 1, 3, 2]


@pytest.mark.parametrize("B,K", [(33001, 2), (65535, 16), (1 << 15, 32)])
def test_many_searches(B, K):
    """More searches, or places, than a launch's second dimension is given."""
    gen = torch.Generator(device=DEV).manual_seed(K)
    parents = torch.randint(0, K, (B, K), device=DEV, generator=gen).int()
    x = torch.arange(B * K, device=DEV).view(B, K)
    y = x.int().clone()
    pool = torch.arange(B * K, device=DEV).float()[:, None].repeat(1, 3)
    ll.ll_beam_reorder(parents, [moved := x.clone(), y])
    want = x.gather(1, parents.long())
    assert torch.equal(moved, want) and torch.equal(y, want.int())
    slots = torch.randperm(B * K, device=DEV, generator=gen).view(B, K).int()
    out, err = torch.empty_like(slots), torch.zeros(1, dtype=torch.int32, device=DEV)
    ll.ll_beam_reorder(parents, [pool], slots=slots, slots_out=out, device_error=err)
    assert err.item() == 0
    assert torch.equal(pool[out.long(), 0], slots.gather(1, parents.long()).float())
