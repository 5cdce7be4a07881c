"""GPU: linear attention, the embedding and beam search captured into graphs.  Every
replay, on new contents of the same buffers and with eager work between, gives the bits of
eager calls on the same inputs; two graphs of one plan take turns."""
import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll
from test_embed_gpu import tokens
from test_linattn_gpu import INS, make as attention, new_outputs
from test_beam_gpu import make as search
from test_operators_graph_gpu import captured

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def same_bits(a, b):
    return torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) and torch.equal(a.isnan(), b.isnan())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [70, 1500])
def test_linear_attention(T, dtype):
    """Whole rows and rows in parts; a second graph of the plan, of the forward alone,
    between the first one's replays."""
    sizes = T, 2, 1, 2, 40, 24
    c = attention(*sizes, dtype, lens=[T, T // 3])
    r, ahead = new_outputs(c, dtype), new_outputs(c, dtype)

    def forward(p, r):
        p.fwd(*[c[n] for n in INS], c["S0"], r["y"], r["ST"])

    def work(p, r):
        forward(p, r)
        p.bwd(*[c[n] for n in INS], c["dy"], c["dST"], r["dq"], r["dk"], r["dv"], r["dS0"])

    with ll.LinattnPlan(*sizes, dtype=dtype) as p, ll.LinattnPlan(*sizes, dtype=dtype) as q:
        g = captured(lambda: work(p, r))
        g2 = captured(lambda: forward(p, ahead))
        for n in range(3):
            new = attention(*sizes, dtype, lens=[T - 7 * n, n], seed=20 + n)
            for name, t in new.items():
                c[name].copy_(t)
            want = new_outputs(c, dtype)
            for t in (*r.values(), *ahead.values()):
                t.fill_(float("nan"))
            work(q, want)
            g2.replay()
            g.replay()
            g2.replay()
            torch.cuda.synchronize()
            assert all(same_bits(r[x], want[x]) for x in r)
            assert all(same_bits(ahead[x], want[x]) for x in ("y", "ST"))
            assert p.status_sync() == q.status_sync() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_token(dtype):
    c = attention(1, 3, 2, 4, 32, 48, dtype)
    ins = [c[n][0].clone() for n in "qkv"] + [c["g"]]
    S = torch.randn(5, 4, 32, 48, device=DEV)
    slots = torch.tensor([4, -1, 1], dtype=torch.int32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    y = torch.zeros_like(ins[2])
    g = captured(lambda: ll.linattn_loop_step(*ins, S, y, slots=slots, device_error=err))
    want = S.clone()
    for n in range(3):
        new = attention(1, 3, 2, 4, 32, 48, dtype, seed=10 + n)
        for a, name in zip(ins, "qkv"):
            a.copy_(new[name][0])
        slots.copy_(torch.tensor([n, 9 if n == 1 else -1, 3], dtype=torch.int32))
        e2, y2 = torch.zeros_like(err), torch.empty_like(y)
        ll.linattn_loop_step(*ins, want, y2, slots=slots, device_error=e2)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(S, want) and torch.equal(y, y2)
        assert e2.item() == (ll.LL_DEVERR_SLOT if n == 1 else 0) and err.item() == (ll.LL_DEVERR_SLOT if n else 0)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N", [50, 3000, 20000])
def test_embedding(N, accumulate):
    """Places sorted by one work-group and by many; what is left of one replay's runs
    must not show in the next one's, which has fewer."""
    V, D = 700, 40
    t, dx = tokens(N, V), torch.randn(N, D, device=DEV)
    table, x, d = torch.randn(V, D, device=DEV), torch.empty(N, D, device=DEV), torch.zeros(V, D, device=DEV)

    def work(p, x, d):
        p.fwd(table, t, x)
        p.bwd(t, dx, d, accumulate=accumulate)

    with ll.EmbedPlan(N, V, D, scale=0.5) as p, ll.EmbedPlan(N, V, D, scale=0.5) as q:
        g = captured(lambda: work(p, x, d))
        for n, kind in enumerate(("one", "text", "all", "none", "text")):
            t.copy_(tokens(N, V, seed=n, kind=kind))
            dx.copy_(torch.randn(N, D, device=DEV))
            x2, d2 = torch.empty_like(x), d.clone()
            work(q, x2, d2)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(x, x2) and torch.equal(d, d2), kind


@pytest.mark.parametrize("shape", [(2, 4, 50001), (40, 8, 1000)], ids=str)
def test_beam_search(shape):
    """Selection with scores, lengths and ends in place, rows moved and a pool's slots
    handed from one array to the other and back: the search goes on from replay to replay."""
    B, K, V = shape
    c = search(B, K, V, "f32", done=0)
    gen = torch.Generator(device=DEV).manual_seed(3)
    history = torch.randint(0, V, (B * K, 12), device=DEV, generator=gen).int()
    pool = torch.randn(B * K + 3, 130, device=DEV, generator=gen)
    s1 = torch.randperm(B * K + 3, device=DEV, generator=gen)[:B * K].view(B, K).int()
    state = dict(scores=c["scores"], finished=c["finished"], lengths=c["lengths"], history=history, pool=pool, s1=s1)
    new = lambda: torch.zeros(B, K, dtype=torch.int32, device=DEV)

    def work(p, s, parents, tokens, s2):
        p.select(c["logits"], s["scores"], s["finished"], s["lengths"], parents, tokens, s["scores"], s["finished"],
                 s["lengths"])
        ll.ll_beam_reorder(parents, [s["history"]])
        ll.ll_beam_reorder(parents, [s["pool"]], slots=s["s1"], slots_out=s2)
        s["s1"].copy_(s2)

    opts = dict(eos=3, length_penalty=0.6)
    with ll.BeamPlan(B, K, V, **opts) as p, ll.BeamPlan(B, K, V, **opts) as q:
        mine = [new(), new(), new()]
        g = captured(lambda: work(p, state, *mine))
        other, theirs = {n: t.clone() for n, t in state.items()}, [new(), new(), new()]
        for n in range(4):
            c["logits"].copy_(search(B, K, V, "f32", seed=5 + n)["logits"])
            work(q, other, *theirs)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(state[x], other[x]) for x in state)
            assert all(torch.equal(a, b) for a, b in zip(mine, theirs))
            assert p.status_sync() == q.status_sync() == 0
            assert all(len(set(row)) == K for row in state["s1"].tolist())
