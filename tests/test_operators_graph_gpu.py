"""GPU: the operators captured into graphs.  Every replay, on new contents of the same
buffers and with eager work between, gives the bits of eager calls on the same inputs."""
import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll
from test_adamw_gpu import HYPER, clone, plan as adamw_plan, tensors
from test_delta_gpu import make
from test_logprob_gpu import logits, targets, weights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def captured(work):
    work()                                   # library and allocator are warm
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        work()
    return g


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_token(dtype):
    """Steps of a pool of states, one of them out of range: states go on from replay to replay."""
    c = make(1, 3, 2, 4, 32, 48, dtype, seed=1)
    ins = [c[n][0].clone() for n in ("q", "k", "v", "g", "beta")]
    pool = torch.randn(5, 4, 32, 48, device=DEV)
    slots = torch.tensor([4, -1, 1], dtype=torch.int32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    S, y = pool.clone(), torch.zeros_like(ins[2])
    g = captured(lambda: ll.delta_loop_step(*ins, S, y, slots=slots, device_error=err))
    S.copy_(pool)
    want = pool.clone()
    for n in range(3):
        new = make(1, 3, 2, 4, 32, 48, dtype, seed=10 + n)
        for a, name in zip(ins, ("q", "k", "v", "g", "beta")):
            a.copy_(new[name][0])
        slots.copy_(torch.tensor([n, 9 if n == 1 else -1, 3], dtype=torch.int32))
        e2, y2 = torch.zeros_like(err), torch.empty_like(y)
        ll.delta_loop_step(*ins, want, y2, slots=slots, device_error=e2)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(S, want) and torch.equal(y, y2)
        assert err.item() == (ll.LL_DEVERR_SLOT if n else 0) and e2.item() == (ll.LL_DEVERR_SLOT if n == 1 else 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 200001, 8), (600, 2000, 4)], ids=str)
@pytest.mark.parametrize("offset", [0.0, 80.0])
def test_log_probabilities(shape, dtype, offset):
    """Split rows (their arrivals are cleared by the kernel) and whole ones; the gradient
    in place too, which sums rows of a large lse beforehand."""
    N, V, top = shape
    x, t = logits(N, V, dtype, seed=2), targets(N, V)
    dl, dh, dt = weights(N, top)
    d, z = torch.empty_like(x), torch.empty_like(x)
    new = lambda: dict(logp=torch.zeros(N, device=DEV), entropy=torch.zeros(N, device=DEV),
                       lse=torch.zeros(N, device=DEV), top_ids=torch.zeros(N, top, dtype=torch.int32, device=DEV),
                       top_logp=torch.zeros(N, top, device=DEV))
    out, both = new(), new()

    def work(p, out, both, d, z):
        p.fwd(x, t, **out)
        p.bwd(x, t, out["lse"], out["entropy"], out["top_ids"], dl, dh, dt, d)
        p.fwd_bwd(x, t, dl, dh, both["logp"], both["entropy"], both["lse"], z)
        z.copy_(x)
        p.bwd(z, t, out["lse"], out["entropy"], out["top_ids"], dl, dh, dt, z)

    with ll.LogprobPlan(N, V, dtype=dtype, top_k=top) as p, ll.LogprobPlan(N, V, dtype=dtype, top_k=top) as q:
        g = captured(lambda: work(p, out, both, d, z))
        for n in range(3):
            x.copy_(logits(N, V, dtype, seed=20 + n) + offset)
            t.copy_(targets(N, V, seed=n))
            for a in (dl, dh, dt):
                a.normal_()
            out2, both2, d2, z2 = new(), new(), torch.empty_like(x), torch.empty_like(x)
            work(q, out2, both2, d2, z2)
            g.replay()
            torch.cuda.synchronize()
            for n_ in out:
                assert torch.equal(out[n_], out2[n_]) and torch.equal(both[n_], both2[n_]), n_
            assert torch.equal(d, d2) and torch.equal(z, z2) and torch.equal(d, z)
        assert p.status_sync() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_repeats_its_hyperparameters(bits):
    """A replay is the call that was captured: the same step number, rate and seed, whatever the program has come to."""
    sizes = [17, 300, 5000]
    d = tensors(sizes, bits, "f32", seed=3)
    e = clone(d)
    scale = torch.ones(1, device=DEV)
    with adamw_plan(d, bits, "f32") as p, adamw_plan(e, bits, "f32") as q:
        g = captured(lambda: p.step(d["g"], grad_scale=scale, seed=5, **HYPER))
        for k, v in clone(e).items():
            if k != "wd":
                for a, b in zip(d[k], v):
                    a.copy_(b)
        for n in range(3):
            for a, b in zip(d["g"], e["g"]):
                a.normal_()
                b.copy_(a)
            scale.fill_(0.5 + n)
            q.step(e["g"], grad_scale=scale, seed=5, **HYPER)
            g.replay()
            torch.cuda.synchronize()
            for k in d:
                if k != "wd":
                    assert all(torch.equal(a, b) for a, b in zip(d[k], e[k])), k
