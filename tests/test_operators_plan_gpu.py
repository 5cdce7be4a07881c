"""GPU: a plan made while the device is busy serves another stream at once: its cleared
arrivals, its tables and its error word are there when its creation returns."""
import pytest
import torch

from paper_1805_01772_amd import lstmloop as ll
from test_adamw_gpu import HYPER, plan as adamw_plan, tensors
from test_logprob_gpu import DEV, check_fwd, fwd, logits, targets

pytestmark = pytest.mark.gpu


def busy():
    a = torch.randn(4096, 4096, device=DEV)
    for _ in range(20):
        a = (a @ a).tanh()
    return a


def test_split_rows_on_another_stream():
    x, t = logits(2, 200001, "f32", seed=1), targets(2, 200001)
    s = torch.cuda.Stream()
    for n in range(4):
        torch.cuda.synchronize()
        hold = busy()
        with torch.cuda.stream(s):
            p, out = fwd(x, t, 8, "f32")
        s.synchronize()
        check_fwd(x, t, out, 8)
        assert p.status_sync() == 0
        p.close()
        del hold


def test_adamw_on_another_stream():
    a, b = tensors([5000] * 40, 32, "f32", seed=2), tensors([5000] * 40, 32, "f32", seed=2)
    with adamw_plan(a, 32, "f32") as p:
        p.step(a["g"], **HYPER)
        torch.cuda.synchronize()
    s = torch.cuda.Stream()
    hold = busy()
    with torch.cuda.stream(s), adamw_plan(b, 32, "f32") as p:
        p.step(b["g"], **HYPER)
        s.synchronize()
    for k in ("p", "m", "v"):
        assert all(torch.equal(x, y) for x, y in zip(a[k], b[k])), k
    del hold
