"""Pins for the oracles of linear attention, the embedding and beam search (CPU):
closed forms, torch.autograd in float64, central differences, search by hand."""
import itertools

import numpy as np
import pytest
import torch

from oracle import beam as ob, embed as oe, linattn as oa


def test_linattn_is_attention_without_softmax():
    """y_t = scale sum_{i <= t} e^{g (t - i)} (q_t.k_i) v_i + scale e^{g (t + 1)} q_t S0."""
    rng = np.random.default_rng(0)
    T, Dk, Dv, g = 6, 3, 2, -0.4
    q, k, v = (rng.standard_normal((T, 1, 1, d)) for d in (Dk, Dk, Dv))
    S0 = rng.standard_normal((1, 1, Dk, Dv))
    y, ST, _ = oa.linattn_forward(q, k, v, [g], S0=S0, scale=0.7)
    t = np.arange(T)
    w = np.where(t[:, None] >= t, np.exp(g * (t[:, None] - t)), 0) * (q[:, 0, 0] @ k[:, 0, 0].T)
    want = 0.7 * (w @ v[:, 0, 0] + np.exp(g * (t + 1))[:, None] * (q[:, 0, 0] @ S0[0, 0]))
    np.testing.assert_allclose(y[:, 0, 0], want, atol=1e-12)
    last = np.exp(g * T) * S0[0, 0] + (k[:, 0, 0] * np.exp(g * (T - 1 - t))[:, None]).T @ v[:, 0, 0]
    np.testing.assert_allclose(ST[0, 0], last, atol=1e-12)


@pytest.mark.parametrize("lens", [None, [5, 0, 3]])
def test_linattn_gradient_against_differences(lens):
    rng = np.random.default_rng(1)
    n = rng.standard_normal
    c = dict(q=n((5, 3, 2, 3)), k=n((5, 3, 2, 3)), v=n((5, 3, 4, 2)), S0=n((3, 4, 3, 2)))
    g = -rng.random(4)
    lens = None if lens is None else np.array(lens)
    dy, dS = n((5, 3, 4, 2)), n((3, 4, 3, 2))

    def loss(x):
        y, S, _ = oa.linattn_forward(x["q"], x["k"], x["v"], g, lens, x["S0"])
        return (y * dy).sum() + (S * dS).sum()

    grads = oa.linattn_backward(oa.linattn_forward(c["q"], c["k"], c["v"], g, lens, c["S0"])[2], dy, dS)
    for name in c:
        got = grads["d" + name]
        assert got.shape == c[name].shape
        for _ in range(12):
            at = tuple(rng.integers(0, m) for m in c[name].shape)
            ends = []
            for s in (1e-5, -1e-5):
                x = {k: a.copy() for k, a in c.items()}
                x[name][at] += s
                ends.append(loss(x))
            assert abs((ends[0] - ends[1]) / 2e-5 - got[at]) < 1e-7, (name, at)


def test_embedding_against_torch():
    rng = np.random.default_rng(2)
    table = torch.from_numpy(rng.standard_normal((7, 3))).requires_grad_()
    tokens = np.array([[3, 0, 3], [6, 3, 1]])
    x = torch.nn.functional.embedding(torch.from_numpy(tokens), table) * 1.5
    np.testing.assert_array_equal(oe.embed_forward(table.detach(), tokens, 1.5), x.detach())
    dx = rng.standard_normal((2, 3, 3))
    want, = torch.autograd.grad(x, table, torch.from_numpy(dx))
    np.testing.assert_allclose(oe.embed_backward(tokens, dx, 7, 1.5), want, atol=1e-14)
    tokens[0, 1] = -1
    tokens[1, 2] = 9
    assert not oe.embed_forward(table.detach(), tokens)[[0, 1], [1, 2]].any()
    old = rng.standard_normal((7, 3))
    got = oe.embed_backward(tokens, dx, 7, 1.5, old)
    np.testing.assert_array_equal(got[[0, 1, 2]], old[[0, 1, 2]])


def test_beam_search_finds_the_best_of_all_sequences():
    """Three steps with as many beams as there are prefixes: every sequence, in order."""
    rng = np.random.default_rng(3)
    V, K = 3, 27
    tables = rng.standard_normal((3, V, V))                  # logits by step and last token
    logp = tables - np.log(np.exp(tables).sum(2, keepdims=True))
    want = sorted(((sum(logp[t, s[t - 1] if t else 0, s[t]] for t in range(3)), s)
                   for s in itertools.product(range(V), repeat=3)), reverse=True)
    scores = np.full((1, K), -np.inf)
    scores[0, 0] = 0
    seqs = [()] * K
    for t in range(3):
        x = np.stack([tables[t, s[-1] if s else 0] for s in seqs])
        r = ob.beam_select(x, scores)
        seqs = [seqs[p] + (int(w),) for p, w in zip(r["parents"][0], r["tokens"][0])]
        scores = r["scores"]
    assert seqs == [s for _, s in want]
    np.testing.assert_allclose(scores[0], [p for p, _ in want], atol=1e-12)


def test_beam_rules():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.1, 0.8]]))
    # a finished beam is one candidate with the score it has; equal ones by token
    r = ob.beam_select(x, [[-1.0, -1.1]], [[0, 1]], [[3, 4]], eos=1)
    assert r["parents"].tolist() == [[1, 0]] and r["tokens"].tolist() == [[1, 0]]
    assert r["finished"].tolist() == [[1, 0]] and r["lengths"].tolist() == [[4, 4]]
    # with a penalty the longer one ranks first although its score is lower
    r = ob.beam_select(np.full((2, 3), -np.inf), [[-1.0, -1.1]], [[1, 1]], [[1, 7]], eos=0, length_penalty=1.0)
    assert r["parents"].tolist() == [[1, 0]]
    # fewer candidates than places
    x[0, 1:] = -np.inf
    r = ob.beam_select(x, [[-2.0, -np.inf]], lengths=[[5, 6]])
    assert r["parents"].tolist() == [[0, 1]] and r["tokens"].tolist() == [[0, -1]]
    assert r["scores"].tolist() == [[-2.0, -np.inf]] and r["lengths"].tolist() == [[6, 6]]


def test_beam_slots():
    out, copies = ob.beam_slots([[2, 2, 0, 2]], [[10, 11, 12, 13]])
    assert out.tolist() == [[12, 11, 10, 13]] and copies == [(12, 11), (12, 13)]
