"""The log probabilities' oracle where the logits share a large offset (CPU)."""
import numpy as np
import pytest

from oracle import logprob as ol


@pytest.mark.parametrize("v", [0.0, 1e6, -3.4e38, 1e300])
def test_equal_logits(v):
    """log p = -log V and the entropy log V, whatever their size."""
    f = ol.logprob_forward(np.full((1, 6), v), np.array([2]), 2)
    np.testing.assert_allclose(f["logp"], -np.log(6), rtol=1e-14)
    np.testing.assert_allclose(f["top_logp"], -np.log(6), rtol=1e-14)
    np.testing.assert_allclose(f["entropy"], np.log(6), rtol=1e-14)
    np.testing.assert_allclose(ol.logprob_backward(f, np.ones(1))[0], np.eye(6)[2] - 1 / 6, rtol=1e-14)
    np.testing.assert_allclose(ol.logprob_backward(f, None, np.ones(1)), 0, atol=1e-15)
