"""GPU: the gradient of g where a token forgets everything.  e^g is 0 there (in float32
below -104, half of its smallest number), so dg is 0, not the rounding of the terms
that cancel; the other gradients are the oracle's.  Tolerances as in the other tests
of the delta rule."""
import math

import pytest
import torch

from test_delta_gpu import check, make, reference, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-math.inf, -1e30, -200.0, -105.0])
def test_a_reset_has_no_gradient(low, dtype):
    c = make(150, 2, 1, 2, 32, 40, dtype, [150, 97], seed=31)
    at = [0, 1, 40, 63, 64, 65, 96, 127, 128, 149]      # first, last and inner ones of the chunks
    c["g"][at, :, 0] = low
    c["g"][70, 0] = low
    got, err = run(c, dtype)
    assert err == 0
    assert not got["dg"][at, :, 0].any() and not got["dg"][70, 0].any()
    check(got, reference({**c, "g": c["g"].clamp(min=-700)}), dtype)
