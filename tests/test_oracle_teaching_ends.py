"""The oracle of the loss over lists where a policy has given up the actions outside its list, against the definition in logarithms."""
import numpy as np
import pytest

from oracle import losses as ol
from oracle import teaching as ot
from tests.test_gpu_distill_ends import _given_up, expected


@pytest.mark.parametrize("T", [1.0, 0.05])
def test_a_rest_that_leaves_float64(T):
    z, ids, lq = _given_up(np.random.default_rng(0), 8, 40, "fp32", (0.0, 40.0, 88.0, 700.0, 740.0, 800.0, 1e4), T)
    out = ot.distill(z, ids, lq, ol.rows_of(8), True, T, "sum")
    values, grad, _ = expected(z, ids, lq, T, float(np.finfo(np.float32).min))
    assert np.allclose(out["values"], values, rtol=1e-12, atol=1e-12)
    assert np.allclose(out["grad"], grad / T, rtol=1e-9, atol=1e-12)
