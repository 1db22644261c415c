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


def _halves(v):
    """Both halves of numbers with a power of two that takes the largest to 2^13 .. 2^14, in fp32."""
    scale = np.float32(2.0 ** (13 - np.floor(np.log2(np.abs(v).max()))))
    hi = (v * scale).astype(np.float16)
    return hi.astype(np.float32), ((v * scale).astype(np.float32) - hi.astype(np.float32)).astype(np.float16).astype(np.float32), scale


def _product(p, q, terms):
    (ph, pl, ps), (qh, ql, qs) = _halves(p), _halves(q)
    parts = {"hi hi": (ph, qh), "hi lo": (ph, ql), "lo hi": (pl, qh)}
    return sum(parts[t][0] @ parts[t][1] for t in terms) / (ps * qs)


ALL = ("hi hi", "hi lo", "lo hi")


@pytest.mark.parametrize("shape", [(16, 211), (64, 64), (60, 700)])
def test_a_lost_product_is_seen(shape):
    """The three products of halves are within what the GPU tests allow; without one of them, in one place of the iteration, they are not."""
    from tests.test_gpu_orthogonal_ends import _factor, allowed
    rng = np.random.default_rng(shape[0])
    x = rng.normal(0, 1, shape)
    x /= np.linalg.norm(x)
    exact = _factor(x, lambda p, q: p @ q)
    error = lambda f: np.linalg.norm(f - exact) / np.linalg.norm(exact)  # noqa: E731
    limit = allowed(error(_factor(x.astype(np.float32), lambda p, q: (p @ q).astype(np.float32))))

    def by_halves(lost, where):
        count = [0]

        def mm(p, q):                                     # in turn X X', A A and B X
            terms = [t for t in ALL if not (t == lost and count[0] % 3 == where)]
            count[0] += 1
            return _product(p.astype(np.float32), q.astype(np.float32), terms)
        return error(_factor(x.astype(np.float32), mm))

    assert by_halves(None, None) <= limit
    for lost in ALL[1:]:
        for where in range(3):
            assert by_halves(lost, where) > 5 * limit, (lost, where, by_halves(lost, where), limit)
