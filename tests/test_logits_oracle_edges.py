"""The oracle of the operators on rows of logits at the ends of what they take (CPU only)."""
import numpy as np
import pytest

from oracle import logits_oracle as lo


@pytest.mark.parametrize("low", [-3.0, -1e30, float(np.finfo(np.float32).min)])
@pytest.mark.parametrize("s1", [1.0, 0.7])
def test_a_list_of_equal_values_is_uniform(low, s1):
    """Wherever they lie: K entries of 1/K each."""
    V, K = 20, 5
    x = np.random.default_rng(1).normal(size=(1, V))
    lq = x[0] - np.log(np.exp(x[0]).sum())
    ids = np.arange(K)[None] * 3
    loss, _, dx, _ = lo.distill(x, ids, np.full((1, K), low), s1, 1.0, False, False)
    assert loss[0] == pytest.approx((np.log(1 / K) - lq[ids[0]]).mean(), rel=1e-12)
    want = np.exp(lq)
    want[ids[0]] -= 1 / K
    np.testing.assert_allclose(dx[0], want, atol=1e-14)
