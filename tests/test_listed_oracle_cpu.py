"""The 64-bit forms of the listed gradients where all other choices are forbidden by a large finite logit: equal scores
have equal shares of the rest."""
import numpy as np
import pytest

from oracle import losses as ref


@pytest.mark.parametrize("low", [-1e4, -1e9, -1e12, -1e30, -3.4028235e38])
def test_forbidden_choices_share_the_rest(low):
    x = np.full((1, 1, 12), low)
    x[0, 0, :3] = 0.0
    ids = np.array([[[2, 0, 1]]])
    d = ref.listed_gradient(x, ids, np.zeros((1, 1, 3)), np.ones((1, 1)), temperature=0.5)
    assert np.allclose(d[0, 0, 3:], 2 / 9, rtol=1e-15, atol=0) and np.allclose(d[0, 0, :3], -2 / 3, rtol=1e-15, atol=0)
    y = np.log(np.array([[[0.3, 0.3, 0.3]]]))
    d = ref.distill_loss(x, ids, y, rest=True)[2]
    assert np.allclose(d[0, 0, 3:], -0.1 / 9, rtol=1e-13, atol=0)
