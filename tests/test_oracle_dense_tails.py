"""The oracle's GELU at arguments whose share of the normal distribution is small: published
values of the distribution (its digits are lost in 1 + erf)."""

import numpy as np

from oracle import dense


def test_gelu_far_out():
    v = np.array([-6.0, -8.0, -10.0])
    share = np.array([9.865876450376981e-10, 6.220960574271786e-16, 7.619853024160527e-24])
    assert np.allclose(dense.activation("gelu", v), v * share, rtol=1e-13, atol=0)
    bell = np.exp(-0.5 * v * v) / np.sqrt(2.0 * np.pi)
    assert np.allclose(dense.activation_grad("gelu", v), share + v * bell, rtol=1e-13, atol=0)
