"""The two forms of the 4-bit reference agree."""
import numpy as np

from tests.quant_ref import quantised, quantised_fast


def test_forms_agree():
    r = np.random.default_rng(1)
    w = r.standard_normal((40, 100)) * np.logspace(-30, 30, 40)[:, None]
    w[3, 5:20] = 0
    w[4] = 0
    w[5, :8] = [7, 6.5, 5, 3.5, 2.5, 1.75, 0.25, 7.0000001]
    w[6, :4] = [28, 26, 20, 14]
    assert np.array_equal(quantised(w), quantised_fast(w))
