"""Group norm of values whose variance is below the smallest normal number of 32 bits, without eps to hide it."""
import numpy as np
import pytest

import test_gpu_seq_norm as norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(3, 1, 512, 2), (2, 49, 64, 4), (1, 9000, 64, 2)], ids=str)
def test_norm_of_tiny_values(shape):
    """Deviations of 2^-65: squares of about 2^-130 keep 2^-149 of absolute precision, 2^-19 of each and less of their sum;
    half of that in rstd, which is 2^65.  1e-5 allowed in the 2-norm, as elsewhere."""
    n, s, c, g = shape
    x = (np.random.default_rng(1).standard_normal((n, s, c)) * 2.0 ** -65).astype(np.float32)
    got, ref = norm.run(shape, 0, True, x=x, eps=0.0)
    for name in ("y", "mean", "rstd"):
        norm.check(got[name], ref[name], 0, name)
    # dx is 2^65 times its terms, dgamma sums xhat
    for name in ("dx", "dgamma", "dbeta"):
        norm.check(got[name], ref[name], 0, name)
