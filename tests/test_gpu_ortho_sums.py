"""The sums of the orthogonalised update's products.  Float32 products leave five steps of 512 x 1024 off by 17 u, u = 2^-24, of the
result; a matrix instruction drops what lies 2^-26 below the sum that it adds to, and sums of 512 terms and more in one register
come to 23 u.  Between the two: 20 u."""
import numpy as np
import pytest

from oracle import ops_oracle as orc
from test_gpu_ortho import EPS, QUINTIC, U, gradient, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", [0, 1, 2])
def test_sums_are_as_near_as_float32_ones(seed):
    G = gradient(512, 1024, seed)
    want = orc.orthogonalize(G, [tuple(float(np.float32(v)) for v in QUINTIC)] * 5, EPS)
    assert np.linalg.norm(run([G], [QUINTIC] * 5)[0] - want) <= 20 * U * np.linalg.norm(want)
