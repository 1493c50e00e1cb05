"""Router and combination where they can go wrong and the tests of every operator do not look."""
import numpy as np
import pytest

from test_gpu_sparse_block import Backward, Routed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k", [(9700, 64, 4), (19300, 16, 3), (38100, 8, 2), (9600, 130, 5)])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_more_tokens_than_lanes_that_take_them(T, E, k, renorm):
    """8 blocks on each of 148 SMs hold 9472 groups of 32 lanes, 18944 of 16, 37888 of 8: some take a second token.  Few experts are
    chosen, so that the two tokens' slots fall on the same ones."""
    rng = np.random.default_rng(T)
    x = rng.standard_normal((T, E)) + np.where(np.arange(E) < k + 1, 4.0, 0.0)
    Backward(Routed(x, "fp32", k, renorm, rng.random(T) < 0.9), rng).check()
