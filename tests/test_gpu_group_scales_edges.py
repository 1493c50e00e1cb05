"""Products with group scales where they can go wrong and the tests of every shape do not look."""
import numpy as np
import pytest

from oracle import sparse_block_oracle as sbo
from test_gpu_group_scales import U16, U32, check, check_grouped, make_weights, run_dense, run_grouped

pytestmark = pytest.mark.gpu

ROWS = [1, 5, 8, 12, 16, 24, 40, 100, 300]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", ROWS)
def test_codes_of_zero_add_nothing(M, group):
    """Every product is zero, so every result is, however large the scales and the tokens."""
    rng = np.random.default_rng(M)
    N, K = 320, 1024
    sg = (1000 * (1 + rng.random((K // group, N)))).astype(np.float16)
    Z = (100 * rng.standard_normal((M, K))).astype(np.float16)
    Z[:, 5] = 60000
    codes = np.zeros((N, K), np.int64)
    for bg in (None, np.zeros_like(sg)):
        assert not run_dense(Z, codes, sg, bg, group).any()
    per = max(1, M // 4)
    ws = [(codes, sg, None)] * 4
    assert not run_grouped(np.resize(Z, (4 * per, K)), ws, None, np.arange(5) * per, 4 * per, group).any()


def one_code_a_row(rng, M, N, K, group):
    """One code of a row is not zero, and the token there is of order one; all others are up to 60000."""
    codes = np.zeros((N, K), np.int64)
    at = rng.integers(0, K // 2, N)                   # so that the large entries are everybody else's
    codes[np.arange(N), at] = rng.choice([-7, -3, 1, 2, 5], N)
    sg = (0.5 + rng.random((K // group, N))).astype(np.float16)
    Z = (1 + rng.random((M, K))).astype(np.float16)
    Z[:, K // 2:] = np.where(rng.random((M, K // 2)) < 0.1, 60000, Z[:, K // 2:])
    exact = Z[:, at].astype(np.float64) * (codes[np.arange(N), at] * sg.astype(np.float64)[at // group, np.arange(N)])
    # the weight rounded to fp16, its product to fp32, the result to fp16
    return codes, sg, Z, exact, np.abs(exact) * (2 * U16 + U16 ** 2 + 2 * U32)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", ROWS)
def test_large_tokens_leave_no_trace_where_the_code_is_zero(M, group):
    codes, sg, Z, exact, tol = one_code_a_row(np.random.default_rng(M + group), M, 320, 2048, group)
    assert np.all(np.abs(run_dense(Z, codes, sg, None, group) - exact) <= tol)
    per = max(1, M // 4)
    ws = [(codes, sg, None)] * 4
    Y = run_grouped(np.resize(Z, (4 * per, 2048)), ws, None, np.arange(5) * per, 4 * per, group)
    assert np.all(np.abs(Y - np.resize(exact, Y.shape)) <= np.resize(tol, Y.shape))
