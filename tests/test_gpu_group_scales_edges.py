"""Products with group scales where they can go wrong and the tests of every shape do not look."""
import numpy as np
import pytest

from gpu_util import Guarded, dev
from oracle import sparse_block_oracle as sbo
from paper_2511_22316_b200 import binding as sq
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


@pytest.mark.parametrize("E,rows", [(257, 3), (300, 9), (609, 2), (700, 10), (1024, 1), (1024, 9)])
def test_more_experts_than_a_block_has_threads(E, rows):
    """Up to 1024 experts, with some 8 rows each (the stream, 256 threads a block) or more (CTA pairs, 608 threads)."""
    rng = np.random.default_rng(E + rows)
    counts = rng.multinomial(rows * E, rng.dirichlet(np.full(E, 0.5)))
    counts[[0, 1, E - 1]] = 0, 2, 3
    offsets = np.concatenate([[0], np.cumsum(counts)])
    M = int(offsets[-1]) + 5
    ws = [make_weights(rng, 66, 96, 32, True) for _ in range(E)]
    Z = rng.standard_normal((50, 96)).astype(np.float16)
    row_token = rng.integers(0, 50, M)
    check_grouped(run_grouped(Z, ws, row_token, offsets, M, 32), Z, ws, row_token, offsets, 32)


@pytest.mark.parametrize("M", [1, 9, 17, 33, 65, 130, 700])
@pytest.mark.parametrize("N,offset", [(200, True), (77, False)])
def test_layer_in_front_of_every_kernel(M, N, offset):
    """The rotation writes what the product behind it reads at once: every kernel as the rotation's dependent, twice in a row."""
    import torch
    n1, n2, group = 16, 32, 64
    K = n1 * n2
    rng = np.random.default_rng(M)
    rot = sq.sq_build_rotation(rng.standard_normal((6, K)).astype(np.float32), n1, n2)
    codes, sg, bg = make_weights(rng, N, K, group, offset)
    w = sbo.weights(codes, sg, bg, group)
    Wq, s, b = dev(sbo.pack_codes(codes)), dev(sg), None if bg is None else dev(bg)
    nb = sq.sq_linear_wo_workspace_bytes(M, K)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    for X in rng.standard_normal((2, M, K)).astype(np.float16):
        x, Y = dev(X), Guarded(M * N * 2)
        sq.sq_linear_gs(rot, x, M, Wq, s, b, N, K, group, ws, nb, Y)
        Z16 = torch.empty(M, K, dtype=torch.float16, device="cuda")
        sq.sq_rotate_act_f16(rot, x, M, Z16)
        assert sq.sq_last_device_status() == sq.SQ_OK
        Y.check()
        check(Y.numpy(np.float16, (M, N)), Z16.cpu().numpy(), w)
    # the same as the layers of two experts, whose rows are the tokens twice, in another order
    rows = np.concatenate([rng.permutation(M), rng.permutation(M)])
    offsets = np.array([0, M // 3, 2 * M], np.int32)
    nb = sq.sq_linear_gs_grouped_workspace_bytes(M, 2 * M, K)
    ws, Y = torch.empty(nb, dtype=torch.uint8, device="cuda"), Guarded(2 * M * N * 2)
    two = lambda t: None if t is None else torch.stack([t, t])
    sq.sq_linear_gs_grouped(rot, x, M, dev(rows.astype(np.int32)), dev(offsets), 2, two(Wq), two(s), two(b), 2 * M, N, K, group, ws, nb, Y)
    assert sq.sq_last_device_status() == sq.SQ_OK
    Y.check()
    check(Y.numpy(np.float16, (2 * M, N)), Z16.cpu().numpy()[rows], w)
    rot.close()


@pytest.mark.parametrize("bits", [4, 3])
@pytest.mark.parametrize("offset", [False, True])
def test_weights_half_a_step_between_codes(bits, offset):
    """The code is floor(fl(fl(fl(w - offset) * fl(1 / step)) + 1/2)) in fp32, as the header says, where a division would take another."""
    top = (1 << (bits - 1)) - 1
    maxima = np.arange(1, 2048, dtype=np.float32) / 4096
    lo = np.float32(0.25) if offset else np.float32(0)
    span = np.float32(2 * top + 1 if offset else top)
    step = (maxima / span).astype(np.float16).astype(np.float32)
    W = np.zeros((len(maxima), 32), np.float16)
    for i, c in enumerate(np.arange(-top, top, dtype=np.float32)):
        W[:, i] = (c + np.float32(0.5)) * step
    if offset:
        W += np.float16(0.25)
    W[:, 30], W[:, 31] = (lo - maxima / 2, lo + maxima / 2) if offset else (0, maxima)
    Wq, s, b = Guarded(W.size // 2), Guarded(len(W) * 2), Guarded(len(W) * 2)
    sq.sq_pack_weight_gs(None, dev(W), len(W), 32, bits, 32, Wq, s, b if offset else None)
    words = Wq.numpy(np.uint32, (len(W), 4))
    codes = np.zeros(W.shape, np.int64)
    for c in range(8):
        codes[:, c::8] = (((words >> np.uint32(4 * sbo.POSITION[c])) & 15) ^ 8).astype(np.int64) - 8
    f = W.astype(np.float32)
    d = s.numpy(np.float16, (len(W), 1)).astype(np.float32)
    o = b.numpy(np.float16, (len(W), 1)).astype(np.float32) if offset else np.float32(0)
    with np.errstate(divide="ignore"):
        inv = np.where(d > 0, np.float32(1) / d, np.float32(0))
    want = np.clip(np.floor((f - o) * inv + np.float32(0.5)), -top - 1, top)
    assert np.array_equal(codes, want)
    # either neighbour is half a step away, 8 steps times 2^-22 for the reciprocal's and the product's roundings; the clamp cuts what the
    # roundings of the step (half a step of fp16, 2^-11, over a range of 2 (top + 1) of them) and of the offset (2^-11 of it) leave outside
    assert np.all(np.abs(f - o - codes * d) <= d * (0.5 + 8 * 2.0 ** -22) + (top + 1) * d * 2.0 ** -10 + np.abs(o) * 2.0 ** -11 + 2.0 ** -25)


def test_products_on_two_streams_at_once():
    """A call of every kernel, beside another one on a stream and in a workspace of its own: the bits of calls one by one."""
    import torch
    N, K, group, E = 512, 1024, 64, 6
    rng = np.random.default_rng(1)
    codes, sg, bg = make_weights(rng, N, K, group, True)
    Wq, s, b = dev(sbo.pack_codes(codes)), dev(sg), dev(bg)
    many = lambda t: torch.stack([t.roll(e, 0) for e in range(E)])
    WqE, sE, bE = many(Wq), many(s), many(b)

    class Call:
        def __init__(self, M, per):
            rows = E * per
            self.M, self.rows = M, rows
            self.Z = dev(rng.standard_normal((M, K)).astype(np.float16))
            self.token = dev(rng.integers(0, M, rows).astype(np.int32))
            self.offsets = dev((np.arange(E + 1) * per).astype(np.int32))
            self.nb = sq.sq_gemm_gs_grouped_workspace_bytes(rows, K)
            self.ws = torch.empty(self.nb, dtype=torch.uint8, device="cuda")
            self.Y, self.YE = (torch.zeros(n, N, dtype=torch.float16, device="cuda") for n in (M, rows))

        def run(self):
            sq.sq_w4a16_gemm_gs(self.Z, Wq, s, b, self.M, N, K, group, self.Y)
            sq.sq_w4a16_gemm_gs_grouped(self.Z, self.M, self.token, self.offsets, E, WqE, sE, bE, self.rows, N, K, group, self.ws, self.nb, self.YE)

    calls = [Call(M, per) for M, per in ((1, 3), (5, 40), (16, 8), (30, 20), (64, 2), (300, 100))]
    torch.cuda.synchronize()
    want = []
    for c in calls:
        c.run()
        torch.cuda.synchronize()
        want.append((c.Y.clone(), c.YE.clone()))
        c.Y.zero_()
        c.YE.zero_()
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(30):
        for c, st in zip(calls, streams):
            with torch.cuda.stream(st):
                c.run()
    torch.cuda.synchronize()
    assert sq.sq_last_device_status() == sq.SQ_OK
    for c, (Y, YE) in zip(calls, want):
        assert torch.equal(c.Y, Y) and torch.equal(c.YE, YE)
