"""Products with 4-bit weights and group scales on the GPU, dense and over the experts of a sparse block."""
import numpy as np
import pytest

from gpu_util import Guarded, dev
from oracle import singlequant_oracle as ora
from oracle import sparse_block_oracle as sbo
from paper_2511_22316_b200 import binding as sq

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -11, 2.0 ** -24       # half a step of fp16 and of fp32, relative


def make_weights(rng, N, K, group, offset, bits=4):
    G = -(-K // group)
    codes = rng.integers(-(1 << (bits - 1)), 1 << (bits - 1), (N, K))
    sg = (0.0043 * (0.5 + rng.random((G, N)))).astype(np.float16)
    bg = (0.02 * (rng.random((G, N)) - 0.5)).astype(np.float16) if offset else None
    return codes, sg, bg


def tolerance(Z, w, Y):
    """|computed - exact| per output.  Every weight may be rounded once to fp16 (U16 of it, or half the smallest subnormal step,
    2^-25), every product is exact in fp32 or rounded (U32), the sum of K terms is in fp32 in some order, by chains that may
    truncate (2 U32 a step); the result is rounded to fp16 (U16 of it, or 2^-25)."""
    A, aw = np.abs(Z.astype(np.float64)), np.abs(w)
    S = A @ aw.T
    K = Z.shape[1]
    return S * (U16 + (2 * K + 2) * U32 + U16 ** 2) + A.sum(1)[:, None] * 2.0 ** -25 + np.abs(Y) * U16 * (1 + 2 * U16) + 2.0 ** -25


def run_dense(Z, codes, sg, bg, group):
    M, K = Z.shape
    N = codes.shape[0]
    Y = Guarded(M * N * 2)
    sq.sq_w4a16_gemm_gs(dev(Z), dev(sbo.pack_codes(codes)), dev(sg), None if bg is None else dev(bg), M, N, K, group, Y)
    assert sq.sq_last_device_status() == sq.SQ_OK
    Y.check()
    return Y.numpy(np.float16, (M, N))


def check(Y, Z, w):
    exact = Z.astype(np.float64) @ w.T
    assert np.all(np.abs(Y.astype(np.float64) - exact) <= tolerance(Z, w, exact))
    # independent roundings: U16 of every weight and U16 of the result bound the relative norm of the error for random signs
    assert np.linalg.norm(Y - exact) <= 2 * U16 * np.linalg.norm(exact) + 1e-12


# M: one token to more than a wide tile; N: odd, even, ragged; K: every alignment that the dispatch looks at
SHAPES = [(1, 8, 8, 32), (1, 130, 40, 32), (3, 33, 72, 64), (1, 512, 512, 32), (2, 514, 256, 128), (4, 1024, 1056, 64), (5, 300, 2016, 128),
          (7, 258, 4096, 128), (8, 1000, 544, 32), (8, 4096, 1024, 128), (9, 640, 1024, 64), (13, 126, 2048, 128), (16, 390, 4128, 32),
          (16, 2048, 512, 128), (17, 512, 512, 64), (31, 257, 640, 128), (33, 768, 1088, 64), (50, 520, 2048, 32), (64, 136, 576, 128),
          (65, 256, 512, 32), (100, 513, 832, 64), (129, 1024, 1024, 128), (200, 384, 320, 32), (257, 130, 4160, 128), (300, 1026, 512, 64),
          (1, 14336, 4096, 128), (6, 4096, 14336, 64), (1, 256, 28672, 32), (16, 128, 28672, 128), (1, 6, 65536, 128), (20, 128, 65536, 32),
          (2, 64, 32, 32), (1, 2, 96, 64), (7, 66, 96, 128), (20, 40, 32, 128), (70, 50, 96, 32), (11, 2048, 2080, 64), (3, 129, 256, 64), (16, 33, 1024, 32), (16, 8192, 4096, 128)]


@pytest.mark.parametrize("offset", [False, True])
@pytest.mark.parametrize("M,N,K,group", SHAPES)
def test_product(M, N, K, group, offset):
    rng = np.random.default_rng(M * 7 + N + K)
    codes, sg, bg = make_weights(rng, N, K, group, offset)
    Z = rng.standard_normal((M, K)).astype(np.float16)
    check(run_dense(Z, codes, sg, bg, group), Z, sbo.weights(codes, sg, bg, group))


@pytest.mark.parametrize("M", [1, 2, 8, 12, 16, 20, 70, 130])
def test_product_twice_gives_the_same_bits(M):
    rng = np.random.default_rng(M)
    codes, sg, bg = make_weights(rng, 1000, 2048, 128, True)
    Z = rng.standard_normal((M, 2048)).astype(np.float16)
    assert np.array_equal(run_dense(Z, codes, sg, bg, 128).view(np.uint16), run_dense(Z, codes, sg, bg, 128).view(np.uint16))


@pytest.mark.parametrize("M", [1, 5, 8, 16, 24, 64, 100, 300])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_a_token_that_is_not_finite_stays_alone(M, value):
    rng = np.random.default_rng(M)
    codes, sg, bg = make_weights(rng, 256, 1024, 64, True)
    codes[codes == 0] = 1
    w = sbo.weights(codes, sg, bg, 64)
    Z = rng.standard_normal((M, 1024)).astype(np.float16)
    Z[M // 2, 77] = value
    Y = run_dense(Z, codes, sg, bg, 64)
    others = np.arange(M) != M // 2
    assert not np.isfinite(Y[M // 2]).any()
    check(Y[others], Z[others], w) if M > 1 else None


def test_product_of_nothing_launches_nothing():
    import torch
    n = sq.sq_kernel_launch_count()
    t = torch.zeros(64, dtype=torch.float16, device="cuda")
    sq.sq_w4a16_gemm_gs(t, t, t, None, 0, 64, 128, 128, t)
    sq.sq_w4a16_gemm_gs(t, t, t, None, 4, 0, 128, 128, t)
    assert sq.sq_kernel_launch_count() == n


def test_many_tokens():
    """A prompt longer than a wave of tiles, against sampled rows."""
    import torch
    rng = np.random.default_rng(11)
    M, N, K = 2500, 1280, 1024
    codes, sg, bg = make_weights(rng, N, K, 128, False)
    Z = rng.standard_normal((M, K)).astype(np.float16)
    check(run_dense(Z, codes, sg, bg, 128), Z, sbo.weights(codes, sg, bg, 128))
    assert torch.cuda.is_available()


# -- packing ---------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("bits", [4, 3])
@pytest.mark.parametrize("offset", [False, True])
@pytest.mark.parametrize("N,K,group", [(1, 8, 32), (5, 72, 64), (33, 1024, 128), (130, 520, 32), (2050, 256, 64)])
def test_packed_without_rotation_are_the_oracles_bits(bits, offset, N, K, group):
    rng = np.random.default_rng(N + K + bits)
    W = (0.02 * rng.standard_normal((N, K)) + (0.01 if offset else 0)).astype(np.float16)
    W[0, :] = 0
    codes, sg, bg = sbo.quantise_groups(W.astype(np.float32), group, bits, offset)
    G = -(-K // group)
    Wq, s, b = Guarded(N * K // 2), Guarded(G * N * 2), Guarded(G * N * 2)
    sq.sq_pack_weight_gs(None, dev(W), N, K, bits, group, Wq, s, b if offset else None)
    for t in (Wq, s, b):
        t.check()
    assert np.array_equal(s.numpy(np.uint16, (G, N)), sg.view(np.uint16))
    if offset:
        assert np.array_equal(b.numpy(np.uint16, (G, N)), bg.view(np.uint16))
    assert np.array_equal(Wq.numpy(np.uint8, (N, K // 2)), sbo.pack_codes(codes))


def pack_on_gpu(rot, W, bits, group, offset):
    import torch
    N, K = W.shape
    G = -(-K // group)
    Wq = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda")
    sg = torch.empty(G, N, dtype=torch.float16, device="cuda")
    bg = torch.empty(G, N, dtype=torch.float16, device="cuda") if offset else None
    nb = sq.sq_pack_weight_gs_workspace_bytes(N, K)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    sq.sq_pack_weight_gs(rot, dev(W), N, K, bits, group, Wq, sg, bg, ws, nb)
    return Wq, sg, bg


@pytest.mark.parametrize("n1,n2,N", [(16, 32, 40), (64, 64, 1100), (12, 128, 33), (136, 64, 20), (10, 24, 9)])
@pytest.mark.parametrize("offset", [False, True])
def test_packed_with_rotation_and_the_layer(n1, n2, N, offset):
    """The rotated weights come back within half a step; the layer is the product of the rotated tokens with them."""
    import torch
    K, group = n1 * n2, 32
    rng = np.random.default_rng(K)
    X = rng.standard_normal((6, K)).astype(np.float16)
    W = (0.02 * rng.standard_normal((N, K))).astype(np.float16)
    rot = sq.sq_build_rotation(X.astype(np.float32), n1, n2, flags=sq.SQ_ROT_DEFAULT if n2 & (n2 - 1) == 0 else sq.SQ_ROT_ART | sq.SQ_ROT_URT)
    R1, R2 = rot.factors()
    Wq, sg, bg = pack_on_gpu(rot, W, 4, group, offset)
    words = Wq.cpu().numpy().view(np.uint32)
    codes = np.zeros((N, K), np.int64)
    for c in range(8):
        codes[:, c::8] = (((words >> np.uint32(4 * sbo.POSITION[c])) & 15) ^ 8).astype(np.int64) - 8
    s, b = sg.cpu().numpy(), None if bg is None else bg.cpu().numpy()
    w, R = sbo.weights(codes, s, b, group), ora.rotate(W, R1, R2)
    g = np.arange(K) // group
    step = s.astype(np.float64)[g].T
    # half a step, the step's and the offset's own rounding over the codes' range, and the rotation's fp32 arithmetic
    slack = 8 * step * 2 * U16 + (0 if b is None else np.abs(b.astype(np.float64))[g].T * 2 * U16) + 1e-5 * np.abs(R).max()
    assert np.all(np.abs(w - R) <= step / 2 + slack)
    for M in (1, 6):
        nb = sq.sq_linear_wo_workspace_bytes(M, K)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        Y = Guarded(M * N * 2)
        sq.sq_linear_gs(rot, dev(X[:M]), M, Wq, sg, bg, N, K, group, ws, nb, Y)
        Y.check()
        Z16 = torch.empty(M, K, dtype=torch.float16, device="cuda")
        sq.sq_rotate_act_f16(rot, dev(X[:M]), M, Z16)
        check(Y.numpy(np.float16, (M, N)), Z16.cpu().numpy(), w)
    with pytest.raises(sq.SingleQuantError) as e:
        sq.sq_linear_gs(rot, dev(X), 6, Wq, sg, bg, N, K + 8, group, ws, nb, Y)
    assert e.value.code == sq.SQ_ERR_SHAPE
    with pytest.raises(sq.SingleQuantError) as e:
        sq.sq_linear_gs(rot, dev(X), 6, Wq, sg, bg, N, K, group, ws, 2 * K, Y)
    assert e.value.code == sq.SQ_ERR_NOMEM
    with pytest.raises(sq.SingleQuantError) as e:
        sq.sq_pack_weight_gs(rot, dev(W), N, K, 4, group, Wq, sg, bg, None, 0)
    assert e.value.code == sq.SQ_ERR_INVALID_ARG
    rot.close()


# -- experts ---------------------------------------------------------------------------------------------------------------


def run_grouped(Z, ws, row_token, offsets, M, group, E=None, stream=None, fill=None):
    """ws: (codes, sg, bg) of every expert."""
    import torch
    N, K = ws[0][0].shape
    Wq = dev(np.stack([sbo.pack_codes(c) for c, _, _ in ws]))
    sg = dev(np.stack([s for _, s, _ in ws]))
    bg = None if ws[0][2] is None else dev(np.stack([b for _, _, b in ws]))
    nb = sq.sq_gemm_gs_grouped_workspace_bytes(M, K)
    work = torch.empty(nb, dtype=torch.uint8, device="cuda")
    Y = Guarded(M * N * 2)
    Y.view.view(torch.int16).fill_(0x1234)
    sq.sq_w4a16_gemm_gs_grouped(dev(Z), Z.shape[0], None if row_token is None else dev(row_token.astype(np.int32)),
                                dev(np.asarray(offsets, np.int32)), len(ws), Wq, sg, bg, M, N, K, group, work, nb, Y)
    assert sq.sq_last_device_status() == sq.SQ_OK
    Y.check()
    return Y.numpy(np.float16, (M, N))


def check_grouped(Y, Z, ws, row_token, offsets, group):
    M = len(Y)
    for e, (c, s, b) in enumerate(ws):
        r = np.arange(min(offsets[e], M), min(offsets[e + 1], M))
        if len(r) == 0:
            continue
        tok = r if row_token is None else row_token[r]
        z = np.where(((tok >= 0) & (tok < len(Z)))[:, None], Z[np.clip(tok, 0, len(Z) - 1)], np.float16(0))
        check(Y[r], z, sbo.weights(c, s, b, group))
    assert np.all(Y[min(offsets[-1], M):].view(np.uint16) == 0x1234)           # rows behind the last expert's


GROUPED = [  # counts per expert, N, K, group
    ([1], 64, 64, 32), ([0, 3, 0, 1], 130, 256, 128), ([2, 2, 2, 2, 0, 1, 0, 5], 1024, 512, 64), ([16, 0, 0, 0], 258, 2048, 128),
    ([8, 9, 17, 1], 512, 1024, 128), ([40, 3, 0, 1, 2, 0, 0, 70], 300, 576, 32), ([130, 1, 129, 0], 384, 512, 128), ([0, 0, 0], 64, 128, 64),
    ([5, 0, 7], 33, 72, 64), ([300, 260, 0, 33], 514, 320, 64), ([1] * 60 + [4] * 4, 176, 1088, 32), ([64, 64], 256, 4096, 128)]


@pytest.mark.parametrize("offset", [False, True])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,N,K,group", GROUPED)
def test_experts(counts, N, K, group, gather, offset):
    rng = np.random.default_rng(sum(counts) + N + K)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    rows, tail = int(offsets[-1]), 3
    M = rows + tail
    ws = [make_weights(rng, N, K, group, offset) for _ in counts]
    T = max(1, rows // 2) if gather else M
    Z = rng.standard_normal((T, K)).astype(np.float16)
    row_token = rng.integers(0, T, M) if gather else None
    check_grouped(run_grouped(Z, ws, row_token, offsets, M, group), Z, ws, row_token, offsets, group)


@pytest.mark.parametrize("per", [1, 12, 40])
def test_experts_with_tokens_outside_and_rows_outside(per):
    """Tokens outside [0, T) count as zeros; offsets that lead beyond M are cut there."""
    rng = np.random.default_rng(per)
    ws = [make_weights(rng, 128, 256, 128, False) for _ in range(4)]
    M = 3 * per + per // 2
    Z = rng.standard_normal((10, 256)).astype(np.float16)
    row_token = rng.integers(0, 10, M)
    row_token[0], row_token[M // 2], row_token[M - 1] = -1, 10, 2 ** 31 - 1
    offsets = np.arange(5) * per
    check_grouped(run_grouped(Z, ws, row_token, offsets, M, 128), Z, ws, row_token, offsets, 128)


@pytest.mark.parametrize("per", [3, 30])
def test_an_experts_token_that_is_not_finite_stays_alone(per):
    rng = np.random.default_rng(5)
    ws = [make_weights(rng, 128, 256, 128, True) for _ in range(3)]
    M = 3 * per
    Z = rng.standard_normal((M, 256)).astype(np.float16)
    row_token = rng.permutation(M)
    bad = per + 1
    Z[row_token[bad], 9] = np.nan
    Y = run_grouped(Z, ws, row_token, np.arange(4) * per, M, 128)
    assert np.isnan(Y[bad]).all()
    Z[row_token[bad]] = 0
    Y[bad] = 0
    for e, (c, s, b) in enumerate(ws):
        r = np.arange(e * per, (e + 1) * per)
        check(Y[r], Z[row_token[r]], sbo.weights(c, s, b, 128))


def test_one_expert_is_the_dense_product():
    rng = np.random.default_rng(8)
    for M in (4, 40, 200):
        w = make_weights(rng, 256, 512, 64, True)
        Z = rng.standard_normal((M, 512)).astype(np.float16)
        check(run_grouped(Z, [w], None, [0, M], M, 64), Z, sbo.weights(*w, 64))
        check(run_dense(Z, *w, 64), Z, sbo.weights(*w, 64))
