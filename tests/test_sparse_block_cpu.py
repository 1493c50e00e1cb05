"""Group scales, router and combination without a GPU: the oracle against independent facts, and every refusal of the C ABI."""
import ctypes

import numpy as np
import pytest

from oracle import sparse_block_oracle as sbo
from paper_2511_22316_b200 import binding as sq
from paper_2511_22316_b200 import build as sqbuild


@pytest.fixture(scope="module")
def lib():
    sqbuild.build()
    return sq.load()


# -- the oracle ------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("offset", [False, True])
@pytest.mark.parametrize("K,group", [(64, 32), (136, 64), (128, 128)])
def test_quantised_groups_are_within_half_a_step(bits, offset, K, group):
    rng = np.random.default_rng(K + bits)
    Z = rng.standard_normal((9, K)).astype(np.float32) * 0.02 + (0.03 if offset else 0.0)
    Z[3] = 0.0
    codes, sg, bg = sbo.quantise_groups(Z, group, bits, offset)
    w = sbo.weights(codes, sg, bg, group)
    step = sg.astype(np.float64)[np.arange(K) // group].T
    # half a step, plus the rounding of the step (2^-11 of it, times the codes' range) and of the offset (2^-11 of it)
    slack = step * (2.0 ** (bits - 1)) * 2.0 ** -10 + (0 if bg is None else np.abs(bg.astype(np.float64))[np.arange(K) // group].T * 2.0 ** -10)
    assert np.all(np.abs(w - Z) <= step / 2 + slack + 1e-7)


def test_packed_words_hold_the_weight_only_order():
    codes = np.array([[0, 1, 2, 3, 4, 5, 6, 7]]) - 4
    word = int(sbo.pack_codes(codes).view(np.uint32)[0, 0])
    order = (0, 2, 4, 6, 1, 3, 5, 7)
    assert [(word >> (4 * i)) & 15 for i in range(8)] == [int(codes[0, c]) & 15 for c in order]


@pytest.mark.parametrize("renorm", [False, True])
def test_oracle_gradient_of_the_router_against_differences(renorm):
    rng = np.random.default_rng(3)
    T, E, k = 5, 7, 3
    x = rng.standard_normal((T, E))
    mask = np.array([1, 1, 0, 1, 1])
    dg, dl = rng.standard_normal((T, k)), 1.7
    base = sbo.route(x, k, renorm, mask)
    grad = sbo.route_backward(base, renorm, dg, dl)

    def value(y):
        r = sbo.route(y, k, renorm, mask)
        assert np.array_equal(r["ids"], base["ids"])
        return dl * r["loss"] + (dg * r["gates"]).sum()
    h = 1e-6
    for t in range(T):
        for e in range(E):
            y, z = x.copy(), x.copy()
            y[t, e] += h
            z[t, e] -= h
            # central difference: error h^2 times a third derivative of order one, rounding 1e-16 / h
            assert abs((value(y) - value(z)) / (2 * h) - grad[t, e]) < 1e-8


def test_oracle_router_sorts_rows_by_expert_and_token():
    rng = np.random.default_rng(4)
    r = sbo.route(rng.standard_normal((20, 6)), 2, True)
    rows = [(e, t) for e in range(6) for t in r["row_token"][r["offsets"][e]:r["offsets"][e + 1]]]
    assert rows == sorted(rows) and len(rows) == 40
    assert np.allclose(r["gates"].sum(1), 1)


# -- refusals --------------------------------------------------------------------------------------------------------------

P = 1 << 20          # a 16-byte aligned address that nothing reads: every call below is refused before a launch
BAD, SHAPE, ALIGN, UNSUP, NOMEM = (sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_SHAPE, sq.SQ_ERR_ALIGN, sq.SQ_ERR_UNSUPPORTED, sq.SQ_ERR_NOMEM)


def _refusals(f, good, cases):
    for change, code in cases:
        args = dict(good)
        assert set(change) <= set(args), change
        args.update(change)
        assert f(*args.values()) == code, (change, code)


def test_product_refusals(lib):
    good = dict(Z=P, Wq=P, sg=P, bg=None, M=4, N=64, K=128, group=128, Y=P, stream=None)
    _refusals(lib.sq_w4a16_gemm_gs, good, [
        (dict(Z=None), BAD), (dict(Wq=None), BAD), (dict(sg=None), BAD), (dict(Y=None), BAD), (dict(M=-1), BAD), (dict(N=-1), BAD),
        (dict(M=1 << 31), BAD), (dict(group=16), BAD), (dict(group=0), BAD), (dict(group=96), BAD), (dict(group=256), BAD),
        (dict(K=4), SHAPE), (dict(K=132), SHAPE), (dict(K=0), SHAPE), (dict(K=65544), UNSUP),
        (dict(Z=P + 8), ALIGN), (dict(Wq=P + 4), ALIGN), (dict(sg=P + 2), ALIGN), (dict(bg=P + 2), ALIGN), (dict(Y=P + 8), ALIGN),
        (dict(M=0), sq.SQ_OK), (dict(N=0), sq.SQ_OK), (dict(M=0, Z=None), sq.SQ_OK)])


def test_grouped_product_refusals(lib):
    good = dict(Z=P, T=4, row_token=P, offsets=P, E=8, Wq=P, sg=P, bg=None, M=8, N=64, K=128, group=32, ws=P, wsb=8 * 256, Y=P, stream=None)
    _refusals(lib.sq_w4a16_gemm_gs_grouped, good, [
        (dict(Z=None), BAD), (dict(offsets=None), BAD), (dict(E=0), BAD), (dict(E=1025), UNSUP), (dict(T=0), BAD), (dict(T=-1), BAD),
        (dict(row_token=None), SHAPE), (dict(row_token=P + 4), ALIGN), (dict(offsets=P + 4), ALIGN), (dict(ws=None), BAD),
        (dict(ws=P + 16), ALIGN), (dict(wsb=8 * 256 - 1), NOMEM), (dict(group=48), BAD), (dict(K=100), SHAPE), (dict(M=0), sq.SQ_OK),
        (dict(N=0), sq.SQ_OK)])
    assert lib.sq_gemm_gs_grouped_workspace_bytes(8, 128) == 8 * 256
    assert lib.sq_gemm_gs_grouped_workspace_bytes(0, 128) == 0
    assert lib.sq_linear_gs_grouped_workspace_bytes(4, 8, 128) == 12 * 256


def test_pack_refusals(lib):
    good = dict(rot=None, W=P, N=64, K=128, bits=4, group=64, Wq=P, sg=P, bg=None, ws=None, wsb=0, stream=None)
    _refusals(lib.sq_pack_weight_gs, good, [
        (dict(W=None), BAD), (dict(Wq=None), BAD), (dict(sg=None), BAD), (dict(bits=5), BAD), (dict(bits=2), BAD), (dict(group=8), BAD),
        (dict(K=12), SHAPE), (dict(K=0), SHAPE), (dict(K=32776), UNSUP), (dict(bg=P + 2), ALIGN), (dict(N=-1), BAD), (dict(N=0), sq.SQ_OK)])
    assert lib.sq_pack_weight_gs_workspace_bytes(3, 128) == 3 * 512 + 256 + 256
    assert lib.sq_pack_weight_gs_workspace_bytes(1 << 20, 128) == lib.sq_pack_weight_gs_workspace_bytes(1024, 128)


def test_layer_refusals(lib):
    assert lib.sq_linear_gs(None, P, 4, P, P, None, 64, 128, 128, P, 1 << 20, P, None) == BAD
    assert lib.sq_linear_gs_grouped(None, P, 4, P, P, 8, P, P, None, 8, 64, 128, 128, P, 1 << 20, P, None) == BAD


def test_route_refusals(lib):
    good = dict(logits=P, dtype=sq.SQ_F32, T=4, E=8, ld=8, k=2, flags=1, mask=None, ids=P, gates=P, counts=P, offsets=P, row_token=P, pos=P,
                loss=None, ws=None, wsb=0, stream=None)
    big = dict(T=100000, ws=P, wsb=1 << 30)
    _refusals(lib.sq_route, good, [
        (dict(logits=None), BAD), (dict(ids=None), BAD), (dict(gates=None), BAD), (dict(counts=None), BAD), (dict(offsets=None), BAD),
        (dict(row_token=None), BAD), (dict(pos=None), BAD), (dict(dtype=3), BAD), (dict(dtype=-1), BAD), (dict(T=-1), BAD),
        (dict(E=0), BAD), (dict(k=0), BAD), (dict(k=9), BAD), (dict(flags=2), BAD), (dict(E=1025, ld=1025), UNSUP),
        (dict(E=64, ld=64, k=33), UNSUP), (dict(T=(1 << 30), ld=8), UNSUP), (dict(ld=7), SHAPE), (dict(logits=P + 8), ALIGN),
        (dict(mask=P + 1), ALIGN), (dict(gates=P + 4), ALIGN), (dict(loss=P + 4), ALIGN), (dict(big, ws=None), BAD),
        (dict(big, ws=P + 128), ALIGN), (dict(big, wsb=16), NOMEM)])
    for E in (1, 8, 60, 256, 1024):
        assert lib.sq_route_workspace_bytes(1 << 20, E) <= 2 << 20
    assert lib.sq_route_workspace_bytes(1, 8) == 0


def test_route_backward_refusals(lib):
    good = dict(logits=P, dtype=sq.SQ_BF16, T=4, E=8, ld=8, k=2, flags=0, mask=None, ids=P, gates=P, counts=P, dgates=P, dloss=None,
                dlogits=P + 4096, ld_d=8, stream=None)
    _refusals(lib.sq_route_backward, good, [
        (dict(logits=None), BAD), (dict(ids=None), BAD), (dict(gates=None), BAD), (dict(counts=None), BAD), (dict(dlogits=None), BAD),
        (dict(ld_d=7), SHAPE), (dict(ld=7), SHAPE), (dict(dlogits=P, ld_d=16), BAD), (dict(dgates=P + 4), ALIGN), (dict(dloss=P + 4), ALIGN),
        (dict(flags=4), BAD), (dict(T=0), sq.SQ_OK)])


def test_combine_refusals(lib):
    good = dict(Y=P, M=8, pos=P, gates=P, T=4, k=2, N=64, out=P + 4096, stream=None)
    _refusals(lib.sq_combine, good, [
        (dict(Y=None), BAD), (dict(pos=None), BAD), (dict(gates=None), BAD), (dict(out=None), BAD), (dict(out=P), BAD), (dict(k=0), BAD),
        (dict(k=33), UNSUP), (dict(T=1 << 30), UNSUP), (dict(M=-1), BAD), (dict(N=-1), BAD), (dict(Y=P + 2), ALIGN), (dict(out=P + 8), ALIGN),
        (dict(T=0), sq.SQ_OK), (dict(N=0), sq.SQ_OK)])
    good = dict(dout=P, Y=P, M=8, pos=P, gates=P, T=4, k=2, N=64, dY=P + 4096, dgates=P, stream=None)
    _refusals(lib.sq_combine_backward, good, [
        (dict(dout=None), BAD), (dict(Y=None), BAD), (dict(pos=None), BAD), (dict(gates=None), BAD), (dict(dY=P), BAD),
        (dict(dgates=P + 4), ALIGN), (dict(k=40), UNSUP), (dict(T=0), sq.SQ_OK), (dict(dY=None, dgates=None), sq.SQ_OK)])


def test_python_binding_raises(lib):
    with pytest.raises(sq.SingleQuantError) as e:
        sq.sq_w4a16_gemm_gs(P, P, P, None, 1, 64, 128, 100, P, stream=0)
    assert e.value.code == BAD
    assert isinstance(ctypes.c_size_t(sq.sq_route_workspace_bytes(4096, 64)).value, int)
