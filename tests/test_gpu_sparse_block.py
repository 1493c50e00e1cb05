"""Router, combination and a whole sparse block on the GPU."""
import numpy as np
import pytest

from gpu_util import Guarded, dev
from oracle import singlequant_oracle as ora
from oracle import sparse_block_oracle as sbo
from paper_2511_22316_b200 import binding as sq

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -11, 2.0 ** -24
DTYPES = {"fp16": (sq.SQ_F16, 2, 2.0 ** -11), "bf16": (sq.SQ_BF16, 2, 2.0 ** -8), "fp32": (sq.SQ_F32, 4, 2.0 ** -24)}


def as_type(x, dtype):
    """(what the device holds, torch tensor; its values in fp64)"""
    import torch
    t = torch.from_numpy(np.asarray(x, np.float32)).to({"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
    return t.cuda(), t.double().numpy()


class Routed:
    def __init__(self, x, dtype, k, renorm, mask=None, ld=None, workspace=None):
        import torch
        T, E = x.shape
        self.ld = ld or E
        wide = np.full((T, self.ld), 99.0, np.float32)          # what lies behind a row must not be read as a logit
        wide[:, :E] = x
        self.t, v = as_type(wide, dtype)
        self.v, self.T, self.E, self.k, self.code, self.renorm = v[:, :E], T, E, k, DTYPES[dtype][0], renorm
        self.mask = None if mask is None else dev(np.asarray(mask, np.uint8))
        self.host_mask = mask
        g = {n: Guarded(max(4, b)) for n, b in dict(ids=4 * T * k, gates=4 * T * k, counts=4 * (E + 1), offsets=4 * (E + 1), row_token=4 * T * k,
                                                    pos=4 * T * k, loss=4).items()}
        for b in g.values():
            b.view.fill_(0x77)
        nb = sq.sq_route_workspace_bytes(T, E)
        self.ws = workspace if workspace is not None else torch.full((max(nb, 256),), 0x5A, dtype=torch.uint8, device="cuda")
        self.g, self.nb = g, nb
        self.run()

    def run(self, stream=None):
        g = self.g
        sq.sq_route(self.t, self.code, self.T, self.E, self.ld, self.k, sq.SQ_ROUTE_RENORM if self.renorm else 0, self.mask, g["ids"], g["gates"],
                    g["counts"], g["offsets"], g["row_token"], g["pos"], g["loss"], self.ws, self.nb, stream=stream)

    def read(self):
        import torch
        torch.cuda.synchronize()
        for b in self.g.values():
            b.check()
        T, E, k = self.T, self.E, self.k
        read = lambda n, kind, shape: self.g[n].numpy(kind, -1)[:int(np.prod(shape))].reshape(shape)          # (T = 0: a buffer of one)
        i = {n: read(n, np.int32, s) for n, s in dict(ids=(T, k), counts=(E + 1,), offsets=(E + 1,), row_token=(T * k,), pos=(T, k)).items()}
        return dict(i, gates=read("gates", np.float32, (T, k)), loss=read("loss", np.float32, (1,))[0])

    def check(self):
        got, want = self.read(), sbo.route(self.v, self.k, self.renorm, self.host_mask)
        for n in ("ids", "counts", "offsets", "pos"):
            assert np.array_equal(got[n], want[n]), n
        rows = want["offsets"][-1]
        assert np.array_equal(got["row_token"][:rows], want["row_token"][:rows])
        assert np.all(got["row_token"][rows:] == 0x77777777)
        # exp: 2 ulp and its argument's rounding (|x - m| U32, where e^-(x-m) matters at all: below 104); the sum over E, one division
        with np.errstate(invalid="ignore"):
            spread = np.nan_to_num(np.where(np.isfinite(self.v), self.v, np.nan).max(1, initial=-1e30, where=np.isfinite(self.v))
                                   - np.where(np.isfinite(self.v), self.v, np.nan).min(1, initial=1e30, where=np.isfinite(self.v)))
        rel = (np.clip(spread, 0, 104) + self.E + 12)[:, None] * 2 * U32
        assert np.all(np.abs(got["gates"] - want["gates"]) <= rel * want["gates"] + 2.0 ** -126)
        assert abs(got["loss"] - want["loss"]) <= ((np.clip(spread, 0, 104).max(initial=0) + self.E + self.T / 64 + 64) * 4 * U32) * abs(want["loss"]) + 1e-30
        return got, want


ROUTES = [(1, 1, 1), (1, 8, 2), (16, 8, 2), (5, 5, 5), (7, 16, 16), (100, 9, 3), (64, 60, 4), (129, 64, 6), (257, 8, 1), (300, 16, 2),
          (700, 32, 8), (1000, 128, 8), (515, 256, 8), (65, 200, 32), (40, 512, 4), (33, 1000, 10), (70, 1024, 32), (3000, 4, 2), (2100, 33, 3)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E,k", ROUTES)
def test_route(T, E, k, renorm, dtype):
    rng = np.random.default_rng(T + E + k)
    x = 1.5 * rng.standard_normal((T, E)) + 0.7 * rng.standard_normal(E)
    mask = rng.random(T) < 0.8 if T % 2 else None
    Routed(x, dtype, k, renorm, mask, ld=E if T % 3 else E + 5).check()


@pytest.mark.parametrize("T,experts,k", [(200, range(17, 64), 2), (20, range(100, 420, 10), 3), (900, range(4, 17), 2), (300, range(257, 400, 7), 2)])
def test_route_with_every_amount_of_shared_memory(T, experts, k):
    """Around the 48 KB up to which a kernel need not ask for its shared memory, and on either side of every shape's border."""
    rng = np.random.default_rng(T)
    for E in experts:
        x = rng.standard_normal((T, E))
        r = Routed(x, "bf16" if E % 2 else "fp32", min(k, E), True)
        got, want = r.read(), sbo.route(r.v, r.k, True)
        for n in ("ids", "counts", "offsets", "pos"):
            assert np.array_equal(got[n], want[n]), (E, n)


def test_route_of_more_slots_than_stay_on_chip():
    """More than 4096 slots of a block: experts and ranks go through the outputs instead."""
    rng = np.random.default_rng(0)
    Routed(rng.standard_normal((90000, 8)) + rng.standard_normal(8), "fp32", 8, False, rng.random(90000) < 0.9).check()


def test_combine_without_rows():
    import torch
    pos, gates, out = dev(np.zeros((3, 2), np.int32)), dev(np.ones((3, 2), np.float32)), Guarded(3 * 16 * 2)
    sq.sq_combine(None, 0, pos, gates, 3, 2, 16, out)
    dg = Guarded(3 * 2 * 4)
    sq.sq_combine_backward(dev(np.ones((3, 16), np.float16)), None, 0, pos, gates, 3, 2, 16, None, dg)
    torch.cuda.synchronize()
    assert not out.numpy(np.uint16, (3, 16)).any() and not dg.numpy(np.uint32, (3, 2)).any()


@pytest.mark.parametrize("E,k", [(8, 3), (16, 4), (40, 8), (300, 5)])
@pytest.mark.parametrize("T", [3, 400])
def test_equal_logits_go_to_the_lowest_index(T, E, k):
    rng = np.random.default_rng(T + E)
    x = rng.integers(-2, 3, (T, E)).astype(np.float32)
    x[0] = 0
    x[1, ::2] = -0.0
    x[1, 1::2] = 0.0
    Routed(x, "fp32", k, True).check()
    Routed(np.zeros((T, E)), "bf16", k, False).check()


@pytest.mark.parametrize("T", [12, 300])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E", [6, 40, 130])
def test_logits_that_are_not_finite_and_masks(T, renorm, E):
    rng = np.random.default_rng(T)
    x = rng.standard_normal((T, E)).astype(np.float32)
    x[0] = -np.inf                            # no expert at all
    x[1] = np.nan
    x[2, 1:] = -np.inf                        # one expert for three slots
    x[3, ::2] = np.nan
    x[4, 2] = np.inf                          # one expert takes all
    x[5, [0, 3]] = np.inf
    x[6] = np.finfo(np.float32).min           # the type's lowest value: finite, all alike
    x[7, 1:] = np.finfo(np.float32).min
    x[8] = np.inf
    mask = np.ones(T)
    mask[9:11] = 0
    r = Routed(x, "fp32", 3, renorm, mask)
    r.check()
    # their gradients are finite and zero where there is no choice
    d = Backward(r, rng).check()
    assert np.isfinite(d).all() and not d[[0, 1, 9, 10]].any()


@pytest.mark.parametrize("T", [0, 1, 200, 900])
def test_no_token_counts(T):
    r = Routed(np.zeros((T, 8), np.float32), "fp32", 2, True, np.zeros(T))
    got = r.read()
    assert not got["counts"].any() and not got["offsets"].any() and got["loss"] == 0
    assert np.all(got["ids"] == -1) and np.all(got["pos"] == -1) and not got["gates"].any()
    if T:
        assert not Backward(r, np.random.default_rng(0)).check().any()


def test_route_twice_gives_the_same_bits_and_a_shared_workspace_needs_no_clearing():
    import torch
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((5000, 64)), rng.standard_normal((4000, 64))
    ws = torch.zeros(sq.sq_route_workspace_bytes(5000, 64), dtype=torch.uint8, device="cuda")
    a = Routed(x, "bf16", 4, False, workspace=ws)
    first, _ = a.check()
    Routed(y, "fp32", 2, True, workspace=ws).check()
    a.run()
    again = a.read()
    for n in first:
        assert np.array_equal(first[n].view(np.uint32) if n == "gates" else first[n], again[n].view(np.uint32) if n == "gates" else again[n]), n


class Backward:
    def __init__(self, r, rng, dgates=True, dloss=True, ld_d=None):
        T, E, k = r.T, r.E, r.k
        self.r, self.ld = r, ld_d or E
        self.dg = rng.standard_normal((T, k)).astype(np.float32) if dgates else None
        self.dl = np.float32(1.0 + rng.random()) if dloss else None
        self.width = 4 if r.code == sq.SQ_F32 else 2
        self.out = Guarded(T * self.ld * self.width)
        self.out.view.fill_(0x33)
        g = r.g
        sq.sq_route_backward(r.t, r.code, T, E, r.ld, k, sq.SQ_ROUTE_RENORM if r.renorm else 0, r.mask, g["ids"], g["gates"], g["counts"],
                             None if self.dg is None else dev(self.dg), None if self.dl is None else dev(np.array([self.dl])), self.out, self.ld)

    def values(self):
        import torch
        torch.cuda.synchronize()
        self.out.check()
        t = self.out.view.cpu()
        kind = {sq.SQ_F16: torch.float16, sq.SQ_BF16: torch.bfloat16, sq.SQ_F32: torch.float32}[self.r.code]
        v = t.view(kind).reshape(self.r.T, self.ld)
        assert (t.view(torch.uint8).reshape(self.r.T, -1)[:, self.r.E * self.width:] == 0x33).all()
        return v[:, :self.r.E].double().numpy()

    def check(self):
        r = self.r
        want = sbo.route(r.v, r.k, r.renorm, r.host_mask)
        dg = np.zeros((r.T, r.k)) if self.dg is None else self.dg.astype(np.float64)
        dl = 0.0 if self.dl is None else float(self.dl)
        exact = sbo.route_backward(want, r.renorm, dg, dl)
        got = self.values()
        u = {sq.SQ_F16: U16, sq.SQ_BF16: 2.0 ** -8, sq.SQ_F32: U32}[r.code]
        # fp32 arithmetic on values up to d = max |dgates| + |loss term|: p is off by (spread + E) roundings, the dot product by E more
        top = (np.abs(dg).max(1, initial=0) + abs(dl) * r.E * want["counts"][:r.E].max() / max(1, r.k * want["counts"][-1]) / max(1, want["counts"][-1]))
        finite = np.where(np.isfinite(r.v), r.v, 0.0)
        spread = np.clip(finite.max(1) - finite.min(1), 0, 104)
        tol = np.abs(exact) * u + ((spread + 2 * r.E + 40) * 8 * U32 * top)[:, None] + (2.0 ** -25 if u == U16 else 1e-38)
        assert np.all(np.abs(got - exact) <= tol)
        return got


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E,k", ROUTES)
def test_route_backward(T, E, k, renorm, dtype):
    rng = np.random.default_rng(T + E + k)
    x = 1.5 * rng.standard_normal((T, E))
    mask = rng.random(T) < 0.8 if T % 2 else None
    r = Routed(x, dtype, k, renorm, mask, ld=E if T % 3 else E + 3)
    Backward(r, rng, ld_d=E if T % 5 else E + 7).check()
    Backward(r, rng, dgates=False).check()
    Backward(r, rng, dloss=False).check()


@pytest.mark.parametrize("renorm", [False, True])
def test_route_backward_against_differences(renorm):
    """The library's own loss and gates, differenced: fp32 values of order one, steps of 2^-7."""
    rng = np.random.default_rng(9)
    T, E, k = 6, 12, 3
    x = np.round(rng.standard_normal((T, E)) * 64) / 64 + np.arange(E) * 0.25          # no two logits of a token nearer than a step
    x = np.argsort(np.argsort(x, 1), 1) * 0.25
    r = Routed(x, "fp32", k, renorm)
    b = Backward(r, rng)
    grad, base, h = b.values(), r.read(), 2.0 ** -7

    def value(y):
        q = Routed(y, "fp32", k, renorm).read()
        assert np.array_equal(q["ids"], base["ids"])
        return float(b.dl) * float(q["loss"]) + float((b.dg.astype(np.float64) * q["gates"]).sum())
    for t in range(T):
        for e in range(E):
            y, z = x.copy(), x.copy()
            y[t, e] += h
            z[t, e] -= h
            # h^2 / 6 times a third derivative (below 1 for a softmax, times k |dgates| + 2), and 2^-23 of values of order ten over 2 h
            bound = h * h / 6 * (np.abs(b.dg[t]).sum() + 2) + 10 * 2.0 ** -23 / (2 * h) * 4
            assert abs((value(y) - value(z)) / (2 * h) - grad[t, e]) <= bound


def test_gradient_in_place():
    rng = np.random.default_rng(2)
    import torch
    r = Routed(rng.standard_normal((700, 64)), "fp32", 2, True)
    b = Backward(r, rng)
    want = b.values()
    g = r.g
    sq.sq_route_backward(r.t, r.code, r.T, r.E, r.ld, r.k, sq.SQ_ROUTE_RENORM, None, g["ids"], g["gates"], g["counts"], dev(b.dg),
                         dev(np.array([b.dl])), r.t, r.ld)
    torch.cuda.synchronize()
    assert np.array_equal(r.t.double().cpu().numpy(), want)


# -- combination -----------------------------------------------------------------------------------------------------------


def slots(rng, T, k, M, some_empty):
    """pos [T, k]: distinct rows, some slots without one."""
    pos = rng.permutation(M)[:T * k].reshape(T, k) if M >= T * k else None
    if some_empty:
        pos = np.where(rng.random((T, k)) < 0.3, -1, pos)
        pos[0] = -1
        pos[-1, -1] = M + 5
    return pos.astype(np.int32)


COMBINE = [(1, 1, 8), (1, 2, 4096), (16, 2, 4096), (5, 3, 33), (7, 4, 1), (33, 5, 264), (20, 8, 2056), (3, 32, 72), (1500, 2, 64), (2, 6, 14336)]


@pytest.mark.parametrize("some_empty", [False, True])
@pytest.mark.parametrize("T,k,N", COMBINE)
def test_combine_and_its_gradient(T, k, N, some_empty):
    import torch
    rng = np.random.default_rng(T + k + N)
    M = T * k + 4
    pos = slots(rng, T, k, M, some_empty)
    Y = rng.standard_normal((M, N)).astype(np.float16)
    unused = np.setdiff1d(np.arange(M), pos)
    Y[unused] = np.nan                                  # rows that no slot names
    gates = rng.random((T, k)).astype(np.float32)
    gates[pos < 0] = np.nan                             # and gates of slots without a row are not used
    out = Guarded(T * N * 2)
    sq.sq_combine(dev(Y), M, dev(pos), dev(gates), T, k, N, out)
    torch.cuda.synchronize()
    out.check()
    exact = sbo.combine(Y, pos, gates)
    size = sbo.combine(np.abs(Y), pos, np.abs(gates))
    # k fused multiply-adds in fp32, one rounding to fp16
    assert np.all(np.abs(out.numpy(np.float16, (T, N)) - exact) <= (k + 1) * U32 * size + U16 * np.abs(exact) * 1.01 + 2.0 ** -25)

    dout = rng.standard_normal((T, N)).astype(np.float16)
    dY, dg = Guarded(M * N * 2), Guarded(T * k * 4)
    dY.view.fill_(0x11)
    sq.sq_combine_backward(dev(dout), dev(Y), M, dev(pos), dev(gates), T, k, N, dY, dg)
    torch.cuda.synchronize()
    dY.check()
    dg.check()
    want, wdg = sbo.combine_backward(dout, Y, pos, gates)
    got = dY.numpy(np.float16, (M, N))
    named = ~np.isnan(want[:, 0])
    assert np.all(np.abs(got[named] - want[named]) <= np.abs(want[named]) * (U16 + 2 * U32) + 2.0 ** -25)
    assert np.all(got[~named].view(np.uint16) == 0x1111)
    g = dg.numpy(np.float32, (T, k))
    _, sz = sbo.combine_backward(np.abs(dout), np.abs(Y), pos, gates)
    assert np.all(np.abs(g - wdg) <= (N + 8) * U32 * sz)
    assert not g[(pos < 0) | (pos >= M)].any()
    # either alone
    one, two = Guarded(M * N * 2), Guarded(T * k * 4)
    one.view.fill_(0x11)
    sq.sq_combine_backward(dev(dout), dev(Y), M, dev(pos), dev(gates), T, k, N, one, None)
    sq.sq_combine_backward(dev(dout), dev(Y), M, dev(pos), dev(gates), T, k, N, None, two)
    torch.cuda.synchronize()
    assert np.array_equal(one.numpy(np.uint16, (M, N)), got.view(np.uint16))
    assert np.array_equal(two.numpy(np.uint32, (T, k)), g.view(np.uint32))


# -- the block ---------------------------------------------------------------------------------------------------------------


class Block:
    """Up and down projection of E experts behind one rotation each, 4-bit weights with group scales, and the router's outputs."""

    def __init__(self, E, k, n1, n2, F, group, T, seed=0, f1=0, f2=0):
        import torch
        rng = np.random.default_rng(seed)
        K = n1 * n2
        self.E, self.k, self.K, self.F, self.group, self.T = E, k, K, F, group, T
        calib = rng.standard_normal((8, K)).astype(np.float32)
        self.rot = sq.sq_build_rotation(calib, n1, n2)
        self.rot2 = sq.sq_build_rotation(rng.standard_normal((8, F)).astype(np.float32), f1, f2)
        def experts(rot, N, Kin):
            G = -(-Kin // group)
            q = torch.empty(E, N, Kin // 2, dtype=torch.uint8, device="cuda")
            s = torch.empty(E, G, N, dtype=torch.float16, device="cuda")
            b = torch.empty(E, G, N, dtype=torch.float16, device="cuda")
            nb = sq.sq_pack_weight_gs_workspace_bytes(N, Kin)
            ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
            for e in range(E):
                W = (rng.standard_normal((N, Kin)) / np.sqrt(Kin)).astype(np.float16)
                sq.sq_pack_weight_gs(rot, dev(W), N, Kin, 4, group, q[e], s[e], b[e], ws, nb)
            return q, s, b
        self.up, self.down = experts(self.rot, F, K), experts(self.rot2, K, F)
        M = T * k
        z = lambda *shape, t=torch.float16: torch.zeros(*shape, dtype=t, device="cuda")
        self.x, self.logits = z(T, K), z(T, E, t=torch.float32)
        self.ids, self.pos, self.row_token = z(T, k, t=torch.int32), z(T, k, t=torch.int32), z(M, t=torch.int32)
        self.gates, self.loss = z(T, k, t=torch.float32), z(1, t=torch.float32)
        self.counts, self.offsets = z(E + 1, t=torch.int32), z(E + 1, t=torch.int32)
        self.h, self.y, self.out = z(M, F), z(M, K), z(T, K)
        self.rws = z(max(256, sq.sq_route_workspace_bytes(T, E)), t=torch.uint8)
        self.nb = max(sq.sq_linear_gs_grouped_workspace_bytes(T, M, K), sq.sq_linear_gs_grouped_workspace_bytes(M, M, F))
        self.ws = z(self.nb, t=torch.uint8)

    def step(self, stream=None):
        T, M, E, k = self.T, self.T * self.k, self.E, self.k
        sq.sq_route(self.logits, sq.SQ_F32, T, E, E, k, sq.SQ_ROUTE_RENORM, None, self.ids, self.gates, self.counts, self.offsets,
                    self.row_token, self.pos, self.loss, self.rws, self.rws.numel(), stream=stream)
        sq.sq_linear_gs_grouped(self.rot, self.x, T, self.row_token, self.offsets, E, *self.up, M, self.F, self.K, self.group, self.ws, self.nb,
                                self.h, stream=stream)
        self.h.relu_()
        sq.sq_linear_gs_grouped(self.rot2, self.h, M, None, self.offsets, E, *self.down, M, self.K, self.F, self.group, self.ws, self.nb, self.y,
                                stream=stream)
        sq.sq_combine(self.y, M, self.pos, self.gates, T, k, self.K, self.out, stream=stream)

    def expected(self):
        def w(packed, e, K):
            q, s, b = (t[e].cpu().numpy() for t in packed)
            words = q.view(np.uint32)
            codes = np.zeros((q.shape[0], K), np.int64)
            for c in range(8):
                codes[:, c::8] = (((words >> np.uint32(4 * sbo.POSITION[c])) & 15) ^ 8).astype(np.int64) - 8
            return sbo.weights(codes, s, b, self.group)
        x = self.x.cpu().numpy()
        r = sbo.route(self.logits.cpu().numpy(), self.k, True)
        z = ora.rotate_f16(x, *self.rot.factors())
        M = self.T * self.k
        h = sbo.experts(z, [w(self.up, e, self.K) for e in range(self.E)], r["row_token"], r["offsets"], M)
        h = np.maximum(h, 0).astype(np.float16)
        z2 = ora.rotate_f16(h, *self.rot2.factors())
        y = sbo.experts(z2, [w(self.down, e, self.F) for e in range(self.E)], np.arange(M), r["offsets"], M)
        return sbo.combine(y, r["pos"], r["gates"]), r


@pytest.mark.parametrize("T,E,k", [(1, 4, 2), (6, 8, 2), (90, 4, 2), (40, 16, 4)])
def test_whole_block(T, E, k):
    import torch
    b = Block(E, k, 8, 32, 512, 32, T, f1=16, f2=32)
    rng = np.random.default_rng(T)
    b.x.copy_(dev(rng.standard_normal((T, b.K)).astype(np.float16)))
    b.logits.copy_(dev(rng.standard_normal((T, E)).astype(np.float32)))
    b.step()
    torch.cuda.synchronize()
    want, r = b.expected()
    assert np.array_equal(b.row_token.cpu().numpy(), r["row_token"]) and np.array_equal(b.counts.cpu().numpy(), r["counts"])
    # six roundings to fp16 on the way (two rotations' results, weights twice, two products) and the last one, each U16 of the norm
    assert np.linalg.norm(b.out.cpu().numpy() - want) <= 8 * U16 * np.linalg.norm(want)


def test_whole_block_captured_and_replayed_with_another_routing():
    import torch
    T, E, k = 12, 8, 2
    b = Block(E, k, 8, 32, 512, 32, T, f1=16, f2=32)
    s = torch.cuda.Stream()
    rng = np.random.default_rng(0)
    def fill(seed):
        q = np.random.default_rng(seed)
        b.x.copy_(dev(q.standard_normal((T, b.K)).astype(np.float16)))
        b.logits.copy_(dev(q.standard_normal((T, E)).astype(np.float32) + (5.0 if seed == 2 else 0.0) * (np.arange(E) < 2)))
    fill(1)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.step()
    for seed in (2, 3):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        want, r = b.expected()
        assert np.array_equal(b.counts.cpu().numpy(), r["counts"])
        assert np.linalg.norm(b.out.cpu().numpy() - want) <= 8 * U16 * np.linalg.norm(want)
    assert rng is not None


def test_the_routing_feeds_the_w4a4_grouped_layer():
    """The rows that sq_route sorts are those that sq_linear_grouped wants, its offsets copied to the host."""
    import torch
    T, E, k, n1, n2, N = 24, 4, 2, 8, 64, 256
    K = n1 * n2
    rng = np.random.default_rng(6)
    r = Routed(rng.standard_normal((T, E)), "fp32", k, True)
    got = r.read()
    X = rng.standard_normal((T, K)).astype(np.float16)
    rot = sq.sq_build_rotation(X.astype(np.float32), n1, n2)
    Ws = [(0.02 * rng.standard_normal((N, K))).astype(np.float16) for _ in range(E)]
    packed = []
    for W in Ws:
        q, s = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda"), torch.empty(N, dtype=torch.float16, device="cuda")
        sq.sq_pack_weight(rot, dev(W), N, K, q, s)
        packed.append((q, s))
    Xs = dev(X)[torch.from_numpy(got["row_token"]).long().cuda()]
    Y = torch.empty(T * k, N, dtype=torch.float16, device="cuda")
    nb = sq.sq_linear_workspace_bytes(T * k, K)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    sq.sq_linear_grouped([rot] * E, got["offsets"], Xs, [q for q, _ in packed], [s for _, s in packed], N, K, ws, nb, Y)
    out = torch.empty(T, N, dtype=torch.float16, device="cuda")
    sq.sq_combine(Y, T * k, r.g["pos"], r.g["gates"], T, k, N, out)
    torch.cuda.synchronize()
    R1, R2 = rot.factors()
    want = ora.linear_grouped(X[got["row_token"]], got["offsets"], Ws, [(R1, R2)] * E).astype(np.float64)
    full = sbo.combine(want, got["pos"], got["gates"])
    assert np.linalg.norm(out.cpu().numpy() - full) <= 1e-2 * np.linalg.norm(full)


def test_two_streams_at_once():
    """Two routings and two products at a time, each with a workspace and outputs of its own."""
    import torch
    blocks = [Block(8, 2, 8, 32, 512, 32, 20, seed=i, f1=16, f2=32) for i in range(2)]
    rng = np.random.default_rng(3)
    for b in blocks:
        b.x.copy_(dev(rng.standard_normal((20, b.K)).astype(np.float16)))
        b.logits.copy_(dev(rng.standard_normal((20, 8)).astype(np.float32)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(20):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b.step()
    torch.cuda.synchronize()
    for b in blocks:
        want, _ = b.expected()
        assert np.linalg.norm(b.out.cpu().numpy() - want) <= 8 * U16 * np.linalg.norm(want)
