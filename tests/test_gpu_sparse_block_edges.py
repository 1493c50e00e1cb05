"""Router and combination where they can go wrong and the tests of every operator do not look."""
import numpy as np
import pytest

from gpu_util import Guarded, dev
from paper_2511_22316_b200 import binding as sq
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


@pytest.mark.parametrize("dloss", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E", [(6, 8), (300, 40)])
def test_tokens_that_do_not_count_have_no_gradient_even_of_an_overflown_loss(T, E, renorm, dloss):
    rng = np.random.default_rng(T)
    x = rng.standard_normal((T, E)).astype(np.float32)
    x[1] = -np.inf
    x[2] = np.nan
    mask = np.ones(T)
    mask[4:] = rng.random(T - 4) < 0.5
    mask[3], mask[4] = 0, 1
    r = Routed(x, "fp32", 2, renorm, mask)
    out, g = Guarded(T * E * 4), r.g
    sq.sq_route_backward(r.t, r.code, T, E, E, 2, sq.SQ_ROUTE_RENORM if renorm else 0, r.mask, g["ids"], g["gates"], g["counts"], None,
                         dev(np.array([dloss], np.float32)), out, E)
    got = out.numpy(np.float32, (T, E))
    counted = (mask > 0) & (np.arange(T) != 1) & (np.arange(T) != 2)
    assert not got[~counted].any() and not np.isfinite(got[counted]).all(1).any()


def test_gradient_of_a_combination_without_channels():
    """Rows of no channels need no memory behind them; the gates' gradients are sums of nothing."""
    dg = Guarded(5 * 2 * 4)
    sq.sq_combine_backward(None, None, 9, dev(np.zeros((5, 2), np.int32)), dev(np.ones((5, 2), np.float32)), 5, 2, 0, None, dg)
    got = dg.numpy(np.uint32, (5, 2))
    dg.check()
    assert not got.any()


@pytest.mark.parametrize("T,E", [(4000000, 49), (2000000, 60), (70000, 7)])
def test_loss_of_many_tokens(T, E):
    """All logits alike: every token has 1 / E of every expert and goes to the first, so the loss is 1.  Each addition of equal numbers
    is off to the same side, which a plain sum of a run of tokens shows."""
    import torch
    x = torch.zeros(T, E, dtype=torch.float16, device="cuda")
    i32 = lambda *n: torch.empty(*n, dtype=torch.int32, device="cuda")
    ids, gates, pos, row_token, counts, offsets = i32(T, 1), i32(T, 1), i32(T, 1), i32(T), i32(E + 1), i32(E + 1)
    loss = torch.empty(1, dtype=torch.float32, device="cuda")
    nb = sq.sq_route_workspace_bytes(T, E)
    sq.sq_route(x, sq.SQ_F16, T, E, E, 1, 0, None, ids, gates, counts, offsets, row_token, pos, loss, torch.empty(nb, dtype=torch.uint8, device="cuda"), nb)
    assert counts.tolist() == [T] + [0] * (E - 1) + [T] and offsets.tolist() == [0] + [T] * E
    run = -(-(-(-T // 148)) // 32)
    # 1 / E once; 64 additions in a register, one for each 64 tokens, at most 24 over the groups of a block, 10 over the blocks; the result
    roundings = 1 + 64 + run // 64 + 1 + 24 + 10 + 1
    assert abs(loss.item() - 1) <= roundings * 2.0 ** -24 * (1 + 2.0 ** -10)


class Gradients:
    """Router, its gradient, the combination and its gradient on buffers that stay."""

    def __init__(self, T, E, k, N):
        import torch
        z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")
        self.T, self.E, self.k, self.N = T, E, k, N
        self.x, self.Y, self.dout, self.dl = z(T, E), z(T * k, N, t=torch.float16), z(T, N, t=torch.float16), z(1)
        i32 = torch.int32
        self.ids, self.pos, self.rows, self.counts, self.offsets = z(T, k, t=i32), z(T, k, t=i32), z(T * k, t=i32), z(E + 1, t=i32), z(E + 1, t=i32)
        self.gates, self.loss, self.out, self.dY, self.dg, self.dx = z(T, k), z(1), z(T, N, t=torch.float16), z(T * k, N, t=torch.float16), z(T, k), z(T, E)
        self.nb = sq.sq_route_workspace_bytes(T, E)
        self.ws = z(max(256, self.nb), t=torch.uint8)

    def fill(self, seed):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (self.x, self.Y, self.dout, self.dl):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))

    def step(self):
        T, E, k, N, M = self.T, self.E, self.k, self.N, self.T * self.k
        sq.sq_route(self.x, sq.SQ_F32, T, E, E, k, 1, None, self.ids, self.gates, self.counts, self.offsets, self.rows, self.pos, self.loss, self.ws, self.nb)
        sq.sq_combine(self.Y, M, self.pos, self.gates, T, k, N, self.out)
        sq.sq_combine_backward(self.dout, self.Y, M, self.pos, self.gates, T, k, N, self.dY, self.dg)
        sq.sq_route_backward(self.x, sq.SQ_F32, T, E, E, k, 1, None, self.ids, self.gates, self.counts, self.dg, self.dl, self.dx, E)

    def results(self):
        import torch
        torch.cuda.synchronize()
        return [t.clone() for t in (self.ids, self.pos, self.rows, self.counts, self.offsets, self.gates, self.loss, self.out, self.dY, self.dg, self.dx)]


@pytest.mark.parametrize("T,E,k,N", [(5, 8, 2, 64), (700, 60, 4, 520), (10000, 40, 2, 64)])
def test_gradients_captured_and_on_two_streams_at_once(T, E, k, N):
    """Bits of a replay on other inputs, and of two of them on streams of their own at the same time, are those of calls one by one."""
    import torch
    one, want = Gradients(T, E, k, N), {}
    for seed in (1, 2, 3):
        one.fill(seed)
        one.step()
        want[seed] = one.results()
    both = [Gradients(T, E, k, N), Gradients(T, E, k, N)]
    streams, graphs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for g, s in zip(both, streams):
        g.fill(1)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            g.step()
        graphs.append(graph)
    for first, second in ((2, 3), (3, 1)):
        both[0].fill(first)
        both[1].fill(second)
        torch.cuda.synchronize()
        for _ in range(20):
            for graph, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    graph.replay()
        for g, seed in zip(both, (first, second)):
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g.results(), want[seed]))
