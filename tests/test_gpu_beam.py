"""One step of a beam search against all candidates in 64 bits: exact ties, masked and infinite logits,
finished and dead beams, fewer tokens than beams, states of any type; the kernels' choices."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from paper_1810_08061_amd import ops
from tests import ops_util as ou
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def _step(m, logits, scores, finished, states=()):
    out = m.step(logits.cuda(), scores.cuda(), finished.cuda(), [s.cuda() for s in states])
    return [t.cpu() for t in out[:4]] + [[s.cpu() for s in out[4]]]


def _check(m, logits, scores, finished, end, states=(), exact=False):
    """Scores within rounding of the 64-bit ones; the choice is the best K's unless candidates are
    nearer than rounding; with `exact` the very order, ties to the lowest index."""
    B, K, V = logits.shape
    got, parent, token, done, out = _step(m, logits, scores, finished, states)
    x, s, f = logits.double().numpy(), scores.double().numpy(), finished.numpy()
    for b in range(B):
        c = ou.beam(x[b], s[b], f[b], end).reshape(-1)
        order = np.argsort(-c, kind="stable")[:K]
        best = c[order]
        fin = np.isfinite(best)
        # the sum of exps and its log 2e-6 (a few times the logarithm's own size), x - lse, and the score's sum
        size = np.abs(s[b][np.isfinite(s[b])]).max(initial=0) + np.abs(best[fin]).max(initial=0)
        tol = 4e-6 + 4 * ou.U * (size + np.abs(x[b][np.isfinite(x[b])]).max(initial=0) + 12)
        at = parent[b].long().numpy() * V + token[b].long().numpy()
        assert ((parent[b] >= 0) & (parent[b] < K) & (token[b] >= 0) & (token[b] < V)).all()
        assert len(set(at.tolist())) == K
        g = got[b].double().numpy()
        assert np.array_equal(np.isfinite(g), fin) and (g[~fin] == -np.inf).all()
        assert (np.abs(g[fin] - best[fin]) <= tol).all() and (np.abs(g[fin] - c[at][fin]) <= tol).all(), b
        assert (np.diff(g[fin]) <= 0).all()
        if exact:
            assert (at == order).all(), (b, at, order)
        assert (done[b].bool().numpy() == ((f[b][parent[b]] != 0) | (token[b].numpy() == end))).all()
        for src, dst in zip(states, out):
            assert (dst[b] == src[b][parent[b].long()]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,V", [
    (1, 1, 1), (1, 1, 2), (2, 3, 3), (1, 4, 63), (3, 2, 64), (1, 5, 65), (2, 8, 1000), (1, 32, 40), (2, 32, 33),
    (1, 3, 255), (1, 16, 4096), (2, 7, 4097), (1, 4, 8193), (1, 2, 50001), (1, 32, 20000), (40, 4, 300),
    (3, 8, 32768), (300, 2, 70)])
def test_beam(B, K, V, dtype):
    import torch
    g = torch.Generator().manual_seed(B + 10 * K + V)
    et = torch.bfloat16 if dtype == "bf16" else torch.float32
    logits = (torch.randn((B, K, V), generator=g) * 3).to(et)
    scores = -5 + torch.randn((B, K), generator=g)
    finished = (torch.rand((B, K), generator=g) < 0.2).to(torch.uint8)
    end = V // 3
    h, c = torch.randn((B, K, 5), generator=g), torch.randn((B, K, 3, 4), generator=g).bfloat16()
    with ld.BeamSearch(B, K, V, dtype, end=end) as m:
        _check(m, logits, scores, finished, end, (h, c))
        assert m.status() == ld.OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,K", [(5, 3), (64, 8), (700, 32), (5000, 16), (40000, 8)])
def test_exact_ties(V, K, dtype):
    """Beams with the same logits in another order and the same score: candidates that are equal to the
    last bit, taken by the lowest index; also where all are equal."""
    import torch
    g = torch.Generator().manual_seed(V)
    et = torch.bfloat16 if dtype == "bf16" else torch.float32
    base = torch.randint(-2, 3, (V,), generator=g).float()
    for logits in (torch.stack([base[torch.randperm(V, generator=g)] for _ in range(K)]),
                   torch.stack([base] * K), torch.zeros((K, V))):
        scores, finished = torch.full((1, K), -3.0), torch.zeros((1, K), dtype=torch.uint8)
        logits = logits[None].to(et)
        with ld.BeamSearch(1, K, V, dtype) as m:
            got, parent, token, _, _ = _step(m, logits, scores, finished)
            flat = logits[0].float().reshape(-1)
            order = torch.sort(flat, descending=True, stable=True).indices[:K]
            # the beams' sums of exps may differ in their last bits where the order of their terms does
            at = parent[0].long() * V + token[0].long()
            if (logits[0] == logits[0, :1]).all():
                assert (at == order).all()
            assert (flat[at] == flat[order]).all()
            for k in range(K):      # within a beam always the lowest tokens
                mine = token[0][parent[0] == k].tolist()
                for t in mine:
                    lower = [j for j in (logits[0, k, :t] == logits[0, k, t]).nonzero().flatten().tolist()]
                    assert all(j in mine for j in lower)


def test_negative_zeros_are_zeros():
    import torch
    V, K = 3000, 8
    g = torch.Generator().manual_seed(1)
    logits = torch.where(torch.rand((1, K, V), generator=g) < 0.5, 0.0, -0.0)
    for et in ("f32", "bf16"):
        with ld.BeamSearch(1, K, V, et) as m:
            x = logits if et == "f32" else logits.bfloat16()
            got, parent, token, _, _ = _step(m, x, torch.zeros((1, K)), torch.zeros((1, K), dtype=torch.uint8))
            assert (parent == 0).all() and token[0].tolist() == list(range(K))


def test_masked_infinite_and_nan_logits():
    import torch
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    V, K = 600, 4
    g = torch.Generator().manual_seed(5)
    logits = torch.randn((6, K, V), generator=g)
    logits[0, 0] = -inf                              # nothing left in a beam
    logits[0, 2, 5:] = -inf                          # fewer tokens than beams
    logits[0, 2, :5] = 1.0
    logits[1, :, ::2] = nan
    logits[2, 1] = low                               # masks of the type's lowest value: all equal
    logits[2, 2, 1:] = low
    logits[3] = -inf                                 # nothing left at all
    logits[4, 0, 7] = inf                            # no candidate of this beam is a number
    logits[5, :, 3:] = -inf
    scores = torch.tensor([[-1.0, -2.0, -1.5, -3.0]]).repeat(6, 1)
    finished = torch.zeros((6, K), dtype=torch.uint8)
    with ld.BeamSearch(6, K, V, "f32", end=2) as m:
        _check(m, logits, scores, finished, 2)
        got, parent, token, done, _ = _step(m, logits, scores, finished)
        assert (got[3] == -inf).all() and (parent[3] == 0).all() and token[3].tolist() == [0, 1, 2, 3]
        assert done[3].tolist() == [0, 0, 1, 0]


def test_finished_and_dead_beams():
    import torch
    inf = float("inf")
    V, K, end = 50, 4, 9
    g = torch.Generator().manual_seed(6)
    logits = torch.randn((5, K, V), generator=g)
    logits[:, 1] = float("nan")                      # a finished beam's logits are not looked at
    scores = torch.tensor([[0.0, -1.0, -2.0, -30.0]]).repeat(5, 1)
    finished = torch.tensor([[0, 1, 0, 0]] * 5).to(torch.uint8)
    finished[1] = 1                                  # all finished: each goes on as itself
    finished[2] = torch.tensor([255, 7, 0, 1])       # any value but zero
    scores[3] = torch.tensor([0.0, -inf, -inf, -inf])    # the first step: one live beam
    scores[4] = torch.tensor([-inf] * 4)
    finished[4] = 0
    logits[4] = torch.randn((K, V), generator=g)
    with ld.BeamSearch(5, K, V, "f32", end=end) as m:
        _check(m, logits, scores, finished, end)
        got, parent, token, done, _ = _step(m, logits, scores, finished)
        assert parent[1].tolist() == [0, 1, 2, 3] and token[1].tolist() == [end] * 4
        assert (got[1] == scores[1]).all() and done[1].all()
        assert (parent[3] == 0).all()
        assert parent[4].tolist() == [0] * 4 and token[4].tolist() == [0, 1, 2, 3]
    with ld.BeamSearch(5, K, V, "f32") as m:         # no end token: a finished beam has no way on
        _check(m, logits, scores, finished, -1)
        assert (_step(m, logits, scores, finished)[0][1] == -inf).all()


def test_fewer_candidates_than_beams_in_a_beam():
    import torch
    g = torch.Generator().manual_seed(8)
    for K, V in ((5, 1), (8, 2), (32, 3)):
        logits = torch.randn((2, K, V), generator=g)
        scores = torch.randn((2, K), generator=g)
        finished = torch.zeros((2, K), dtype=torch.uint8)
        finished[1, ::2] = 1
        with ld.BeamSearch(2, K, V, "f32", end=0) as m:
            _check(m, logits, scores, finished, 0)


@pytest.mark.parametrize("shape,dt", [((1,), "uint8"), ((3,), "uint8"), ((16,), "uint8"), ((5,), "bfloat16"),
                                      ((7,), "float32"), ((8,), "float32"), ((3, 5, 4), "float32"), ((1000,), "float64")])
def test_states(shape, dt):
    import torch
    B, K, V = 3, 5, 40
    g = torch.Generator().manual_seed(9)
    logits, scores = torch.randn((B, K, V), generator=g), torch.randn((B, K), generator=g)
    s = torch.randint(0, 200, (B, K, *shape), generator=g).to(getattr(torch, dt))
    with ld.BeamSearch(B, K, V, "f32") as m:
        _check(m, logits, scores, torch.zeros((B, K), dtype=torch.uint8), -1, [s] * 8)
        _check(m, logits, scores, torch.zeros((B, K), dtype=torch.uint8), -1)
        with pytest.raises(ValueError):
            _step(m, logits, scores, torch.zeros((B, K), dtype=torch.uint8), [s] * 9)
        with pytest.raises(ValueError):
            _step(m, logits, scores, torch.zeros((B, K), dtype=torch.uint8), [s[:2]])
        c = s.cuda()
        with pytest.raises(ld.LstmDynError):         # in place
            m.step(logits.cuda(), scores.cuda(), torch.zeros((B, K), dtype=torch.uint8).cuda(), [c], [c])
        with pytest.raises(TypeError):
            m.step(logits.cuda(), scores.cuda(), torch.zeros((B, K), dtype=torch.bool).cuda())


def test_graph_replay_and_streams():
    import torch
    B, K, V = 3, 6, 9000
    g = torch.Generator().manual_seed(10)
    logits = [torch.randn((B, K, V), generator=g).bfloat16().cuda() for _ in range(4)]
    scores, fin = torch.randn((B, K), generator=g).cuda(), torch.zeros((B, K), dtype=torch.uint8).cuda()
    h = torch.randn((B, K, 64), generator=g).cuda()
    with ld.BeamSearch(B, K, V, "bf16", end=1) as m, ld.BeamSearch(B, K, V, "bf16", end=1) as m2:
        x = logits[0].clone()
        m.step(x, scores, fin, [h])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = m.step(x, scores, fin, [h])
        s = torch.cuda.Stream()
        for i in range(4):
            x.copy_(logits[i])
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                want = m2.step(x, scores, fin, [h])
            s.synchronize()
            assert all((a == b).all() for a, b in zip(out[:4], want[:4])) and (out[4][0] == want[4][0]).all(), i
