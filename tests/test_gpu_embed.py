"""The token table's rows and its gradient against their definitions: sizes around the sort's and the
sums' pieces, one token for everything, every token once, tokens out of range, lengths, streams, replay."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from paper_1810_08061_amd import ops
from tests import ops_util as ou
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def _tokens(kind, g, B, T, V):
    import torch
    if kind == "same":
        return torch.full((B, T), V // 2, dtype=torch.int32)
    if kind == "distinct":
        return (torch.randperm(max(V, B * T), generator=g)[:B * T] % V).int().reshape(B, T)
    if kind == "skewed":
        return (V ** torch.rand((B, T), generator=g, dtype=torch.float64) - 1).int().clamp(0, V - 1)
    return torch.randint(0, V, (B, T), generator=g, dtype=torch.int32)


def _check(B, T, V, D, dtype, grad, kind, lengths=None, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed + B + T + V + D)
    et, gt = (torch.bfloat16 if d == "bf16" else torch.float32 for d in (dtype, grad))
    tok, scale = _tokens(kind, g, B, T, V), 1.75
    table, dx = torch.randn((V, D), generator=g).to(et), torch.randn((B, T, D), generator=g).to(gt)
    if lengths is None:
        L = torch.randint(0, T + 1, (B,), generator=g).int()
        L[0] = T
    elif lengths == "full":
        L = None
    else:
        L = torch.tensor(lengths, dtype=torch.int32)
    Ln = np.full(B, T) if L is None else L.numpy()
    want, mag, cnt = ou.embed_grad(tok.numpy(), Ln, dx.double().numpy(), V, scale)
    on = torch.arange(T)[None, :] < torch.as_tensor(Ln)[:, None]
    x = torch.where(on[..., None], (table[tok.long()].float() * scale).to(et), torch.zeros((), dtype=et))
    tok[~on], dx[~on] = -7, float("nan")
    tok, table, dx = tok.cuda(), table.cuda(), dx.cuda()
    L = None if L is None else L.cuda()
    with ld.TokenEmbed(B, T, V, D, dtype, scale=scale) as m:
        assert (m.forward(tok, L, table).cpu() == x).all()          # one product, rounded once: exact
        out = torch.full((V, D), float("nan"), device="cuda")
        got = m.backward(tok, L, dx, out=out)
        err = np.abs(got.double().cpu().numpy() - want)
        bound = (cnt[:, None] + 2) * ou.U * mag                      # a sum's roundings, and the scale's
        say(f"d_table: max error {err.max():.3g}, largest bound {bound.max():.3g}")
        assert (err <= bound).all()
        assert (m.backward(tok, L, dx) == got).all()                 # the same bits again
        assert m.status() == ld.OK


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("B,T,V,D,kind", [
    (1, 1, 1, 1, "any"), (1, 1, 100, 64, "any"), (2, 3, 5, 7, "any"), (3, 21, 1000, 33, "skewed"),
    (1, 63, 4, 130, "any"), (1, 64, 3, 256, "any"), (1, 65, 2, 258, "same"), (4, 500, 511, 20, "skewed"),
    (4, 512, 512, 12, "skewed"), (5, 700, 600, 40, "same"), (2, 1025, 70000, 16, "distinct"),
    (7, 1400, 300, 9, "any"), (3, 3000, 40000, 8, "skewed")])
def test_embed(B, T, V, D, dtype, grad, kind):
    _check(B, T, V, D, dtype, grad, kind)


@pytest.mark.parametrize("lengths", ["full", [0, 0, 0], [0, 130, 1], [130, 130, 130]])
def test_lengths(lengths):
    _check(3, 130, 50, 24, "bf16", "f32", "any", lengths)


def test_large_vocabulary():
    _check(2, 40, 300000, 4, "f32", "f32", "any")      # three digits of the sort


def test_tokens_and_lengths_out_of_range():
    import torch
    B, T, V, D = 2, 70, 30, 20
    g = torch.Generator().manual_seed(4)
    tok = torch.randint(0, V, (B, T), generator=g, dtype=torch.int32)
    table, dx = torch.randn((V, D), generator=g).cuda(), torch.randn((B, T, D), generator=g).cuda()
    L = torch.tensor([T, T], dtype=torch.int32).cuda()
    bad = tok.clone()
    bad[0, 3], bad[0, 69], bad[1, 0], bad[1, 8] = V, -1, 2 ** 31 - 1, -2 ** 31
    masked = dx.clone()
    masked[(bad != tok).cuda()] = 0
    with ld.TokenEmbed(B, T, V, D, "f32", scale=0.5) as m:
        x, want = m.forward(tok.cuda(), L, table), m.backward(tok.cuda(), L, masked)
        assert m.status() == ld.OK
        xb = m.forward(bad.cuda(), L, table)
        assert m.status() == ops.ERR_BAD_TOKENS and m.status() == ld.OK
        diff = (bad != tok).cuda()
        assert (xb[diff] == 0).all() and (xb[~diff] == x[~diff]).all()
        got = m.backward(bad.cuda(), L, dx)
        assert m.status() == ops.ERR_BAD_TOKENS
        assert torch.allclose(got, want, rtol=0, atol=140 * ou.U * 8)   # the sums' pieces differ
        m.forward(tok.cuda(), L + 1, table)
        assert m.status() == ld.ERR_BAD_LENGTHS
        with pytest.raises(TypeError):
            m.forward(tok.long().cuda(), L, table)
        with pytest.raises(ValueError):
            m.forward(tok.cuda(), L, table[:-1])
        with pytest.raises(TypeError):
            m.backward(tok.cuda(), L, dx.double())


def test_gradient_against_differences():
    """The lookup is linear in the table: differences are exact up to rounding."""
    import torch
    B, T, V, D = 3, 90, 17, 12
    g = torch.Generator().manual_seed(6)
    tok = torch.randint(0, V, (B, T), generator=g, dtype=torch.int32).cuda()
    L = torch.tensor([90, 31, 0], dtype=torch.int32).cuda()
    table, v, dx = (torch.randn(s, generator=g).cuda() for s in ((V, D), (V, D), (B, T, D)))
    with ld.TokenEmbed(B, T, V, D, "f32", scale=3.0) as m:
        loss = lambda t: float((m.forward(tok, L, t).double() * dx.double()).sum())
        want = float((m.backward(tok, L, dx).double() * v).sum())
        got = (loss(table + v) - loss(table - v)) / 2
        size = float((m.forward(tok, L, table.abs() + v.abs()) * dx.abs()).sum())
        assert abs(got - want) <= 8 * ou.U * size


def test_graph_replay_and_streams():
    import torch
    B, T, V, D = 4, 600, 900, 36
    g = torch.Generator().manual_seed(8)
    toks = [torch.randint(0, V, (B, T), generator=g, dtype=torch.int32).cuda() for _ in range(4)]
    dx = torch.randn((B, T, D), generator=g).cuda()
    L = torch.tensor([600, 599, 1, 0], dtype=torch.int32).cuda()
    with ld.TokenEmbed(B, T, V, D, "f32") as m, ld.TokenEmbed(B, T, V, D, "f32") as m2:
        m.backward(toks[0], L, dx)
        t, out = toks[0].clone(), torch.empty((V, D), device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.backward(t, L, dx, out=out)
        s = torch.cuda.Stream()
        for i in range(4):
            t.copy_(toks[i])
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                want = m2.backward(t, L, dx)
            s.synchronize()
            assert (out == want).all(), i
