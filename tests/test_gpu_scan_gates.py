"""The gated scan's states where a gate is nearly shut or an operand is at the end of its type's range,
element by element against the definition in 64 bits with running bounds.

A gate's smaller side is e / (1 + e), e = exp(-|x|): the exponent's rounding is |x| U, the hardware's exp
and reciprocal, the sum and the product are a few U: eps(x) = (3 |x| + 12) U of itself, which the larger
side, 1 minus it, has too.  A state is a sum over paths of products of gates; every step adds
its gate's eps and four roundings to each path, and the joins of runs and shares 64: with M the sum of the
paths' magnitudes, B_t = a B_{t-1} + (eps + 4 U) (a M_{t-1} + k |v|), and B_t + 64 U M_t bounds the error."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from tests import ops_util as ou
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

U = ou.U


def _eps(x):
    return (3 * np.abs(x) + 12) * U


def _states(f, v, h0):
    """h [T + 1, ...] and bounds of it, from gates and candidates [T, ...] in 64 bits."""
    a, k = ou.sigmoid(f), ou.sigmoid(-f)
    h, M, B = [h0], [np.abs(h0)], [np.zeros_like(h0)]
    for t in range(len(f)):
        h.append(a[t] * h[-1] + k[t] * v[t])
        B.append(a[t] * B[-1] + (_eps(f[t]) + 4 * U) * (a[t] * M[-1] + k[t] * np.abs(v[t])))
        M.append(a[t] * M[-1] + k[t] * np.abs(v[t]))
    return np.stack(h), np.stack(B) + 64 * U * np.stack(M)


def _inputs(T, H, dtype, seed, low, high):
    """Gates in [low, high] to either side; states and candidates of sizes from 1e-3 to 1e6."""
    import torch
    g = torch.Generator().manual_seed(seed)
    et = torch.bfloat16 if dtype == "bf16" else torch.float32
    sign = lambda *s: torch.randint(0, 2, s, generator=g) * 2.0 - 1
    size = lambda *s: sign(*s) * 10 ** (torch.rand(s, generator=g) * 9 - 3)
    gate = lambda: sign(1, T, H) * (low + (high - low) * torch.rand((1, T, H), generator=g))
    z = torch.cat([gate(), size(1, T, H), gate()], 2).to(et)
    return z, torch.tensor([T], dtype=torch.int32), size(1, H), size(1, T, H).to(et), size(1, H)


def _within(name, got, want, bound, rel=0.0):
    got = got.double().cpu().numpy()
    err = np.abs(got - want)
    bound = bound + rel * (np.abs(want) + bound) + 1e-37
    assert np.isfinite(got).all(), name
    say(f"{name}: largest error {np.max(err / bound):.3g} of its bound")
    assert (err <= bound).all(), (name, np.max(err / bound))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low,high", [(0, 4), (4, 12), (12, 20), (20, 40)])
@pytest.mark.parametrize("T,H", [(1, 33), (7, 64), (40, 10), (700, 20)])
def test_states(T, H, low, high, dtype):
    z, L, h0, _, _ = _inputs(T, H, dtype, 100 * T + low, low, high)
    f, v, o = (q[0] for q in np.split(z.double().numpy(), 3, 2))
    h, bound = _states(f, v, h0[0].double().numpy())
    s = ou.sigmoid(o)
    rel = 2.0 ** -8 if dtype == "bf16" else 0.0
    with ld.GatedScan(1, H, T, dtype) as m:
        y, last = m.forward(z.cuda(), L.cuda(), h0.cuda())
        _within("y", y[0], s * h[1:], s * bound[1:] + (_eps(o) + 2 * U) * s * np.abs(h[1:]), rel)
        _within("h", last[0], h[-1], bound[-1])
        y2, last2 = m.forward_train(z.cuda(), L.cuda(), h0.cuda())
        assert (y2 == y).all() and (last2 == last).all()
        # one step after another
        x = h0.cuda()
        for t in range(min(T, 40)):
            yt, x = m.step(z[:, t].contiguous().cuda(), x)
            _within(f"step {t}", x[0], h[t + 1], bound[t + 1])
            _within(f"step {t}, y", yt[0], s[t] * h[t + 1], s[t] * bound[t + 1] + (_eps(o[t]) + 2 * U) * s[t] * np.abs(h[t + 1]), rel)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 300, 1500])
def test_infinite_states_stay(T, dtype):
    """An infinite state or candidate makes the state infinite from there on, as the definition does step
    by step (no product of gates underflows here), in its channel alone."""
    import torch
    H = 24
    g = torch.Generator().manual_seed(T)
    et = torch.bfloat16 if dtype == "bf16" else torch.float32
    z = torch.randn((2, T, 3 * H), generator=g)
    z[..., :H] = 4 + z[..., :H].abs()           # a >= 0.98
    h0 = torch.randn((2, H), generator=g)
    L = torch.tensor([T, (T + 1) // 2], dtype=torch.int32)
    inf = float("inf")
    start = {2: inf, 3: -inf, 10: inf}
    for c, x in start.items():
        h0[:, c] = x
    at = T // 3
    z[0, at, H + 5], z[0, at, H + 6] = inf, -inf
    z = z.to(et)
    dev = [t.cuda() for t in (z, L, h0)]
    plain = z.clone()
    plain[0, at, H + 5:H + 7] = 0.0
    h0p = torch.where(h0.isinf(), torch.zeros(()), h0)
    with ld.GatedScan(2, H, T, dtype) as m:
        y0, l0 = (t.cpu() for t in m.forward(plain.cuda(), L.cuda(), h0p.cuda()))
        steps, x = [], dev[2]
        for t in range(min(T, 40)):
            yt, x = m.step(dev[0][:, t].contiguous(), x)
            steps.append((yt.cpu(), x.cpu()))
        for f in (m.forward, m.forward_train):
            y, last = (t.cpu() for t in f(*dev))
            for b in range(2):
                for c, x in start.items():
                    assert (y[b, :L[b], c] == x).all() and last[b, c] == x, (b, c)
                for c, x in ((5, inf), (6, -inf)) if b == 0 else ():
                    assert (y[b, at:, c] == x).all() and last[b, c] == x
                    y[b, at:, c], last[b, c] = y0[b, at:, c], l0[b, c]
                for c in start:
                    y[b, :, c], last[b, c] = y0[b, :, c], l0[b, c]
            assert (y == y0).all() and (last == l0).all()
        for t, (yt, x) in enumerate(steps):
            for c, want in start.items():
                assert (x[:, c] == want).all() and (yt[:, c] == want).all(), (t, c)
            for c, want in ((5, inf), (6, -inf)):
                assert (x[0, c] == want) == (t >= at)


def test_operands_at_the_ends_of_the_range():
    """States and candidates of 3e38 with opposite signs: their difference has no fp32, the state has."""
    import torch
    T, H = 40, 32
    g = torch.Generator().manual_seed(1)
    f, o = torch.randn((2, 1, T, H), generator=g)
    sign = torch.randint(0, 2, (1, T + 1, H), generator=g) * 2.0 - 1
    v, h0 = 3e38 * sign[:, 1:], 3e38 * sign[:, 0]
    z = torch.cat([f, v, o], 2)
    h, bound = _states(f[0].double().numpy(), v[0].double().numpy(), h0[0].double().numpy())
    with ld.GatedScan(1, H, T, "f32") as m:
        y, last = m.forward(z.cuda(), torch.tensor([T], dtype=torch.int32).cuda(), h0.cuda())
        _within("h", last[0], h[-1], bound[-1])
        x = h0.cuda()
        for t in range(T):
            _, x = m.step(z[:, t].contiguous().cuda(), x)
            _within(f"step {t}", x[0], h[t + 1], bound[t + 1])


def _gradients(f, v, o, h, hb, dy, dh):
    """dz (its three blocks) and dh0 with their bounds, in 64 bits: the gradient carried back is bounded as
    the states are, a product by the sum of its factors' relative errors and its roundings."""
    a, k, s, s1 = ou.sigmoid(f), ou.sigmoid(-f), ou.sigmoid(o), ou.sigmoid(-o)
    e, ME, BE = dh, np.abs(dh), np.zeros_like(dh)
    dz, bounds = np.zeros((3,) + f.shape), np.zeros((3,) + f.shape)
    for t in reversed(range(len(f))):
        q = s[t] * np.abs(dy[t])
        g, MG, BG = s[t] * dy[t] + e, q + ME, BE + (_eps(o[t]) + 3 * U) * q
        B, slope = BG + 64 * U * MG, a[t] * k[t]
        d = h[t] - v[t]
        dz[:, t] = g * d * slope, g * k[t], dy[t] * h[t + 1] * s[t] * s1[t]
        bounds[:, t] = ((B + np.abs(g) * (2 * _eps(f[t]) + 8 * U)) * np.abs(d) * slope + (np.abs(g) + B) * slope * hb[t],
                        B * k[t] + np.abs(g) * k[t] * (_eps(f[t]) + 2 * U),
                        np.abs(dy[t]) * s[t] * s1[t] * (hb[t + 1] + np.abs(h[t + 1]) * (2 * _eps(o[t]) + 8 * U)))
        e, ME = a[t] * g, a[t] * MG
        BE = a[t] * (BG + MG * (_eps(f[t]) + 3 * U))
    return dz, bounds * (1 + 1e-4), e, BE + 64 * U * ME


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low,high", [(0, 4), (4, 12), (8, 20), (20, 40)])
@pytest.mark.parametrize("T,H", [(1, 33), (7, 64), (40, 10), (700, 20)])
def test_gradients(T, H, low, high, dtype):
    z, L, h0, dy, dh = _inputs(T, H, dtype, 100 * T + high, low, high)
    f, v, o = (q[0] for q in np.split(z.double().numpy(), 3, 2))
    h, hb = _states(f, v, h0[0].double().numpy())
    dz, bz, dh0, bh = _gradients(f, v, o, h, hb, dy[0].double().numpy(), dh[0].double().numpy())
    rel = 2.0 ** -8 if dtype == "bf16" else 0.0
    dev = [t.cuda() for t in (z, L, h0, dy, dh)]
    with ld.GatedScan(1, H, T, dtype) as m:
        m.forward_train(*dev[:3])
        d = m.backward(*dev)
        for i, name in enumerate(("dzf", "dzv", "dzo")):
            _within(name, d["dz"][0, :, i * H:(i + 1) * H], dz[i], bz[i], rel)
        _within("dh0", d["dh0"][0], dh0, bh)
