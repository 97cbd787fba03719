"""Linear attention where a row of the time axis is cut into shares of several chunks; the state in place, beside other work."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
import workloads
from tests.gpu_util import say, to_device
from tests.test_gpu_attend import _compare, _inputs, _lengths

pytestmark = pytest.mark.gpu


def _shares(m):
    """The shares that a handle cuts its rows into, from its workspace: two states a row, head and share behind the tables."""
    up = lambda n: (n + 255) // 256 * 256
    states = m.query(ld.ops.OPS_Q_WORKSPACE_BYTES) - 256 - up(4 * 65 * m.heads) - up(8 * m.heads)
    each = 8 * m.B * m.heads * m.Dk * m.Dv
    assert states % each == 0
    return max(1, states // each)


# rows and heads that are and are no multiple of eight, over which a row's shares lie on one chiplet or on several; shares of
# one chunk and of more; lengths that end in the first share, at the end of one and behind it
IN_PLACE = [("bf16", 1, 1, 64, 64, 2100, [2100]), ("f32", 1, 3, 16, 24, 1000, [999]), ("bf16", 3, 1, 128, 128, 700, [700, 64, 65]),
            ("bf16", 2, 4, 32, 48, 4000, [4000, 33]), ("f32", 5, 3, 50, 75, 301, [301, 0, 32, 33, 160]), ("f32", 20, 5, 16, 16, 300, None),
            ("bf16", 10, 30, 16, 16, 2500, None), ("bf16", 1, 16, 128, 128, 4200, [4200]), ("f32", 4, 2, 128, 128, 1300, [1300, 700, 1, 0])]


@pytest.mark.parametrize("dtype,B,heads,Dk,Dv,T,L", IN_PLACE)
def test_in_place_gives_the_same_bits_beside_other_work(dtype, B, heads, Dk, Dv, T, L):
    """The first share has the given state whenever it runs: also where the time loop, on a stream of its own, holds its place
    while the share that writes the state runs."""
    import torch
    say("in place", dtype, B, heads, Dk, Dv, T)
    r = np.random.default_rng(T + B)
    s = _inputs(r, dtype, B, T, heads, Dk, Dv)
    L = _lengths(L if L is not None else [int(x) for x in r.integers(0, T + 1, B)])
    side = torch.cuda.Stream()
    loop = ld.LstmDyn(40, 32, 256, 50, "bf16", "persistent")
    loop.set_option(ld.OPT_TIMEOUT_US, 500000)
    dev = to_device(workloads.random_case(9900, 40, 32, 256, 50, dtype="bf16"))
    alone = loop.forward(*dev)
    with ld.LinearAttention(B, heads, Dk, Dv, T, [0.9, 1.0, 0.99][:heads] if heads < 4 else 0.99, dtype) as m:
        assert _shares(m) > 1
        y, S = m.forward(s["z"], L, s["S0"])
        states = [s["S0"].clone() for _ in range(10)]
        torch.cuda.synchronize()
        for state in states:
            with torch.cuda.stream(side):
                h, c = loop.forward(*dev)
            y2, out = m.forward(s["z"], L, state, out_S=state)
            assert out is state
            torch.cuda.synchronize()
            assert (state == S).all() and (y2 == y).all()
            assert (h == alone[0]).all() and (c == alone[1]).all()
        assert m.status() == ld.OK and loop.query(ld.Q_LAST_STATUS) == ld.OK
    loop.close()


# Shares of several chunks each: states carried from chunk to chunk behind a row's first share, additions that several
# chunks form, decays over whole shares of several chunks; lengths inside, at and just past a share of `span` steps.
SEVERAL = [("f32", 20, 5, 16, 16, 300, 128), ("f32", 7, 16, 24, 9, 300, 128), ("f32", 2, 16, 128, 128, 700, 96),
           ("bf16", 10, 30, 16, 16, 2500, 1024), ("bf16", 2, 16, 128, 128, 1100, 128), ("bf16", 2, 16, 128, 100, 1100, 128),
           ("bf16", 5, 30, 20, 33, 1400, 256)]


@pytest.mark.parametrize("dtype,B,heads,Dk,Dv,T,span", SEVERAL)
def test_shares_of_several_chunks(dtype, B, heads, Dk, Dv, T, span):
    say("several", dtype, B, heads, Dk, Dv, T)
    r = np.random.default_rng(T + B)
    last = (T - 1) // span * span
    L = [T, last + 1, span, span + 1, 0, last, span - 1, 1, 2 * span, T - 1, *(int(x) for x in r.integers(0, T + 1, 10))][:B]
    decay = [0.9, 1.0, 0.0, 0.999, 0.99, 0.5] * 5
    s = _inputs(r, dtype, B, T, heads, Dk, Dv)
    with ld.LinearAttention(B, heads, Dk, Dv, T, decay[:heads], dtype) as m:
        assert _shares(m) == (T - 1) // span + 1 > 1          # and a share is several chunks of 32 or 64 steps
        assert span > (64 if dtype == "bf16" else 32)
        y, S = m.forward(s["z"], _lengths(L), s["S0"])
        got = m.backward(s["z"], _lengths(L), s["S0"], s["dy"], s["dS"])
        _compare(dict(got, y=y, S=S), s, L, decay[:heads], Dk, Dv, dtype)
        assert m.status() == ld.OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_state_that_replays_carry_on(dtype):
    """A captured call whose result lies in its given state, over several shares: every replay goes on from the one before, with
    eager calls of the same handle between."""
    import torch
    B, heads, Dk, Dv, T = 3, 2, 48, 64, 900
    r = np.random.default_rng(3)
    s = _inputs(r, dtype, B, T, heads, Dk, Dv)
    L = _lengths([900, 70, 0])
    with ld.LinearAttention(B, heads, Dk, Dv, T, [0.99, 1.0], dtype) as m:
        assert _shares(m) > 1
        state = s["S0"].clone()
        y = torch.empty((B, T, heads * Dv), dtype=s["z"].dtype, device="cuda")
        m.forward(s["z"], L, s["S0"])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.forward(s["z"], L, state, out_S=state, out_y=y)
        want = s["S0"]
        for i in range(4):
            s["z"].mul_(-0.75)
            want_y, want = m.forward(s["z"], L, want)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert (state == want).all() and (y == want_y).all(), i
        del graph
