"""Layer norm on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from tests import layer_util
from tests.layer_util import HALF, U

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _dev(a, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _np(t):
    return t.detach().double().cpu().numpy()


def _lengths(L):
    import torch
    return torch.tensor(L, dtype=torch.int32, device="cuda")


def _check(got, want, bound, dtype):
    for k, g in got.items():
        rounding = HALF[dtype[k]] if k in dtype else 0.0
        g = _np(g)
        assert np.isfinite(g).all(), k
        over = np.abs(g - want[k]) - (bound[k] * (1 + rounding) + rounding * np.abs(want[k]) + 1e-37)
        assert (over <= 0).all(), (k, over.max())


# one vector, where a wave's, four waves' and sixteen waves' elements end, odd sizes
WIDTHS = [1, 2, 7, 64, 255, 256, 257, 333, 512, 513, 1000, 1024, 1025, 1032, 2048, 2056, 4096, 4097, 4104, 8192, 8200, 16383, 16384, 16392, 32767, 32768]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_forward_and_backward(dtype, grad, D):
    r = np.random.default_rng(D)
    L = [3, 0, 2] if D > 4096 else [9, 0, 1, 5]
    B, T = len(L), L[0]
    x = _dev(r.standard_normal((B, T, D)) * 2 + r.standard_normal((B, T, 1)), dtype)
    dy = _dev(r.standard_normal((B, T, D)), grad)
    w, b = _dev(1 + 0.3 * r.standard_normal(D)), _dev(r.standard_normal(D))
    want, bound = layer_util.norm(_np(x), L, _np(w), _np(b), EPS, _np(dy))
    with ld.LayerNorm(B, T, D, dtype, eps=EPS) as m:
        got = dict(m.backward(x, _lengths(L), w, dy), y=m.forward(x, _lengths(L), w, b))
        _check(got, want, bound, {"y": dtype, "dx": grad})
        for i, n in enumerate(L):
            assert (got["y"][i, n:] == 0).all() and (got["dx"][i, n:] == 0).all()
        assert m.status() == ld.OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 15, 16, 17, 4097, 20000])
def test_numbers_of_rows(dtype, rows):
    """From one row to more than the workgroups hold at once: each gets its own, and the sums all of them."""
    r = np.random.default_rng(rows)
    D = 40
    x, dy = _dev(r.standard_normal((1, rows, D)), dtype), _dev(r.standard_normal((1, rows, D)), dtype)
    w = _dev(r.standard_normal(D))
    want, bound = layer_util.norm(_np(x), [rows], _np(w), None, EPS, _np(dy))
    with ld.LayerNorm(1, rows, D, dtype, eps=EPS) as m:
        _check(dict(m.backward(x, None, w, dy), y=m.forward(x, None, w)), want, bound, {"y": dtype, "dx": dtype})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_optional_arguments(dtype):
    import torch
    r = np.random.default_rng(3)
    B, T, D = 2, 4, 96
    x, dy = _dev(r.standard_normal((B, T, D)), dtype), _dev(r.standard_normal((B, T, D)), dtype)
    one, zero = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    with ld.LayerNorm(B, T, D, dtype) as m:
        full = _lengths([T, T])
        assert (m.forward(x) == m.forward(x, full, one, zero)).all()
        a, b = m.backward(x, None, None, dy), m.backward(x, full, one, dy)
        assert all((a[k] == b[k]).all() for k in a)
        want = m.forward(x, None, one, zero)
        there = x.clone()                       # in place
        assert (m.forward(there, None, one, zero, out_y=there) == want).all()
        g = dy.clone()
        out = {"dx": g, "dweight": torch.empty_like(one), "dbias": torch.empty_like(one)}
        m.backward(x, None, None, g, out=out)
        assert all((a[k] == out[k]).all() for k in a)


@pytest.mark.parametrize("D", [96, 5000, 20000])
def test_in_place_over_waves(D):
    r = np.random.default_rng(D)
    x = _dev(r.standard_normal((1, 7, D)))
    with ld.LayerNorm(1, 7, D, "f32") as m:
        want = m.forward(x)
        assert (m.forward(x, out_y=x) == want).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [100.0, 30000.0])
def test_rows_far_from_zero(dtype, offset):
    """The deviations are formed from the mean, so a large one costs only the rounding of x itself."""
    r = np.random.default_rng(4)
    x = _dev(r.standard_normal((1, 6, 500)) + offset, dtype)
    dy, w = _dev(r.standard_normal((1, 6, 500)), dtype), _dev(r.standard_normal(500))
    want, bound = layer_util.norm(_np(x), [6], _np(w), None, EPS, _np(dy))
    with ld.LayerNorm(1, 6, 500, dtype, eps=EPS) as m:
        _check(dict(m.backward(x, None, w, dy), y=m.forward(x, None, w)), want, bound, {"y": dtype, "dx": dtype})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_deviation(dtype):
    r = np.random.default_rng(5)
    x = _dev(np.full((1, 3, 64), 0.5), dtype)
    b, dy = _dev(r.standard_normal(64)), _dev(r.standard_normal((1, 3, 64)), dtype)
    with ld.LayerNorm(1, 3, 64, dtype, eps=EPS) as m:
        assert (m.forward(x, None, None, b) == b.to(x.dtype)).all()
        got = m.backward(x, None, None, dy)
        assert (got["dweight"] == 0).all() and got["dx"].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 3000])
def test_nothing_behind_a_sequence_counts(dtype, D):
    r = np.random.default_rng(6)
    L, T = [5, 2, 0], 5
    x, dy, w, b = _dev(r.standard_normal((3, T, D)), dtype), _dev(r.standard_normal((3, T, D)), dtype), _dev(r.standard_normal(D)), _dev(r.standard_normal(D))
    with ld.LayerNorm(3, T, D, dtype) as m:
        both = lambda: dict(m.backward(x, _lengths(L), w, dy), y=m.forward(x, _lengths(L), w, b))
        want = both()
        for bad in (float("nan"), float("inf")):
            for i, n in enumerate(L):
                x[i, n:] = bad
                dy[i, n:] = bad
            got = both()
            assert all((got[k] == want[k]).all() for k in want)


def test_a_bad_row_is_its_own():
    """NaN and infinity in a row make that row, and the sums over rows, not numbers."""
    r = np.random.default_rng(7)
    x = _dev(r.standard_normal((1, 9, 70)))
    with ld.LayerNorm(1, 9, 70, "f32") as m:
        want = m.forward(x)
        x[0, 2, 3], x[0, 5, 69] = float("nan"), float("inf")
        got = m.forward(x)
        keep = [i for i in range(9) if i not in (2, 5)]
        assert (got[0, keep] == want[0, keep]).all() and got[0, [2, 5]].isnan().all()


def test_bad_lengths_are_clamped_and_reported():
    r = np.random.default_rng(8)
    x = _dev(r.standard_normal((3, 6, 30)))
    with ld.LayerNorm(3, 6, 30, "f32") as m:
        want = m.forward(x, _lengths([6, 0, 4]))
        assert m.status() == ld.OK
        assert (m.forward(x, _lengths([7, -1, 4])) == want).all()
        assert m.status() == ld.ERR_BAD_LENGTHS and m.status() == ld.OK


def test_gradients_against_differences():
    r = np.random.default_rng(9)
    B, T, D, L, h = 2, 3, 20, [3, 2], 1e-2
    x, dy, w, b = _dev(r.standard_normal((B, T, D))), _dev(r.standard_normal((B, T, D))), _dev(r.standard_normal(D)), _dev(r.standard_normal(D))
    with ld.LayerNorm(B, T, D, "f32", eps=1e-3) as m:
        loss = lambda: float((_np(m.forward(x, _lengths(L), w, b)) * _np(dy)).sum())
        got = m.backward(x, _lengths(L), w, dy)
        for t, g in ((x, got["dx"]), (w, got["dweight"]), (b, got["dbias"])):
            for _ in range(10):
                i = tuple(int(r.integers(0, n)) for n in t.shape)
                old = float(t[i])
                values, at = [], []
                for s in (h, -h):
                    t[i] = old + s
                    at.append(float(t[i]))
                    values.append(loss())
                t[i] = old
                slope = (values[0] - values[1]) / (at[0] - at[1])
                # h^2 / 6 times a third derivative of some tens; rounding of 60 terms over h
                assert abs(slope - float(g[i])) <= 1e-4 * 50 + 60 * 4 * U * 3 / h, i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_call_same_bits_and_replays(dtype):
    import torch
    r = np.random.default_rng(10)
    B, T, D = 40, 50, 200
    L = _lengths([int(n) for n in r.integers(0, T + 1, B)])
    x, dy, w, b = _dev(r.standard_normal((B, T, D)), dtype), _dev(r.standard_normal((B, T, D)), dtype), _dev(r.standard_normal(D)), _dev(r.standard_normal(D))
    m, other = ld.LayerNorm(B, T, D, dtype), ld.LayerNorm(B, T, D, dtype)
    both = lambda m: dict(m.backward(x, L, w, dy), y=m.forward(x, L, w, b))
    both(m)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(m)
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        dy.copy_(torch.randn(x.shape, device="cuda"))
        want, again = both(other), both(other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all((out[k] == want[k]).all() and (again[k] == want[k]).all() for k in want), i
    del graph
    m.close(), other.close()


@pytest.mark.parametrize("D,dtype", [(4096, "bf16"), (4097, "bf16"), (4104, "f32"), (40, "f32"), (41, "bf16")])
@pytest.mark.parametrize("rows", [1, 5, 1023, 5000])
def test_sums_stay_in_the_workspace(D, dtype, rows):
    """The workgroups' sums for every number of rows and shape of a row: as many as the handle made room for, and the
    same as over the rows one by one (of ones and signs, whose sums are exact)."""
    import torch
    x = torch.ones((1, rows, D), device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    x[..., ::2] = -1
    with ld.LayerNorm(1, rows, D, dtype, eps=0.0) as m:
        got = m.backward(x, None, None, torch.ones_like(x))
        room = m.query(ld.ops.OPS_Q_WORKSPACE_BYTES)
    assert (got["dbias"] == rows).all()
    assert room <= 256 + 8 * D * min((rows + 3) // 4, 1024)
    if D % 2 == 0:
        assert (got["dweight"][::2] == -rows).all() and (got["dweight"][1::2] == rows).all()
