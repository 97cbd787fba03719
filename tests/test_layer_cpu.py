"""The C ABI of the layer's operators without a GPU: every declared function is exported, and bad arguments are
refused by the checks each call makes first; the definitions that the GPU tests use, against differences."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_1810_08061_amd as ld
from paper_1810_08061_amd import layer, ops
from tests import layer_util
from tests.test_ops_cpu import _place, _refusals

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED = ld.OK, ld.ERR_INVALID, ld.ERR_UNSUPPORTED
TYPES = [(ld.F32, 4), (ld.BF16, 2)]


def test_library_exports_every_declared_operator():
    with open(os.path.join(ROOT, "include", "lstm_dyn_layer.h")) as f:
        names = re.findall(r"^int\s+(lstm_dyn_\w+)\s*\(", f.read(), re.M)
    assert len(names) == 25
    lib = ctypes.CDLL(ld.library_path())
    for n in names:
        assert hasattr(lib, n) and hasattr(layer, n), n


@pytest.mark.parametrize("dtype,e", TYPES)
def test_norm_refusals(dtype, e):
    B, T, D = 3, 5, 24
    n = B * T * D
    sizes = [n * e, 4 * B, 4 * D, 4 * D, n * e]
    chk = lambda *q: ops._lib().lstm_dyn_check_norm_args(B, T, D, dtype, 1e-5, *q, 0, 0, 0, 0, 0)
    p = _place(sizes)
    _refusals(chk, p, sizes, (4,), optional=(1, 2, 3), same={(4, 0)})
    for dy, ge in TYPES:
        sizes = [n * e, 4 * B, 4 * D, n * ge, n * ge, 4 * D, 4 * D]
        chk = lambda x, L, w, d, dx, dw, db: layer.lstm_dyn_check_norm_args(B, T, D, dtype, 1e-5, x, L, w, 0, 0, d, dy, dx, dw, db)
        p = _place(sizes)
        _refusals(chk, p, sizes, (4, 5, 6), optional=(1, 2), same={(4, 3)})
        for i in (0, 3, 4):
            q = list(p)
            q[i] += 8
            assert chk(*q) == INVALID
    big = 1 << 40
    full = lambda B, T, D, dtype, eps: layer.lstm_dyn_check_norm_args(B, T, D, dtype, eps, big, 0, 0, 0, 2 * big, 0, 0, 0, 0, 0)
    assert full(1, 1, 32768, dtype, 0.0) == OK
    for bad in ((0, 1, 1, dtype, 0.0), (1, 0, 1, dtype, 0.0), (1, 1, 0, dtype, 0.0), (1, 1, 1, 7, 0.0), (1, 1, 1, dtype, -1.0),
                (1, 1, 1, dtype, float("nan")), (1, 1, 1, dtype, float("inf"))):
        assert full(*bad) == INVALID, bad
    assert full(1, 1, 32769, dtype, 0.0) == UNSUPPORTED and full(1 << 16, 1 << 15, 1, dtype, 0.0) == UNSUPPORTED


@pytest.mark.parametrize("dtype,e", TYPES)
def test_clip_refusals(dtype, e):
    n = [100, 0, 7]
    g, out, result = [1 << 20, 0, 1 << 21], [1 << 22, 0, 1 << 23], 1 << 24
    chk = lambda g=g, result=result, out=out: layer.lstm_dyn_check_clip_args(n, g, dtype, result, out)
    assert chk() == OK and chk(out=None) == OK and chk(out=g) == OK
    assert layer.lstm_dyn_check_clip_args(n) == OK
    assert chk(g=[0, 0, g[2]]) == INVALID and chk(out=[out[0], 0, 0]) == INVALID and chk(result=0) == INVALID
    assert chk(g=[g[0] + e // 2, 0, g[2]]) == INVALID and chk(result=result + 2) == INVALID
    assert chk(result=g[0] + 16) == INVALID and chk(result=out[2]) == INVALID       # on a gradient, on an output
    assert chk(out=[g[2], 0, out[2]]) == INVALID          # on another gradient
    assert chk(out=[out[0], 0, out[0] + 50 * e]) == INVALID and chk(out=[g[0] + 50 * e, 0, out[2]]) == INVALID
    assert chk(g=[g[0], 0, g[0]], out=None) == OK         # one gradient twice is read twice
    assert chk(g=[g[0], 0, g[0]], out=[g[0], 0, out[2]]) == INVALID   # but not while it is written
    assert layer.lstm_dyn_check_clip_args([]) == INVALID and layer.lstm_dyn_check_clip_args([-1]) == INVALID
    assert layer.lstm_dyn_check_clip_args([1 << 36]) == UNSUPPORTED and layer.lstm_dyn_check_clip_args([1 << 40]) == UNSUPPORTED
    assert layer.lstm_dyn_check_clip_args([1 << 35]) == OK
    assert layer.lstm_dyn_check_clip_args(n, g, 5, result, out) == INVALID


@pytest.mark.parametrize("dtype,e", TYPES)
def test_sample_refusals(dtype, e):
    N, V = 8, 33
    sizes = [N * V * e, 4 * N, 4 * N, 4 * N]
    p = _place(sizes)
    chk = lambda x, u, t, l: layer.lstm_dyn_check_sample_args(N, V, dtype, x, u, None, t, l)
    _refusals(chk, p, sizes, (2, 3))
    assert chk(p[0] + e, *p[1:]) == OK and chk(p[0] + e // 2, *p[1:]) == INVALID
    f = layer.SampleFilter()
    full = lambda: layer.lstm_dyn_check_sample_args(N, V, dtype, p[0], p[1], ctypes.byref(f), p[2], p[3])
    for name in ("temperatures", "top_ps", "min_ps", "top_ks"):
        setattr(f, name, 1 << 30)
        assert full() == OK
        for bad in ((1 << 30) + 2, p[2], p[3]):      # misaligned, on an output
            setattr(f, name, bad)
            assert full() == INVALID, (name, bad)
        setattr(f, name, p[1])                       # inputs may be the same
        assert full() == OK
        setattr(f, name, None)
    args = lambda N, V, d: layer.lstm_dyn_check_sample_args(N, V, d, 1 << 45, 1 << 30, None, 1 << 31, 1 << 32)
    assert args(1, (1 << 27) - 1, dtype) == OK
    assert args(0, 1, dtype) == INVALID and args(1, 0, dtype) == INVALID and args(1, 1, 9) == INVALID
    assert args(1, 1 << 27, dtype) == UNSUPPORTED and args(1 << 22, 1, dtype) == UNSUPPORTED


@pytest.mark.parametrize("dtype,e", TYPES)
def test_attend_refusals(dtype, e):
    B, heads, Dk, Dv, T = 2, 3, 8, 12, 5
    a = [0.5, 1.0, 0.0]
    nz, ny, ns = B * T * heads * (2 * Dk + Dv) * e, B * T * heads * Dv * e, 4 * B * heads * Dk * Dv
    head = (B, heads, Dk, Dv, T, dtype, a)
    sizes = [nz, 4 * B, ns, ns, ny]
    chk = lambda *q: layer.lstm_dyn_check_attend_args(*head, *q, 0, 0, 0, 0)
    p = _place(sizes)
    assert chk(*p) == OK
    for i in (1, 2, 3, 4):                  # (without z the check is of the sizes alone)
        assert chk(*[0 if j == i else x for j, x in enumerate(p)]) == (OK if i == 1 else INVALID)
    for i in (3, 4):
        for j in range(5):
            if j != i:
                assert chk(*[p[j] if k == i else x for k, x in enumerate(p)]) == (OK if (i, j) == (3, 2) else INVALID), (i, j)
    assert chk(p[0] + e, *p[1:]) == OK and chk(p[0] + e // 2, *p[1:]) == INVALID
    sizes = [nz, 4 * B, ns, ny, ns, nz, ns]
    back = lambda z, L, S, dy, dS, dz, dS0: layer.lstm_dyn_check_attend_args(*head, z, L, S, 0, 0, dy, dS, dz, dS0)
    p = _place(sizes)
    for i in range(1, 7):
        assert back(*[0 if j == i else x for j, x in enumerate(p)]) == (OK if i in (1, 4) else INVALID), i
    for i in (5, 6):
        for j in range(7):
            if j != i:
                assert back(*[p[j] if k == i else x for k, x in enumerate(p)]) == INVALID, (i, j)
    size = lambda *s: layer.lstm_dyn_check_attend_args(*s, *[0] * 9)
    assert size(*head) == OK and size(1, 1, 128, 128, 1, dtype, [1.0]) == OK
    for bad in ((0, 1, 1, 1, 1, dtype, [1.0]), (1, 1, 0, 1, 1, dtype, [1.0]), (1, 1, 1, 0, 1, dtype, [1.0]), (1, 1, 1, 1, 0, dtype, [1.0]),
                (1, 1, 1, 1, 1, 4, [1.0]), (1, 1, 1, 1, 1, dtype, None), (1, 1, 1, 1, 1, dtype, [1.5]), (1, 1, 1, 1, 1, dtype, [-0.1]),
                (1, 2, 1, 1, 1, dtype, [1.0, float("nan")])):
        assert size(*bad) == INVALID, bad
    for bad in ((1, 1, 129, 1, 1), (1, 1, 1, 129, 1), (1 << 20, 1, 1, 1, 1), (4, 1, 1, 1, 1 << 29), (1, 1, 1, 1, 1 << 30)):
        assert size(*bad, dtype, [1.0]) == UNSUPPORTED, bad


def test_handles_are_refused_before_any_work():
    for call in (lambda: layer.lstm_dyn_norm_forward(0, 1, 0, 0, 0, 1), lambda: layer.lstm_dyn_norm_backward(0, 1, 0, 0, 1, 0, 1, 1, 1),
                 lambda: layer.lstm_dyn_clip_norm(0, None, 0, 1.0, 1.0, 16), lambda: layer.lstm_dyn_clip_apply(0, None, 0, 16, None),
                 lambda: layer.lstm_dyn_sample_step(0, 1, 1, None, 1, 1), lambda: layer.lstm_dyn_attend_forward(0, 1, 0, 1, 1, 1),
                 lambda: layer.lstm_dyn_attend_backward(0, 1, 0, 1, 1, 0, 1, 1), lambda: layer.lstm_dyn_attend_step(0, 1, 1, 1, 1, 1),
                 lambda: layer.lstm_dyn_adamw_step_clipped(0, None, 0, 0.1, 0.9, 0.9, 0.0, 16, 1)):
        with pytest.raises(ld.LstmDynError) as error:
            call()
        assert error.value.code == INVALID


def test_definition_of_attention_against_differences():
    """The loss is linear in every single entry, so a central difference of any step is exact."""
    r = np.random.default_rng(0)
    B, T, heads, Dk, Dv = 2, 5, 2, 3, 4
    z, S0 = r.standard_normal((B, T, heads * (2 * Dk + Dv))), r.standard_normal((B, heads, Dk, Dv))
    dy, dS = r.standard_normal((B, T, heads * Dv)), r.standard_normal(S0.shape)
    L, a = np.array([5, 3]), [0.7, 1.0]

    def loss():
        o = layer_util.attend(z, L, S0, a, Dk, Dv)
        return (o["y"] * dy).sum() + (o["S"] * dS).sum()
    want = layer_util.attend(z, L, S0, a, Dk, Dv, dy, dS)
    for x, g in ((z, want["dz"]), (S0, want["dS0"])):
        for i in np.ndindex(x.shape):
            old = x[i]
            x[i] = old + 1
            up = loss()
            x[i] = old - 1
            down = loss()
            x[i] = old
            assert abs((up - down) / 2 - g[i]) < 1e-10


def test_definition_of_the_norm_against_differences():
    r = np.random.default_rng(1)
    B, T, D, eps, h = 2, 3, 7, 1e-3, 1e-4
    x, w, b, dy = r.standard_normal((B, T, D)), r.standard_normal(D), r.standard_normal(D), r.standard_normal((B, T, D))
    L = np.array([3, 1])
    loss = lambda: (layer_util.norm(x, L, w, b, eps)[0]["y"] * dy).sum()
    want = layer_util.norm(x, L, w, b, eps, dy)[0]
    for v, g in ((x, want["dx"]), (w, want["dweight"]), (b, want["dbias"])):
        for i in np.ndindex(v.shape):
            old = v[i]
            v[i] = old + h
            up = loss()
            v[i] = old - h
            down = loss()
            v[i] = old
            assert abs((up - down) / (2 * h) - g[i]) < 1e-6     # h^2 times a third derivative of some ten
