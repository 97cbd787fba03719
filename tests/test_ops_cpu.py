"""The C ABI of the operators around the loop without a GPU: every declared function is exported, and
bad arguments are refused by the checks each call makes first."""
import ctypes
import os
import re

import pytest

import paper_1810_08061_amd as ld
from paper_1810_08061_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED = ld.OK, ld.ERR_INVALID, ld.ERR_UNSUPPORTED


def test_library_exports_every_declared_operator():
    with open(os.path.join(ROOT, "include", "lstm_dyn_ops.h")) as f:
        names = re.findall(r"^int\s+(lstm_dyn_\w+)\s*\(", f.read(), re.M)
    assert len(names) == 25
    lib = ctypes.CDLL(ld.library_path())
    for n in names:
        assert hasattr(lib, n) and hasattr(ops, n), n


def _place(sizes):
    p, at = [], 1 << 20
    for s in sizes:
        p.append(at)
        at += (s + 255) // 256 * 256 + 256
    return p


def _refusals(chk, p, sizes, written, optional=(), same=()):
    """chk accepts p; refuses NULL, misaligned and overlapping buffers one at a time."""
    assert chk(*p) == OK
    for i in range(len(p)):
        q = list(p)
        q[i] = 0
        assert chk(*q) == (OK if i in optional else INVALID), i
    for i in written:
        for j in range(len(p)):
            if j == i:
                continue
            q = list(p)
            q[i] = q[j]
            assert chk(*q) == (OK if (i, j) in same else INVALID), (i, j)
            if sizes[j] > 16:
                q[i] = p[j] + (sizes[j] - 1) // 16 * 16     # on the last bytes of another
                assert chk(*q) == INVALID, (i, j)


@pytest.mark.parametrize("dtype,e", [(ld.F32, 4), (ld.BF16, 2)])
def test_scan_refusals(dtype, e):
    B, H, T = 3, 24, 5
    n = B * T * H
    sizes = [3 * n * e, 4 * B, 4 * B * H, 4 * B * H, n * e]
    p = _place(sizes)
    chk = lambda *q: ops.lstm_dyn_check_scan_args(B, H, T, dtype, *q, 0, 0, 0, 0)
    _refusals(chk, p, sizes, (3, 4), same={(3, 2)})
    sizes = [3 * n * e, 4 * B, 4 * B * H, n * e, 4 * B * H, 3 * n * e, 4 * B * H]
    p = _place(sizes)
    chk = lambda z, L, h0, dy, dh, dz, dh0: ops.lstm_dyn_check_scan_args(B, H, T, dtype, z, L, h0, 0, 0, dy, dh, dz, dh0)
    _refusals(chk, p, sizes, (5, 6), optional=(4,))
    for i, off in ((0, 8), (3, 4), (5, 8), (1, 2), (6, 2)):
        q = list(p)
        q[i] += off
        assert chk(*q) == INVALID, i
    for bad in ((0, H, T, dtype), (B, 0, T, dtype), (B, H, 0, dtype), (B, H, T, 2)):
        assert ops.lstm_dyn_check_scan_args(*bad, p[0], p[1], p[2], 0, 0, p[3], 0, p[5], p[6]) == INVALID
    assert ops.lstm_dyn_check_scan_args(1 << 16, H, 1 << 16, dtype, p[0], p[1], p[2], 0, 0, p[3], 0, p[5], p[6]) == UNSUPPORTED


def test_embed_refusals():
    B, T, V, D = 3, 5, 40, 12
    sizes = [4 * B * T, 4 * B, 2 * V * D, 2 * B * T * D]
    p = _place(sizes)
    chk = lambda *q: ops.lstm_dyn_check_embed_args(B, T, V, D, ld.BF16, *q, 0, ld.F32, 0)
    _refusals(chk, p, sizes, (3,), optional=(1,))
    sizes = [4 * B * T, 4 * B, 4 * B * T * D, 4 * V * D]
    p = _place(sizes)
    chk = lambda t, L, dx, dt: ops.lstm_dyn_check_embed_args(B, T, V, D, ld.BF16, t, L, 0, 0, dx, ld.F32, dt)
    _refusals(chk, p, sizes, (3,), optional=(1,))
    assert ops.lstm_dyn_check_embed_args(B, T, V, D, ld.BF16, p[0], p[1], 0, 0, p[2], 7, p[3]) == INVALID
    for bad in ((0, T, V, D), (B, 0, V, D), (B, T, 0, D), (B, T, V, 0)):
        assert ops.lstm_dyn_check_embed_args(*bad, ld.BF16, p[0], p[1], 0, 0, p[2], ld.F32, p[3]) == INVALID
    for big in ((1 << 15, 1 << 15, V, D), (B, T, 1 << 27, D), (B, T, V, 1 << 21)):
        assert ops.lstm_dyn_check_embed_args(*big, ld.BF16, p[0], p[1], 0, 0, p[2], ld.F32, p[3]) == UNSUPPORTED


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_refusals(bits):
    ns, e = (300, 0, 7), (4 if bits == 32 else 1)
    tensors, sizes = [], []
    for n in ns:
        b = -(-n // 256)
        sizes.append([4 * n, 2 * n, e * n, e * n, b, b])
    place = iter(_place([s for row in sizes for s in row] + [4 * n for n in ns]))
    for n in ns:
        a = [next(place) for _ in range(6)]
        if bits == 32:
            a[4] = a[5] = 0
        tensors.append(a)
    grads = [next(place) for _ in ns]

    def chk(t, g=grads, dt=ld.F32, b=bits):
        return ops.lstm_dyn_check_adamw_args([ops.AdamwTensor(*row, n, 0.01) for row, n in zip(t, ns)], b, g, dt)

    def change(i, j, value):
        t = [list(r) for r in tensors]
        t[i][j] = value
        return t

    assert chk(tensors) == OK
    assert chk(change(0, 1, 0)) == OK                                   # no copy
    assert chk([tensors[0], [0] * 6, tensors[2]], [grads[0], 0, grads[2]]) == OK   # an empty tensor
    for j in (0, 2, 3) + ((4, 5) if bits == 8 else ()):
        assert chk(change(0, j, 0)) == INVALID, j
    assert chk(change(0, 0, tensors[0][0] + 2)) == INVALID
    assert chk(change(0, 1, tensors[0][1] + 1)) == INVALID
    for j in (0, 1, 2, 3):
        assert chk(change(0, j, tensors[2][0])) == INVALID, j           # on another tensor's parameters
    assert chk(change(0, 2, tensors[0][0] + 4 * 299)) == INVALID        # on its own last parameter
    assert chk(tensors, [0] + grads[1:]) == INVALID
    assert chk(tensors, [tensors[2][2]] + grads[1:]) == INVALID         # a gradient on a state
    assert chk(tensors, [grads[0] + 2] + grads[1:]) == INVALID
    assert chk(tensors, [grads[0] + 2] + grads[1:], ld.BF16) == OK
    assert chk(tensors, grads, 5) == INVALID
    assert chk(tensors, None, ld.F32, 16) == INVALID
    assert ops.lstm_dyn_check_adamw_args([], bits) == INVALID
    assert ops.lstm_dyn_check_adamw_args([ops.AdamwTensor(*tensors[0], -1, 0.0)], bits) == INVALID
    assert ops.lstm_dyn_check_adamw_args([ops.AdamwTensor(*tensors[0], 300, float("nan"))], bits) == INVALID


def test_beam_refusals():
    B, K, V, w = 2, 3, 50, 20
    n = B * K
    sizes = [n * V * 2, 4 * n, n, 4 * n, 4 * n, 4 * n, n, n * w, n * w]
    p = _place(sizes)

    def chk(*q, ns=1):
        st = (ops.BeamState * 1)(ops.BeamState(q[7], q[8], w))
        return ops.lstm_dyn_check_beam_args(B, K, V, ld.BF16, *q[:7], st, ns)

    _refusals(chk, p, sizes, (3, 4, 5, 6, 8))
    assert chk(*p, ns=0) == OK and chk(*p, ns=-1) == INVALID and chk(*p, ns=9) == INVALID
    assert ops.lstm_dyn_check_beam_args(B, K, V, ld.BF16, *p[:7], None, 1) == INVALID
    st = (ops.BeamState * 1)(ops.BeamState(p[7], p[8], 0))
    assert ops.lstm_dyn_check_beam_args(B, K, V, ld.BF16, *p[:7], st, 1) == INVALID
    for bad in ((0, K, V), (B, 0, V), (B, K, 0)):
        assert ops.lstm_dyn_check_beam_args(*bad, ld.BF16, *p[:7], None, 0) == INVALID
    assert ops.lstm_dyn_check_beam_args(B, 33, V, ld.BF16, *p[:7], None, 0) == UNSUPPORTED


def test_null_handles():
    lib = ops._lib()
    assert lib.lstm_dyn_scan_forward(None, 0, 0, 0, 0, 0, 0) == INVALID
    assert lib.lstm_dyn_embed_forward(None, 0, 0, 0, 1.0, 0, 0) == INVALID
    assert lib.lstm_dyn_adamw_step(None, None, 0, 0, 0, 0, 0, 0, 1, 0) == INVALID
    assert lib.lstm_dyn_beam_step(None, 0, 0, 0, 0, 0, 0, 0, 0, None, 0, 0) == INVALID
    for kind in ("scan", "embed", "adamw", "beam"):
        assert getattr(lib, f"lstm_dyn_{kind}_destroy")(None) == OK
        assert getattr(lib, f"lstm_dyn_{kind}_query")(None, 0, None) == INVALID
    for kind, args in (("scan", (0, 4, 4, 0)), ("embed", (1, 1, 0, 4, 0)), ("beam", (1, 0, 4, 0))):
        h = ctypes.c_void_p(5)
        assert getattr(lib, f"lstm_dyn_{kind}_create")(ctypes.byref(h), *args) == INVALID and not h.value
    assert ld.lstm_dyn_strerror(ops.ERR_BAD_TOKENS) != "unknown status"
