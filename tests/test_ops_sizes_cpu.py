"""Sizes at which the operators' indexes or a launch's threads would pass 32 bits: refused by the checks
each call makes first, and the last ones before them accepted."""
import pytest

import paper_1810_08061_amd as ld
from paper_1810_08061_amd import ops
from tests.test_ops_cpu import _place

OK, UNSUPPORTED = ld.OK, ld.ERR_UNSUPPORTED


def _scan(B, H, T, dtype):
    e, n = (2 if dtype == ld.BF16 else 4), B * T * H
    z, L, h0, out_h, y, dy, dz, dh0 = _place([3 * n * e, 4 * B, 4 * B * H, 4 * B * H, n * e, n * e, 3 * n * e, 4 * B * H])
    f = ops.lstm_dyn_check_scan_args(B, H, T, dtype, z, L, h0, out_h, y, 0, 0, 0, 0)
    assert ops.lstm_dyn_check_scan_args(B, H, T, dtype, z, L, h0, 0, 0, dy, 0, dz, dh0) == f
    return f


@pytest.mark.parametrize("dtype", [ld.F32, ld.BF16])
def test_scan(dtype):
    # one row: with bf16 data its steps and a share of 256, with fp32 its threads, four a step
    last = 2 ** 31 - 1 - 256 if dtype == ld.BF16 else 2 ** 30 - 128
    assert _scan(1, 1, last, dtype) == OK
    for T in (last + 1, 2 ** 31 - 129, 2 ** 31 - 17, 2 ** 31 - 2, 2 ** 31 - 1):
        assert _scan(1, 1, T, dtype) == UNSUPPORTED, T
    # 64 threads a row and 64 or 128 channels
    for H, tiles in ((1, 1), (64, 1), (65, 2), (128, 1), (129, 3), (130, 2)):
        rows = (2 ** 32 - 1) // (64 * tiles)
        assert _scan(rows, H, 1, dtype) == OK, H
        assert _scan(rows + 1, H, 1, dtype) == UNSUPPORTED, H
    # many shares: two or four threads a step for each 64 channels, 32 of odd H
    rows = 2 ** 32 // (2 ** 22 * (2 if dtype == ld.BF16 else 4))
    T = 2 ** 22 - 1
    for H, tiles in ((1, 1), (64, 1), (65, 3), (130, 3)):
        assert _scan(rows // tiles - (tiles == 1), H, T, dtype) == OK, H
        assert _scan(rows // tiles + (tiles > 1), H, T, dtype) == UNSUPPORTED, H


def test_scan_step():
    lib = ops._lib()
    step = lambda rows, H, dtype=ld.F32: lib.lstm_dyn_scan_step(rows, H, dtype, *_place([12 * rows * H, 4 * rows * H, 4 * rows * H, 4 * rows * H]), 0)
    assert step(2 ** 31 - 1, 3) == UNSUPPORTED
    assert step(2 ** 17, 2 ** 15 + 1) == UNSUPPORTED
    assert step(2 ** 30, 16) == UNSUPPORTED           # four elements a thread
    assert step(4, 2 ** 18) == UNSUPPORTED
    assert step(0, 4) == step(4, 0) == step(4, 4, 9) == ld.ERR_INVALID


@pytest.mark.parametrize("D,tiles", [(1, 1), (64, 1), (65, 2), (67, 2), (130, 2), (260, 2), (513, 9), (2048, 8)])
def test_embed(D, tiles):
    def chk(N):
        V = 5
        tok, table, x, dx, dt = _place([4 * N, 2 * V * D, 2 * N * D, 2 * N * D, 4 * V * D])
        if N < 2 ** 30:     # the lookup has no such launch
            assert ops.lstm_dyn_check_embed_args(1, N, V, D, ld.BF16, tok, 0, table, x, 0, ld.BF16, 0) == OK
        return ops.lstm_dyn_check_embed_args(1, N, V, D, ld.BF16, tok, 0, 0, 0, dx, ld.BF16, dt)
    last = min(2 ** 30 - 1, 32 * ((2 ** 26 - 2 ** 16 - 1) // tiles))
    assert chk(last) == OK and chk(last + 1) == UNSUPPORTED
