"""Sampling where a row's workgroup changes with its length and with the number of rows; every row's outputs are written."""
import ctypes

import numpy as np
import pytest

import paper_1810_08061_amd as ld
from paper_1810_08061_amd import layer
from tests import layer_util
from tests.gpu_util import say
from tests.layer_util import U
from tests.test_gpu_sample import FILTERS, _dev, _sample

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(3, 100), (9, 8200), (700, 1000), (600, 16385)])     # workgroups of 512, 1024, 256 and 512
def test_every_row_is_written(dtype, N, V):
    """Rows from flat to steep with u at both ends of the unit interval, where a running sum that missed its target by one unit
    would leave the row as it was."""
    import torch
    say("written", dtype, N, V)
    r = np.random.default_rng(N + V)
    ends = [0.0, 2.0 ** -24, 2.0 ** -149, 1.0 - 2.0 ** -24, 1.0 - 2.0 ** -23, 1.0, 0.5]
    x = _dev(r.standard_normal((N, V)) * np.exp(r.uniform(-9, 3, (N, 1))), dtype)
    T = _dev(np.exp(r.uniform(-3, 3, N)))
    m = ld.TokenSample(N, V, dtype)
    stream = torch.cuda.current_stream().cuda_stream
    for k, p, q in FILTERS:
        for shift in range(len(ends)):
            u = _dev(np.resize(np.roll(ends, shift), N))
            f = layer.SampleFilter(1.0, 1.0, 0.0, 0, T.data_ptr(), None, None, None)
            keep = [_dev(np.exp(r.uniform(0, np.log(V), N)).astype(np.int32)), _dev(r.uniform(0.001, 1.0, N)), _dev(np.exp(r.uniform(-14, 0, N)))]
            f.top_ks, f.top_ps, f.min_ps = (t.data_ptr() if on else None for t, on in zip(keep, (k, p, q)))
            token = torch.full((N,), -7, dtype=torch.int32, device="cuda")
            logp = torch.full((N,), 9.0, device="cuda")
            layer.lstm_dyn_sample_step(m.handle, x.data_ptr(), u.data_ptr(), ctypes.byref(f), token.data_ptr(), logp.data_ptr(), stream)
            torch.cuda.synchronize()
            assert ((token >= 0) & (token < V)).all() and (logp <= 0).all(), (k, p, q, shift)
    assert m.status() == ld.OK
    m.close()


# 512 threads hand over to 1024 behind 8192 tokens, and with more rows than two a CU 256 to 512 behind 16384
@pytest.mark.parametrize("N,V", [(12, 8191), (12, 8192), (12, 8193), (520, 16383), (520, 16384), (520, 16385)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,p,m", FILTERS)
def test_where_workgroups_change(dtype, N, V, k, p, m):
    """Twelve of the rows against the definition; rows in which rounding decides are passed over, and log p is held to the bound
    that the other sizes are held to."""
    r = np.random.default_rng(V * 8 + 4 * k + 2 * p + m)
    x = _dev(r.standard_normal((N, V)) * 2.5, dtype)
    f32 = lambda a: a.astype(np.float32).astype(np.float64)
    u, T = f32(r.random(N)), f32(r.uniform(0.4, 1.3, N))
    ks = r.integers(0, 300, N).astype(np.int32) if k else None
    ps = f32(r.uniform(0.2, 0.99, N)) if p else None
    ms = f32(np.exp(r.uniform(-7, -1, N))) if m else None
    token, logp = _sample(x, u, temperature=T, top_k=ks, top_p=ps, min_p=ms)
    seen = 0
    for n in range(0, N, N // 12):
        row = x[n].double().cpu().numpy()
        want, lp, near = layer_util.sample(row, u[n], T[n], ks[n] if k else 0, ps[n] if p else 1.0, ms[n] if m else 0.0)
        if near < 1e-6:
            continue
        seen += 1
        assert token[n] == want, (n, near)
        assert abs(logp[n] - lp) <= 1e-6 + 2 * U * abs(lp), n
    assert seen >= 6
