"""The layer's calls that name their stream: what they allocate belongs to that stream, and the results are those of the
current stream's calls.  And sizes beyond 2^31 elements."""
import pytest

import paper_1810_08061_amd as ld
from tests.gpu_util import say
from tests.test_gpu_ops_streams import _flat, _pool

pytestmark = pytest.mark.gpu


def _calls():
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    B, T, h, D = 3, 300, 2, 24
    L = torch.tensor([T, 7, 0], dtype=torch.int32, device="cuda")
    z, S0, dy, dS, z1 = normal(B, T, 3 * h * D), normal(B, h, D, D), normal(B, T, h * D), normal(B, h, D, D), normal(B, 3 * h * D)
    m = ld.LinearAttention(B, h, D, D, T, [0.9, 0.99], "f32")
    yield m, [lambda **k: m.forward(z, L, S0, **k), lambda **k: m.backward(z, L, S0, dy, dS, **k), lambda **k: m.step(z1, S0, **k)]
    x, gx, w, b = normal(B, T, D), normal(B, T, D), normal(D), normal(D)
    n = ld.LayerNorm(B, T, D, "f32")
    yield n, [lambda **k: n.forward(x, L, w, b, **k), lambda **k: n.backward(x, L, w, gx, **k)]
    grads = [normal(1000), normal(7, 5)]
    p = [normal(1000), normal(7, 5)]
    start = [q.clone() for q in p]
    c, opt = ld.GradClip(grads, 1.0), ld.AdamW(p)

    def step(**k):
        for q, s in zip(p, start):
            q.copy_(s)
        for s in opt.m + opt.v:
            s.zero_()
        opt.steps_done = 0
        torch.cuda.synchronize()
        return opt.step(grads, 0.1, clip=c, **k)

    def clip(**k):
        mine = [q.clone() for q in grads]
        torch.cuda.synchronize()
        return c.clip(mine, **k)
    yield c, [lambda **k: c.norm(grads, **k), clip, step]
    logits, u = normal(5, 5000), torch.rand((5,), generator=g, device="cuda")
    s = ld.TokenSample(5, 5000, "f32")
    yield s, [lambda **k: s.sample(logits, u, top_k=40, top_p=0.9, **k)]


@pytest.mark.parametrize("address", [False, True])
def test_results_belong_to_the_stream_that_is_named(address):
    import torch
    stream = torch.cuda.Stream()
    for handle, calls in _calls():
        with handle:
            want = [[t.clone() for t in _flat(f())] for f in calls]
            torch.cuda.synchronize()
            for i, f in enumerate(calls):
                got = _flat(f(stream=stream.cuda_stream if address else stream))
                assert torch.cuda.current_stream() != stream
                stream.synchronize()
                assert all(_pool(t) == stream.cuda_stream for t in got), (type(handle).__name__, i)
                assert all((a == b).all() for a, b in zip(got, want[i])), (type(handle).__name__, i)
            assert handle.status() == ld.OK


def test_more_than_2_31_elements():
    """Each against a part of itself: rows far behind give what they give alone."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    x = new(1, 70000, 32000)
    say("norm")
    with ld.LayerNorm(1, 70000, 32000, "bf16") as m, ld.LayerNorm(1, 100, 32000, "bf16") as small:
        y = m.forward(x)
        assert (y[:, -100:] == small.forward(x[:, -100:].contiguous())).all()
        y = m.backward(x, None, None, x, out={"dx": y, "dweight": torch.empty(32000, device="cuda"), "dbias": torch.empty(32000, device="cuda")})["dx"]
        tail = x[:, -100:].contiguous()
        assert (y[:, -100:] == small.backward(tail, None, None, tail)["dx"]).all()
    say("clip")
    flat = x.view(-1)
    with ld.GradClip([flat], 1.0) as m:
        norm = float(m.clip([flat], out=[y.view(-1)])[0])
        want = sum(float(x[0, i:i + 7000].double().square().sum()) for i in range(0, 70000, 7000)) ** 0.5
        assert abs(norm - want) <= 1e-6 * want
        f = torch.tensor(1.0, device="cuda", dtype=torch.float64) / want
        # the factor's last bit may be another than that of `want`
        a, b = y.view(-1)[-1000:].double(), flat[-1000:].double() * f
        assert ((a - b).abs() <= b.abs() * 2.0 ** -8).all() and (a != 0).any()
    say("sample")
    del y
    u = torch.rand((70000,), generator=g, device="cuda")
    with ld.TokenSample(70000, 32000, "bf16") as m, ld.TokenSample(50, 32000, "bf16") as small:
        token, logp = m.sample(x[0], u, top_p=0.9)
        t2, l2 = small.sample(x[0, -50:].contiguous(), u[-50:].contiguous(), top_p=0.9)
        assert (token[-50:] == t2).all() and (logp[-50:] == l2).all() and (token >= 0).all() and (token < 32000).all()
    del x
    say("attend")
    # 3 rows of 2^16 steps of 16 heads of 3 x 256 bytes: the third row starts beyond 2^31 bytes, its end beyond 2^31 elements
    B, T, h, D = 6, 65536, 16, 120
    z = new(B, T, 3 * h * D)
    assert z.numel() > 1 << 31
    z[..., h * D:2 * h * D] *= 0.1
    S0 = torch.randn((B, h, D, D), generator=g, device="cuda")
    dy = new(B, T, h * D)
    L = torch.full((B,), 777, dtype=torch.int32, device="cuda")
    with ld.LinearAttention(B, h, D, D, T, 0.9, "bf16") as m, ld.LinearAttention(1, h, D, D, T, 0.9, "bf16") as small:
        y, S = m.forward(z, L, S0)
        grads = m.backward(z, L, S0, dy)
        y1, S1 = small.forward(z[-1:].contiguous(), L[:1], S0[-1:].contiguous())
        g1 = small.backward(z[-1:].contiguous(), L[:1], S0[-1:].contiguous(), dy[-1:].contiguous())
        # the same chunks, but shares of another length: roundings of sums over 777 steps
        for a, b in ((y[-1:], y1), (S[-1:], S1), (grads["dz"][-1:], g1["dz"]), (grads["dS0"][-1:], g1["dS0"])):
            a, b = a.double(), b.double()
            assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 1e-3 * b.abs().max()).all()
            assert float(b.abs().max()) > 0
        assert (y[-1, 777:] == 0).all() and (grads["dz"][-1, 777:] == 0).all()
