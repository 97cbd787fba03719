"""The gradients' norm and clipping on the GPU, alone and on the way into AdamW."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from tests.layer_util import HALF, U

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().double().cpu().numpy()


def _tensors(r, sizes, dtype, size=1.0):
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    return [torch.from_numpy((size * r.standard_normal(s)).astype(np.float32)).cuda().to(t) for s in sizes]


def _want(grads, max_norm, gs=1.0):
    norm = abs(gs) * np.sqrt(sum((_np(g) ** 2).sum() for g in grads))
    return norm, gs * (1.0 if norm <= max_norm else max_norm / norm)


def _check(result, out, grads, max_norm, dtype, gs=1.0):
    norm, f = _want(grads, max_norm, gs)
    got = _np(result)
    # sums in 64 bits; each of the two rounded once
    assert abs(got[0] - norm) <= U * norm * 1.001 and abs(got[1] - f) <= U * abs(f) * 1.001
    for o, g in zip(out, grads):
        w = _np(g) * f
        assert (np.abs(_np(o) - w) <= (2 * U * 1.001 + HALF[dtype] * 1.001) * np.abs(w) + 2.0 ** -149).all()


# around a workgroup's elements (16384), nothing, one, odd; many tensors and few
SETS = [[(1,)], [(0,), (5,)], [(16383,), (16384,), (16385,), (3, 7)], [(100, 1000), (0,), (32768,), (33, 5, 7)], [(1 << 20,), (1,)],
        [(i % 13,) for i in range(700)], [(9,)] * 256, [(9,)] * 257, [(3,)] * 129]


@pytest.mark.parametrize("sizes", SETS, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_norm_and_clip(dtype, sizes, max_norm):
    import torch
    r = np.random.default_rng(len(sizes))
    g = _tensors(r, sizes, dtype)
    with ld.GradClip(g, max_norm) as m:
        out = [torch.empty_like(x) for x in g]
        result = m.clip(g, out=out)
        _check(result, out, g, max_norm, dtype)
        assert (m.norm(g) == result).all()
        mine = [x.clone() for x in g]              # in place
        assert (m.clip(mine) == result).all() and all((a == b).all() for a, b in zip(mine, out))
        assert (m.norm(g) == result).all()         # the same call, the same bits
        if max_norm > 1:
            assert all((a == b).all() for a, b in zip(out, g))
        result = m.clip(g, grad_scale=-0.25, out=out)
        _check(result, out, g, max_norm, dtype, -0.25)
        assert m.status() == ld.OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_off_their_alignment(dtype):
    import torch
    r = np.random.default_rng(1)
    base = _tensors(r, [(40001,), (16384 + 1,)], dtype)
    g = [b[1:] for b in base]
    with ld.GradClip(g, 1.0) as m:
        out = [torch.empty_like(b)[1:] for b in base]
        _check(m.clip(g, out=out), out, g, 1.0, dtype)


@pytest.mark.parametrize("size", [1e-30, 1e25, 3e38])
def test_the_ends_of_the_range(size):
    """Squares far outside fp32's range: the sum is formed in 64 bits."""
    import torch
    g = [torch.full((3,), size, device="cuda"), torch.full((1,), -size, device="cuda")]
    with ld.GradClip(g, 1.0) as m:
        result = _np(m.norm(g))
        norm = 2 * float(np.float32(size))
        if norm > 3.5e38:
            assert result[0] == np.inf
            assert abs(result[1] - 1 / norm) <= 2.0 ** -149     # a subnormal factor
        else:
            assert abs(result[0] - norm) <= U * norm * 1.001


def test_what_is_not_a_number():
    import torch
    g = [torch.ones(5, device="cuda"), torch.ones(20000, device="cuda")]
    with ld.GradClip(g, 1.0) as m:
        g[1][17000] = float("inf")
        result = m.norm(g)
        assert result[0] == float("inf") and result[1] == 0
        g[1][17000] = float("nan")
        assert m.norm(g).isnan().all()
        g[1][17000] = 1.0
        zero = [torch.zeros_like(x) for x in g]
        result = m.norm(zero)
        assert result[0] == 0 and result[1] == 1
        assert all((x == 0).all() for x in zero)
    with ld.GradClip(g, 0.0) as m:
        assert m.norm(g)[1] == 0 and m.norm(zero)[1] == 1
    with ld.GradClip(g, float("inf")) as m:
        assert m.norm(g)[1] == 1
        with pytest.raises(ld.LstmDynError):
            m.norm(g, grad_scale=float("nan"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_the_step_clipped_is_the_step_of_clipped_gradients(dtype, bits):
    """The factor taken along is the same multiplication as grad_scale's: bit for bit where the
    factor is the same number."""
    import torch
    r = np.random.default_rng(2)
    sizes = [(50, 70), (333,), (0,), (4096 * 5 + 3,)]
    p = _tensors(r, sizes, "f32")
    a, b = [x.clone() for x in p], [x.clone() for x in p]
    one, two = ld.AdamW(a, state_bits=bits), ld.AdamW(b, state_bits=bits)
    clip = ld.GradClip(p, 0.7)
    for step in range(3):
        g = _tensors(r, sizes, dtype, 10.0 ** (1 - 3 * step))
        result = one.step(g, 0.01, grad_scale=0.5, clip=clip)
        two.step(g, 0.01, grad_scale=float(result[1]))
        assert one.steps_done == two.steps_done == step + 1
        torch.cuda.synchronize()
        assert all((x == y).all() for x, y in zip(a, b))
        for x, y in zip(one.m + one.v, two.m + two.v):
            assert (x.view(torch.uint8) == y.view(torch.uint8)).all()
        norm, f = _want(g, 0.7, 0.5)
        assert abs(float(result[1]) - f) <= U * abs(f) * 1.001
    one.close(), two.close(), clip.close()


def test_nothing_to_add():
    import torch
    g = [torch.empty(0, device="cuda"), torch.empty(3, 0, device="cuda")]
    with ld.GradClip(g, 1.0) as m:
        for _ in range(2):
            assert m.clip(g, grad_scale=0.5).tolist() == [0.0, 0.5]


def test_wrong_lists_are_refused():
    import torch
    g = [torch.ones(4, device="cuda"), torch.ones(2, 3, device="cuda")]
    with ld.GradClip(g, 1.0) as m:
        with pytest.raises(ValueError):
            m.norm(g[:1])
        with pytest.raises(ValueError):
            m.norm([g[0], g[0]])
        with pytest.raises(TypeError):
            m.norm([g[0], g[1].bfloat16()])
        with pytest.raises(TypeError):
            m.norm([x.half() for x in g])
        with pytest.raises(ValueError):
            m.clip(g, out=g[:1])
        both = torch.empty(10, device="cuda")        # an output that lies on another one's memory
        with pytest.raises(ld.LstmDynError):
            m.clip(g, out=[both[:4], both[2:8].view(2, 3)])
    with pytest.raises(ValueError):
        ld.GradClip([], 1.0)


def test_replays_of_a_graph():
    """Norm, clipping and the clipped step captured; the counter of workgroups is left as it was found."""
    import torch
    r = np.random.default_rng(4)
    sizes = [(300, 300), (17,), (16384 * 3 + 5,)]
    g, p = _tensors(r, sizes, "f32"), _tensors(r, sizes, "f32")
    start = [x.clone() for x in p]
    q = [x.clone() for x in p]
    one, two = ld.AdamW(p), ld.AdamW(q)
    clip, other = ld.GradClip(p, 1.0), ld.GradClip(p, 1.0)
    out, want = [torch.empty_like(x) for x in g], [torch.empty_like(x) for x in g]
    one.step(g, 0.1, clip=clip)
    clip.clip(g, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = clip.clip(g, out=out)
        one.steps_done = 0
        one.step(g, 0.1, clip=clip)
    for i in range(4):
        for x in g:
            x.copy_(torch.randn(x.shape, device="cuda") * 10.0 ** -i)
        for opt, params in ((one, p), (two, q)):
            for a, b in zip(params, start):
                a.copy_(b)
            for x in opt.m + opt.v:
                x.zero_()
        two.steps_done = 0
        expected = other.clip(g, out=want)
        two.step(g, 0.1, clip=other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (result == expected).all()
        assert all((a == b).all() for a, b in zip(out + p, want + q)), i
    del graph
    for h in (one, two, clip, other):
        h.close()
