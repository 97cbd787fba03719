"""Linear attention on the GPU against its definition in 64 bits, step by step."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from tests import layer_util
from tests.gpu_util import say
from tests.layer_util import HALF, U

pytestmark = pytest.mark.gpu


def _torch_type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _dev(a, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(_torch_type(dtype))


def _np(t):
    return t.detach().double().cpu().numpy()


def _inputs(r, dtype, B, T, heads, Dk, Dv):
    z = _dev(r.standard_normal((B, T, heads * (2 * Dk + Dv))), dtype)
    return {"z": z, "S0": _dev(r.standard_normal((B, heads, Dk, Dv))), "dy": _dev(r.standard_normal((B, T, heads * Dv)), dtype),
            "dS": _dev(r.standard_normal((B, heads, Dk, Dv)))}


def _compare(got, s, L, decay, Dk, Dv, dtype, train=True, tight=True):
    """Element by element within the bounds; and on the whole, since roundings are independent, within
    four times the root of their number."""
    z, S0 = _np(s["z"]), _np(s["S0"])
    dy, dS = (_np(s["dy"]), _np(s["dS"]) if s["dS"] is not None else None) if train else (None, None)
    valid = np.arange(z.shape[1])[None, :, None] < np.asarray(L)[:, None, None]
    z = np.where(valid, z, 0)
    dy = np.where(valid, dy, 0) if train else None
    a = np.float32(decay).astype(np.float64)
    want = layer_util.attend(z, L, S0, a, Dk, Dv, dy, dS)
    bound, mag, n = layer_util.attend_bounds(z, L, S0, a, Dk, Dv, dtype, dy, dS)
    for k, w in want.items():
        if k not in got:
            continue
        g = _np(got[k])
        assert np.isfinite(g).all(), k
        rounding = HALF[dtype] if k in ("y", "dz") else 0.0
        err = np.abs(g - w)
        assert (err <= bound[k] * (1 + rounding) + rounding * np.abs(w) + 1e-37).all(), (k, (err - bound[k]).max())
        if tight and rounding == 0:
            assert np.linalg.norm(err) <= 4 * np.sqrt(n) * U * np.linalg.norm(mag[k]) + 1e-37, k


def _lengths(L):
    import torch
    return torch.tensor(L, dtype=torch.int32, device="cuda")


SHAPES = [(1, 1, 1), (8, 12, 3), (16, 16, 2), (32, 32, 1), (33, 31, 2), (64, 64, 2), (50, 75, 3), (65, 8, 1), (128, 128, 1), (127, 128, 2),
          (8, 128, 1), (120, 40, 2)]


@pytest.mark.parametrize("Dk,Dv,heads", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_and_backward(dtype, Dk, Dv, heads):
    r = np.random.default_rng(Dk * 1000 + Dv)
    T, L = 70, [70, 0, 1, 33, 64]
    s = _inputs(r, dtype, len(L), T, heads, Dk, Dv)
    decay = [0.9, 1.0, 0.0][:heads] if heads > 1 else [0.97]
    with ld.LinearAttention(len(L), heads, Dk, Dv, T, decay, dtype) as m:
        y, S = m.forward(s["z"], _lengths(L), s["S0"])
        got = m.backward(s["z"], _lengths(L), s["S0"], s["dy"], s["dS"])
        _compare(dict(got, y=y, S=S), s, L, decay, Dk, Dv, dtype)
        assert m.status() == ld.OK
    for b, n in enumerate(L):       # zeros behind a sequence; one without steps passes its states on
        assert (y[b, n:] == 0).all() and (got["dz"][b, n:] == 0).all()
        if n == 0:
            assert (S[b] == s["S0"][b]).all() and (got["dS0"][b] == s["dS"][b]).all()


# around a chunk (32 or 64 steps), a share of four chunks and more
@pytest.mark.parametrize("T", [1, 2, 31, 32, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths(dtype, T):
    r = np.random.default_rng(T)
    L = [T, max(0, T - 1), T // 2, 0]
    Dk, Dv, heads = 16, 24, 2
    s = _inputs(r, dtype, 4, T, heads, Dk, Dv)
    decay = [1.0, 0.99]
    with ld.LinearAttention(4, heads, Dk, Dv, T, decay, dtype) as m:
        y, S = m.forward(s["z"], _lengths(L), s["S0"])
        got = m.backward(s["z"], _lengths(L), s["S0"], s["dy"], s["dS"])
        _compare(dict(got, y=y, S=S), s, L, decay, Dk, Dv, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_wide_heads_over_shares(dtype):
    r = np.random.default_rng(7)
    L, T, Dk, Dv, heads = [700, 300, 257], 700, 128, 100, 2
    s = _inputs(r, dtype, 3, T, heads, Dk, Dv)
    decay = [0.999, 0.8]
    with ld.LinearAttention(3, heads, Dk, Dv, T, decay, dtype) as m:
        y, S = m.forward(s["z"], _lengths(L), s["S0"])
        got = m.backward(s["z"], _lengths(L), s["S0"], s["dy"], s["dS"])
        _compare(dict(got, y=y, S=S), s, L, decay, Dk, Dv, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_take_one_share_each(dtype):
    r = np.random.default_rng(8)
    B, T, Dk, Dv, heads = 150, 90, 8, 8, 4       # 600 rows and heads
    L = [int(x) for x in r.integers(0, T + 1, B)]
    s = _inputs(r, dtype, B, T, heads, Dk, Dv)
    decay = [0.9, 0.5, 1.0, 0.99]
    with ld.LinearAttention(B, heads, Dk, Dv, T, decay, dtype) as m:
        y, S = m.forward(s["z"], _lengths(L), s["S0"])
        got = m.backward(s["z"], _lengths(L), s["S0"], s["dy"], s["dS"])
        _compare(dict(got, y=y, S=S), s, L, decay, Dk, Dv, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [40, 600])
def test_optional_arguments(dtype, T):
    import torch
    r = np.random.default_rng(9)
    Dk, Dv, heads = 16, 32, 1
    s = _inputs(r, dtype, 2, T, heads, Dk, Dv)
    with ld.LinearAttention(2, heads, Dk, Dv, T, 0.9, dtype) as m:
        full = _lengths([T, T])
        a, b = m.forward(s["z"], full, s["S0"]), m.forward(s["z"], None, s["S0"])
        assert (a[0] == b[0]).all() and (a[1] == b[1]).all()
        zero = torch.zeros_like(s["dS"])
        a, b = m.backward(s["z"], full, s["S0"], s["dy"], zero), m.backward(s["z"], None, s["S0"], s["dy"])
        assert (a["dz"] == b["dz"]).all() and (a["dS0"] == b["dS0"]).all()
        S = s["S0"].clone()                      # the state in place
        y, out = m.forward(s["z"], None, S, out_S=S)
        want = m.forward(s["z"], None, s["S0"])
        assert out is S and (S == want[1]).all() and (y == want[0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,Dk,Dv", [(100, 8, 12), (600, 64, 64)])
def test_nothing_behind_a_sequence_counts(dtype, T, Dk, Dv):
    import torch
    r = np.random.default_rng(10)
    L, heads = [T, T // 3, 0], 2
    s = _inputs(r, dtype, 3, T, heads, Dk, Dv)
    with ld.LinearAttention(3, heads, Dk, Dv, T, [0.9, 1.0], dtype) as m:
        def both():
            y, S = m.forward(s["z"], _lengths(L), s["S0"])
            return dict(m.backward(s["z"], _lengths(L), s["S0"], s["dy"], s["dS"]), y=y, S=S)
        want = both()
        for bad in (float("nan"), float("inf")):
            for b, n in enumerate(L):
                s["z"][b, n:] = bad
                s["dy"][b, n:] = bad
            got = both()
            torch.cuda.synchronize()
            for k in want:
                assert (got[k] == want[k]).all(), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bad_lengths_are_clamped_and_reported(dtype):
    r = np.random.default_rng(11)
    T, Dk, Dv, heads = 300, 8, 8, 1
    s = _inputs(r, dtype, 3, T, heads, Dk, Dv)
    with ld.LinearAttention(3, heads, Dk, Dv, T, 0.9, dtype) as m:
        want = m.forward(s["z"], _lengths([T, 0, 5]), s["S0"])
        assert m.status() == ld.OK
        got = m.forward(s["z"], _lengths([T + 9, -4, 5]), s["S0"])
        assert m.status() == ld.ERR_BAD_LENGTHS and m.status() == ld.OK
        assert (got[0] == want[0]).all() and (got[1] == want[1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(1, 1), (8, 12), (64, 64), (50, 75), (128, 128), (33, 4), (3, 128)])
@pytest.mark.parametrize("R", [1, 5])
def test_step(dtype, Dk, Dv, R):
    import torch
    r = np.random.default_rng(Dk + Dv)
    heads, decay = 3, [0.9, 1.0, 0.0]
    s = _inputs(r, dtype, R, 1, heads, Dk, Dv)
    with ld.LinearAttention(2, heads, Dk, Dv, 4, decay, dtype) as m:       # any number of rows
        y, S = m.step(s["z"][:, 0].contiguous(), s["S0"])
        _compare({"y": y[:, None], "S": S}, s, [1] * R, decay, Dk, Dv, dtype, train=False)
        again = s["S0"].clone()
        y2, S2 = m.step(s["z"][:, 0].contiguous(), again, out_S=again)
        torch.cuda.synchronize()
        assert S2 is again and (again == S).all() and (y2 == y).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_and_sequences_agree(dtype):
    """A prompt as a whole, then single tokens, against the definition over all of it."""
    r = np.random.default_rng(12)
    T, P, Dk, Dv, heads = 80, 70, 24, 40, 2
    decay = [0.95, 1.0]
    s = _inputs(r, dtype, 2, T, heads, Dk, Dv)
    with ld.LinearAttention(2, heads, Dk, Dv, P, decay, dtype) as m:
        y, S = m.forward(s["z"][:, :P].contiguous(), None, s["S0"])
        ys = [y]
        for t in range(P, T):
            y1, S = m.step(s["z"][:, t].contiguous(), S, out_S=S)
            ys.append(y1[:, None])
        import torch
        _compare({"y": torch.cat(ys, 1), "S": S}, s, [T, T], decay, Dk, Dv, dtype, train=False)


def test_gradients_against_differences():
    """The loss is linear in every single entry: a difference of steps of one is exact but for rounding."""
    r = np.random.default_rng(13)
    B, T, Dk, Dv, heads, L = 2, 300, 10, 6, 2, [300, 111]
    s = _inputs(r, "f32", B, T, heads, Dk, Dv)
    with ld.LinearAttention(B, heads, Dk, Dv, T, [0.9, 0.8], "f32") as m:
        def loss():
            y, S = m.forward(s["z"], _lengths(L), s["S0"])
            return float((_np(y) * _np(s["dy"])).sum() + (_np(S) * _np(s["dS"])).sum())
        got = m.backward(s["z"], _lengths(L), s["S0"], s["dy"], s["dS"])
        size = np.abs(_np(m.forward(s["z"], _lengths(L), s["S0"])[0]) * _np(s["dy"])).sum()
        for key, g in (("z", got["dz"]), ("S0", got["dS0"])):
            x = s[key]
            for _ in range(12):
                i = tuple(int(r.integers(0, n)) for n in x.shape)
                if key == "z":
                    i = (i[0], int(r.integers(0, L[i[0]])), i[2])
                old = float(x[i])
                values = []
                for h in (1.0, -1.0):
                    x[i] = old + h
                    values.append(loss())
                x[i] = old
                # each y is off by some 100 roundings of a magnitude a few times its size
                assert abs((values[0] - values[1]) / 2 - float(g[i])) <= 300 * U * size, (key, i)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_call_same_bits(dtype):
    r = np.random.default_rng(14)
    T, Dk, Dv, heads = 900, 64, 64, 2
    s = _inputs(r, dtype, 3, T, heads, Dk, Dv)
    L = _lengths([900, 430, 77])
    with ld.LinearAttention(3, heads, Dk, Dv, T, [0.9, 0.99], dtype) as m:
        def both():
            y, S = m.forward(s["z"], L, s["S0"])
            return dict(m.backward(s["z"], L, s["S0"], s["dy"], s["dS"]), y=y, S=S)
        want = both()
        for _ in range(3):
            got = both()
            assert all((got[k] == want[k]).all() for k in want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_operands_off_their_alignment(dtype):
    """Buffers that start at any element give the bits of aligned ones."""
    import torch
    r = np.random.default_rng(15)
    T, Dk, Dv, heads = 100, 16, 32, 2
    s = _inputs(r, dtype, 2, T, heads, Dk, Dv)

    def off(t):
        big = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        big[1:] = t.flatten()
        return big[1:].view(t.shape)
    with ld.LinearAttention(2, heads, Dk, Dv, T, [0.9, 0.99], dtype) as m:
        L = _lengths([T, 41])
        y, S = m.forward(s["z"], L, s["S0"])
        g = m.backward(s["z"], L, s["S0"], s["dy"], s["dS"])
        y2, S2 = m.forward(off(s["z"]), L, off(s["S0"]), out_S=off(s["S0"]), out_y=off(y))
        g2 = m.backward(off(s["z"]), L, off(s["S0"]), off(s["dy"]), off(s["dS"]), out={k: off(v) for k, v in g.items()})
        assert (y == y2).all() and (S == S2).all() and all((g[k] == g2[k]).all() for k in g)
        z1 = s["z"][:, 0].contiguous()
        a, b = m.step(z1, s["S0"]), m.step(off(z1), off(s["S0"]), out_S=off(s["S0"]))
        # a state off its alignment goes by single columns: rows are added in another order
        assert (a[1] == b[1]).all()
        mag = layer_util.attend(np.abs(_np(z1))[:, None], [1, 1], np.abs(_np(s["S0"])), np.float32([0.9, 0.99]), Dk, Dv)["y"][:, 0]
        assert (np.abs(_np(a[0]) - _np(b[0])) <= 2 * Dk * U * mag + 2 * HALF[dtype] * np.abs(_np(a[0]))).all()


def test_infinite_states_stay_in_their_columns():
    """fp32: an infinity in S0 reaches what its row and column reach, and nothing else."""
    r = np.random.default_rng(16)
    s = _inputs(r, "f32", 1, 40, 1, 8, 8)
    with ld.LinearAttention(1, 1, 8, 8, 40, 0.9, "f32") as m:
        y, S = m.forward(s["z"], None, s["S0"])
        s["S0"][0, 0, 3, 5] = float("inf")
        y2, S2 = m.forward(s["z"], None, s["S0"])
    assert S2[0, 0, 3, 5] == float("inf")
    keep = [i for i in range(8) if i != 5]
    assert (y2[..., keep] == y[..., keep]).all() and not y2[..., 5].isfinite().any()
    S2[0, 0, 3, 5] = S[0, 0, 3, 5]
    assert (S2 == S).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replays_of_a_graph(dtype):
    """Forward, backward and step captured, replayed with eager calls of another handle between, on new inputs."""
    import torch
    r = np.random.default_rng(17)
    T, Dk, Dv, heads = 600, 32, 48, 2
    s, fresh = _inputs(r, dtype, 2, T, heads, Dk, Dv), _inputs(r, dtype, 2, T, heads, Dk, Dv)
    L = _lengths([T, 222])
    m, other = (ld.LinearAttention(2, heads, Dk, Dv, T, [0.9, 0.99], dtype) for _ in range(2))
    z1 = s["z"][:, 0].contiguous()

    def calls(m, s, z1):
        y, S = m.forward(s["z"], L, s["S0"])
        g = m.backward(s["z"], L, s["S0"], s["dy"], s["dS"])
        return [y, S, g["dz"], g["dS0"], *m.step(z1, S)]
    calls(m, s, z1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(m, s, z1)
    for i in range(4):
        for k in s:
            s[k].copy_(fresh[k] if i % 2 else -fresh[k] * (i + 1))
        z1.copy_(s["z"][:, 1])
        want = calls(other, s, z1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all((a == b).all() for a, b in zip(out, want)), i
    del graph
    say(m.query(ld.ops.OPS_Q_WORKSPACE_BYTES))
    m.close(), other.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_products_under_the_mask_may_overflow(dtype):
    """q of early steps and k of late ones, whose product no step forms, are far apart in size: it overflows, and
    every result is finite."""
    import torch
    Dk, Dv, T = 16, 16, 60
    r = np.random.default_rng(18)
    s = _inputs(r, dtype, 1, T, 1, Dk, Dv)
    s["z"][:, :30, :Dk] *= 1e20               # q
    s["z"][:, 30:, Dk:2 * Dk] *= 1e20         # k
    s["z"][:, 30:, :Dk] *= 1e-20
    with ld.LinearAttention(1, 1, Dk, Dv, T, 0.9, dtype) as m:
        y, S = m.forward(s["z"], None, s["S0"])
        got = m.backward(s["z"], None, s["S0"], s["dy"], s["dS"])
        torch.cuda.synchronize()
        _compare(dict(got, y=y, S=S), s, [T], [0.9], Dk, Dv, dtype, tight=False)
