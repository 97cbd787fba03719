"""Sampling on the GPU against its definition in 64 bits, and where its weights are whole numbers exactly."""
import math

import numpy as np
import pytest

import paper_1810_08061_amd as ld
from tests import layer_util
from tests.layer_util import U

pytestmark = pytest.mark.gpu
INF = float("inf")


def _dev(a, dtype="f32"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if a.dtype == np.int32 else t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _sample(x, u, dtype="f32", **k):
    """Token and logp of rows x [N, V] (device or host); per-row filters given as lists go as tensors."""
    import torch
    x = x if isinstance(x, torch.Tensor) else _dev(np.asarray(x, np.float64), dtype)
    u = _dev(np.asarray(u, np.float64)) if not isinstance(u, torch.Tensor) else u
    for n, v in k.items():
        if isinstance(v, (list, np.ndarray)):
            k[n] = _dev(np.asarray(v, np.int32 if n == "top_k" else np.float64))
    with ld.TokenSample(x.shape[0], x.shape[1], "bf16" if x.dtype == torch.bfloat16 else "f32") as m:
        token, logp = m.sample(x, u, **k)
        assert m.status() == ld.OK
        return token.cpu().numpy(), logp.double().cpu().numpy()


FILTERS = [(a, b, c) for a in (0, 1) for b in (0, 1) for c in (0, 1)]


# one token, a piece of 16 bytes, a wave's, where 256 threads hand over to 1024, odd sizes
@pytest.mark.parametrize("V", [1, 2, 3, 8, 9, 63, 64, 65, 1000, 4095, 4096, 4097, 10007, 32768, 65537])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,p,m", FILTERS)
def test_against_the_definition(dtype, V, k, p, m):
    """Rows in which rounding decides (a sum or a ratio nearer than 1e-6 to what it is compared with) are passed over:
    weights are off by 2 roundings of their exponent (below 2^6: 2^-17 of a weight that is 2^-64; for one of 1e-3 of
    the largest 2^-20) and sums by less, as errors of single weights."""
    r = np.random.default_rng(V * 8 + 4 * k + 2 * p + m)
    N = 12
    x = _dev(r.standard_normal((N, V)) * 2.5, dtype)
    f32 = lambda a: a.astype(np.float32).astype(np.float64)
    u, T = f32(r.random(N)), f32(r.uniform(0.4, 1.3, N))
    ks = r.integers(0, min(V, 300) + 1, N).astype(np.int32) if k else None
    ps = f32(r.uniform(0.2, 0.99, N)) if p else None
    ms = f32(np.exp(r.uniform(-7, -1, N))) if m else None
    T[3] = 0.0
    token, logp = _sample(x, u, temperature=T, top_k=ks, top_p=ps, min_p=ms)
    xs, seen = x.double().cpu().numpy(), 0
    for n in range(N):
        want, lp, near = layer_util.sample(xs[n], u[n], T[n], ks[n] if k else 0, ps[n] if p else 1.0, ms[n] if m else 0.0)
        if near < 1e-6 and V > 1:
            continue
        seen += 1
        assert token[n] == want, (n, near)
        assert abs(logp[n] - lp) <= 1e-6 + 2 * U * abs(lp), n
    assert seen >= N // 2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 8, 64, 4096, 8192, 65536])
def test_equal_logits_are_exact(dtype, V):
    """V equal weights, V a power of two: the token is exactly u V rounded down, and every filter cuts by index."""
    r = np.random.default_rng(V)
    j = np.unique(np.concatenate([[0, V - 1, V // 2], r.integers(0, V, 20)]))
    u = j / V
    x = np.full((len(j), V), -1.25)
    assert (_sample(x, u, dtype)[0] == j).all()
    below = np.nextafter(np.float32(u), np.float32(0)).astype(np.float64)
    got = _sample(x, np.maximum(below, 0), dtype)[0]
    assert (got == np.maximum(np.where(u > 0, j - 1, 0), 0)).all()
    for n in (1, 2, 3, V // 2, V - 1):
        if 0 < n < V:
            got, lp = _sample(x, u, dtype, top_k=n)
            assert (got == np.floor(u * n)).all()              # u n has few bits: exact
            assert np.abs(lp + math.log(n)).max() <= 2 * U * math.log(V) + 1e-7
    if V >= 8:
        assert (_sample(x, u, dtype, top_p=0.5)[0] == np.floor(u * (V // 2))).all()
        assert (_sample(x, u, dtype, top_p=float(np.nextafter(np.float32(0.5), np.float32(1))))[0]
                == np.floor(u * (V // 2 + 1))).all()
        assert (_sample(x, u, dtype, top_k=V // 2, top_p=0.5)[0] == np.floor(u * (V // 4))).all()
        assert (_sample(x, u, dtype, min_p=1.0)[0] == j).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 20000])
def test_ties_at_the_cut_go_to_the_lowest_index(dtype, V):
    """Few distinct logits, many of each: top_k cuts inside a group of equal ones."""
    r = np.random.default_rng(V)
    x = r.integers(0, 4, (1, V)).astype(np.float64)
    order = np.lexsort((np.arange(V), -x[0]))
    for k in (1, 2, 5, V // 4 + 3, V // 2, V - 1):
        kept = np.sort(order[:k])
        w = np.exp(x[0, kept])
        c = np.cumsum(w) / w.sum()
        mid = np.float32((c + np.concatenate([[0], c[:-1]])) / 2).astype(np.float64)   # the middle of each token's share
        at = r.integers(0, k, 30)
        got = _sample(np.repeat(x, 30, 0), mid[at], dtype, top_k=k)[0]
        assert (got == kept[at]).all(), k


def test_ends_of_the_unit_interval():
    x = np.array([[-INF, 0.0, 1.0, -INF]] * 5)
    token, _ = _sample(x, [0.0, -1.0, 1.0, 2.0, float("nan")])
    assert token.tolist() == [1, 1, 2, 2, 1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 700, 9000])
def test_masked_rows(dtype, V):
    """-inf, NaN and the type's lowest value in masked places; nothing left; all but one left."""
    lowest = -3.3895314e38
    r = np.random.default_rng(V)
    for mask in (-INF, float("nan"), lowest, -1e9):
        x = r.standard_normal((4, V))
        x[0, :] = mask
        x[1, :] = mask
        x[1, V // 2] = -7.0
        x[2, ::2] = mask
        token, logp = _sample(x, [0.5] * 4, dtype)
        if mask == mask and mask > -INF:
            assert token[0] == V // 2 or V == 5 or abs(token[0] - V / 2) <= 1     # all equal
        else:
            assert token[0] == -1 and logp[0] == -INF
        assert token[1] == V // 2 and abs(logp[1]) <= 1e-6
        assert token[2] % 2 == 1 and 0 <= token[3] < V
        # every filter leaves the same
        token, logp = _sample(x, [0.5] * 4, dtype, top_k=3, top_p=0.9, min_p=0.1)
        assert token[1] == V // 2 and (token[0] == -1) == (not mask > -INF) and token[2] % 2 == 1


def test_infinite_logits_share():
    x = np.zeros((4, 40))
    x[:, [3, 17]] = INF
    token, logp = _sample(x, [0.0, 0.49, 0.5, 0.99])
    assert token.tolist() == [3, 3, 17, 17] and np.abs(logp + math.log(2)).max() <= 1e-6
    assert _sample(x, [0.9] * 4, top_k=1)[0].tolist() == [3] * 4
    assert _sample(x, [0.9] * 4, top_p=0.5)[0].tolist() == [3] * 4
    assert _sample(x, [0.9] * 4, temperature=0.0)[0].tolist() == [3] * 4


@pytest.mark.parametrize("V", [50, 6000])
def test_filters_out_of_range(V):
    import torch
    r = np.random.default_rng(V)
    x, u = r.standard_normal((6, V)), np.float32(r.random(6)).astype(np.float64)
    nan = float("nan")
    plain = _sample(x, u)[0]
    for k in ({"top_k": 0}, {"top_k": -5}, {"top_k": V}, {"top_k": V + 9}, {"top_p": 1.0}, {"top_p": 7.0}, {"top_p": nan}, {"min_p": 0.0},
              {"min_p": -1.0}, {"min_p": nan}, {"temperature": 1.0}):
        assert (_sample(x, u, **k)[0] == plain).all(), k
        n, v = next(iter(k.items()))
        assert (_sample(x, u, **{n: [v] * 6})[0] == plain).all(), k
    best = x.argmax(1)
    for k in ({"top_k": 1}, {"top_p": 0.0}, {"top_p": -1.0}, {"min_p": 1.0}, {"min_p": 5.0}, {"temperature": 0.0}, {"temperature": -2.0},
              {"temperature": nan}, {"temperature": 1e-45}, {"temperature": 1e-7}):
        token, logp = _sample(x, u, **k)
        assert (token == best).all() and (logp == 0).all(), k
    token, logp = _sample(x, np.arange(6) / 8, temperature=INF)    # all alike
    assert (np.abs(token - np.arange(6) / 8 * V) <= 1).all() and np.abs(logp + math.log(V)).max() < 1e-6


def test_far_apart_and_large_logits():
    """A constant on all logits changes nothing; a lone best token takes all."""
    r = np.random.default_rng(3)
    x = np.round(r.standard_normal((8, 5000)) * 64) / 64
    u = np.float32(r.random(8)).astype(np.float64)
    want = _sample(x, u, top_p=0.9)[0]
    assert (_sample(x + 2.0 ** 17, u, top_p=0.9)[0] == want).all()      # exact in fp32
    x[:, 77] = 300.0
    token, logp = _sample(x, u)
    assert (token == 77).all() and (logp == 0).all()


@pytest.mark.parametrize("T", [1e-30, 1e-36, 1.9e-37, 1.7e-37, 1e-37, 1e-38, 5e-39])
@pytest.mark.parametrize("filters", [{}, {"top_p": 0.9}, {"top_k": 6}, {"top_k": 9, "top_p": 0.8, "min_p": 0.01}])
def test_temperatures_near_the_end_of_fp32(T, filters):
    """Down to where 1 / T is no fp32 number, the differences of logits count in multiples of T. Weights are off by 2^-22
    (an exponential and its correction), log p by twice as much and its own rounding (below 16: 2^-21)."""
    r = np.random.default_rng(5)
    N, V = 24, 200
    x = np.full((N, V), -1.0)
    x[:, ::9] = -T * r.integers(0, 40, (N, 23)) / 8
    x = _dev(x)
    u, t = np.float32(r.random(N)).astype(np.float64), float(np.float32(T))
    token, logp = _sample(x, u, temperature=t, **filters)
    xs, seen = x.double().cpu().numpy(), 0
    f32 = lambda v: float(np.float32(v))
    for n in range(N):
        want, lp, near = layer_util.sample(xs[n], u[n], t, filters.get("top_k", 0), f32(filters.get("top_p", 1.0)),
                                           f32(filters.get("min_p", 0.0)))
        if near < 1e-6:
            continue
        seen += 1
        assert token[n] == want and abs(logp[n] - lp) <= 2.0 ** -20, (n, token[n], want, logp[n], lp)
    assert seen > N // 2


@pytest.mark.parametrize("top", [1, 2, 63, 64, 65, 127, 128, 129, 300, 513])
@pytest.mark.parametrize("spread", [0.0, 0.01, 3.0])
@pytest.mark.parametrize("V", [2000, 9001])
def test_few_and_more_tokens_far_above_the_others(top, spread, V):
    """As many as can be compared one by one, one more, and fewer, in one range of the histogram and in several,
    with the cuts of every filter in them and behind. Tolerance of log p: that of the temperatures above."""
    r = np.random.default_rng(top)
    x = np.full((1, V), -30.0) - r.random((1, V))
    x[0, r.permutation(V)[:top]] = 4 - spread * np.arange(top) / top
    x = np.repeat(np.float32(x).astype(np.float64), 12, 0)
    u = np.float32(r.random(12)).astype(np.float64)
    f32, seen = lambda v: float(np.float32(v)), 0
    for f in ({"top_k": top}, {"top_k": max(top - 1, 2)}, {"top_k": top + 1}, {"top_p": 0.61}, {"top_p": 0.999}, {"top_k": top + 9, "top_p": 0.53},
              {"top_k": max(top // 2, 2), "top_p": 0.37, "min_p": 0.2}, {"top_p": 0.77, "min_p": 0.3}):
        token, logp = _sample(x, u, **f)
        for n in range(12):
            want, lp, near = layer_util.sample(x[n], u[n], 1.0, f.get("top_k", 0), f32(f.get("top_p", 1.0)), f32(f.get("min_p", 0.0)))
            if near < 1e-6:
                continue
            seen += 1
            assert token[n] == want and abs(logp[n] - lp) <= 2.0 ** -20, (f, n, token[n], want, logp[n], lp)
    assert seen > 48


def _nan_rows(V):
    x = np.full((5, V), float("nan"))
    x[0, V // 2] = 1.0
    x[1, ::3] = np.arange(len(x[1, ::3])) % 5
    x[2, :] = np.where(np.arange(V) % 2, x[2], -INF)
    x[3, V - 1] = x[3, 0] = -3e38
    x[4, :7] = 3e38
    return x


@pytest.mark.parametrize("V", [9, 1001, 5000])
@pytest.mark.parametrize("filters", [{}, {"top_p": 0.7}, {"top_k": 3}, {"top_k": 8, "top_p": 0.6}, {"min_p": 0.1}])
def test_no_numbers_are_never_taken(V, filters):
    """Rows of NaN but for a few logits, among them the largest and smallest finite ones."""
    x, u = _nan_rows(V), [0.3, 0.55, 0.3, 0.8, 0.45]
    token, logp = _sample(x, u, **filters)
    xs = np.float32(x).astype(np.float64)
    for n in range(5):
        want, lp, near = layer_util.sample(xs[n], float(np.float32(u[n])), 1.0, filters.get("top_k", 0),
                                           float(np.float32(filters.get("top_p", 1.0))), float(np.float32(filters.get("min_p", 0.0))))
        assert near > 1e-6 and token[n] == want, (n, token[n], want)
        assert logp[n] == lp or abs(logp[n] - lp) < 2.0 ** -20 * max(1.0, abs(lp)), (n, logp[n], lp)


@pytest.mark.parametrize("V", [700, 9000, 17001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,p,m", FILTERS)
def test_a_row_gives_the_same_in_any_batch(dtype, V, k, p, m):
    """Workgroups differ with the number of rows; sums are of whole numbers, so tokens and log p do not."""
    import torch
    r = np.random.default_rng(V + 4 * k + 2 * p + m)
    N = 700
    x, u = _dev(r.standard_normal((N, V)) * 3, dtype), _dev(r.random(N))
    f = {"temperature": _dev(r.uniform(0.3, 1.2, N))}
    if k:
        f["top_k"] = _dev(r.integers(0, 600, N).astype(np.int32))
    if p:
        f["top_p"] = _dev(r.uniform(0.2, 1.0, N))
    if m:
        f["min_p"] = _dev(r.uniform(0.0, 0.2, N))
    token, logp = _sample(x, u, **f)
    for n in (300, 9):
        at = torch.arange(n, device="cuda") * (N // n)
        some = _sample(x[at], u[at], **{name: v[at] for name, v in f.items()})
        assert (some[0] == token[at.cpu().numpy()]).all() and (some[1] == logp[at.cpu().numpy()]).all(), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_off_their_alignment(dtype):
    """Odd V: every row starts elsewhere; and a buffer that starts at any element."""
    import torch
    r = np.random.default_rng(4)
    for V in (33, 5001):
        x = _dev(r.standard_normal((9, V)), dtype)
        u = _dev(r.random(9))
        big = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")
        big[1:] = x.flatten()
        for k in ({}, {"top_k": 7}, {"top_p": 0.7}):
            a, b = _sample(x, u, **k), _sample(big[1:].view(x.shape), u, **k)
            assert (a[0] == b[0]).all() and (a[1] == b[1]).all()
            each = np.concatenate([_sample(x[n:n + 1].clone(), u[n:n + 1].clone(), **k)[0] for n in range(9)])
            assert (a[0] == each).all()


def test_shares_follow_the_probabilities():
    """u on a fine grid: each token as often as its probability says, to one point of the grid at either end."""
    r = np.random.default_rng(5)
    x = np.repeat(r.standard_normal((1, 20)), 4096, 0)
    token, logp = _sample(x, np.arange(4096) / 4096, top_k=11, temperature=0.8)
    n = np.bincount(token, minlength=20)
    order = np.argsort(-x[0])[:11]
    p = np.zeros(20)
    p[order] = np.exp(x[0, order] / 0.8)
    p /= p.sum()
    assert (np.abs(n - 4096 * p) <= 1).all()
    assert np.abs(logp - np.log(p[token])).max() <= 1e-6


def test_wide_vocabulary():
    """More tokens than one piece a lane of every segment: V of 2^20 and more."""
    V = (1 << 20) + 3
    x = np.zeros((2, V), np.float32)
    u = np.float32([0.25, 0.75]).astype(np.float64)
    assert (_sample(x, u)[0] == np.floor(u * V)).all()
    assert (_sample(x, u, top_k=1 << 19)[0] == np.floor(u * (1 << 19))).all()
    got = _sample(x, u, top_p=0.5)[0]
    assert (got == np.floor(u * ((V + 1) // 2))).all()


def test_replays_of_a_graph():
    import torch
    g = torch.Generator(device="cuda").manual_seed(6)
    x, u, p = torch.randn((20, 9000), generator=g, device="cuda"), torch.rand((20,), generator=g, device="cuda"), torch.full((20,), 0.8, device="cuda")
    m, other = ld.TokenSample(20, 9000, "f32"), ld.TokenSample(20, 9000, "f32")
    call = lambda m: m.sample(x, u, top_k=100, top_p=p, min_p=0.01)
    call(m)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(m)
    m.sample(x, u)                  # other filters on the handle do not reach the captured call
    for _ in range(4):
        x.normal_(generator=g)
        u.uniform_(generator=g)
        want = call(other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (out[0] == want[0]).all() and (out[1] == want[1]).all()
    del graph
    m.close(), other.close()
