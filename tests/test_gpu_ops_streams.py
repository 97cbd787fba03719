"""The loop's and the operators' calls that name their stream: what they allocate belongs to that stream (torch's
allocator would hand memory of the current stream out again while the named one still uses it, and
may give the call memory that the current stream's earlier work still uses), and the results
are those of the current stream's calls."""
import pytest

import paper_1810_08061_amd as ld

pytestmark = pytest.mark.gpu


def _pool(t):
    """The address of the stream that owns a tensor's memory."""
    import torch
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no such memory")


def _flat(x):
    if isinstance(x, dict):
        x = list(x.values())
    return [t for q in x for t in _flat(q)] if isinstance(x, (list, tuple)) else [x]


def _calls():
    """Per operator: its handle and calls, each a function of the stream that returns what it allocated."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    B, T, H, V, K = 3, 40, 24, 50, 4
    L = torch.tensor([T, 7, 0], dtype=torch.int32, device="cuda")
    z, h0, dy, dh, zs = normal(B, T, 3 * H), normal(B, H), normal(B, T, H), normal(B, H), normal(B, 3 * H)
    scan = ld.GatedScan(B, H, T, "f32")
    yield scan, [lambda **k: scan.forward(z, L, h0, **k), lambda **k: scan.forward_train(z, L, h0, **k),
                 lambda **k: scan.backward(z, L, h0, dy, dh, **k), lambda **k: scan.step(zs, h0, **k)]
    tok = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    table = normal(V, H)
    embed = ld.TokenEmbed(B, T, V, H, "f32")
    yield embed, [lambda **k: embed.forward(tok, L, table, **k), lambda **k: embed.backward(tok, L, dy, **k)]
    p = [normal(1000), normal(7, 5)]
    grads = [normal(1000), normal(7, 5)]
    opt = ld.AdamW(p, state_bits=8)

    def adamw(**k):
        with torch.no_grad():
            for q, i in zip(p, (1.0, 2.0)):
                q.fill_(i)
            for s in opt.m + opt.v:
                s.view(torch.uint8).zero_()
        opt.steps_done = 0
        torch.cuda.synchronize()
        opt.step(grads, 0.1, **k)
        return opt.states(**k)
    yield opt, [adamw]
    logits, scores, fin = normal(B, K, V), normal(B, K), torch.zeros((B, K), dtype=torch.uint8, device="cuda")
    state = normal(B, K, 9)
    D = 8
    w = [normal(B, T, D), L, normal(D, 4 * H) * 0.2, normal(H, 4 * H) * 0.2, normal(4 * H), h0, dh]
    loop = ld.LstmDyn(B, D, H, T, "f32")
    stop = normal(H)
    yield loop, [lambda **k: loop.forward(*w, **k), lambda **k: loop.forward_seq(*w, **k),
                 lambda **k: loop.forward_stop(*w, stop, -0.5, with_seq=True, **k),
                 lambda **k: loop.forward_train(*w, with_seq=True, **k),
                 lambda **k: loop.backward(*w, dh, h0, dy, **k)]
    beams = ld.BeamSearch(B, K, V, "f32", end=3)
    yield beams, [lambda **k: beams.step(logits, scores, fin, [state], **k)]


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
            assert not hasattr(handle, "status") or handle.status() == ld.OK


def test_the_default_stream_by_its_address():
    import torch
    other = torch.cuda.Stream()
    for handle, calls in _calls():
        with handle:
            want = [[t.clone() for t in _flat(f())] for f in calls]
            torch.cuda.synchronize()
            with torch.cuda.stream(other):
                for i, f in enumerate(calls):
                    got = _flat(f(stream=0))
                    torch.cuda.synchronize()
                    assert all(_pool(t) == 0 for t in got), (type(handle).__name__, i)
                    assert all((a == b).all() for a, b in zip(got, want[i])), (type(handle).__name__, i)
