"""The operators where offsets pass 32 bits: more than 2^31 elements in an operand, checked against the
same rows in small calls."""
import pytest

import paper_1810_08061_amd as ld

pytestmark = pytest.mark.gpu


def _enough(gib):
    import torch
    free, _ = torch.cuda.mem_get_info()
    if free < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_scan():
    import torch
    _enough(24)
    B, T, H = 3, 16384, 16384
    g = torch.Generator(device="cuda").manual_seed(0)
    z1 = torch.empty((1, T, 3 * H), device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    dy1 = torch.empty((1, T, H), device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    h1 = torch.empty((1, H), device="cuda").normal_(generator=g)
    L = torch.tensor([0, T, T], dtype=torch.int32, device="cuda")
    with ld.GatedScan(1, H, T, "bf16") as m:
        y1, e1 = m.forward_train(z1, L[1:2], h1)
        d1 = m.backward(z1, L[1:2], h1, dy1, h1)
    z, dy, h = z1.expand(B, -1, -1).contiguous(), dy1.expand(B, -1, -1).contiguous(), h1.expand(B, -1).contiguous()
    assert z.numel() > 2 ** 31
    with ld.GatedScan(B, H, T, "bf16") as m:
        y, e = m.forward_train(z, L, h)
        d = m.backward(z, L, h, dy, h)
        assert m.status() == ld.OK
    for b in (1, 2):
        assert (y[b] == y1[0]).all() and (e[b] == e1[0]).all()
        assert (d["dz"][b] == d1["dz"][0]).all() and (d["dh0"][b] == d1["dh0"][0]).all()
    assert (y[0] == 0).all() and (e[0] == h1[0]).all() and (d["dz"][0] == 0).all() and (d["dh0"][0] == h1[0]).all()


def test_embed():
    import torch
    _enough(20)
    B, T, V, D = 2, 40, 70000, 32768
    g = torch.Generator(device="cuda").manual_seed(1)
    table = torch.empty((V, D), device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    assert table.numel() > 2 ** 31
    tok = torch.randint(V - 20, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    tok[0, 0], tok[1, 39] = V - 1, 0
    dx = torch.randint(-4, 5, (B, T, D), generator=g, device="cuda").float()     # sums are exact
    with ld.TokenEmbed(B, T, V, D, "bf16", scale=2.0) as m:
        assert (m.forward(tok, None, table) == table[tok.long()] * 2).all()
        d = m.backward(tok, None, dx)
        assert m.status() == ld.OK
    seen = tok.unique()
    for v in seen.tolist():
        assert (d[v] == 2 * dx[tok == v].sum(0)).all()
    d[seen.long()] = 0
    assert d.abs().amax() == 0


def test_more_places_than_the_sort_has_tiles():
    """Over a million places: every block of the sort takes several tiles, one after another."""
    import torch
    B, T, V, D = 3, 500001, 5003, 4
    g = torch.Generator(device="cuda").manual_seed(4)
    tok = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    tok[1] = torch.arange(T, device="cuda", dtype=torch.int32) // 200 % V       # long runs of one token
    L = torch.tensor([T, T - 7, 300000], dtype=torch.int32, device="cuda")
    dx = torch.randint(-4, 5, (B, T, D), generator=g, device="cuda").float()     # sums are exact
    on = torch.arange(T, device="cuda")[None] < L[:, None]
    want = torch.zeros((V, D), dtype=torch.float64, device="cuda")
    want.index_add_(0, tok[on].long(), dx[on].double())
    with ld.TokenEmbed(B, T, V, D, "f32", scale=0.5) as m:
        assert (m.backward(tok, L, dx).double() == want * 0.5).all()
        assert m.status() == ld.OK


def test_beam():
    """The largest vocabulary and number of beams: indices up to 2^32, most logits equal."""
    import torch
    _enough(20)
    K, V = 32, 2 ** 27 - 1
    g = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.zeros((1, K, V), device="cuda", dtype=torch.bfloat16)
    at = torch.randint(1, V - 1, (K,), generator=g, device="cuda").tolist()
    for k, t in enumerate(at):
        logits[0, k, t] = 1.0 + k          # the last beam's is the best
    logits[0, 31, V - 1] = 40.0            # the very last candidate
    scores = torch.zeros((1, K), device="cuda")
    with ld.BeamSearch(1, K, V, "bf16") as m:
        _, parent, token, _, _ = m.step(logits, scores, torch.zeros((1, K), dtype=torch.uint8, device="cuda"))
    # the tokens above the zeros, one a beam and two in the last, by score - log(sum of exps)
    import math
    tops = [{at[k]: 1.0 + k} for k in range(K)]
    tops[31][V - 1] = 40.0
    want = []
    for k in range(K):
        lse = math.log(V - len(tops[k]) + sum(math.exp(x) for x in tops[k].values()))
        want += [(x - lse, k, t) for t, x in tops[k].items()]
    want.sort(key=lambda q: -q[0])
    assert list(zip(parent[0].tolist(), token[0].tolist())) == [q[1:] for q in want[:K]]


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw(bits):
    import torch
    _enough(60)
    n, tail = 2 ** 31 + 4099, 5000
    p = torch.zeros(n, device="cuda")
    grad = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(3)
    first = n - tail - (n - tail) % 256       # a block's start
    grad[first:].normal_(generator=g)
    small, sg = p[first:].clone(), grad[first:].clone()
    with ld.AdamW([p], state_bits=bits) as a, ld.AdamW([small], state_bits=bits) as b:
        for _ in range(2):
            a.step([grad], 0.1)
            b.step([sg], 0.1)
        assert (p[first:] == small).all() and p[:first].abs().amax() == 0
        assert all((x[0][first:] == y[0]).all() for x, y in zip(a.states(), b.states()))
