"""A beam search step over vocabularies masked with large finite values (whole waves, whole slices and
all but one token) and with logits that lie anywhere, against all candidates in 64 bits, in the very order.

The bound knows the logits that are not masked only.  The terms' exponents are within a few units of U of their size, and
those of 2^-30 and less do not matter: 30 x 4 U of a term, 64 of a thread added one by one, then ten
additions of sums: 4e-6 and 80 U of the sum, which its log has absolutely; then roundings of that log (at most 18 for
2^24 tokens), of the logit and of the score, and the sums'."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from tests import ops_util as ou
from tests.gpu_util import say
from tests.test_gpu_beam import _step

pytestmark = pytest.mark.gpu


def _candidates(x, scores):
    """[K V] in 64 bits; the largest logit and the log apart, so that no size of the logits is lost."""
    m = x.max(1, keepdims=True)
    with np.errstate(over="ignore"):
        log = np.log(np.exp(x - m).sum(1, keepdims=True))
        return (scores[:, None] + ((x - m) - log)).reshape(-1)


def _check_order(m, logits, scores, spread, name):
    """spread: the largest distance from its beam's largest logit of one that is not masked."""
    import torch
    B, K, V = logits.shape
    got, parent, token, done, _ = _step(m, logits, scores, torch.zeros((B, K), dtype=torch.uint8))
    x, s = logits.double().numpy(), scores.double().numpy()
    compared = 0
    for b in range(B):
        c = _candidates(x[b], s[b])
        order = np.argsort(-c, kind="stable")[:K + 1]
        best = c[order]
        tol = 4e-6 + 80 * ou.U + 4 * ou.U * (spread + 18 + np.abs(s[b]).max() + np.abs(best[:K]).max())
        at = parent[b].long().numpy() * V + token[b].long().numpy()
        g = got[b].double().numpy()
        err = np.abs(g - best[:K]).max()
        say(f"{name} {b}: max error {err:.3g}, bound {tol:.3g}")
        assert err <= tol, (name, b)
        assert (np.abs(c[at] - best[:K]) <= 2 * tol).all(), (name, b)
        # the very order, where rounding cannot change it; equal logits of one beam are ties
        gaps = best[:-1] - best[1:]
        if ((gaps > 2 * tol) | (gaps == 0)).all():
            assert (at == order[:K]).all(), (name, b)
            compared += 1
    assert compared >= B - B // 4, (name, compared)
    assert not done.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", ["lowest", -1e38, -1e30, -1e10, -3e9, -1e6, 1e38])
@pytest.mark.parametrize("V,K", [(600, 4), (4096, 8), (16384, 3), (70000, 2), (5003, 16)])
def test_large_masks(V, K, mask, dtype):
    """mask 1e38: a token far above all others (its beam has no other candidate above -1e38)."""
    import torch
    g = torch.Generator().manual_seed(V + K)
    et = torch.float32 if dtype == "f32" else torch.bfloat16
    value = torch.finfo(et).min if mask == "lowest" else mask
    B = 8
    logits = (torch.randn((B, K, V), generator=g) * 3).to(et).float()
    scores = -5 + torch.randn((B, K), generator=g) * 2
    if mask == 1e38:
        at = torch.randint(0, V, (B, K, 1), generator=g)
        one = torch.zeros((B, K, V), dtype=torch.bool).scatter_(2, at, True)
        logits = torch.where(one, value, logits).to(et)      # one candidate a beam: its score
        with ld.BeamSearch(B, K, V, dtype) as m:
            got, parent, token, _, _ = _step(m, logits, scores, torch.zeros((B, K), dtype=torch.uint8))
        order = scores.argsort(1, descending=True)
        assert (parent.long() == order).all() and (got == scores.gather(1, order)).all()
        assert (token.long() == at[..., 0].gather(1, order)).all()
        return
    t = torch.arange(V)
    best = logits.argmax(2, keepdim=True)
    masked = {
        "waves": ((t // 256) % 2 == 1).expand(B, K, V),                       # every other 256 tokens
        "range": (t >= V // 5).expand(B, K, V),                              # all from a token on: whole waves, slices
        "tail": (t < V - V // 7).expand(B, K, V),
        "beams": (t[None] // 512 % 3 == (torch.arange(K) % 3)[:, None]).expand(B, K, V),
        "one": torch.ones((B, K, V), dtype=torch.bool).scatter(2, best, False),
    }
    with ld.BeamSearch(B, K, V, dtype) as m:
        for name, where in masked.items():
            x = torch.where(where, value, logits)
            # one token in [0, 2 K) of each beam stays: there is always a choice
            keep = torch.randint(0, min(V, 2 * K), (B, K, 1), generator=g)
            if name != "one":
                x.scatter_(2, keep, logits.gather(2, keep))
            _check_order(m, x.to(et), scores, 40.0, name)
        assert m.status() == ld.OK


@pytest.mark.parametrize("V,K", [(600, 4), (16384, 3), (70000, 2), (5003, 16)])
@pytest.mark.parametrize("offset", [100.0, -300.0, 1000.0, -60000.0, 2.0 ** 17, -2.0 ** 19])
def test_a_constant_on_a_beams_logits_changes_nothing(V, K, offset):
    """Every beam's logits lie elsewhere.  The logits are multiples of 2^-3, so the shifted ones are exact."""
    import torch
    g = torch.Generator().manual_seed(V + K)
    B = 8
    logits = (torch.randn((B, K, V), generator=g) * 24).round() / 8
    scores = -5 + torch.randn((B, K), generator=g) * 2
    shifted = logits + (offset * torch.arange(K) / K).round()[None, :, None]
    with ld.BeamSearch(B, K, V, "f32") as m:
        _check_order(m, shifted, scores, 40.0, f"offset {offset:g}")
        fin = torch.zeros((B, K), dtype=torch.uint8)
        a, b = _step(m, logits, scores, fin), _step(m, shifted, scores, fin)
        assert (a[1] == b[1]).all() and (a[2] == b[2]).all()
        assert m.status() == ld.OK


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_beam_with_all_its_tokens_masked(dtype):
    """Equal logits are equal chances, whatever their value: score - log V, the lowest tokens first."""
    import torch
    et = torch.float32 if dtype == "f32" else torch.bfloat16
    K = 6
    for V in (40, 3000, 33000):
        logits = torch.zeros((1, K, V))
        for k, x in enumerate((0.0, 40.0, -1e6, -1e10, -1e30, torch.finfo(et).min)):
            logits[0, k] = x
        scores = torch.tensor([[-1.0, -1.5, -2.0, -2.5, -3.0, -3.5]])
        with ld.BeamSearch(1, K, V, dtype) as m:
            for shift in range(K):      # each beam is the best one once
                s = scores.roll(shift, 1)
                _check_order(m, logits.to(et), s, 0.0, f"all masked, V {V}")
                got, parent, token, _, _ = _step(m, logits.to(et), s, torch.zeros((1, K), dtype=torch.uint8))
                assert (parent[0] == shift).all() and token[0].tolist() == list(range(K))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,V", [(1, 1), (1, 2), (3, 3), (4, 63), (2, 64), (5, 65), (8, 1000), (32, 33), (3, 255), (16, 4096),
                                 (7, 4097), (4, 8193), (2, 50001), (32, 20000), (8, 32768), (4, 300)])
def test_the_very_order(K, V, dtype):
    """Ordinary logits: each sequence's choice in order, equal logits of a beam by the lowest token."""
    import torch
    g = torch.Generator().manual_seed(10 * K + V)
    logits = (torch.randn((6, K, V), generator=g) * 3).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    scores = -5 + torch.randn((6, K), generator=g)
    with ld.BeamSearch(6, K, V, dtype) as m:
        _check_order(m, logits, scores, 40.0, "order")
        assert m.status() == ld.OK
