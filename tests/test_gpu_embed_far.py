"""Lookups on both sides of the size from which their stores bypass the caches: rows are copied exactly."""
import pytest

import paper_1810_08061_amd as ld

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [("bf16", 1024), ("bf16", 1022), ("bf16", 1023), ("f32", 512), ("f32", 510), ("f32", 511)])
@pytest.mark.parametrize("mib", [200, 300])
def test_lookup(dtype, D, mib):
    import torch
    et = torch.bfloat16 if dtype == "bf16" else torch.float32
    B, V = 5, 1000
    T = (mib << 20) // (B * D * (2 if dtype == "bf16" else 4))
    g = torch.Generator(device="cuda").manual_seed(mib + D)
    table = torch.randn((V, D), generator=g, device="cuda").to(et)
    tok = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    L = torch.tensor([T, 0, 1, T - 1, T // 2], dtype=torch.int32, device="cuda")
    with ld.TokenEmbed(B, T, V, D, dtype, scale=2.0) as m:
        x = m.forward(tok, L, table)
        for b in range(B):
            n = int(L[b])
            assert (x[b, :n] == table[tok[b, :n].long()] * 2).all() and not x[b, n:].any()
        assert m.status() == ld.OK
