"""The first forward for training of a scan allocates: under a capture it is refused by name, and the
capture goes on; after an eager call it is captured like any other."""
import pytest

import paper_1810_08061_amd as ld

pytestmark = pytest.mark.gpu


def test_the_first_forward_for_training_under_a_capture():
    import torch
    B, T, H = 3, 300, 40
    g = torch.Generator(device="cuda").manual_seed(0)
    z = torch.randn((B, T, 3 * H), generator=g, device="cuda")
    L = torch.tensor([T, 0, 17], dtype=torch.int32, device="cuda")
    h0, dy = torch.randn((B, H), generator=g, device="cuda"), torch.randn((B, T, H), generator=g, device="cuda")
    x = torch.ones(100, device="cuda")
    with ld.GatedScan(B, H, T, "f32") as m:
        graph, code = torch.cuda.CUDAGraph(), None
        with torch.cuda.graph(graph):
            y, h = m.forward(z, L, h0)
            try:
                m.forward_train(z, L, h0)
            except ld.LstmDynError as e:
                code = e.code
            x2 = x * 2
        assert code == ld.ERR_INVALID
        for i in range(3):
            x.fill_(i)
            z.mul_(0.9)
            graph.replay()
            torch.cuda.synchronize()
            want, wh = m.forward(z, L, h0)
            assert (y == want).all() and (h == wh).all() and (x2 == 2 * i).all()
        m.forward_train(z, L, h0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, h = m.forward_train(z, L, h0)
            d = m.backward(z, L, h0, dy)
        for i in range(3):
            z.mul_(0.9)
            graph.replay()
            torch.cuda.synchronize()
            want, wh = m.forward_train(z, L, h0)
            assert (y == want).all() and (h == wh).all()
            w = m.backward(z, L, h0, dy)
            assert all((d[k] == w[k]).all() for k in w)
        assert m.status() == ld.OK
