"""The layer's wrappers refuse a tensor of another GPU than their handle's, argument by argument, before any call of
the library.  The tensors are CPU tensors that say which device they are on; the library is not called."""
import pytest
import torch

import paper_1810_08061_amd as ld
from tests.test_ops_devices_cpu import F, I, _tensor, no_library  # noqa: F401  (a fixture)

B, T, h, Dk, Dv, D, N, V = 2, 3, 2, 4, 5, 6, 3, 7
W = h * (2 * Dk + Dv)
SHAPES = {"z": ((B, T, W), F), "lengths": ((B,), I), "S0": ((B, h, Dk, Dv), F), "out_S": ((B, h, Dk, Dv), F), "out_y": ((B, T, h * Dv), F),
          "dy": ((B, T, h * Dv), F), "dS": ((B, h, Dk, Dv), F), "dz": ((B, T, W), F), "dS0": ((B, h, Dk, Dv), F), "z1": ((B, W), F),
          "y1": ((B, h * Dv), F), "x": ((B, T, D), F), "w": ((D,), F), "b": ((D,), F), "y": ((B, T, D), F), "g": ((B, T, D), F),
          "dx": ((B, T, D), F), "dw": ((D,), F), "db": ((D,), F), "g1": ((4,), F), "g2": ((2, 3), F), "o1": ((4,), F), "o2": ((2, 3), F),
          "logits": ((N, V), F), "u": ((N,), F), "t": ((N,), F), "k": ((N,), I), "p": ((N,), F), "m": ((N,), F)}
attend = lambda: ld.LinearAttention(B, h, Dk, Dv, T, 0.5, "f32")
norm = lambda: ld.LayerNorm(B, T, D, "f32")
clip = lambda: ld.GradClip([torch.empty(4), torch.empty(2, 3)], 1.0)


def _adamw(_, a, b):
    p = [_tensor((4,)), _tensor((2, 3))]
    return ld.AdamW(p).step([a, b], 0.1, clip=clip())


CALLS = {
    "attend forward": (attend, "z lengths S0 out_S out_y", lambda m, *a: m.forward(*a)),
    "attend backward": (attend, "z lengths S0 dy dS dz dS0",
                        lambda m, z, L, S, dy, dS, dz, dS0: m.backward(z, L, S, dy, dS, out={"dz": dz, "dS0": dS0})),
    "attend step": (attend, "z1 S0 out_S y1", lambda m, *a: m.step(*a)),
    "norm forward": (norm, "x lengths w b y", lambda m, *a: m.forward(*a)),
    "norm backward": (norm, "x lengths w g dx dw db",
                      lambda m, x, L, w, g, dx, dw, db: m.backward(x, L, w, g, out={"dx": dx, "dweight": dw, "dbias": db})),
    "clip norm": (clip, "g1 g2", lambda m, *a: m.norm(a)),
    "clip clip": (clip, "g1 g2 o1 o2", lambda m, a, b, c, d: m.clip([a, b], out=[c, d])),
    "adamw clip": (lambda: None, "g1 g2", _adamw),
    "sample": (lambda: ld.TokenSample(N, V, "f32"), "logits u t k p m", lambda m, x, u, t, k, p, q: m.sample(x, u, t, k, p, q)),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_tensor_of_another_device_is_refused(name, no_library):  # noqa: F811
    make, args, call = CALLS[name]
    args = args.split()
    call(make(), *[_tensor(*SHAPES[a]) for a in args])
    runs = [n for n in no_library if not n.endswith(("create", "destroy"))]
    assert len(runs) == (2 if name in ("clip clip", "adamw clip") else 1), no_library
    for i, a in enumerate(args):
        others = [_tensor(*SHAPES[x]) for x in args]
        others[i].number = 1
        m = make()
        del no_library[:]
        with pytest.raises(ValueError, match="device"):
            call(m, *others)
        assert not [n for n in no_library if not n.endswith(("create", "destroy"))], a
