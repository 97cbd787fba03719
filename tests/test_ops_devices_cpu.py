"""The loop's and the operators' wrappers refuse a tensor of another GPU than their handle's, argument by argument, before
any call of the library: its address would be read by kernels of the handle's GPU.  The tensors
here are CPU tensors that say which device they are on; the library is not called."""
import types

import pytest
import torch

import paper_1810_08061_amd as ld
from paper_1810_08061_amd import ops


class OnDevice(torch.Tensor):
    number = 0
    is_cuda = True

    def get_device(self):
        return self.number


def _tensor(shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


F, I = torch.float32, torch.int32
B, T, H, V, K = 2, 3, 4, 5, 2
SHAPES = {"z": ((B, T, 3 * H), F), "lengths": ((B,), I), "h0": ((B, H), F), "out_h": ((B, H), F), "out_y": ((B, T, H), F),
          "dy": ((B, T, H), F), "d_out_h": ((B, H), F), "z1": ((B, 3 * H), F), "h": ((B, H), F), "y1": ((B, H), F),
          "tokens": ((B, T), I), "table": ((V, H), F), "out_x": ((B, T, H), F), "dx": ((B, T, H), F),
          "out": ((V, H), F), "dz": ((B, T, 3 * H), F), "dh0": ((B, H), F), "logits": ((B, K, V), F),
          "scores": ((B, K), F), "finished": ((B, K), torch.uint8), "state": ((B, K, 3), F), "dst": ((B, K, 3), F),
          "p": ((7,), F), "copy": ((7,), torch.bfloat16), "g": ((7,), F)}

scan = lambda: ld.GatedScan(B, H, T, "f32")
embed = lambda: ld.TokenEmbed(B, T, V, H, "f32")
CALLS = {
    "scan forward": (scan, "z lengths h0 out_h out_y", lambda m, *a: m.forward(*a)),
    "scan forward_train": (scan, "z lengths h0 out_h out_y", lambda m, *a: m.forward_train(*a)),
    "scan backward": (scan, "z lengths h0 dy d_out_h dz dh0",
                      lambda m, z, L, h, dy, dh, dz, dh0: m.backward(z, L, h, dy, dh, out={"dz": dz, "dh0": dh0})),
    "scan step": (scan, "z1 h out_h y1", lambda m, *a: m.step(*a)),
    "embed forward": (embed, "tokens lengths table out_x", lambda m, *a: m.forward(*a)),
    "embed backward": (embed, "tokens lengths dx out", lambda m, *a: m.backward(*a)),
    "adamw": (lambda: None, "p copy g", lambda _, p, c, g: ld.AdamW([p], [c]).step([g], 0.1)),
    "beam": (lambda: ld.BeamSearch(B, K, V, "f32"), "logits scores finished state dst",
             lambda m, x, s, f, a, b: m.step(x, s, f, [a], [b])),
}


@pytest.fixture
def no_library(monkeypatch):
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0
    ops._t()
    monkeypatch.setattr(ops, "_ready", Library())
    monkeypatch.setattr(ops, "_stream", lambda device: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return called


@pytest.mark.parametrize("name", CALLS)
def test_a_tensor_of_another_device_is_refused(name, no_library):
    make, args, call = CALLS[name]
    args = args.split()
    tensors = [_tensor(*SHAPES[a]) for a in args]
    call(make(), *tensors)
    kind = name.split()[0]
    runs = [n for n in no_library if n.startswith(f"lstm_dyn_{kind}_") and not n.endswith(("create", "destroy"))]
    assert len(runs) == 1, no_library         # with all of them on the handle's device it goes through
    for i, a in enumerate(args):
        others = list(tensors)
        others[i] = _tensor(*SHAPES[a])
        others[i].number = 1
        m = make()
        del no_library[:]
        with pytest.raises(ValueError, match="device"):
            call(m, *others)
        assert not [n for n in no_library if not n.endswith(("create", "destroy"))], a


def test_the_loops_wrapper_refuses_them_too(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ld, "lstm_dyn_create_cell", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: types.SimpleNamespace(cuda_stream=0))
    called = []
    for f in ("lstm_dyn_forward", "lstm_dyn_forward_seq", "lstm_dyn_forward_train", "lstm_dyn_backward", "lstm_dyn_forward_stop"):
        monkeypatch.setattr(ld, f, lambda *a, f=f: called.append(f))
    D = 3
    m = ld.LstmDyn(B, D, H, T, "f32")
    weights = {"x": (B, T, D), "lengths": (B,), "W": (D, 4 * H), "U": (H, 4 * H), "b": (4 * H,), "h0": (B, H), "c0": (B, H)}
    outs = {"out_h": (B, H), "out_c": (B, H)}
    seq = {"out_seq": (B, T, H)}
    back = dict(weights, d_out_h=(B, H), d_out_c=(B, H), d_seq=(B, T, H))
    grads = {"dx": (B, T, D), "dW": (D, 4 * H), "dU": (H, 4 * H), "db": (4 * H,), "dh0": (B, H), "dc0": (B, H)}
    for call, shapes, extra in ((m.forward, dict(weights, **outs), {}), (m.forward_seq, dict(weights, **outs, **seq), {}),
                                (m.forward_train, dict(weights, **outs, **seq), {}),
                                (m.forward_stop, dict(weights, stop_v=(H,), **outs, out_steps=(B,), **seq), {"stop_c": 0.0}),
                                (m.backward, back, {}), (m.backward, dict(back, **grads), {})):
        for odd in [None] + list(shapes):
            t = {n: _tensor(s, I if n in ("lengths", "out_steps") else F) for n, s in shapes.items()}
            if odd:
                t[odd].number = 1
            if grads.keys() <= t.keys():
                t["out"] = {n: t.pop(n) for n in grads}
            del called[:]
            if odd is None:
                call(**t, **extra)
                assert len(called) == 1
                continue
            with pytest.raises(ValueError, match="device"):
                call(**t, **extra)
            assert not called, odd
