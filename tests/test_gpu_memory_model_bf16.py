"""The example's model in bf16: its gradients against the same chain of operators in 64 bits, rounded where the model rounds.

Where an fp32 sum and the 64-bit one lie on two sides of a rounding, the two chains part by a step, and what follows meets other
roundings: at most, each is a draw of its own of the same errors.  Two such draws are sqrt 2 times as far apart as one of them is
from the chain without roundings (E), and over the 32 values of the smallest tensor that distance spreads by 1 / sqrt(64).  Twice
E is 3.3 such spreads beyond it; an operator that is off by more than the roundings of its place, or one more rounding of some
tensor's whole size, is not within it."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from examples import memory_model as mm
from tests import layer_util
from tests.test_gpu_memory_model import _setup

pytestmark = pytest.mark.gpu


def _norm(x, lengths, w, b, dy=None):
    return layer_util.norm(x, lengths, w, b, 1e-5, dy)[0]


def _chain(params, tokens, targets, lengths, R):
    """Loss, logits and gradients on the host, every tensor that the model keeps in bf16 passed through R."""
    table, nw, nb, Wz, hw, hb, Wo, lw, lb, Wl = params
    N, P = tokens.shape
    H, Dk, Dv, D = mm.HEADS, mm.DK, mm.DV, mm.D
    on = (np.arange(P)[None] < lengths[:, None])[..., None]
    a = np.float32(mm.DECAY).astype(np.float64)
    S0 = np.zeros((N, H, Dk, Dv))
    x = np.where(on, table[tokens], 0.0)
    n = R(_norm(x, lengths, nw, nb)["y"])
    z = R(n @ Wz)
    y = R(layer_util.attend(z, lengths, S0, a, Dk, Dv)["y"])
    of_heads = lambda t: t.reshape(N, P * H, Dv)
    u = R(_norm(of_heads(y), lengths * H, hw, hb)["y"]).reshape(N, P, H * Dv)
    r = R(x + R(u @ Wo))
    m = R(_norm(r, lengths, lw, lb)["y"])
    logits = R(m @ Wl)
    e = np.exp(logits - logits.max(2, keepdims=True))
    p = e / e.sum(2, keepdims=True)
    hit = np.eye(mm.V)[targets]
    share = on / lengths.sum()
    loss = -(np.log((p * hit).sum(2, keepdims=True)) * share).sum()
    d = R((p - hit) * share)
    flat = lambda t: t.reshape(N * P, -1)
    dWl = R(flat(m).T @ flat(d))
    last = _norm(r, lengths, lw, lb, R(d @ Wl.T))
    dr = R(last["dx"])
    dWo = R(flat(u).T @ flat(dr))
    head = _norm(of_heads(y), lengths * H, hw, hb, of_heads(R(dr @ Wo.T)))
    dy = R(head["dx"]).reshape(N, P, H * Dv)
    dz = R(layer_util.attend(z, lengths, S0, a, Dk, Dv, dy, np.zeros_like(S0))["dz"])
    dWz = R(flat(n).T @ flat(dz))
    first = _norm(x, lengths, nw, nb, R(dz @ Wz.T))
    dx = R(dr + R(first["dx"]))
    dtable = np.zeros_like(table)
    np.add.at(dtable, tokens[on[..., 0]], dx[on[..., 0]])
    return loss, logits, [dtable, first["dweight"], first["dbias"], dWz, head["dweight"], head["dbias"], dWo, last["dweight"], last["dbias"], dWl]


def test_bf16_gradients_are_the_rounded_chains():
    import torch
    params, inputs, targets, lengths = _setup()
    weights = [q.bfloat16() if q.dim() == 2 else q for q in params]
    model = mm.Model(6, mm.T, "bf16")
    logits, _, kept = model.forward(weights, inputs, lengths)
    loss, dlogits = mm.loss_of(logits, targets, lengths)
    grads = model.backward(weights, inputs, lengths, kept, dlogits)
    assert model.status() == ld.OK
    host = lambda t: t.detach().double().cpu().numpy()
    args = [host(q) for q in weights], inputs.long().cpu().numpy(), targets.long().cpu().numpy(), lengths.long().cpu().numpy()
    rounded = _chain(*args, lambda t: torch.from_numpy(t).to(torch.bfloat16).double().numpy())
    exact = _chain(*args, lambda t: t)
    on = (np.arange(mm.T)[None] < args[3][:, None])[..., None]
    far = lambda a, b: float(np.linalg.norm(np.asarray(a) - np.asarray(b)))
    apart = np.abs((host(logits) - rounded[1]) * on).max()
    assert abs(float(loss) - rounded[0]) <= 2 * apart + 1e-5 * rounded[0]      # log softmax changes by twice a logit's change
    assert far(host(logits) * on, rounded[1] * on) <= 2 * far(rounded[1] * on, exact[1] * on)
    for name, g, w, e in zip(mm.NAMES, grads, rounded[2], exact[2]):
        assert far(host(g), w) <= 2 * far(w, e), (name, far(host(g), w), far(w, e))
