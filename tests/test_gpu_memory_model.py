"""The layer's operators together, as the example uses them: its gradients against a plain model in 64 bits, its steps
in a captured graph, its answers token by token against the whole sequence."""
import numpy as np
import pytest

import paper_1810_08061_amd as ld
from examples import memory_model as mm

pytestmark = pytest.mark.gpu


def _plain(params, tokens, lengths, targets):
    """The loss in 64 bits on the CPU; params require gradients."""
    import torch
    table, nw, nb, Wz, hw, hb, Wo, lw, lb, Wl = params
    N, P = tokens.shape
    H, Dk, Dv = mm.HEADS, mm.DK, mm.DV
    norm = lambda x, w, b: (x - x.mean(-1, keepdim=True)) / (x.var(-1, keepdim=True, unbiased=False) + 1e-5).sqrt() * w + b
    x = table[tokens]
    z = norm(x, nw, nb) @ Wz
    q, k, v = (t.reshape(N, P, H, -1) for t in z.split([H * Dk, H * Dk, H * Dv], 2))
    a = torch.tensor(mm.DECAY, dtype=torch.float32).double()[None, :, None, None]
    S, ys = torch.zeros((N, H, Dk, Dv), dtype=torch.float64), []
    for t in range(P):
        S = a * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        ys.append((q[:, t, :, :, None] * S).sum(2))
    u = norm(torch.stack(ys, 1), hw, hb).reshape(N, P, H * Dv)
    logits = norm(x + u @ Wo, lw, lb) @ Wl
    on = (torch.arange(P)[None] < lengths[:, None])
    logp = torch.log_softmax(logits, 2).gather(2, targets[..., None])[..., 0]
    return -(logp * on).sum() / lengths.sum(), logits


def _setup(N=6, seed=3):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    tok, lengths = mm.batch(g)
    tok, lengths = tok[:N].contiguous(), lengths[:N].contiguous()
    lengths[0] = mm.T
    params = mm.new_params(seed)
    return params, tok[:, :mm.T].contiguous(), tok[:, 1:].contiguous(), lengths


# A gradient is a sum of some 10^4 products that pass some 100 roundings each, of magnitudes some ten times
# what is left: 1e-4 of the largest; taken over all of a gradient, where roundings are independent, a quarter of that.
# (In bf16 some fifteen tensors on the way are rounded, whose gains no arithmetic gives: there each operator
# is held to its own bound, in its own test.)
def test_gradients_of_the_whole_model():
    import torch
    tol = 1e-4
    params, inputs, targets, lengths = _setup()
    model = mm.Model(6, mm.T, "f32")
    logits, _, kept = model.forward(params, inputs, lengths)
    loss, dlogits = mm.loss_of(logits, targets, lengths)
    grads = model.backward(params, inputs, lengths, kept, dlogits)
    assert model.status() == ld.OK
    plain = [q.detach().double().cpu().requires_grad_() for q in params]
    want, _ = _plain(plain, inputs.long().cpu(), lengths.cpu(), targets.long().cpu())
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= tol * float(want.detach())
    for name, g, w in zip(mm.NAMES, grads, plain):
        err = (g.double().cpu() - w.grad).abs().max() / w.grad.abs().max()
        whole = (g.double().cpu() - w.grad).norm() / w.grad.norm()
        assert float(err) <= tol and float(whole) <= tol / 4, (name, float(err), float(whole))


def test_a_training_step_replayed():
    """Forward, backward, norm and the clipped step in one graph, on new batches, against eager steps of another model."""
    import torch
    runs = []
    for _ in range(2):
        params, inputs, targets, lengths = _setup()
        runs.append((params, inputs, targets, lengths, mm.Model(6, mm.T, "f32"), ld.AdamW(params), ld.GradClip(params, 0.5)))

    def step(params, inputs, targets, lengths, model, opt, clip):
        logits, _, kept = model.forward(params, inputs, lengths)
        loss, dlogits = mm.loss_of(logits, targets, lengths)
        return loss, opt.step(model.backward(params, inputs, lengths, kept, dlogits), lr=0.01, clip=clip)
    for r in runs:
        step(*r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, result = step(*runs[0])
    g = torch.Generator(device="cuda").manual_seed(9)
    for i in range(4):
        tok, lengths = mm.batch(g)
        for r in runs:
            r[1].copy_(tok[:6, :mm.T])
            r[2].copy_(tok[:6, 1:])
            r[3].copy_(lengths[:6])
        runs[1][5].steps_done = 1          # the captured step's number
        want_loss, want = step(*runs[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (loss == want_loss).all() and (result == want).all(), i
        assert all((a == b).all() for a, b in zip(runs[0][0], runs[1][0])), i
    del graph


def test_answers_token_by_token():
    """Greedy answers from single steps are those of the whole sequence, prompt and answer together."""
    import torch
    params = [q.bfloat16() if q.dim() == 2 else q for q in mm.new_params(5)]
    prompt = torch.randint(2, mm.V, (7, 5), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
    tokens, logps = mm.answer(params, prompt, 6, temperature=0.0)
    assert (logps == 0).all()
    whole = torch.cat([prompt, tokens], 1)
    logits, _, _ = mm.Model(7, 11, "bf16").forward(params, whole, None)
    at = logits[:, 4:-1].float()
    best = at.max(2).values
    chosen = at.gather(2, tokens[..., None].long())[..., 0]
    # the same logits, but for the roundings on two ways to them: six tensors of 2^-8 each
    assert (best - chosen <= 6 * 2.0 ** -8 * at.abs().max()).all()
    again, _ = mm.answer(params, prompt, 6, temperature=0.0)
    assert (again == tokens).all()


def test_the_example_runs():
    losses, tokens, logps = mm.main(20)
    assert len(losses) == 20 and np.isfinite(losses).all()
    assert tokens.shape == (2, 8) and ((tokens >= 0) & (tokens < mm.V)).all() and (logps <= 0).all()
