"""A small token model trained and decoded with the operators around the loop.

    python examples/token_model.py [steps]

tokens -> TokenEmbed -> x W_z -> GatedScan -> y W_out -> cross entropy, its
gradients back through the same operators, one AdamW step over all tensors
(fp32 parameters with bf16 copies for the products, states in 8 bits); then
a beam search that takes one token of every beam at a time.

The sequences alternate between two tokens and end with END, so the next token
is the one before the last: the recurrence has to remember it.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1810_08061_amd as ld

V, D, H, B, T, K = 48, 64, 128, 64, 20, 4
START, END = 0, 1


def batch(g):
    """tokens int32 [B, T + 1]: START, a, b, a, b, ..., END; lengths int32 [B] of the inputs (END is a target)."""
    a = torch.randint(2, V, (B, 1), generator=g, device="cuda")
    b = torch.randint(2, V, (B, 1), generator=g, device="cuda")
    t = torch.arange(T + 1, device="cuda")[None]
    n = torch.randint(6, T + 1, (B, 1), generator=g, device="cuda")
    tok = torch.where(t == 0, START, torch.where(t % 2 == 1, a, b))
    tok = torch.where(t >= n, END, tok)
    return tok.int(), n[:, 0].int()


def train(steps, seed=0):
    """Returns the bf16 weights and the mean loss of every step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    params = [normal(V, D) / D ** 0.5, normal(D, 3 * H) / D ** 0.5, normal(H, V) / H ** 0.5]
    table, Wz, Wo = copies = [p.bfloat16() for p in params]
    embed = ld.TokenEmbed(B, T, V, D, "bf16", scale=D ** 0.5)
    scan = ld.GatedScan(B, H, T, "bf16")
    opt = ld.AdamW(params, copies=copies, state_bits=8, weight_decay=0.001)
    h0 = torch.zeros((B, H), device="cuda")
    losses = []
    for _ in range(steps):
        tok, lengths = batch(g)
        inputs, targets = tok[:, :T].contiguous(), tok[:, 1:].long()
        x = embed.forward(inputs, lengths, table)
        z = (x.view(B * T, D) @ Wz).view(B, T, 3 * H)
        y, _ = scan.forward_train(z, lengths, h0)
        logp = torch.log_softmax((y.view(B * T, H) @ Wo).float(), 1)
        on = (torch.arange(T, device="cuda")[None] < lengths[:, None]).flatten()
        hit = torch.nn.functional.one_hot(targets.flatten(), V)
        losses.append((-(logp * hit).sum(1) * on).sum() / on.sum())
        dlogits = ((logp.exp() - hit) * (on / on.sum())[:, None]).bfloat16()
        dWo = y.view(B * T, H).t() @ dlogits
        dy = (dlogits @ Wo.t()).view(B, T, H)
        dz = scan.backward(z, lengths, h0, dy)["dz"].view(B * T, 3 * H)
        dWz = x.view(B * T, D).t() @ dz
        dtable = embed.backward(inputs, lengths, (dz @ Wz.t()).view(B, T, D))
        opt.step([dtable, dWz.float(), dWo.float()], lr=0.01)
    assert embed.status() == scan.status() == opt.status() == ld.OK
    return (table, Wz, Wo), torch.stack(losses).tolist()


def decode(weights, prompt, steps):
    """The best continuations of prompt int32 [N, P] (all of one length): tokens [N, K, steps], scores [N, K]."""
    table, Wz, Wo = weights
    N, P = prompt.shape
    # the prompt, through the whole-sequence forms
    embed, scan = ld.TokenEmbed(N, P, V, D, "bf16", scale=D ** 0.5), ld.GatedScan(N, H, P, "bf16")
    lengths = torch.full((N,), P, dtype=torch.int32, device="cuda")
    z = (embed.forward(prompt, None, table).view(N * P, D) @ Wz).view(N, P, 3 * H)
    y, h = scan.forward(z, lengths, torch.zeros((N, H), device="cuda"))
    # then one token of every beam at a time; at first one beam is alive
    beams = ld.BeamSearch(N, K, V, "bf16", end=END)
    one = ld.TokenEmbed(N, K, V, D, "bf16", scale=D ** 0.5)
    logits = (y[:, -1] @ Wo)[:, None].expand(N, K, V).contiguous()
    h = h[:, None].expand(N, K, H).contiguous()
    scores = torch.full((N, K), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    finished = torch.zeros((N, K), dtype=torch.uint8, device="cuda")
    history = torch.zeros((N, K, steps), dtype=torch.int32, device="cuda")
    for i in range(steps):
        scores, _, token, finished, (h, history) = beams.step(logits, scores, finished, [h, history])
        history[:, :, i] = token
        z = one.forward(token, None, table).view(N * K, D) @ Wz
        y, hn = scan.step(z, h.view(N * K, H))
        h, logits = hn.view(N, K, H), (y @ Wo).view(N, K, V)
    return history, scores


def main(steps=300):
    weights, losses = train(steps)
    print(f"loss of the first step {losses[0]:.3f}, mean of the last ten {sum(losses[-10:]) / 10:.3f}")
    prompt = torch.tensor([[START, 5, 9, 5], [START, 30, 41, 30]], dtype=torch.int32, device="cuda")
    tokens, scores = decode(weights, prompt, 8)
    for n in range(2):
        print(f"after {prompt[n].tolist()}:")
        for k in range(K):
            print(f"  {scores[n, k]:8.3f}  {tokens[n, k].tolist()}")
    return losses, tokens, scores


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 300)
