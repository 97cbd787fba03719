"""A small token model whose layer is a matrix memory, trained under a clipped gradient, answering by sampling.

    python examples/memory_model.py [steps]

tokens -> TokenEmbed -> LayerNorm -> x W_z -> LinearAttention -> LayerNorm of each head -> y W_o, added to
the embedded tokens -> LayerNorm -> logits; the gradients back through the same operators, AdamW from gradients
clipped on their way; then answers token by token, each layer in its form for single tokens, from TokenSample.

The sequences alternate between two tokens and end with END, so the next token
is the one before the last: the memory has to hold it.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1810_08061_amd as ld

V, D, HEADS, DK, DV, B, T = 48, 64, 4, 16, 32, 64, 20
WIDTH = HEADS * (2 * DK + DV)
DECAY = [0.5, 0.8, 0.95, 1.0]
START, END = 0, 1
NAMES = ["table", "norm_w", "norm_b", "Wz", "head_w", "head_b", "Wo", "last_w", "last_b", "Wl"]


def batch(g):
    """tokens int32 [B, T + 1]: START, a, b, a, b, ..., END; lengths int32 [B] of the inputs (END is a target)."""
    a = torch.randint(2, V, (B, 1), generator=g, device="cuda")
    b = torch.randint(2, V, (B, 1), generator=g, device="cuda")
    t = torch.arange(T + 1, device="cuda")[None]
    n = torch.randint(6, T + 1, (B, 1), generator=g, device="cuda")
    tok = torch.where(t == 0, START, torch.where(t % 2 == 1, a, b))
    return torch.where(t >= n, END, tok).int(), n[:, 0].int()


def new_params(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    ones, zeros = lambda n: torch.ones(n, device="cuda"), lambda n: torch.zeros(n, device="cuda")
    return [normal(V, D), ones(D), zeros(D), normal(D, WIDTH) / D ** 0.5, ones(DV), zeros(DV),
            normal(HEADS * DV, D) / (HEADS * DV) ** 0.5, ones(D), zeros(D), normal(D, V) / D ** 0.5]


class Model:
    """The layer's handles for N rows of P tokens in a type."""

    def __init__(self, N, P, dtype):
        self.N, self.P = N, P
        self.embed = ld.TokenEmbed(N, P, V, D, dtype)
        self.norm, self.last = ld.LayerNorm(N, P, D, dtype), ld.LayerNorm(N, P, D, dtype)
        self.attend = ld.LinearAttention(N, HEADS, DK, DV, P, DECAY, dtype)
        self.head = ld.LayerNorm(N, P * HEADS, DV, dtype)      # a head of a step is a row of its own
        self.S0 = torch.zeros((N, HEADS, DK, DV), device="cuda")

    def forward(self, p, tokens, lengths):
        """The logits [N, P, V], the state after each row, and what the gradients need."""
        table, nw, nb, Wz, hw, hb, Wo, lw, lb, Wl = p
        N, P = self.N, self.P
        x = self.embed.forward(tokens, lengths, table)
        n = self.norm.forward(x, lengths, nw, nb)
        z = (n.view(N * P, D) @ Wz).view(N, P, WIDTH)
        y, S = self.attend.forward(z, lengths, self.S0)
        of_heads = None if lengths is None else lengths * HEADS
        u = self.head.forward(y.view(N, P * HEADS, DV), of_heads, hw, hb).view(N, P, HEADS * DV)
        r = x + (u.view(N * P, HEADS * DV) @ Wo).view(N, P, D)
        m = self.last.forward(r, lengths, lw, lb)
        return (m.view(N * P, D) @ Wl).view(N, P, V), S, (x, n, z, y, of_heads, u, r, m)

    def backward(self, p, tokens, lengths, kept, dlogits):
        """The gradients of all parameters, float32."""
        table, nw, nb, Wz, hw, hb, Wo, lw, lb, Wl = p
        x, n, z, y, of_heads, u, r, m = kept
        N, P = self.N, self.P
        flat = lambda t: t.reshape(N * P, -1)
        d = flat(dlogits)
        dWl = flat(m).t() @ d
        last = self.last.backward(r, lengths, lw, (d @ Wl.t()).view(N, P, D))
        dr = last["dx"]
        dWo = flat(u).t() @ flat(dr)
        head = self.head.backward(y.view(N, P * HEADS, DV), of_heads, hw, (flat(dr) @ Wo.t()).view(N, P * HEADS, DV))
        dz = self.attend.backward(z, lengths, self.S0, head["dx"].view(N, P, HEADS * DV))["dz"]
        dWz = flat(n).t() @ flat(dz)
        first = self.norm.backward(x, lengths, nw, (flat(dz) @ Wz.t()).view(N, P, D))
        dtable = self.embed.backward(tokens, lengths, dr + first["dx"])
        return [dtable, first["dweight"], first["dbias"], dWz.float(), head["dweight"], head["dbias"], dWo.float(),
                last["dweight"], last["dbias"], dWl.float()]

    def status(self):
        return max(h.status() for h in (self.embed, self.norm, self.last, self.attend, self.head))


def loss_of(logits, targets, lengths):
    """Mean cross entropy over the rows' steps, and its gradient."""
    N, P, _ = logits.shape
    logp = torch.log_softmax(logits.float(), 2)
    on = (torch.arange(P, device=logits.device)[None] < lengths[:, None])[..., None] / lengths.sum()
    hit = torch.nn.functional.one_hot(targets.long(), V)
    return -(logp * hit * on).sum(), ((logp.exp() - hit) * on).to(logits.dtype)


def train(steps, seed=0):
    """Returns the weights as the layers take them and the loss of every step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    params = new_params(seed)
    # matrices in bf16 for the products; the norms' weights stay float32
    copies = [q.bfloat16() if q.dim() == 2 else None for q in params]
    weights = [q if c is None else c for q, c in zip(params, copies)]
    model, opt = Model(B, T, "bf16"), ld.AdamW(params, copies=copies, weight_decay=0.001)
    clip, losses, norms = ld.GradClip(params, 1.0), [], []
    for _ in range(steps):
        tok, lengths = batch(g)
        inputs = tok[:, :T].contiguous()
        logits, _, kept = model.forward(weights, inputs, lengths)
        loss, dlogits = loss_of(logits, tok[:, 1:], lengths)
        norms.append(opt.step(model.backward(weights, inputs, lengths, kept, dlogits), lr=0.01, clip=clip)[0])
        losses.append(loss)
    assert model.status() == opt.status() == clip.status() == ld.OK
    return weights, torch.stack(losses).tolist(), torch.stack(norms).tolist()


def answer(weights, prompt, steps, seed=0, **filters):
    """Continuations of prompt int32 [N, P], sampled: tokens [N, steps] and their log probabilities."""
    table, nw, nb, Wz, hw, hb, Wo, lw, lb, Wl = weights
    N, P = prompt.shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    logits, S, _ = Model(N, P, "bf16").forward(weights, prompt, None)
    one, sample = Model(N, 1, "bf16"), ld.TokenSample(N, V, "bf16")
    logits, tokens, logps = logits[:, -1].contiguous(), [], []
    for _ in range(steps):
        u = torch.rand((N,), generator=g, device="cuda")
        token, logp = sample.sample(logits, u, **filters)
        tokens.append(token)
        logps.append(logp)
        x = one.embed.forward(token[:, None], None, table)
        z = one.norm.forward(x, None, nw, nb).view(N, D) @ Wz
        y, S = one.attend.step(z, S, out_S=S)
        v = one.head.forward(y.view(N, HEADS, DV), None, hw, hb).view(N, HEADS * DV)
        r = x + (v @ Wo).view(N, 1, D)
        logits = one.last.forward(r, None, lw, lb).view(N, D) @ Wl
    return torch.stack(tokens, 1), torch.stack(logps, 1)


def main(steps=300):
    weights, losses, norms = train(steps)
    print(f"loss of the first step {losses[0]:.3f}, mean of the last ten {sum(losses[-10:]) / 10:.3f}; "
          f"gradient norm {norms[0]:.2f}, then {norms[-1]:.2f}")
    prompt = torch.tensor([[START, 5, 9, 5], [START, 30, 41, 30]], dtype=torch.int32, device="cuda")
    tokens, logps = answer(weights, prompt, 8, temperature=0.8, top_k=20, top_p=0.95, min_p=0.02)
    for n in range(2):
        print(f"after {prompt[n].tolist()}: {tokens[n].tolist()}, log probability {float(logps[n].sum()):.3f}")
    return losses, tokens, logps


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 300)
