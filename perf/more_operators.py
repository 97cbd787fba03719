"""Performance cases of the operators of a layer around the time loop, of its training and of
its answers: what is timed, on which inputs, and what comes out.

A case is a dict of plain values; "op" names the operator and its direction:
  attend_step, attend_forward, attend_train   linear attention with a decay for each head: one
                           token per row, the whole sequence, the sequence and its gradients
  norm_forward, norm_train layer norm; and its gradients with those of weight and bias
  clip                     the global norm of the gradients, and the gradients clipped to it
  clip_step                the same norm, and an AdamW step from gradients clipped to it
  sample                   one token a row: temperature, top-k, top-p, min-p, from given numbers

With `own` false, run() computes the operators in elementary torch operations
in 32 bits (sampling's sums, which decide whole numbers, in 64); with `own`
true it calls the framework.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_NORM_EPS = 1e-5
_BETA1, _BETA2, _EPS, _WD, _LR = 0.9, 0.999, 1e-8, 0.01, 1e-3


# --- cases ------------------------------------------------------------------

def _attend(op, dtype, B, T, heads, Dk, Dv, ragged):
    return {"op": op, "dtype": dtype, "B": B, "T": T, "heads": heads, "Dk": Dk, "Dv": Dv, "ragged": ragged}


def _norm(op, dtype, grad, B, T, D, ragged):
    return {"op": op, "dtype": dtype, "grad": grad, "B": B, "T": T, "D": D, "ragged": ragged}


def _clip(op, dtype, max_norm, layers, D, H, V):
    return {"op": op, "dtype": dtype, "max_norm": max_norm, "layers": layers, "D": D, "H": H, "V": V}


def _sample(dtype, N, V, top_k, top_p, min_p):
    return {"op": "sample", "dtype": dtype, "N": N, "V": V, "top_k": top_k, "top_p": top_p, "min_p": min_p}


def listed():
    named = {
        # one generated token for each of a few rows: a launch and its latency
        "attend_step_b16": _attend("attend_step", "bf16", 16, 1, 8, 64, 64, False),
        # one long prompt: few heads, so the time axis has to be split
        "attend_prompt_t32768": _attend("attend_forward", "bf16", 1, 32768, 16, 128, 128, False),
        # a training batch at sizes that are no multiple of any tile, fp32
        "attend_train_odd_f32": _attend("attend_train", "f32", 5, 301, 3, 50, 75, True),
        # the largest training batch: long documents of different lengths
        "attend_train_large": _attend("attend_train", "bf16", 8, 4096, 16, 128, 128, True),
        # serving: the rows of one new token for each of 64 sequences
        "norm_forward_b64": _norm("norm_forward", "bf16", "bf16", 64, 1, 512, False),
        # a small odd training batch, fp32
        "norm_train_odd_f32": _norm("norm_train", "f32", "f32", 21, 45, 333, True),
        # the largest: the loop's input normalised, its gradient in fp32 as the loop's backward gives it
        "norm_train_large": _norm("norm_train", "bf16", "f32", 256, 1000, 1024, True),
        # the gradients of a stack of ordinary fp32 layers, clipped as a call of its own
        "clip_5x256": _clip("clip", "f32", 1.0, 5, 256, 256, 1000),
        # a wide model with a large token table: the clipped step
        "clip_step_large": _clip("clip_step", "f32", 1.0, 3, 1024, 2048, 65536),
        # one sequence answered over a small vocabulary, every filter on
        "sample_b1_v1000": _sample("f32", 1, 1000, True, True, True),
        # an ordinary decoding batch
        "sample_b16_v32768": _sample("bf16", 16, 32768, True, True, False),
        # the largest: many rows, a large vocabulary, no limit on the number of tokens kept
        "sample_b256_v65536": _sample("bf16", 256, 65536, False, True, True),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, low, high):
    """A whole number, spread over the logarithm of its range."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _width(rng, low, high):
    """A layer's width: a multiple of 32 as often as any number."""
    w = _log(rng, low, high)
    return w // 160 * 160 if rng.random() < 0.5 and w >= 160 else w


def _head(rng):
    """A head's width: one of the usual ones as often as any number."""
    return rng.choice([32, 64, 128]) if rng.random() < 0.5 else rng.randint(8, 128)


def draw(rng):
    op = rng.choice(["attend_step", "attend_forward", "attend_train", "norm_forward", "norm_train", "clip",
                     "clip_step", "sample", "sample"])
    dtype = rng.choice(["f32", "bf16"])
    ragged = rng.random() < 0.5
    if op.startswith("attend"):
        heads, Dk = _log(rng, 1, 16), _head(rng)
        Dv = Dk if rng.random() < 0.5 else _head(rng)
        if op == "attend_step":
            return _attend(op, dtype, _log(rng, 1, 512), 1, heads, Dk, Dv, False)
        B, T = _log(rng, 1, 64), _log(rng, 2, 32768)
        most = 1 << (26 if op == "attend_forward" else 25)
        if dtype == "f32":
            most >>= 2
        T = max(2, min(T, most // (B * heads * max(Dk, Dv))))
        return _attend(op, dtype, B, T, heads, Dk, Dv, ragged)
    if op.startswith("norm"):
        B, T, D = _log(rng, 1, 256), _log(rng, 1, 1000), _width(rng, 16, 8192)
        T = max(1, min(T, (1 << 27) // (B * D)))
        return _norm(op, dtype, rng.choice(["f32", dtype]), B, T, D, ragged)
    if op.startswith("clip"):
        return _clip(op, dtype, rng.choice([0.25, 1.0, 1000.0]), rng.randint(1, 5), _width(rng, 16, 1024),
                     _width(rng, 16, 1024), _log(rng, 64, 16384))
    N, V = _log(rng, 1, 256), _log(rng, 64, 65536)
    return _sample(dtype, N, V, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5)


# --- inputs -----------------------------------------------------------------

def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, mean=0.0, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(mean, std, generator=g)


def _uniform(g, shape, low=0.0, high=1.0, dtype=torch.float32):
    return torch.empty(shape, device="cuda", dtype=dtype).uniform_(low, high, generator=g)


def _lengths(g, B, T, ragged):
    if not ragged:
        return torch.full((B,), T, dtype=torch.int32, device="cuda")
    L = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    L[0] = T
    return L


def _decay(heads):
    """Memories from eight steps to two thousand, each head's own."""
    return [1.0 - 2.0 ** -(3.0 + 8.0 * i / max(1, heads - 1)) for i in range(heads)]


def _shapes(case):
    """An LSTM stack's tensors (W, U, b of each layer) and a token table."""
    D, H = case["D"], case["H"]
    one = [(H, 4 * H), (H, 4 * H), (4 * H,)]
    return [(case["V"], D)] + [(D, 4 * H)] + one[1:] + one * (case["layers"] - 1)


def _inputs(case, seed):
    """The tensors of a case, from its seed alone."""
    g, op = _rng(seed), case["op"]
    if op.startswith("attend"):
        B, T, heads, Dk, Dv, dt = case["B"], case["T"], case["heads"], case["Dk"], case["Dv"], _DT[case["dtype"]]
        z = _normal(g, (B, T, heads * (2 * Dk + Dv)), dtype=dt)
        z[..., heads * Dk:2 * heads * Dk] *= Dk ** -0.5
        s = {"z": z, "S0": _normal(g, (B, heads, Dk, Dv), std=0.5), "lengths": _lengths(g, B, T, case["ragged"]),
             "decay": _decay(heads)}
        if op == "attend_step":
            s["z"] = z[:, 0].contiguous()
        if op == "attend_train":
            s["dy"] = _normal(g, (B, T, heads * Dv), dtype=dt)
            s["dS"] = _normal(g, (B, heads, Dk, Dv), std=0.1)
        return s
    if op.startswith("norm"):
        B, T, D, dt = case["B"], case["T"], case["D"], _DT[case["dtype"]]
        x = _normal(g, (B, T, D)) * torch.exp(_normal(g, (B, T, 1), std=0.5)) + _normal(g, (B, T, 1))
        s = {"x": x.to(dt), "lengths": _lengths(g, B, T, case["ragged"]), "weight": _normal(g, (D,), 1.0, 0.2),
             "bias": _normal(g, (D,), std=0.2)}
        if op == "norm_train":
            s["dy"] = _normal(g, (B, T, D), dtype=_DT[case["grad"]])
        return s
    if op.startswith("clip"):
        s = {"g": [], "max_norm": case["max_norm"], "t": 100}
        for shape in _shapes(case):
            size = torch.exp(_normal(g, (shape[-1],), mean=-7.0))       # columns differ in the size of their gradients
            s["g"].append((_normal(g, shape) * size).to(_DT[case["dtype"]]))
        if op == "clip":
            s["out"] = [torch.empty_like(x) for x in s["g"]]
            return s
        s.update(p=[_normal(g, x.shape, std=x.shape[-1] ** -0.5) for x in s["g"]],
                 m=[x.float() * 0.3 for x in s["g"]],
                 v=[(x.float() * _normal(g, x.shape, 1.0, 0.2)).square() for x in s["g"]])
        return s
    N, V = case["N"], case["V"]
    s = {"logits": _normal(g, (N, V), std=2.5, dtype=_DT[case["dtype"]]),
         "temperature": _uniform(g, (N,), 0.5, 1.2), "u": _uniform(g, (N,)),
         "top_k": torch.exp(_uniform(g, (N,), 0.0, math.log(min(V, 1000)))).int() if case["top_k"] else None,
         "top_p": _uniform(g, (N,), 0.3, 0.98) if case["top_p"] else None,
         "min_p": torch.exp(_uniform(g, (N,), math.log(1e-3), math.log(0.2))) if case["min_p"] else None}
    s["logits"][:, 0] = -math.inf                                # a token that is never to be chosen
    s["temperature"][N // 2::7] = 0.0                            # some rows take their best token
    if case["top_k"]:
        s["top_k"][N // 3::5] = 0                                # and some have no such limit
    _spread_sample(s)
    return s


def _spread_sample(s):
    """Move top_p, min_p and u to the middle of the gap between the sums (or values) that they fall
    between, so that rounding does not decide which tokens are kept or chosen."""
    T = torch.where(s["temperature"] > 0, s["temperature"], 1.0).double()[:, None]
    x, at = s["logits"].double().sort(dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / T)
    N, V = w.shape
    place = torch.arange(V, device=w.device)
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
        w = torch.where(place < k, w, 0.0)
    if s["top_p"] is not None:
        c = w.cumsum(1) / w.sum(1, keepdim=True)
        i = (c < s["top_p"].double()[:, None]).sum(1, keepdim=True).clamp(max=V - 1)
        high = c.gather(1, i)
        low = torch.where(i > 0, c.gather(1, (i - 1).clamp(min=0)), 0.0)
        s["top_p"] = ((low + high) / 2)[:, 0].float()
        w = torch.where(place <= i, w, 0.0)
    if s["min_p"] is not None:
        m = s["min_p"].double()[:, None]
        r = torch.exp((x - x[:, :1]) / T)
        low = torch.where(r < m, r, 0.0).amax(1)
        high = torch.where(r >= m, r, 2.0).amin(1)
        s["min_p"] = torch.where(low > 0, (low * high).sqrt(), high / 2).float()
        w = torch.where(r < m, 0.0, w)
    w = torch.zeros_like(w).scatter_(1, at, w)
    c = w.cumsum(1) / w.sum(1, keepdim=True)
    i = (c <= s["u"].double()[:, None]).sum(1, keepdim=True).clamp(max=V - 1)
    high = c.gather(1, i)
    low = torch.where(i > 0, c.gather(1, (i - 1).clamp(min=0)), 0.0)
    s["u"] = ((low + high) / 2)[:, 0].float()


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if not own:
        return s
    import paper_1810_08061_amd as ld
    op = case["op"]
    if op.startswith("attend"):
        s["handle"] = ld.LinearAttention(case["B"], case["heads"], case["Dk"], case["Dv"], case["T"], s["decay"],
                                         case["dtype"])
    elif op.startswith("norm"):
        s["handle"] = ld.LayerNorm(case["B"], case["T"], case["D"], case["dtype"], eps=_NORM_EPS)
    elif op == "clip":
        s["handle"] = ld.GradClip(s["g"], s["max_norm"])
    elif op == "clip_step":
        s["handle"] = ld.GradClip(s["p"], s["max_norm"])
        s["adamw"] = ld.AdamW(s["p"], betas=(_BETA1, _BETA2), eps=_EPS, weight_decay=_WD, steps_done=s["t"])
        s["adamw"].load_state(s["m"], s["v"])
        s["m"] = s["v"] = None
    else:
        s["handle"] = ld.TokenSample(case["N"], case["V"], case["dtype"])
    return s


# --- one pass ---------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    op, h = s["case"]["op"], s["handle"]
    if op == "attend_step":
        y, S = h.step(s["z"], s["S0"])
        return {"y": y, "S": S}
    if op == "attend_forward":
        y, S = h.forward(s["z"], s["lengths"], s["S0"])
        return {"y": y, "S": S}
    if op == "attend_train":
        y, S = h.forward(s["z"], s["lengths"], s["S0"])
        return dict(h.backward(s["z"], s["lengths"], s["S0"], s["dy"], s["dS"]), y=y, S=S)
    if op == "norm_forward":
        return h.forward(s["x"], s["lengths"], s["weight"], s["bias"])
    if op == "norm_train":
        y = h.forward(s["x"], s["lengths"], s["weight"], s["bias"])
        return dict(h.backward(s["x"], s["lengths"], s["weight"], s["dy"]), y=y)
    if op == "clip":
        result = h.clip(s["g"], out=s["out"])
        return {"result": result, "g": s["out"]}
    if op == "clip_step":
        result = s["adamw"].step(s["g"], _LR, clip=h)
        m, v = s["adamw"].states()
        return {"result": result, "p": s["p"], "m": m, "v": v}
    token, logp = h.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                           min_p=s["min_p"])
    return {"token": token, "logp": logp}


def _run_plain(s):
    op = s["case"]["op"]
    if op.startswith("attend"):
        return _plain_attend(s, op)
    if op.startswith("norm"):
        return _plain_norm(s, op)
    return _plain_sample(s) if op == "sample" else _plain_clip(s, op)


def _valid(lengths, T):
    return torch.arange(T, device=lengths.device) < lengths[:, None]


def _split(z, heads, Dk, Dv):
    """q, k [B, heads, T, Dk] and v [B, heads, T, Dv] of z [B, T, heads (2 Dk + Dv)]."""
    B, T = z.shape[:2]
    q, k, v = z.split([heads * Dk, heads * Dk, heads * Dv], 2)
    return [t.reshape(B, T, heads, -1).transpose(1, 2) for t in (q, k, v)]


_CHUNK = 64


def _chunked(x, y, z, a, S, on, skip):
    """out_i = sum_{j <= i} a^(i-j) (x_i . y_j) z_j + a^(i+1-skip) x_i S over the steps that are `on`, and the state
    after the last: inside a chunk as a product under a mask of decays, between chunks through the state.
    skip = 0: the state decays before a step adds to it; skip = 1: after (the way back).  x, y and z are
    zero where a step is not on; such a step leaves the state."""
    B, h, T, _ = x.shape
    n = -(-T // _CHUNK)
    cut = lambda t: torch.nn.functional.pad(t, (0, 0, 0, n * _CHUNK - T)).reshape(B, h, n, _CHUNK, -1)
    x, y, z = cut(x), cut(y), cut(z)
    count = torch.nn.functional.pad(on.int(), (0, n * _CHUNK - T)).reshape(B, 1, n, _CHUNK).cumsum(3)   # within the chunk
    power = lambda e: a[:, None, None] ** e.clamp(min=0)
    order = torch.tril(torch.ones((_CHUNK, _CHUNK), device=x.device))
    mask = a[:, None, None, None] ** (count[..., None] - count[..., None, :]).clamp(min=0) * order
    out = torch.matmul(torch.matmul(x, y.transpose(3, 4).contiguous()) * mask, z)
    total = count[..., -1:]
    add = torch.matmul((y * power(total - count + skip)[..., None]).transpose(3, 4).contiguous(), z)
    keep = power(total)[..., None]
    starts = []
    for c in range(n):
        starts.append(S)
        S = keep[:, :, c] * S + add[:, :, c]
    out = out + torch.matmul(x * power(count - skip)[..., None], torch.stack(starts, 2))
    return out.reshape(B, h, n * _CHUNK, -1)[:, :, :T], S


def _packed(t):
    """[B, heads, T, D] as [B, T, heads D]."""
    return t.transpose(1, 2).flatten(2)


def _plain_attend(s, op):
    c = s["case"]
    heads, Dk, Dv, dt, S0 = c["heads"], c["Dk"], c["Dv"], s["z"].dtype, s["S0"]
    a = torch.tensor(s["decay"], dtype=torch.float32, device=S0.device)
    if op == "attend_step":
        q, k, v = [t[:, :, 0] for t in _split(s["z"].float()[:, None], heads, Dk, Dv)]
        S = a[:, None, None] * S0 + k[..., None] * v[..., None, :]
        return {"y": (q[..., None] * S).sum(2).flatten(1).to(dt), "S": S}
    B, T = s["z"].shape[:2]
    on = _valid(s["lengths"], T)
    q, k, v = _split(torch.where(on[..., None], s["z"].float(), 0.0), heads, Dk, Dv)
    y, S = _chunked(q, k, v, a, S0, on, 0)
    out = {"y": _packed(y).to(dt), "S": S}
    if op == "attend_forward":
        return out
    d = torch.where(on[..., None], s["dy"].float(), 0.0).reshape(B, T, heads, Dv).transpose(1, 2)
    dq, _ = _chunked(d, v, k, a, S0.transpose(2, 3), on, 0)
    q, k, v, d, on = q.flip(2), k.flip(2), v.flip(2), d.flip(2), on.flip(1)
    dv, dS0 = _chunked(k, q, d, a, s["dS"], on, 1)
    dk, _ = _chunked(v, d, q, a, s["dS"].transpose(2, 3), on, 1)
    return dict(out, dz=torch.cat([_packed(dq), _packed(dk.flip(2)), _packed(dv.flip(2))], 2).to(dt), dS0=dS0)


def _plain_norm(s, op):
    x, w = s["x"].float(), s["weight"]
    on = _valid(s["lengths"], x.shape[1])[..., None]
    x = torch.where(on, x, 0.0)
    d = x - x.mean(2, keepdim=True)
    r = 1.0 / torch.sqrt((d * d).mean(2, keepdim=True) + _NORM_EPS)
    n = d * r
    y = torch.where(on, n * w + s["bias"], 0.0).to(s["x"].dtype)
    if op == "norm_forward":
        return y
    dy = torch.where(on, s["dy"].float(), 0.0)
    g = dy * w
    dx = r * (g - g.mean(2, keepdim=True) - n * (g * n).mean(2, keepdim=True))
    return {"y": y, "dx": dx.to(s["dy"].dtype), "dweight": (dy * n).sum((0, 1)), "dbias": dy.sum((0, 1))}


def _plain_clip(s, op):
    total = sum((g.float() ** 2).sum() for g in s["g"])
    norm = torch.sqrt(total)
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    result = torch.stack([norm, scale])
    if op == "clip":
        for g, out in zip(s["g"], s["out"]):
            out.copy_(g.float() * scale)
        return {"result": result, "g": s["out"]}
    s["t"] += 1
    for i, p in enumerate(s["p"]):
        g = s["g"][i].float() * scale
        s["m"][i] = m = _BETA1 * s["m"][i] + (1 - _BETA1) * g
        s["v"][i] = v = _BETA2 * s["v"][i] + (1 - _BETA2) * g * g
        mhat, vhat = m / (1 - _BETA1 ** s["t"]), v / (1 - _BETA2 ** s["t"])
        p.copy_(p - _LR * (mhat / (torch.sqrt(vhat) + _EPS) + _WD * p))
    return {"result": result, "p": s["p"], "m": list(s["m"]), "v": list(s["v"])}


def _plain_sample(s):
    greedy = ~(s["temperature"] > 0)
    T = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]
    x, at = s["logits"].double().sort(dim=1, descending=True, stable=True)      # stable: ties to the lowest index
    w = torch.exp((x - x[:, :1]) / T)
    ratio, (N, V) = w, w.shape
    place = torch.arange(V, device=w.device)
    if s["top_k"] is not None:
        w = torch.where(place < torch.where(s["top_k"] > 0, s["top_k"], V)[:, None], w, 0.0)
    if s["top_p"] is not None:
        c = w.cumsum(1)
        w = torch.where(c - w < s["top_p"].double()[:, None] * w.sum(1, keepdim=True), w, 0.0)
    if s["min_p"] is not None:
        w = torch.where(ratio < s["min_p"].double()[:, None], 0.0, w)
    w = torch.where(greedy[:, None], (place == 0).double(), w)
    w = torch.zeros_like(w).scatter_(1, at, w)
    total = w.sum(1, keepdim=True)
    token = (w.cumsum(1) <= s["u"].double()[:, None] * total).sum(1, keepdim=True).clamp(max=V - 1)
    token = torch.where(greedy[:, None], at[:, :1], token)
    logp = torch.log(w.gather(1, token) / total)
    return {"token": token[:, 0].int(), "logp": logp[:, 0].float()}


# --- what a pass cannot do without ------------------------------------------

def work(case):
    op = case["op"]
    if op.startswith("attend"):
        e, heads, Dk, Dv = _SIZE[case["dtype"]], case["heads"], case["Dk"], case["Dv"]
        N, state = case["B"] * case["T"], 4 * case["B"] * heads * Dk * Dv
        n = N / 2 if case["ragged"] else N        # valid steps (expected)
        row, products = heads * (2 * Dk + Dv), heads * Dk * Dv
        moved = n * row * e + N * heads * Dv * e + 2 * state
        if op == "attend_train":
            moved += n * (row + heads * Dv) * e + N * row * e + 3 * state
        # the state's update and its reading; back: state and its gradient formed once, read for dq, dk and dv
        return {"bytes": moved, "flops": n * products * (14 if op == "attend_train" else 4)}
    if op.startswith("norm"):
        e, D, N = _SIZE[case["dtype"]], case["D"], case["B"] * case["T"]
        n = N / 2 if case["ragged"] else N
        moved = n * D * e + N * D * e + 8 * D
        if op == "norm_train":
            ge = _SIZE[case["grad"]]
            moved += n * D * (e + ge) + N * D * ge + 12 * D
        return {"bytes": moved, "flops": n * D * (22 if op == "norm_train" else 8)}
    if op.startswith("clip"):
        n = sum(math.prod(x) for x in _shapes(case))
        e = _SIZE[case["dtype"]]
        each = 3 * e if op == "clip" else 2 * e + 24       # the norm has to be known before the second reading
        return {"bytes": n * each, "flops": n * (3 if op == "clip" else 18)}
    N, V = case["N"], case["V"]
    return {"bytes": N * (V * _SIZE[case["dtype"]] + 28), "flops": 6 * N * V}


# --- the operators' definitions in 64 bits ----------------------------------

def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op.startswith("attend"):
        return _exact_attend(s, case)
    if op.startswith("norm"):
        return _exact_norm(s, op)
    return _exact_sample(s) if op == "sample" else _exact_clip(s, op)


def _exact_attend(s, case):
    """Step by step, a row's state only in its own steps."""
    heads, Dk, Dv, T = case["heads"], case["Dk"], case["Dv"], case["T"]
    z = s["z"] if s["z"].dim() == 3 else s["z"][:, None]
    B = z.shape[0]
    a = torch.tensor(s["decay"], dtype=torch.float32, device="cuda").double()[:, None, None]

    def parts(t):
        r = z[:, t].double()
        return (r[:, :heads * Dk].reshape(B, heads, Dk), r[:, heads * Dk:2 * heads * Dk].reshape(B, heads, Dk),
                r[:, 2 * heads * Dk:].reshape(B, heads, Dv))

    train = case["op"] == "attend_train"
    S, y = s["S0"].double(), torch.zeros((B, T, heads, Dv), device="cuda", dtype=torch.float64)
    dz = torch.zeros(z.shape, device="cuda", dtype=torch.float64) if train else None
    grad = (lambda t: s["dy"][:, t].double().reshape(B, heads, Dv)) if train else None
    for t in range(T):
        q, k, v = parts(t)
        on = (t < s["lengths"])[:, None, None]
        S = torch.where(on[..., None], a * S + k[..., None] * v[..., None, :], S)
        y[:, t] = torch.where(on, (q[..., None] * S).sum(2), 0.0)
        if train:
            dz[:, t, :heads * Dk] = torch.where(on, (S * grad(t)[:, :, None]).sum(3), 0.0).flatten(1)
    out = {"y": y.flatten(2), "S": S}
    if case["op"] == "attend_step":
        return {"y": out["y"][:, 0], "S": S}
    if not train:
        return out
    R = s["dS"].double()
    for t in reversed(range(T)):
        q, k, v = parts(t)
        on = (t < s["lengths"])[:, None, None]
        new = R + q[..., None] * grad(t)[:, :, None]
        dk, dv = (new * v[:, :, None]).sum(3), (new * k[..., None]).sum(2)
        dz[:, t, heads * Dk:] = torch.cat([torch.where(on, dk, 0.0).flatten(1), torch.where(on, dv, 0.0).flatten(1)], 1)
        R = torch.where(on[..., None], a * new, R)
    return dict(out, dz=dz, dS0=R)


def _exact_norm(s, op):
    on = _valid(s["lengths"], s["x"].shape[1])
    x, w = s["x"][on].double(), s["weight"].double()
    centred = x - x.mean(1, keepdim=True)
    std = (centred.square().mean(1, keepdim=True) + _NORM_EPS).sqrt()
    unit = centred / std
    y = torch.zeros(s["x"].shape, device="cuda", dtype=torch.float64)
    y[on] = unit * w + s["bias"].double()
    if op == "norm_forward":
        return y
    dy = s["dy"][on].double()
    dweight, dbias = (dy * unit).sum(0), dy.sum(0)
    dy *= w
    proj = unit * (dy * unit).mean(1, keepdim=True)
    dx = torch.zeros(s["x"].shape, device="cuda", dtype=torch.float64)
    dx[on] = (dy - dy.mean(1, keepdim=True) - proj) / std
    return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}


def _exact_clip(s, op):
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in s["g"]))
    scale = min(1.0, s["max_norm"] / norm)
    out = {"result": torch.tensor([norm, scale], dtype=torch.float64, device="cuda")}
    if op == "clip":
        return dict(out, g=[g.double() * scale for g in s["g"]])
    t, out = s["t"] + 1, dict(out, p=[], m=[], v=[])
    for i, p in enumerate(s["p"]):
        g, m, v = s["g"][i].double() * scale, s["m"][i].double(), s["v"][i].double()
        m += (g - m) * (1 - _BETA1)
        v += (g * g - v) * (1 - _BETA2)
        root = (v / (1 - _BETA2 ** t)) ** 0.5
        out["p"].append(p.double() * (1 - _LR * _WD) - _LR * (m / (1 - _BETA1 ** t)) / (root + _EPS))
        out["m"].append(m)
        out["v"].append(v)
    return out


def _exact_sample(s):
    """Row by row on the host: the tokens in order, cut after each filter."""
    host = {k: (t.float().cpu().numpy().astype(np.float64) if t is not None else None)
            for k, t in s.items() if k in ("logits", "u", "temperature", "top_k", "top_p", "min_p")}
    tokens, logps = [], []
    for n, x in enumerate(host["logits"]):
        order = np.lexsort((np.arange(len(x)), -x))
        if not host["temperature"][n] > 0:
            tokens.append(order[0])
            logps.append(0.0)
            continue
        if host["top_k"] is not None and host["top_k"][n] > 0:
            order = order[:int(host["top_k"][n])]
        p = np.exp((x[order] - x[order[0]]) / host["temperature"][n])
        if host["top_p"] is not None:
            keep = 1 + int(np.searchsorted(np.cumsum(p), host["top_p"][n] * p.sum()))
            order, p = order[:keep], p[:keep]
        if host["min_p"] is not None:
            order, p = order[p >= host["min_p"][n] * p[0]], p[p >= host["min_p"][n] * p[0]]
        by_index = np.argsort(order)
        order, p = order[by_index], p[by_index]
        c = np.cumsum(p)
        j = int(np.searchsorted(c, host["u"][n] * c[-1], side="right"))
        tokens.append(order[j])
        logps.append(math.log(p[j] / c[-1]))
    return {"token": torch.tensor(np.array(tokens), dtype=torch.int32, device="cuda"),
            "logp": torch.tensor(logps, dtype=torch.float64, device="cuda")}
