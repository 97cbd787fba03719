"""Performance cases of the operators around the time loop: what is timed, on
which inputs, and what comes out.

A case is a dict of plain values; "op" names the operator and its direction:
  scan_step, scan_forward, scan_train    gated linear recurrence: one token per row,
           the whole sequence, the sequence and its gradients
  embed_lookup, embed_train              rows of a token table; and the table's gradient
  adamw                                  one optimizer step over many tensors
  beam                                   one selection of a beam search, states reordered

With `own` false, run() computes the operators in elementary torch operations
in 32 bits; with `own` true it calls the framework.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_BLOCK = 256      # elements that share the exponent of an 8-bit state
_BETA1, _BETA2, _EPS, _WD, _LR = 0.9, 0.999, 1e-8, 0.01, 1e-3


# --- cases ------------------------------------------------------------------

def _scan(op, dtype, B, T, H, ragged):
    return {"op": op, "dtype": dtype, "B": B, "T": T, "H": H, "ragged": ragged}


def _embed(op, dtype, grad, B, T, V, D, ragged):
    return {"op": op, "dtype": dtype, "grad": grad, "B": B, "T": T, "V": V, "D": D, "ragged": ragged}


def _adamw(bits, copies, layers, D, H, V):
    return {"op": "adamw", "bits": bits, "copies": copies, "layers": layers, "D": D, "H": H, "V": V}


def _beam(dtype, B, K, V, H):
    return {"op": "beam", "dtype": dtype, "B": B, "K": K, "V": V, "H": H}


def listed():
    named = {
        # one generated token for each of a few rows: a launch and its latency
        "scan_step_b16_h512": _scan("scan_step", "bf16", 16, 1, 512, False),
        # one long prompt: few channels, so the time axis has to be split
        "scan_prompt_t32768": _scan("scan_forward", "bf16", 1, 32768, 2048, False),
        # a training batch at sizes that are no multiple of any tile, fp32
        "scan_train_odd_f32": _scan("scan_train", "f32", 37, 301, 750, True),
        # the largest training batch: long documents of different lengths
        "scan_train_large": _scan("scan_train", "bf16", 32, 4096, 2048, True),
        # serving: the row of one new token for each of 64 sequences
        "embed_lookup_b64": _embed("embed_lookup", "bf16", "bf16", 64, 1, 32768, 512, False),
        # a small odd training batch, fp32: most rows of the table get no gradient
        "embed_train_odd_f32": _embed("embed_train", "f32", "f32", 21, 45, 10007, 333, True),
        # the largest: long rows, a large table, some tokens far more frequent than others,
        # the gradient in fp32 as the time loop's backward gives it
        "embed_train_large": _embed("embed_train", "bf16", "f32", 256, 1000, 65536, 1024, True),
        # a stack of ordinary fp32 layers
        "adamw_5x256": _adamw(32, False, 5, 256, 256, 1000),
        # a wide bf16 model with a large token table, its states held in 8 bits
        "adamw_large_8bit": _adamw(8, True, 3, 1024, 2048, 65536),
        # one sequence decoded with a few beams over a small vocabulary
        "beam_b1_k4": _beam("f32", 1, 4, 1000, 256),
        # an ordinary decoding batch
        "beam_b16_k8": _beam("bf16", 16, 8, 32768, 512),
        # the largest: many sequences, many beams, a large vocabulary, wide states
        "beam_b64_k16": _beam("bf16", 64, 16, 65536, 2048),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, low, high):
    """A whole number, spread over the logarithm of its range."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _width(rng, low, high):
    """A layer's width: a multiple of 32 as often as any number."""
    w = _log(rng, low, high)
    return w // 160 * 160 if rng.random() < 0.5 and w >= 160 else w


def draw(rng):
    op = rng.choice(["scan_step", "scan_forward", "scan_train", "embed_lookup", "embed_train", "adamw", "beam"])
    dtype = rng.choice(["f32", "bf16"])
    ragged = rng.random() < 0.5
    if op == "scan_step":
        return _scan(op, dtype, _log(rng, 1, 512), 1, _width(rng, 16, 2560), False)
    if op in ("scan_forward", "scan_train"):
        B, H, T = _log(rng, 1, 256), _width(rng, 16, 2560), _log(rng, 2, 32768)
        T = max(2, min(T, (1 << (28 if dtype == "bf16" else 27)) // (B * H)))
        return _scan(op, dtype, B, T, H, ragged)
    if op in ("embed_lookup", "embed_train"):
        V, D = _log(rng, 64, 65536), _width(rng, 16, 2048)
        V = min(V, (1 << 26) // D)
        B, T = _log(rng, 1, 256), _log(rng, 1, 1000)
        T = max(1, min(T, (1 << 27) // (B * D)))
        return _embed(op, dtype, rng.choice(["f32", "bf16"]), B, T, V, D, ragged)
    if op == "adamw":
        return _adamw(rng.choice([32, 8]), rng.random() < 0.5, rng.randint(1, 5), _width(rng, 16, 1024),
                      _width(rng, 16, 1024), _log(rng, 64, 16384))
    B, K, V = _log(rng, 1, 64), _log(rng, 1, 16), _log(rng, 64, 65536)
    return _beam(dtype, B, K, max(64, min(V, (1 << (26 if dtype == "bf16" else 25)) // (B * K))),
                 _width(rng, 16, 2048))


# --- inputs -----------------------------------------------------------------

def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, mean=0.0, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(mean, std, generator=g)


def _lengths(g, B, T, ragged):
    if not ragged:
        return torch.full((B,), T, dtype=torch.int32, device="cuda")
    L = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    L[0] = T
    return L


def _tokens(g, B, T, V):
    """Token ids whose frequency falls as one over their rank; the ranks are scattered over the ids."""
    rank = torch.exp(torch.rand((B, T), generator=g, device="cuda", dtype=torch.float64) * math.log(V)).long().clamp_(1, V) - 1
    return ((rank * 40503 + 17) % V).int()


def _shapes(case):
    """An LSTM stack's tensors (W, U, b of each layer) and a token table."""
    D, H = case["D"], case["H"]
    one = [(H, 4 * H), (H, 4 * H), (4 * H,)]
    return [(case["V"], D)] + [(D, 4 * H)] + one[1:] + one * (case["layers"] - 1)


def _inputs(case, seed):
    """The tensors of a case, from its seed alone."""
    g, op = _rng(seed), case["op"]
    if op.startswith("scan"):
        B, T, H, dt = case["B"], case["T"], case["H"], _DT[case["dtype"]]
        z = _normal(g, (B, T, 3 * H), dtype=dt)
        z[..., :H] += 2.0                       # a forget gate's usual bias: memories of some ten steps
        s = {"z": z, "h0": _normal(g, (B, H), std=0.5), "lengths": _lengths(g, B, T, case["ragged"])}
        if op == "scan_step":
            s["z"] = z[:, 0].contiguous()
        if op == "scan_train":
            s["dy"] = _normal(g, (B, T, H), dtype=dt)
            s["dh"] = _normal(g, (B, H))
        return s
    if op.startswith("embed"):
        B, T, V, D = case["B"], case["T"], case["V"], case["D"]
        s = {"table": _normal(g, (V, D), std=D ** -0.5, dtype=_DT[case["dtype"]]),
             "tokens": _tokens(g, B, T, V), "lengths": _lengths(g, B, T, case["ragged"]), "scale": math.sqrt(D)}
        if op == "embed_train":
            s["dx"] = _normal(g, (B, T, D), dtype=_DT[case["grad"]])
        return s
    if op == "adamw":
        s = {"p": [], "g": [], "m": [], "v": [], "mexp": [], "vexp": [], "copy": [], "t": 100}
        for shape in _shapes(case):
            n, last = math.prod(shape), shape[-1]
            size = torch.exp(_normal(g, (last,), mean=-7.0))       # columns differ in the size of their gradients
            s["p"].append(_normal(g, shape, std=last ** -0.5))
            s["g"].append(_normal(g, shape) * size)
            m = (_normal(g, shape) * size * 0.3).reshape(-1)
            r = ((_normal(g, shape, std=0.2) + 1.0).abs() * size).reshape(-1)
            if case["bits"] == 8:
                (m, me), (r, re) = _to8(m), _to8(r, True)
                s["m"].append(m), s["v"].append(r), s["mexp"].append(me), s["vexp"].append(re)
            else:
                s["m"].append(m.reshape(shape)), s["v"].append((r * r).reshape(shape))
            if case["copies"]:
                s["copy"].append(s["p"][-1].bfloat16())
        return s
    B, K, V, H = case["B"], case["K"], case["V"], case["H"]
    s = {"logits": _normal(g, (B, K, V), std=2.0, dtype=_DT[case["dtype"]]), "end": 2,
         "scores": -10.0 + _normal(g, (B, K)).sort(1, descending=True).values,
         "finished": (torch.rand((B, K), generator=g, device="cuda") < 0.1).to(torch.uint8),
         "h": _normal(g, (B, K, H), std=0.3), "c": _normal(g, (B, K, H))}
    s["logits"][..., 0] = -math.inf                                # a token that is never to be chosen
    _spread_scores(s, g)
    return s


def _spread_scores(s, g):
    """Draw again the scores of sequences in which two of the best candidates are nearer than
    rounding in 32 bits can tell apart; equal logits of one beam stay as they are (ties)."""
    B, K, V = s["logits"].shape
    x = s["logits"].double()
    logp = x - torch.logsumexp(x, 2, keepdim=True)
    best, at = logp.topk(min(V, K + 1), 2)
    live = s["finished"] == 0
    for _ in range(20):
        sc = s["scores"].double()
        c = torch.where(live[..., None], sc[..., None] + best, -math.inf)
        c = torch.cat([c.flatten(1), torch.where(live, -math.inf, sc)], 1).sort(1, descending=True).values[:, :K + 1]
        gap = c[:, :-1] - c[:, 1:]
        near = ((gap < 5e-5) & (gap > 1e-12)).any(1)
        s["scores"] = torch.where(near[:, None], -10.0 + _normal(g, (B, K)).sort(1, descending=True).values, s["scores"])


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if not own:
        return s
    import paper_1810_08061_amd as ld
    op = case["op"]
    if op.startswith("scan"):
        s["handle"] = ld.GatedScan(case["B"], case["H"], case["T"], case["dtype"])
    elif op.startswith("embed"):
        s["handle"] = ld.TokenEmbed(case["B"], case["T"], case["V"], case["D"], case["dtype"], scale=s["scale"])
    elif op == "adamw":
        s["handle"] = ld.AdamW(s["p"], copies=s["copy"] or None, state_bits=case["bits"], betas=(_BETA1, _BETA2),
                               eps=_EPS, weight_decay=_WD, steps_done=s["t"])
        s["handle"].load_state(s["m"], s["v"], s["mexp"] or None, s["vexp"] or None)
        s["m"] = s["v"] = s["mexp"] = s["vexp"] = None
    else:
        s["handle"] = ld.BeamSearch(case["B"], case["K"], case["V"], case["dtype"], end=s["end"])
    return s


# --- one pass ---------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    op, h = s["case"]["op"], s["handle"]
    if op == "scan_step":
        y, out_h = h.step(s["z"], s["h0"])
        return {"y": y, "h": out_h}
    if op == "scan_forward":
        y, out_h = h.forward(s["z"], s["lengths"], s["h0"])
        return {"y": y, "h": out_h}
    if op == "scan_train":
        y, out_h = h.forward_train(s["z"], s["lengths"], s["h0"])
        return dict(h.backward(s["z"], s["lengths"], s["h0"], s["dy"], s["dh"]), y=y, h=out_h)
    if op == "embed_lookup":
        return h.forward(s["tokens"], s["lengths"], s["table"])
    if op == "embed_train":
        return {"x": h.forward(s["tokens"], s["lengths"], s["table"]),
                "dtable": h.backward(s["tokens"], s["lengths"], s["dx"])}
    if op == "adamw":
        h.step(s["g"], _LR)
        m, v = h.states()
        return {"p": s["p"], "copy": s["copy"], "m": m, "v": v}
    scores, parent, token, finished, (hh, cc) = h.step(s["logits"], s["scores"], s["finished"], [s["h"], s["c"]])
    return {"scores": scores, "parent": parent, "token": token, "finished": finished, "h": hh, "c": cc}


def _valid(lengths, T):
    return torch.arange(T, device=lengths.device) < lengths[:, None]


def _scan_doubling(a, u):
    """h_t = a_t h_{t-1} + u_t along dim 1 from h_{-1} = 0: after the pass with distance d, u_t is the sum over the last 2 d steps."""
    d, T = 1, a.shape[1]
    while d < T:
        u = torch.cat([u[:, :d], torch.addcmul(u[:, d:], a[:, d:], u[:, :-d])], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return u


def _run_plain(s):
    op = s["case"]["op"]
    if op.startswith("scan"):
        return _plain_scan(s, op)
    if op.startswith("embed"):
        return _plain_embed(s, op)
    return _plain_adamw(s) if op == "adamw" else _plain_beam(s)


def _plain_scan(s, op):
    dt, h0 = s["z"].dtype, s["h0"]
    if op == "scan_step":
        f, v, o = s["z"].float().chunk(3, 1)
        h = h0 + torch.sigmoid(-f) * (v - h0)
        return {"y": (torch.sigmoid(o) * h).to(dt), "h": h}
    f, v, o = s["z"].float().chunk(3, 2)
    T = f.shape[1]
    valid = _valid(s["lengths"], T)[..., None]
    # a step past a row's length keeps the state: a = 1, nothing added
    a = torch.where(valid, torch.sigmoid(f), 1.0)
    b = torch.where(valid, torch.sigmoid(-f), 0.0)
    u = torch.where(valid, b * v, 0.0)
    u[:, 0] += a[:, 0] * h0
    h = _scan_doubling(a, u)
    so = torch.sigmoid(o)
    y = torch.where(valid, so * h, 0.0).to(dt)
    out = {"y": y, "h": h[:, -1].contiguous()}
    if op == "scan_forward":
        return out
    dy = torch.where(valid, s["dy"].float(), 0.0)
    q = torch.where(valid, so, 0.0) * dy
    q[:, -1] += s["dh"]
    # from the last step back: g_t = q_t + a_{t+1} g_{t+1}
    an = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    g = _scan_doubling(an.flip(1), q.flip(1)).flip(1)
    hp = torch.cat([h0[:, None], h[:, :-1]], 1)
    dz = torch.cat([torch.where(valid, g * (hp - v) * a * b, 0.0), torch.where(valid, g * b, 0.0),
                    torch.where(valid, dy * h * so * (1.0 - so), 0.0)], 2).to(dt)
    return dict(out, dz=dz, dh0=a[:, 0] * g[:, 0])


def _plain_embed(s, op):
    table, tokens = s["table"], s["tokens"].long()
    valid = _valid(s["lengths"], tokens.shape[1])[..., None]
    x = torch.where(valid, table[tokens].float() * s["scale"], 0.0).to(table.dtype)
    if op == "embed_lookup":
        return x
    dx = torch.where(valid, s["dx"].float(), 0.0)
    dtable = torch.zeros(table.shape, device=table.device)
    dtable.index_add_(0, tokens.flatten(), dx.flatten(0, 1))
    return {"x": x, "dtable": dtable * s["scale"]}


def _pow2(e):
    return ((e.int() + 127) << 23).view(torch.float32)


def _to8(x, up=False):
    """x in e4m3 with one power of two per 256 elements, the smallest for which the block's largest is at most 448
    (at least 2^-100); `up`: what is not zero is not rounded to zero. Gives the codes and the exponents + 127."""
    n = x.numel()
    w = torch.nn.functional.pad(x, (0, -n % _BLOCK)).reshape(-1, _BLOCK)
    frac, e = torch.frexp(w.abs().amax(1))
    e = torch.where(frac <= 0.875, e - 9, e - 8).clamp(min=-100)
    e = torch.where(frac == 0, -100, e)
    w = w * _pow2(-e)[:, None]
    if up:
        w = torch.where(w > 0, w.clamp(min=2.0 ** -9), w)
    return w.to(torch.float8_e4m3fn).reshape(-1)[:n], (e + 127).to(torch.uint8)


def _from8(code, exp, dtype=torch.float32):
    n = code.numel()
    w = torch.nn.functional.pad(code.to(dtype), (0, -n % _BLOCK)).reshape(-1, _BLOCK)
    return (w * _pow2(exp.int() - 127)[:, None]).reshape(-1)[:n]


def _adamw_math(p, g, m, v, t):
    m = _BETA1 * m + (1 - _BETA1) * g
    v = _BETA2 * v + (1 - _BETA2) * g * g
    mhat, vhat = m / (1 - _BETA1 ** t), v / (1 - _BETA2 ** t)
    return p - _LR * (mhat / (torch.sqrt(vhat) + _EPS) + _WD * p), m, v


def _plain_adamw(s):
    s["t"] += 1
    ms, vs = [], []
    for i, p in enumerate(s["p"]):
        m, v, g = s["m"][i], s["v"][i], s["g"][i]
        if s["case"]["bits"] == 8:
            m = _from8(m, s["mexp"][i]).reshape(p.shape)
            v = _from8(v, s["vexp"][i]).reshape(p.shape).square()
        new, m, v = _adamw_math(p, g, m, v, s["t"])
        p.copy_(new)
        if s["case"]["copies"]:
            s["copy"][i].copy_(new)
        if s["case"]["bits"] == 8:
            s["m"][i], s["mexp"][i] = _to8(m.reshape(-1))
            s["v"][i], s["vexp"][i] = _to8(v.sqrt().reshape(-1), True)
            m = _from8(s["m"][i], s["mexp"][i]).bfloat16().reshape(p.shape)       # exact: 4 bits and a power of two
            v = _from8(s["v"][i], s["vexp"][i]).bfloat16().reshape(p.shape)
        else:
            s["m"][i], s["v"][i] = m, v
        ms.append(m)
        vs.append(v)
    return {"p": s["p"], "copy": s["copy"], "m": ms, "v": vs}


def _plain_beam(s):
    x, end = s["logits"].float(), s["end"]
    B, K, V = x.shape
    top = x.amax(2, keepdim=True)
    logp = x - (top + torch.log(torch.exp(x - top).sum(2, keepdim=True)))
    is_end = torch.arange(V, device=x.device) == end
    logp = torch.where(s["finished"][..., None] != 0, torch.where(is_end, 0.0, -math.inf), logp)
    cand = (s["scores"][..., None] + logp).flatten(1)
    best, at = torch.sort(cand, dim=1, descending=True, stable=True)        # stable: ties to the lowest index
    best, at = best[:, :K].contiguous(), at[:, :K]
    parent, token = at // V, at % V
    finished = ((s["finished"].gather(1, parent) != 0) | (token == end)).to(torch.uint8)
    rows = parent[..., None].expand(B, K, s["h"].shape[2])
    return {"scores": best, "parent": parent.int(), "token": token.int(), "finished": finished,
            "h": s["h"].gather(1, rows), "c": s["c"].gather(1, rows)}


# --- what a pass cannot do without ------------------------------------------

def work(case):
    op = case["op"]
    if op.startswith("scan"):
        e, H, N = _SIZE[case["dtype"]], case["H"], case["B"] * case["T"]
        n = N / 2 if case["ragged"] else N        # valid steps (expected)
        state = 8 * case["B"] * H
        moved = (3 * n + N) * H * e + state
        if op == "scan_train":
            moved += (4 * n + 3 * N) * H * e + state
        return {"bytes": moved, "flops": n * H * (40 if op == "scan_train" else 12)}
    if op.startswith("embed"):
        e, D, N = _SIZE[case["dtype"]], case["D"], case["B"] * case["T"]
        n = N / 2 if case["ragged"] else N
        moved = 4 * n + min(n, case["V"]) * D * e + N * D * e
        if op == "embed_train":
            moved += 4 * n + n * D * _SIZE[case["grad"]] + case["V"] * D * 4
        return {"bytes": moved, "flops": n * D * (2 if op == "embed_train" else 1)}
    if op == "adamw":
        n = sum(math.prod(x) for x in _shapes(case))
        # 8 bits: the states are read and written in 8 bits, and come out as the values they stand for
        each = (28 if case["bits"] == 32 else 12 + 4 + 4) + (2 if case["copies"] else 0)
        return {"bytes": n * each, "flops": 16 * n}
    B, K, V, H = (case[k] for k in "BKVH")
    return {"bytes": B * K * (V * _SIZE[case["dtype"]] + 16 * H), "flops": 4 * B * K * V}


# --- the operators' definitions in 64 bits ----------------------------------

def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op.startswith("scan"):
        return _exact_scan(s, op, case["T"])
    if op.startswith("embed"):
        return _exact_embed(s, op)
    return _exact_adamw(s, case) if op == "adamw" else _exact_beam(s)


def _exact_scan(s, op, T):
    """Step by step."""
    z, L = s["z"], s["lengths"]
    H = s["h0"].shape[1]
    if op == "scan_step":
        z = z[:, None]

    def gates(t):
        f, v, o = z[:, t].double().split(H, 1)
        return 1 / (1 + torch.exp(-f)), v, 1 / (1 + torch.exp(-o))

    # the forward keeps every 64th state; the backward goes back over the steps between
    h, y, kept = s["h0"].double(), torch.zeros(z.shape[:2] + (H,), device="cuda", dtype=torch.float64), []
    for t in range(T):
        if t % 64 == 0:
            kept.append(h)
        a, v, so = gates(t)
        on = (t < L)[:, None]
        h = torch.where(on, a * h + (1 - a) * v, h)
        y[:, t] = torch.where(on, so * h, 0.0)
    if op == "scan_step":
        return {"y": y[:, 0], "h": h}
    out = {"y": y, "h": h}
    if op == "scan_forward":
        return out
    g, dz = s["dh"].double(), torch.zeros(z.shape, device="cuda", dtype=torch.float64)
    for c in reversed(range(len(kept))):
        hs = [kept[c]]
        for t in range(64 * c, min(T, 64 * c + 64)):
            a, v, _ = gates(t)
            hs.append(torch.where((t < L)[:, None], a * hs[-1] + (1 - a) * v, hs[-1]))
        for t in reversed(range(64 * c, min(T, 64 * c + 64))):
            a, v, so = gates(t)
            on, hp, hn = (t < L)[:, None], hs[t - 64 * c], hs[t - 64 * c + 1]
            dy = s["dy"][:, t].double()
            gt = g + so * dy
            dz[:, t] = torch.where(on, torch.cat([gt * (hp - v) * a * (1 - a), gt * (1 - a),
                                                  dy * hn * so * (1 - so)], 1), 0.0)
            g = torch.where(on, a * gt, g)
    return dict(out, dz=dz, dh0=g)


def _exact_embed(s, op):
    V, D = s["table"].shape
    on = _valid(s["lengths"], s["tokens"].shape[1])
    x = torch.zeros(s["tokens"].shape + (D,), device="cuda", dtype=torch.float64)
    x[on] = s["table"].double()[s["tokens"][on].long()] * s["scale"]
    if op == "embed_lookup":
        return x
    order = s["tokens"][on].long().argsort()
    counts = torch.bincount(s["tokens"][on].long(), minlength=V)
    ends = counts.cumsum(0)
    dtable = torch.zeros((V, D), device="cuda", dtype=torch.float64)
    for j in range(0, D, 64):       # sums of the sorted rows, as differences of their running sum
        run_sum = s["dx"][..., j:j + 64][on][order].double().cumsum(0)
        run_sum = torch.cat([run_sum.new_zeros((1, run_sum.shape[1])), run_sum])
        dtable[:, j:j + 64] = (run_sum[ends] - run_sum[ends - counts]) * s["scale"]
    return {"x": x, "dtable": dtable}


def _exact_adamw(s, case):
    t, out = s["t"] + 1, {"p": [], "copy": [], "m": [], "v": []}
    for i, p in enumerate(s["p"]):
        g, eight = s["g"][i].double().reshape(-1), case["bits"] == 8
        m = _from8(s["m"][i], s["mexp"][i], torch.float64) if eight else s["m"][i].double().reshape(-1)
        v = _from8(s["v"][i], s["vexp"][i], torch.float64) ** 2 if eight else s["v"][i].double().reshape(-1)
        m += (g - m) * (1 - _BETA1)
        v += (g * g - v) * (1 - _BETA2)
        root = (v / (1 - _BETA2 ** t)) ** 0.5
        new = p.double().reshape(-1) * (1 - _LR * _WD) - _LR * (m / (1 - _BETA1 ** t)) / (root + _EPS)
        if eight:
            m, v = _from8(*_to8(m)), _from8(*_to8(v ** 0.5, True))
        for k, x in (("p", new), ("copy", new), ("m", m), ("v", v)):
            if k != "copy" or case["copies"]:
                out[k].append(x.reshape(p.shape))
    return out


def _exact_beam(s):
    x, end = s["logits"].double(), s["end"]
    B, K, V = x.shape
    cand = s["scores"].double()[..., None] + torch.log_softmax(x, 2)
    done = s["finished"] != 0
    cand[done] = -math.inf
    cand[..., end] = torch.where(done, s["scores"].double(), cand[..., end])
    cand = cand.flatten(1)
    index = torch.arange(K * V, device="cuda")
    scores, at = [], []
    for _ in range(K):
        best = cand.amax(1, keepdim=True)
        i = torch.where(cand == best, index, K * V).amin(1, keepdim=True)
        cand.scatter_(1, i, -math.inf)     # every beam has a finite candidate: K of them are found
        scores.append(best)
        at.append(i)
    scores, at = torch.cat(scores, 1), torch.cat(at, 1)
    parent, token = at // V, at % V
    finished = (done.gather(1, parent) | (token == end)).to(torch.uint8)
    pick = torch.arange(B, device="cuda")[:, None]
    return {"scores": scores, "parent": parent.int(), "token": token.int(), "finished": finished,
            "h": s["h"][pick, parent].double(), "c": s["c"][pick, parent].double()}
