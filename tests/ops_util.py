"""Plain 64-bit definitions of the operators around the loop, on the CPU, for their tests."""
import numpy as np

U = 2.0 ** -24   # half a unit in the last place of a number in [1, 2), in fp32


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def scan(z, lengths, h0, dy=None, dh=None):
    """z [B, T, 3H] float64; returns a dict of y, h and (with dy) dz, dh0, and the sizes the bounds need."""
    B, T, H3 = z.shape
    H = H3 // 3
    y, out_h = np.zeros((B, T, H)), h0.copy()
    dz, dh0 = np.zeros_like(z), np.zeros((B, H))
    info = {"n": 1.0, "M": 1e-30, "G": 1e-30, "Q": 1e-30, "D": 1e-30}
    for b in range(B):
        L = int(lengths[b])
        f, v, o = np.split(z[b, :L], 3, axis=1)
        a, k, s = sigmoid(f), sigmoid(-f), sigmoid(o)
        hs = [h0[b]]
        for t in range(L):
            hs.append(a[t] * hs[-1] + k[t] * v[t])
            y[b, t] = s[t] * hs[-1]
        out_h[b] = hs[-1]
        info["M"] = max(info["M"], np.abs(np.stack(hs)).max(initial=0.0), np.abs(v).max(initial=0.0))
        if L:  # errors live for 1 / k steps, at most L
            info["n"] = max(info["n"], min(L, 1 / max(k.min(), 1e-30)))
        if dy is None:
            continue
        e = dh[b].copy() if dh is not None else np.zeros(H)
        for t in reversed(range(L)):
            d = dy[b, t]
            g = s[t] * d + e
            dz[b, t] = np.concatenate([g * (hs[t] - v[t]) * a[t] * k[t], g * k[t], d * hs[t + 1] * s[t] * (1 - s[t])])
            e = a[t] * g
            info["G"] = max(info["G"], np.abs(g).max())
            info["Q"] = max(info["Q"], np.abs(hs[t] - v[t]).max())
            info["D"] = max(info["D"], np.abs(d).max())
        dh0[b] = e
    out = {"y": y, "h": out_h, "info": info}
    return out if dy is None else dict(out, dz=dz, dh0=dh0)


def scan_bounds(info, bf16):
    """Largest errors of the kernels' fp32 arithmetic.  The hardware's exp and reciprocal leave a gate
    within 3e-6 of itself (gates' arguments up to 20).  A step adds that times its own share and two
    roundings of the state, and an error dies out over n steps; a piece's product of
    gates and its join with the carried state double the roundings."""
    n, M, G, Q, D = (info[k] for k in "nMGQD")
    h = M * (4e-6 + 4 * U * n)
    g = G * (4e-6 + 8 * U * n)
    out = {"h": h, "y": h + 4e-6 * M, "dh0": g,
           "dz": max(0.25 * (g * Q + G * h + 8e-6 * G * Q), g + 4e-6 * G, 0.25 * (D * h + 8e-6 * D * M))}
    return out, (2.0 ** -8 if bf16 else 0.0)   # relative, where the result is rounded to bf16


def embed_grad(tokens, lengths, dx, V, scale):
    """d_table and the sums of magnitudes and counts its rounding is bounded by."""
    B, T = tokens.shape
    d, mag, cnt = np.zeros((V, dx.shape[2])), np.zeros((V, dx.shape[2])), np.zeros(V)
    for b in range(B):
        for t in range(int(lengths[b])):
            v = int(tokens[b, t])
            if 0 <= v < V:
                d[v] += scale * dx[b, t]
                mag[v] += abs(scale) * np.abs(dx[b, t])
                cnt[v] += 1
    return d, mag, cnt


def beam(logits, scores, finished, end):
    """All candidates [K V] of one sequence; -inf where there is none."""
    x = logits.astype(np.float64).copy()
    x[np.isnan(x)] = -np.inf
    K, V = x.shape
    c = np.full((K, V), -np.inf)
    for k in range(K):
        if finished[k]:
            if 0 <= end < V:
                c[k, end] = scores[k]
            continue
        m = x[k].max()
        if not np.isfinite(m) or not scores[k] > -np.inf:
            continue
        c[k] = scores[k] + (x[k] - (m + np.log(np.exp(x[k] - m).sum())))
    c[np.isnan(c)] = -np.inf
    return c


def e4m3_values():
    """The values of the codes 0 .. 126 in order."""
    v = []
    for c in range(127):
        e, m = c >> 3, c & 7
        v.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)
