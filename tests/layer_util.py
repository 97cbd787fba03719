"""Plain 64-bit definitions of the layer's operators, on the CPU, for their tests."""
import numpy as np

U = 2.0 ** -24      # half a unit in the last place of a number in [1, 2), in fp32
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}   # rounding to the data's type, relative


def attend(z, lengths, S0, decay, Dk, Dv, dy=None, dS=None):
    """z [B, T, heads (2 Dk + Dv)] float64, step by step; a dict of y, S and (with dy) dz, dS0."""
    B, T, _ = z.shape
    heads = len(decay)
    q, k, v = (x.reshape(B, T, heads, -1) for x in np.split(z, [heads * Dk, 2 * heads * Dk], axis=2))
    a = np.asarray(decay)[:, None, None]
    y, out_S = np.zeros((B, T, heads, Dv)), S0.copy()
    dq, dk, dv, dS0 = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros_like(S0)
    for b in range(B):
        S, L = S0[b], int(lengths[b])
        for t in range(L):
            S = a * S + k[b, t][:, :, None] * v[b, t][:, None, :]
            y[b, t] = np.einsum("hk,hkv->hv", q[b, t], S)
            if dy is not None:
                dq[b, t] = np.einsum("hkv,hv->hk", S, dy[b, t].reshape(heads, Dv))
        out_S[b] = S
        if dy is None:
            continue
        R = dS[b] if dS is not None else np.zeros_like(S)
        for t in reversed(range(L)):
            R = R + q[b, t][:, :, None] * dy[b, t].reshape(heads, 1, Dv)
            dk[b, t] = np.einsum("hkv,hv->hk", R, v[b, t])
            dv[b, t] = np.einsum("hkv,hk->hv", R, k[b, t])
            R = a * R
        dS0[b] = R
    flat = lambda x: x.reshape(B, T, -1)
    out = {"y": flat(y), "S": out_S}
    return out if dy is None else dict(out, dz=np.concatenate([flat(dq), flat(dk), flat(dv)], 2), dS0=dS0)


def attend_bounds(z, lengths, S0, decay, Dk, Dv, dtype, dy=None, dS=None):
    """What rounding may do to attend's results, element by element: every result is a sum of products, so the same
    formula over magnitudes (m) bounds it.  A product meets at most 3 roundings a step of the
    sums that it is added to (three parts in bf16), Dk or Dv in the sum over the state's rows, and some 200 in a
    chunk's sums and decays.  bf16: two parts of a state or a masked product leave 2^-17 of it."""
    ab = np.abs
    m = attend(ab(z), lengths, ab(S0), decay, Dk, Dv, None if dy is None else ab(dy), None if dS is None else ab(dS))
    n = 3 * z.shape[1] + max(Dk, Dv) + 200
    two = 2.0 ** -17 if dtype == "bf16" else 0.0
    return {k: x * (n * U + (two if k in ("y", "dz") else 0.0)) for k, x in m.items()}, m, n


def norm(x, lengths, w, b, eps, dy=None):
    """x [B, T, D] float64; y and (with dy) dx, dweight, dbias, and bounds of each for fp32 arithmetic.

    A sum over a row passes at most 32 additions of a thread, 6 over lanes and 16 over waves: 54 roundings,
    60 with those of its terms.  With A the row's largest |x| and s its deviation, d = x - mean is off by 60 U A,
    its square sum relatively by twice that over s, so n by 60 U (A / s + 1) (1 + |n|)."""
    B, T, D = x.shape
    w = np.ones(D) if w is None else w
    b = np.zeros(D) if b is None else b
    out = {"y": np.zeros_like(x)}
    bound = {"y": np.zeros_like(x)}
    if dy is not None:
        for k, shape in (("dx", x.shape), ("dweight", (D,)), ("dbias", (D,))):
            out[k], bound[k] = np.zeros(shape), np.zeros(shape)
    rows, mag_w, mag_b = 0, np.zeros(D), np.zeros(D)
    for i in range(B):
        for t in range(int(lengths[i])):
            r = x[i, t]
            d = r - r.mean()
            s = np.sqrt((d * d).mean() + eps)
            n = d / s
            e = 60 * U * (np.abs(r).max() / s + 1)
            en = e * (1 + np.abs(n))
            out["y"][i, t] = n * w + b
            bound["y"][i, t] = np.abs(w) * en + 2 * U * (np.abs(n * w) + np.abs(b))
            if dy is None:
                continue
            g = dy[i, t] * w
            m0, m1 = g.mean(), (g * n).mean()
            out["dx"][i, t] = (g - m0 - n * m1) / s
            G, N = np.abs(g).max(), np.abs(n).max()
            bound["dx"][i, t] = (G * (70 * U * (1 + N * N) + 2 * N * en.max()) + en * abs(m1)) / s + np.abs(out["dx"][i, t]) * e
            out["dweight"] += dy[i, t] * n
            out["dbias"] += dy[i, t]
            mag_w += np.abs(dy[i, t] * n)
            mag_b += np.abs(dy[i, t])
            bound["dweight"] += np.abs(dy[i, t]) * en
            rows += 1
    if dy is not None:
        bound["dweight"] += (rows + 64) * U * mag_w
        bound["dbias"] += (rows + 64) * U * mag_b
    return out, bound


def sample(x, u, T, top_k, top_p, min_p):
    """One row's token, its log probability, and how near rounding was to deciding either (the least distance
    of top_p and u from a sum that they are compared with, as a share of all; of min_p from a ratio)."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    order = np.lexsort((np.arange(len(x)), -x))
    if not x[order[0]] > -np.inf:
        return -1, -np.inf, 1.0
    if not T > 0:
        return int(order[0]), 0.0, 1.0
    near = 1.0
    if 0 < top_k < len(x):
        order = order[:top_k]
    with np.errstate(invalid="ignore"):
        d = np.where(x[order] == x[order[0]], 0.0, x[order] - x[order[0]])
    p = np.exp(d / T)
    ratio = p.copy()
    if top_p < 1:
        c = np.cumsum(p) / p.sum()
        keep = 1 + int(np.searchsorted(c, top_p)) if top_p > 0 else 1
        near = min(near, np.abs(c[p > 0] - top_p).min())
        order, p, ratio = order[:keep], p[:keep], ratio[:keep]
    if min_p > 0:
        near = min(near, np.abs(ratio / min(min_p, 1.0) - 1)[ratio < 1].min(initial=1.0))
        order, p = order[ratio >= min(min_p, 1.0)], p[ratio >= min(min_p, 1.0)]
    by = np.argsort(order)
    order, p = order[by], p[by]
    c = np.cumsum(p) / p.sum()
    j = int(np.searchsorted(c, u, side="right"))
    near = min(near, np.abs(c[:-1][p[:-1] > 0] - u).min(initial=1.0))
    return int(order[j]), float(np.log(p[j] / p.sum())), near
