"""Plain 64-bit references of the ragged-batch calls and of the norms of queries and
keys, and the comparison their tests use."""
import numpy as np
import torch

# half a rounding step relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def f64(t):
    return None if t is None else t.detach().to("cpu").double().numpy()


def close(name, X, R, delta):
    """|X - R| <= half a step of X's type at R + delta RMS(R), element by element: what
    the output's own rounding takes, and `delta` for everything before it."""
    r = f64(X) if isinstance(X, torch.Tensor) else np.asarray(X)
    R = np.asarray(R)
    assert r.shape == R.shape, f"{name}: {r.shape} != {R.shape}"
    if not R.size:
        return
    assert np.isfinite(r).all(), f"{name}: not finite"
    rms = float(np.sqrt(np.mean(R * R)))
    over = np.abs(r - R) - HALF[X.dtype] * (np.abs(R) + delta * rms)
    worst = float(over.max()) / max(rms, 1e-300)
    print(f"  {name:8s} beyond rounding: {worst:.2e} rms (allowed {delta:g})", flush=True)
    assert worst <= delta, f"{name}: {worst:.3e} > {delta}"


def sequences(lens, T=None, before=0):
    cu = np.cumsum([before] + list(lens))
    return cu, (int(cu[-1]) if T is None else T)


def gdn(q, k, v, g, beta, state, cu, slots, fresh=None):
    """Token by token.  Returns (o, written, state): `written` marks the rows of o that
    belong to a sequence with a slot."""
    q, k, v, g, beta = (f64(x) for x in (q, k, v, g, beta))
    state = f64(state).copy()
    T, Hv, Dv = v.shape
    group = Hv // q.shape[1]
    o, written = np.zeros((T, Hv, Dv)), np.zeros(T, bool)
    for i in range(len(cu) - 1):
        slot = i if slots is None else int(slots[i])
        b, e = (min(max(int(x), 0), T) for x in cu[i:i + 2])
        if e <= b or not 0 <= slot < len(state):
            continue
        S = np.zeros_like(state[slot]) if fresh is not None and fresh[i] else state[slot]
        for t in range(b, e):
            kt, qt = np.repeat(k[t], group, 0), np.repeat(q[t], group, 0)
            S = np.exp(g[t])[:, None, None] * S
            u = beta[t][:, None] * (v[t] - np.einsum("hkv,hk->hv", S, kt))
            S = S + kt[:, :, None] * u[:, None, :]
            o[t] = np.einsum("hkv,hk->hv", S, qt)
        written[b:e] = True
        state[slot] = S
    return o, written, state


def conv(x, w, tails, cu, slots, fresh=None, act="silu"):
    x, w = f64(x), f64(w)
    T, C = x.shape
    W = w.shape[1]
    tails = np.zeros((1 << 30 if slots is None else int(max(slots)) + 1, 0, C)) if W == 1 else f64(tails).copy()
    y, written = np.zeros((T, C)), np.zeros(T, bool)
    for i in range(len(cu) - 1):
        slot = i if slots is None else int(slots[i])
        b, e = (min(max(int(c), 0), T) for c in cu[i:i + 2])
        if e <= b or slot < 0 or slot >= len(tails):
            continue
        tail = np.zeros((W - 1, C)) if fresh is not None and fresh[i] else tails[slot]
        xe = np.concatenate([tail, x[b:e]])
        u = sum(xe[j:j + e - b] * w[:, j] for j in range(W))
        with np.errstate(over="ignore"):
            y[b:e] = u / (1 + np.exp(-u)) if act == "silu" else u
        written[b:e] = True
        if W > 1:
            tails[slot] = xe[e - b:]
    return y, written, tails


def _turn(x, ang, inter):
    """Rows x [..., D] turned by ang [..., R / 2]."""
    n = ang.shape[-1]
    out = x.copy()
    ia, ib = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if inter else (np.arange(n), np.arange(n, 2 * n))
    a, b, c, s = x[..., ia], x[..., ib], np.cos(ang), np.sin(ang)
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    return out


def _one(x, w, norm, eps, scale, ang, inter, dy=None):
    D = x.shape[-1]
    c = {"none": 0.0, "l2": 1.0, "rms": 1.0 / D}[norm]
    r = np.ones(x.shape[:-1] + (1,)) if norm == "none" else 1 / np.sqrt(c * (x * x).sum(-1, keepdims=True) + eps)
    wt = np.ones(D) if w is None else w
    if dy is None:
        z = wt * (r * x)
        return scale * (z if ang is None else _turn(z, ang, inter))
    dz = scale * (dy if ang is None else _turn(dy, -ang, inter))
    h = wt * dz
    dx = r * h - c * r ** 3 * (h * x).sum(-1, keepdims=True) * x
    terms = dz * r * x
    return dx, terms.sum((0, 1, 2)), np.abs(terms).sum((0, 1, 2))


def qk(q, k, *, norm="l2", q_weight=None, k_weight=None, eps=1e-6, q_scale=1.0, inv_freq=None, pos=None, pos0=0,
       interleaved=False, dyq=None, dyk=None):
    """Forward: (q', k'); with dyq, dyk: ((dq, dwq, sum |terms of dwq|), the same of k)."""
    B, L = q.shape[:2]
    ang = None
    if inv_freq is not None and inv_freq.numel():
        p = f64(pos) if pos is not None else np.broadcast_to(pos0 + np.arange(L, dtype=np.float64), (B, L))
        ang = (p[..., None] * f64(inv_freq))[:, :, None]
    return tuple(_one(f64(x), f64(w), norm, eps, s, ang, interleaved, f64(dy))
                 for x, w, s, dy in ((q, q_weight, q_scale, dyq), (k, k_weight, 1.0, dyk)))
