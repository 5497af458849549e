"""CPU oracle of the training operators -- TEST INFRASTRUCTURE, NOT THE PRODUCT.

Plain fp64 numpy statements of the gradients of both softmax attentions and of layer norm, from their formulas; imports
nothing from the package.  Pins: tests/test_oracle_pins_gradients.py (torch's automatic differentiation of the forward
definition, central differences, closed forms).

    P = RowSoftmax(scale Q K^T),  dP = dO V^T,  dS = P (dP - rowsum(P dP))
    dV = P^T dO,  dQ = scale dS K,  dK = scale dS^T Q

Every gradient of the attentions comes with a *magnitude*: the same sum with every term's absolute value and every product's
factors likewise, which is what roundings of single terms and of sums are relative to.
"""
from __future__ import annotations

import numpy as np

F64 = np.float64


def attention_backward(Q, K, V, dO, H: int, scale=None, own=None):
    """Gradients of multi-head RowSoftmax(scale Q K^T) V: dict of dQ [n, d], dK, dV [L, d], and with own = (K', V') [n, d] (one more
    key and value of each row's own) dKs, dVs [n, d].  Keys with "|..|" hold the magnitudes, "A" the largest sum of |products| of a
    score."""
    Q, K, V, dO = (np.asarray(a, dtype=F64) for a in (Q, K, V, dO))
    n, d = Q.shape
    dh = d // H
    scale = 1.0 / np.sqrt(dh) if not scale else scale
    names = ("dQ", "dK", "dV") + (("dKs", "dVs") if own is not None else ())
    like = {"dQ": Q, "dK": K, "dV": V, "dKs": Q, "dVs": Q}
    out = {k: np.zeros_like(like[k]) for k in names}
    out |= {f"|{k}|": np.zeros_like(like[k]) for k in names}
    out["A"] = 0.0
    L = K.shape[0]
    if L == 0 and own is None:
        return out
    for h in range(H):
        c = slice(h * dh, (h + 1) * dh)
        q, k, v, do = Q[:, c], K[:, c], V[:, c], dO[:, c]
        s, dp, t = scale * (q @ k.T), do @ v.T, np.abs(do) @ np.abs(v).T
        out["A"] = max(out["A"], (scale * (np.abs(q) @ np.abs(k).T)).max(initial=0.0))
        if own is not None:
            ks, vs = (np.asarray(o, dtype=F64)[:, c] for o in own)
            s = np.concatenate([s, scale * (q * ks).sum(1, keepdims=True)], 1)
            dp = np.concatenate([dp, (do * vs).sum(1, keepdims=True)], 1)
            t = np.concatenate([t, (np.abs(do) * np.abs(vs)).sum(1, keepdims=True)], 1)
            out["A"] = max(out["A"], (scale * (np.abs(q) * np.abs(ks)).sum(1)).max())
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        ds = p * (dp - (p * dp).sum(1, keepdims=True))
        m = p * (t + (p * t).sum(1, keepdims=True))              # magnitude of ds
        out["dQ"][:, c], out["|dQ|"][:, c] = scale * ds[:, :L] @ k, scale * m[:, :L] @ np.abs(k)
        out["dK"][:, c], out["|dK|"][:, c] = scale * ds[:, :L].T @ q, scale * m[:, :L].T @ np.abs(q)
        out["dV"][:, c], out["|dV|"][:, c] = p[:, :L].T @ do, p[:, :L].T @ np.abs(do)
        if own is not None:
            out["dQ"][:, c] += scale * ds[:, L:] * ks
            out["|dQ|"][:, c] += scale * m[:, L:] * np.abs(ks)
            out["dKs"][:, c], out["|dKs|"][:, c] = scale * ds[:, L:] * q, scale * m[:, L:] * np.abs(q)
            out["dVs"][:, c], out["|dVs|"][:, c] = p[:, L:] * do, p[:, L:] * np.abs(do)
    return out


def summarize_backward(X, offsets, Q, W_k, W_v, dO, H: int, scale=None, self_term=False):
    """Per user the gradients of stage 1 with respect to queries and projected keys and values (a list of dicts of
    attention_backward; users without history have zeros)."""
    X, Wk, Wv = (np.asarray(a, dtype=F64) for a in (X, W_k, W_v))
    got = []
    for b in range(len(offsets) - 1):
        x = X[offsets[b]:offsets[b + 1]]
        q = np.asarray(Q[b] if Q.ndim == 3 else Q, dtype=F64)
        own = (q @ Wk, q @ Wv) if self_term and len(x) else None
        g = attention_backward(q, x @ Wk, x @ Wv, dO[b], H, scale, own)
        # the projections' own sums
        g["A"] = max([g["A"]] + [float((np.abs(q[:, c]) @ (np.abs(x) @ np.abs(Wk[:, c])).T).max() * (scale or (q.shape[1] // H) ** -0.5))
                                 for c in (slice(h * q.shape[1] // H, (h + 1) * q.shape[1] // H) for h in range(H)) if len(x)])
        if self_term and own is None:
            g |= {k: np.zeros_like(q) for k in ("dKs", "dVs", "|dKs|", "|dVs|")}
        got.append(g)
    return got


def target_attend_backward(T, Y, dO, H: int, scale=None, self_term=False):
    """One user's candidates T [C, d] over summaries Y [S, d], which are keys and values at once: dict of dT, dY, magnitudes, A."""
    g = attention_backward(T, Y, Y, dO, H, scale, (T, T) if self_term else None)
    out = {"dT": g["dQ"], "|dT|": g["|dQ|"], "dY": g["dK"] + g["dV"], "|dY|": g["|dK|"] + g["|dV|"], "A": g["A"]}
    if self_term:                                  # the candidate as its own key and value
        out["dT"] = out["dT"] + g["dKs"] + g["dVs"]
        out["|dT|"] = out["|dT|"] + g["|dKs|"] + g["|dVs|"]
    return out


def layer_norm(x, w=None, b=None, eps=1e-6):
    """(x - mean) / sqrt(var + eps) * w + b over the last axis."""
    x = np.asarray(x, dtype=F64)
    z = x - x.mean(-1, keepdims=True)
    z = z / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
    z = z if w is None else z * np.asarray(w, dtype=F64)
    return z if b is None else z + np.asarray(b, dtype=F64)


def layer_norm_backward(x, w, dy, eps=1e-6):
    """(dx, dw, db); w may be None (ones)."""
    x, dy = np.asarray(x, dtype=F64), np.asarray(dy, dtype=F64)
    c = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    z = c * r
    g = dy if w is None else dy * np.asarray(w, dtype=F64)
    dx = r * (g - g.mean(-1, keepdims=True) - z * (g * z).mean(-1, keepdims=True))
    rows = tuple(range(x.ndim - 1))
    return dx, (dy * z).sum(rows), dy.sum(rows)
