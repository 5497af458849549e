"""Pins of oracle/gradients.py on the CPU: automatic differentiation of the forward definitions in fp64, central
differences, closed forms."""
import numpy as np
import pytest
import torch

from oracle import gradients as G
from oracle import vista_oracle as O

CASES = [(7, 5, 6, 2), (1, 1, 4, 1), (3, 9, 15, 3), (4, 1, 8, 2)]


def rnd(seed, *shapes):
    g = np.random.default_rng(seed)
    return [g.normal(size=s) for s in shapes]


def forward(q, k, v, H, own=None):
    outs, dh = [], q.shape[1] // H
    for h in range(H):
        c = slice(h * dh, (h + 1) * dh)
        s = q[:, c] @ k[:, c].T
        if own is not None:
            s = torch.cat([s, (q[:, c] * own[0][:, c]).sum(1, keepdim=True)], 1)
        p = torch.softmax(s / dh ** 0.5, 1)
        outs.append(p[:, :k.shape[0]] @ v[:, c] + (p[:, k.shape[0]:] * own[1][:, c] if own is not None else 0))
    return torch.cat(outs, 1)


@pytest.mark.parametrize("self_term", [False, True])
@pytest.mark.parametrize("n,L,d,H", CASES)
def test_attention_gradients_against_automatic_differentiation(n, L, d, H, self_term):
    q, k, v, do, ks, vs = rnd(1, (n, d), (L, d), (L, d), (n, d), (n, d), (n, d))
    own = (ks, vs) if self_term else None
    at = [torch.from_numpy(a).requires_grad_(True) for a in ((q, k, v) + (own or ()))]
    o = forward(at[0], at[1], at[2], H, tuple(at[3:]) or None)
    want = torch.autograd.grad(o, at, torch.from_numpy(do))
    got = G.attention_backward(q, k, v, do, H, own=own)
    for name, w in zip(("dQ", "dK", "dV", "dKs", "dVs"), want):
        np.testing.assert_allclose(got[name], w.numpy(), rtol=1e-10, atol=1e-13)
        assert np.all(np.abs(got[name]) <= got[f"|{name}|"] * (1 + 1e-12) + 1e-15)


def test_stage1_gradients_by_central_differences():
    d, H, S = 6, 2, 3
    X, Q, Wk, Wv, dO = rnd(2, (5, d), (S, d), (d, d), (d, d), (3, S, d))
    off = np.array([0, 4, 4, 5])
    got = G.summarize_backward(X, off, Q, Wk, Wv, dO, H, self_term=False)
    step = 1e-5
    f = lambda q: (O.summarize(X, off, q, Wk, Wv, H) * dO).sum()
    for i, c in [(0, 0), (1, 5), (2, 3)]:
        e = np.zeros_like(Q)
        e[i, c] = step
        assert abs((f(Q + e) - f(Q - e)) / (2 * step) - sum(g["dQ"][i, c] for g in got)) < 1e-8
    # dX = dK W_k^T + dV W_v^T
    fx = lambda x: (O.summarize(x, off, Q, Wk, Wv, H) * dO).sum()
    for i, c in [(0, 1), (3, 4), (4, 0)]:
        e = np.zeros_like(X)
        e[i, c] = step
        g, r = (got[0], i) if i < 4 else (got[2], 0)
        want = (g["dK"][r] @ Wk.T + g["dV"][r] @ Wv.T)[c]
        assert abs((fx(X + e) - fx(X - e)) / (2 * step) - want) < 1e-8
    assert not got[1]["dQ"].any() and got[1]["dK"].shape == (0, d)


@pytest.mark.parametrize("self_term", [False, True])
def test_stage2_gradients_by_central_differences(self_term):
    d, H, S, C = 4, 2, 3, 5
    T, Y, dO = rnd(3, (1, C, d), (1, S, d), (1, C, d))
    got = G.target_attend_backward(T[0], Y[0], dO[0], H, self_term=self_term)
    f = lambda t, y: (O.target_attend(t, y, H, self_term=self_term) * dO).sum()
    step = 1e-5
    for i in range(3):
        for c in range(d):
            e, k = np.zeros_like(T), np.zeros_like(Y)
            e[0, i, c] = k[0, i, c] = step
            assert abs((f(T + e, Y) - f(T - e, Y)) / (2 * step) - got["dT"][i, c]) < 1e-8
            assert abs((f(T, Y + k) - f(T, Y - k)) / (2 * step) - got["dY"][i, c]) < 1e-8


def test_one_key_has_no_score_gradient():
    q, k, v, do = rnd(4, (3, 4), (1, 4), (1, 4), (3, 4))
    got = G.attention_backward(q, k, v, do, 2)
    assert np.abs(got["dQ"]).max() < 1e-15 and np.abs(got["dK"]).max() < 1e-15
    np.testing.assert_allclose(got["dV"][0], do.sum(0))


@pytest.mark.parametrize("affine", [False, True])
def test_layer_norm_against_automatic_differentiation(affine):
    x, w, b, dy = rnd(5, (4, 3, 7), (7,), (7,), (4, 3, 7))
    at = [torch.from_numpy(a).requires_grad_(True) for a in ((x, w, b) if affine else (x,))]
    y = torch.nn.functional.layer_norm(at[0], (7,), *at[1:], eps=1e-6)
    want = torch.autograd.grad(y, at, torch.from_numpy(dy))
    np.testing.assert_allclose(G.layer_norm(x, *((w, b) if affine else ())), y.detach().numpy(), rtol=1e-11, atol=1e-13)
    got = G.layer_norm_backward(x, w if affine else None, dy)
    for g, t in zip(got, want):
        np.testing.assert_allclose(g, t.numpy(), rtol=1e-9, atol=1e-12)


def test_layer_norm_gradient_by_central_differences():
    x, w, dy = rnd(6, (2, 5), (5,), (2, 5))
    dx = G.layer_norm_backward(x, w, dy, eps=1e-3)[0]
    f = lambda a: (G.layer_norm(a, w, eps=1e-3) * dy).sum()
    for i in range(2):
        for c in range(5):
            e = np.zeros_like(x)
            e[i, c] = 1e-6
            assert abs((f(x + e) - f(x - e)) / 2e-6 - dx[i, c]) < 1e-7
