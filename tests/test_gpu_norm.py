"""Layer norm and its gradients against the fp64 oracle, alone and as part of a training step.

Bounds, per element: fp32 sums of d terms are off by d 2^-24 of the sum of absolute terms at most; z then by (d + 8) 2^-24 of
(|x| + mean |x|) r, and by the output's rounding (2^-8 of the value in bf16)."""
import numpy as np
import pytest
import torch

from oracle import gradients as G
from oracle import vista_oracle as O
from paper_2510_22049_amd import binding as V
from paper_2510_22049_amd import inputs as I
from tests.helpers import dev, host64, torch_dtype

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def rnd(g, shape, dtype, std=1.0, shift=0.0):
    return I.round_to((g.normal(size=shape) * std + shift).astype(np.float32), dtype)


def place(a, dtype, odd):
    """On the device; odd: one element behind an aligned address."""
    if a is None or not odd:
        return None if a is None else dev(a, dtype)
    return torch.empty(a.size + 1, device="cuda", dtype=torch_dtype(dtype))[1:].view(a.shape).copy_(dev(a, dtype))


WIDTHS = [1, 2, 3, 7, 8, 31, 32, 64, 100, 128, 255, 256, 300, 512, 513, 1000, 1023, 1024]


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm_and_gradients(d, dtype, odd):
    for rows, shift, affine in ((1, 0.0, True), (67, 3.0, True), (9, -50.0, False)):
        g = np.random.default_rng(d)
        x, dy = rnd(g, (rows, d), dtype, 1.0, shift), rnd(g, (rows, d), dtype)
        w, b = (rnd(g, (d,), dtype, 0.3, 1.0), rnd(g, (d,), dtype)) if affine else (None, None)
        X, W, Bt, DY = (place(a, dtype, odd) for a in (x, w, b, dy))
        y, dx = (torch.full((rows * d + 16,), 7.0, device="cuda", dtype=torch_dtype(dtype)) for _ in range(2))
        at = slice(1, 1 + rows * d) if odd else slice(0, rows * d)
        sums = [torch.full((d,), float("nan"), device="cuda", dtype=torch_dtype(dtype)) for _ in range(2)]
        print(f"layer norm: {rows} x {d} {dtype} odd={odd}", flush=True)
        V.vista_layer_norm(X, W, Bt, y[at].view(rows, d), eps=1e-3)
        V.vista_layer_norm_backward(X, W, DY, dx[at].view(rows, d), *sums, eps=1e-3)
        torch.cuda.synchronize()
        assert bool((y[rows * d + 1:] == 7).all()) and bool((dx[rows * d + 1:] == 7).all())
        u = HALF[dtype]
        c = x.astype(np.float64) - x.astype(np.float64).mean(-1, keepdims=True)
        r = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + 1e-3)
        ez = (2 * d + 16) * 2.0 ** -24 * (np.abs(x) + np.abs(x).mean(-1, keepdims=True)) * r * (1 + np.abs(c * r))
        aw = np.ones(d) if w is None else np.abs(w).astype(np.float64)
        want = G.layer_norm(x, w, b, 1e-3)
        got = host64(y[at].view(rows, d))
        bound = ez * aw + 2.0 ** -23 * (np.abs(c * r) * aw + (0 if b is None else np.abs(b))) + u * np.abs(want) + 1e-37
        assert (np.abs(got - want) <= bound).all(), "y"
        dxw, dww, dbw = G.layer_norm_backward(x, w, dy, 1e-3)
        gm = np.abs(dy) * aw
        z = np.abs(c * r)
        mag = r * (gm + gm.mean(-1, keepdims=True) + z * (gm * z).mean(-1, keepdims=True))
        more = r * (ez * (gm * z).mean(-1, keepdims=True) + z * (gm * ez).mean(-1, keepdims=True)) + \
            mag * (ez * z).mean(-1, keepdims=True)
        got = host64(dx[at].view(rows, d))
        assert (np.abs(got - dxw) <= (2 * d + 32) * 2.0 ** -24 * mag + 2 * more + u * np.abs(dxw) + 1e-37).all(), "dx"
        for name, s, wsum, m in (("dw", sums[0], dww, (np.abs(dy) * (z * (rows + 8) * 2.0 ** -24 + ez)).sum(0)),
                                 ("db", sums[1], dbw, (rows + 8) * 2.0 ** -24 * np.abs(dy).sum(0))):
            assert (np.abs(host64(s) - wsum) <= m + u * np.abs(wsum) + 1e-37).all(), name


def test_many_rows_sum_in_place_and_repeatable():
    """More rows than workgroups: partial sums of every one; outputs over the inputs; equal bits again."""
    g = np.random.default_rng(3)
    rows, d = 40_013, 96
    x, dy, w = rnd(g, (rows, d), "bf16"), rnd(g, (rows, d), "bf16"), rnd(g, (d,), "bf16", 0.3, 1.0)
    X, DY, W = dev(x, "bf16"), dev(dy, "bf16"), dev(w, "bf16")
    sums = lambda: [torch.empty(d, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    (dw, db), (dw2, db2) = sums(), sums()
    dx = torch.empty_like(DY)
    ws = V.vista_layer_norm_backward(X, W, DY, dx, dw, db)
    V.vista_layer_norm_backward(X, W, DY, DY, dw2, db2, workspace=ws.fill_(255))
    y, z = torch.empty_like(X), X.clone()
    V.vista_layer_norm(X, W, None, y)
    V.vista_layer_norm(z, W, None, z)
    torch.cuda.synchronize()
    assert torch.equal(dx, DY) and torch.equal(dw, dw2) and torch.equal(db, db2) and torch.equal(y, z)
    dxw, dww, dbw = G.layer_norm_backward(x, w, dy)
    for got, want in ((dx, dxw), (dw, dww), (db, dbw)):
        # one rounding to bf16, 2^-8 / sqrt(3) at most in the root mean square
        assert np.linalg.norm(host64(got) - want) <= 2.4e-3 * np.linalg.norm(want)


@pytest.mark.parametrize("dtype,d", [("bf16", 211), ("bf16", 999), ("f32", 67), ("bf16", 9)])
def test_rows_that_are_no_whole_chunks_in_place(dtype, d):
    """A row's last chunk overlaps the one before: in place it has been read before either is stored."""
    g = np.random.default_rng(d)
    rows = 5003
    x, w, b, dy = (rnd(g, s, dtype) for s in ((rows, d), (d,), (d,), (rows, d)))
    X, W, Bt, DY = (dev(a, dtype) for a in (x, w, b, dy))
    y, dx = torch.empty_like(X), torch.empty_like(X)
    sums = [torch.empty_like(W) for _ in range(4)]
    V.vista_layer_norm(X, W, Bt, y)
    V.vista_layer_norm_backward(X, W, DY, dx, *sums[:2])
    V.vista_layer_norm_backward(X, W, DY, DY, *sums[2:])
    V.vista_layer_norm(X, W, Bt, X)
    assert torch.equal(X, y) and torch.equal(DY, dx) and torch.equal(sums[0], sums[2]) and torch.equal(sums[1], sums[3])


def test_rows_of_one_value_and_rows_that_are_not_finite():
    x = torch.randn(6, 128, device="cuda")
    clean = torch.empty_like(x)
    V.vista_layer_norm(x, None, None, clean)
    x[1] = 5.0
    x[3, 7] = float("nan")
    x[4, 0] = float("inf")
    y = torch.empty_like(x)
    V.vista_layer_norm(x, None, None, y)
    torch.cuda.synchronize()
    assert torch.equal(y[[0, 2, 5]], clean[[0, 2, 5]])
    assert bool((y[1] == 0).all()) and bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[4]).any())


def test_no_rows():
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.zeros((0, 48), device="cuda", dtype=dtype)
        dw, db = (torch.full((48,), float("nan"), device="cuda", dtype=dtype) for _ in range(2))
        V.vista_layer_norm(x, None, None, x)
        V.vista_layer_norm_backward(x, None, x, x, dw, db)
        torch.cuda.synchronize()
        assert not dw.any() and not db.any()


def step(t, off, H, out):
    """One training step of a layer: norm, summaries, candidates; gradients back to the raw items.  Every call is the
    framework's; the projections' own backward is two matrix products."""
    V.vista_layer_norm(t["X"], t["w"], t["b"], out["Z"])
    V.vista_summarize(out["Z"], off, t["Q"], t["Wk"], t["Wv"], out["Y"], H=H, workspace=out["ws0"])
    V.vista_target_attend(t["T"], out["Y"], out["O"], H=H, self_term=True)
    V.vista_target_attend_backward(t["T"], out["Y"], t["dO"], out["dT"], out["dY"], H=H, self_term=True, workspace=out["ws1"])
    V.vista_summarize_backward(out["Z"], off, t["Q"], t["Wk"], t["Wv"], out["dY"], out["dQ"], out["dK"], out["dV"], H=H,
                               workspace=out["ws2"])
    out["dZ"].copy_(out["dK"].float() @ t["Wk"].float().T + out["dV"].float() @ t["Wv"].float().T)
    V.vista_layer_norm_backward(t["X"], t["w"], out["dZ"], out["dX"], out["dw"], out["db"], workspace=out["ws3"])


def make_step(seed, lens, C, d, H, S, dtype):
    import ctypes
    g, dt = np.random.default_rng(seed), torch_dtype(dtype)
    off, B = I.offsets_from_lengths(lens), len(lens)
    N = int(off[-1])
    h = {"X": rnd(g, (N, d), dtype, 2.0, 0.5), "w": rnd(g, (d,), dtype, 0.1, 1.0), "b": rnd(g, (d,), dtype, 0.1),
         "Q": rnd(g, (S, d), dtype), "Wk": rnd(g, (d, d), dtype, d ** -0.5), "Wv": rnd(g, (d, d), dtype, d ** -0.5),
         "T": rnd(g, (B, C, d), dtype), "dO": rnd(g, (B, C, d), dtype)}
    shapes = {"Z": (N, d), "Y": (B, S, d), "O": (B, C, d), "dT": (B, C, d), "dY": (B, S, d), "dQ": (B, S, d), "dK": (N, d),
              "dV": (N, d), "dZ": (N, d), "dX": (N, d), "dw": (d,), "db": (d,)}
    out = {k: torch.full(s, float("nan"), device="cuda", dtype=dt) for k, s in shapes.items()}
    code = V.VISTA_BF16 if dtype == "bf16" else V.VISTA_F32
    sd = V.summarize_desc(B, S, d, H, code, N)
    ad = V.AttendDesc(B=B, C=C, S=S, d=d, H=H, dtype=code, scale=0.0, flags=V.VISTA_FLAG_SELF_TERM)
    L, ref = V.lib(), ctypes.byref
    for i, n in enumerate((V.vista_summarize_workspace_bytes(sd), L.vista_target_attend_backward_workspace_bytes(ref(ad)),
                           L.vista_summarize_backward_workspace_bytes(ref(sd)),
                           L.vista_layer_norm_backward_workspace_bytes(ref(V.NormDesc(rows=N, d=d, dtype=code, eps=0.0))))):
        out[f"ws{i}"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return h, off, {k: dev(v, dtype) for k, v in h.items()}, torch.from_numpy(off).cuda(), out


def reference_step(h, off, H):
    """The same in fp64 by automatic differentiation of the forward definitions."""
    t = {k: torch.from_numpy(v.astype(np.float64)).requires_grad_(k in ("X", "w", "b", "Q", "T")) for k, v in h.items()}
    d = h["X"].shape[1]
    dh = d // H
    z = torch.nn.functional.layer_norm(t["X"], (d,), t["w"], t["b"], eps=1e-6)
    loss = 0.0
    for b in range(len(off) - 1):
        x = z[off[b]:off[b + 1]]
        k, v = x @ t["Wk"], x @ t["Wv"]
        for c in (slice(i * dh, (i + 1) * dh) for i in range(H)):
            y = torch.softmax(t["Q"][:, c] @ k[:, c].T / dh ** 0.5, 1) @ v[:, c] if len(x) else torch.zeros_like(t["Q"][:, c])
            q = t["T"][b][:, c]
            s = torch.cat([q @ y.T, (q * q).sum(1, keepdim=True)], 1) / dh ** 0.5
            p = torch.softmax(s, 1)
            loss = loss + ((p[:, :-1] @ y + p[:, -1:] * q) * t["dO"][b][:, c]).sum()
    return dict(zip(("dX", "dw", "db", "dQ", "dT"), (g.numpy() for g in torch.autograd.grad(loss, [t[k] for k in ("X", "w", "b", "Q", "T")]))))


@pytest.mark.parametrize("dtype,d,H,S", [("f32", 64, 2, 16), ("bf16", 128, 4, 64), ("bf16", 128, 4, 100)])
def test_a_training_step(dtype, d, H, S):
    h, off, t, doff, out = make_step(31, [90, 0, 1, 333], 70, d, H, S, dtype)
    step(t, doff, H, out)
    torch.cuda.synchronize()
    want = reference_step(h, off, H)
    # bf16: a gradient passes up to five stored tensors and their roundings (Z, Y, dY, dK / dV, dZ) and the operands of three
    # attentions; each is 2^-8 / sqrt(3) of the 2-norm at most, twelve of them independent 8e-3.  fp32: 1e-5 as for one call.
    tol = 1.2e-2 if dtype == "bf16" else 1e-5
    for k, w in want.items():
        got = host64(out[k]).sum(0) if k == "dQ" else host64(out[k])
        err = np.linalg.norm(got - w) / np.linalg.norm(w)
        assert err <= tol, f"{k}: {err:.2e}"


@pytest.mark.parametrize("dtype,d,H,S", [("f32", 64, 2, 16), ("bf16", 128, 4, 64)])
def test_a_training_step_captured_and_replayed(dtype, d, H, S):
    """A captured step, replayed with new inputs and with eager work and synchronisation between: every replay against the
    eager result; on a stream that is not the default one."""
    h, off, t, doff, out = make_step(32, [90, 0, 1, 333], 70, d, H, S, dtype)
    eager = {k: v.clone() for k, v in out.items()}
    keys = ("Z", "Y", "O", "dT", "dY", "dQ", "dK", "dV", "dX", "dw", "db")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(t, doff, H, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(t, doff, H, out)
    for n in range(4):
        for k in ("X", "T", "dO"):
            t[k].mul_(0.5 if n % 2 else 2.0)
        for k in keys:
            out[k].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        step(t, doff, H, eager)
        torch.cuda.synchronize()
        for k in keys:
            assert torch.equal(out[k], eager[k]), f"replay {n}: {k}"
