"""Gradients of softmax attention, both stages, against the fp64 oracle.

Bounds.  A rounding to bf16 is off by at most 2^-8 of the value (half a step), fp32 arithmetic by 2^-24.  Per element, against the
magnitudes of oracle/gradients.py (sums of absolute terms):
  * a probability is off by 2 kappa A relative, A the largest sum of |products| of a score and kappa the error of one score:
    (d + dh + 8) 2^-24 where everything is fp32, 2^-16 + that where keys are two bf16 terms;
  * dV, dVs: that, one rounding of P to bf16 on the bf16 matrix cores;  dK, dKs: three times that (P, dP, delta), one rounding
    of dS;  dQ: likewise and one of K;  and the output's own rounding.
Over a whole tensor roundings are independent: one of bf16 has the root mean square 2^-8 / sqrt(3) at most, so four of them stay
below 5e-3 of the 2-norm (the 2-norm test is the sharp one); in fp32 1e-5 covers sums of some hundred terms."""
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
NORM = {"bf16": 5e-3, "f32": 1e-5}


def rnd(g, shape, dtype, std=1.0):
    return I.round_to((g.normal(size=shape) * std).astype(np.float32), dtype)


def guarded(shape, dtype):
    """An output full of NaN between two rows of a value that has to stay."""
    n = int(np.prod(shape))
    pad = 64
    buf = torch.full((n + 2 * pad,), 7.0, device="cuda", dtype=torch_dtype(dtype))
    buf[pad:pad + n] = float("nan")
    return buf, buf[pad:pad + n].view(shape)


def check_guards(buf, what):
    assert bool((buf[:64] == 7).all()) and bool((buf[-64:] == 7).all()), f"{what}: written past its end"


def close(got, want, mag, A, d, dh, dtype, terms, what):
    assert np.all(np.isfinite(got)), f"{what}: non-finite"
    kappa = (d + dh + 8) * 2.0 ** -24 + (2.0 ** -16 if dtype == "bf16" else 0)
    times, roundings = terms
    rel = times * 2 * kappa * max(A, 1.0) + roundings * HALF[dtype] + (len(want) + 64) * 2.0 ** -24
    bound = rel * mag + HALF[dtype] * np.abs(want) + 1e-37
    worst = (np.abs(got - want) / bound).max(initial=0.0)
    assert worst <= 1.0, f"{what}: {worst:.2f} of the bound of an element"
    norm = np.linalg.norm(want)
    # where everything cancels (one key a row) there is no result to be relative to
    if norm > 1e-3 * np.linalg.norm(mag):
        err = np.linalg.norm(got - want) / norm
        assert err <= NORM[dtype] * max(1.0, A / 8), f"{what}: 2-norm error {err:.2e}"


TERMS = {"dV": (1, 1), "dVs": (1, 1), "dK": (3, 1), "dKs": (3, 1), "dQ": (3, 2), "dT": (3, 2), "dY": (3, 1)}


class History:
    def __init__(self, seed, lens, d, H, S, dtype, per_user=False, self_term=False, scale=0.0, std_q=1.0):
        g = np.random.default_rng(seed)
        self.lens, self.d, self.H, self.S, self.dtype = lens, d, H, S, dtype
        self.self_term, self.scale = self_term, scale
        self.off = I.offsets_from_lengths(lens)
        B = len(lens)
        self.X, self.Q = rnd(g, (self.off[-1], d), dtype), rnd(g, (B, S, d) if per_user else (S, d), dtype, std_q)
        self.Wk, self.Wv = rnd(g, (d, d), dtype, d ** -0.5), rnd(g, (d, d), dtype, d ** -0.5)
        self.dO = rnd(g, (B, S, d), dtype)

    def run(self, seg=0, host=True, shift=False, ws=None):
        """Device call; returns a dict of outputs.  shift: every tensor one element away from any alignment."""
        B, S, d = self.dO.shape
        place = lambda a: dev(a, self.dtype)
        if shift:
            def place(a):
                t = torch.empty(a.size + 1, device="cuda", dtype=torch_dtype(self.dtype))[1:].view(a.shape)
                return t.copy_(dev(a, self.dtype))
        names = {"dQ": (B, S, d), "dK": self.X.shape, "dV": self.X.shape}
        if self.self_term:
            names |= {"dKs": (B, S, d), "dVs": (B, S, d)}
        bufs = {k: guarded(v, self.dtype) for k, v in names.items()}
        out = {k: b[1] for k, b in bufs.items()}
        if shift:
            bufs = {k: (torch.full((int(np.prod(v)) + 1,), float("nan"), device="cuda", dtype=torch_dtype(self.dtype)),) for k, v in names.items()}
            out = {k: bufs[k][0][1:].view(v) for k, v in names.items()}
        print(f"history gradient: lens={self.lens[:12]} d={d} H={self.H} S={S} {self.dtype} seg={seg} shift={shift}", flush=True)
        self.ws = V.vista_summarize_backward(place(self.X), torch.from_numpy(self.off).cuda(), place(self.Q), place(self.Wk),
                                             place(self.Wv), place(self.dO), out["dQ"], out["dK"], out["dV"], H=self.H,
                                             scale=self.scale, segment_items=seg, workspace=ws,
                                             offsets_host=torch.from_numpy(self.off) if host else None,
                                             d_self_keys=out.get("dKs"), d_self_values=out.get("dVs"))
        torch.cuda.synchronize()
        assert int(self.ws[:4].view(torch.int32).item()) == 0
        if not shift:
            for k, b in bufs.items():
                check_guards(b[0], k)
        return out

    def check(self, out):
        want = G.summarize_backward(self.X, self.off, self.Q, self.Wk, self.Wv, self.dO, self.H, self.scale or None, self.self_term)
        got = {k: host64(t) for k, t in out.items()}
        for b, w in enumerate(want):
            r = slice(self.off[b], self.off[b + 1])
            for k in got:
                mine = got[k][r] if k in ("dK", "dV") else got[k][b]
                if self.lens[b] == 0:
                    assert not mine.any(), f"user {b} has no history, {k} is not zero"
                else:
                    close(mine, w[k], w[f"|{k}|"], w["A"], self.d, self.d // self.H, self.dtype, TERMS[k], f"user {b} {k}")


JAGGED = [700, 0, 1, 31, 32, 33, 1100, 64, 0, 95, 2, 65]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,H,S,per_user,self_term,seg", [
    (64, 1, 16, False, False, 0), (64, 2, 100, True, True, 0), (128, 4, 256, False, False, 96), (15, 3, 7, True, True, 0),
    (96, 4, 33, False, True, 32), (66, 2, 1, False, False, 64), (256, 8, 130, True, False, 0), (32, 8, 65, False, True, 0)])
def test_history_gradients(dtype, d, H, S, per_user, self_term, seg):
    p = History(1, JAGGED, d, H, S, dtype, per_user, self_term)
    p.check(p.run(seg, host=seg == 0))


@pytest.mark.parametrize("d,H,S,per_user,self_term,seg", [
    (64, 2, 512, False, True, 0), (64, 2, 1, True, False, 0), (128, 4, 31, True, True, 0), (128, 4, 300, False, False, 0),
    (128, 4, 512, True, False, 64), (256, 8, 512, False, False, 0), (256, 8, 64, True, True, 160), (512, 16, 96, False, False, 0),
    (32, 1, 288, False, False, 0)])
def test_history_gradients_of_heads_of_width_32(d, H, S, per_user, self_term, seg):
    p = History(2, [5, 2500, 0, 129, 64, 1, 127], d, H, S, "bf16", per_user, self_term)
    p.check(p.run(seg, host=seg == 0))


@pytest.mark.parametrize("dtype,d,H,S", [("bf16", 128, 4, 64), ("bf16", 40, 5, 9), ("f32", 64, 2, 24)])
def test_history_gradients_of_element_aligned_tensors(dtype, d, H, S):
    p = History(3, [70, 0, 300, 1], d, H, S, dtype, True, True)
    p.check(p.run(shift=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("std_q,scale", [(30.0, 0.0), (1.0, 4.0), (0.0, 0.0)])
def test_history_gradients_of_large_and_equal_scores(dtype, std_q, scale):
    """Scores of some hundreds (a row's weight lies on a few items), and queries of zeros (every item weighs the same)."""
    p = History(4, [300, 1, 65, 1000], 64, 2, 48, dtype, std_q=std_q, scale=scale)
    p.check(p.run())


@pytest.mark.parametrize("dtype,d,H,S", [("f32", 64, 2, 24), ("bf16", 128, 4, 64), ("bf16", 128, 4, 100)])
def test_history_gradients_without_any_items(dtype, d, H, S):
    p = History(5, [0, 0, 0], d, H, S, dtype, self_term=True)
    out = p.run()
    assert all(not t.any() for t in out.values())


@pytest.mark.parametrize("dtype,d,H,S", [("f32", 64, 2, 24), ("bf16", 128, 4, 256), ("bf16", 64, 2, 40)])
def test_what_is_not_finite_keeps_to_its_user(dtype, d, H, S):
    lens = [40, 33, 0, 50, 7]
    p = History(6, lens, d, H, S, dtype, per_user=True)
    clean = p.run()
    p.X[50, 3] = np.nan                     # user 1
    p.dO[3, 0, 1] = np.inf                  # user 3
    dirty = p.run()
    for b in (0, 2, 4):
        r = slice(p.off[b], p.off[b + 1])
        assert torch.equal(clean["dQ"][b], dirty["dQ"][b])
        assert torch.equal(clean["dK"][r], dirty["dK"][r]) and torch.equal(clean["dV"][r], dirty["dV"][r])
    assert bool(torch.isnan(dirty["dQ"][1]).any()) and not bool(torch.isfinite(dirty["dV"][p.off[3]:p.off[4]]).all())


@pytest.mark.parametrize("dtype,d,H,S", [("f32", 64, 2, 24), ("bf16", 128, 4, 256)])
def test_offsets_that_are_wrong_are_reported(dtype, d, H, S):
    p = History(7, [100, 60, 40], d, H, S, dtype)
    p.off = np.array([0, 160, 100, 200])
    with pytest.raises(V.VistaError, match="OFFSETS"):
        p.run(host=True)
    with pytest.raises(AssertionError):     # the status word; every row index stays inside [0, N)
        p.run(host=False)
    assert int(p.ws[:4].view(torch.int32).item()) == V.VISTA_ERR_OFFSETS


@pytest.mark.parametrize("d,H,S,self_term", [(64, 2, 40, False), (128, 4, 256, False), (128, 4, 100, True), (256, 8, 512, False), (48, 3, 20, False)])
def test_history_gradients_of_many_short_histories(d, H, S, self_term):
    g = np.random.default_rng(40)
    p = History(10, [int(x) for x in g.integers(0, 66, size=60)] + [200], d, H, S, "bf16", self_term=self_term)
    a = p.run()
    p.check(a)
    b = p.run(ws=p.ws.fill_(255))
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_history_gradients_of_long_histories():
    """More segments than the device has places for, one user over many of them: split, joined, repeatable."""
    p = History(8, [50_000, 3, 9000], 128, 4, 64, "bf16")
    a = p.run()
    p.check(a)
    b = p.run(ws=p.ws.fill_(255))           # whatever the workspace held
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("d,H,S", [(64, 2, 100), (64, 2, 384), (128, 4, 256), (128, 4, 20), (256, 8, 70), (256, 8, 512)])
@pytest.mark.parametrize("less", [0, 1])
def test_history_gradients_on_either_side_of_an_average_of_4_d_items(d, H, S, less):
    p = History(9, [7 * d - less, d], d, H, S, "bf16", per_user=True)
    p.check(p.run())


# ------------------------------------------------------------------------------------------------ stage 2
class Candidates:
    def __init__(self, seed, B, C, d, H, S, dtype, self_term=False, scale=0.0, std=1.0):
        g = np.random.default_rng(seed)
        self.T, self.Y, self.dO = rnd(g, (B, C, d), dtype, std), rnd(g, (B, S, d), dtype), rnd(g, (B, C, d), dtype)
        self.H, self.dtype, self.self_term, self.scale = H, dtype, self_term, scale

    def run(self, shift=False, ws=None):
        place, B = (lambda a: dev(a, self.dtype)), self.T.shape[0]
        if shift:
            def place(a):
                t = torch.empty(a.size + 1, device="cuda", dtype=torch_dtype(self.dtype))[1:].view(a.shape)
                return t.copy_(dev(a, self.dtype))
        a, b = guarded(self.T.shape, self.dtype), guarded(self.Y.shape, self.dtype)
        print(f"candidates' gradient: {self.T.shape} S={self.Y.shape[1]} H={self.H} {self.dtype} self={self.self_term}", flush=True)
        self.ws = V.vista_target_attend_backward(place(self.T), place(self.Y), place(self.dO), a[1], b[1], H=self.H,
                                                 scale=self.scale, self_term=self.self_term, workspace=ws)
        torch.cuda.synchronize()
        check_guards(a[0], "dT")
        check_guards(b[0], "dY")
        return {"dT": a[1], "dY": b[1]}

    def check(self, out, users=None):
        d = self.T.shape[2]
        got = {k: host64(t) for k, t in out.items()}
        for b in range(self.T.shape[0]) if users is None else users:
            w = G.target_attend_backward(self.T[b], self.Y[b], self.dO[b], self.H, self.scale or None, self.self_term)
            for k in got:
                close(got[k][b], w[k], w[f"|{k}|"], w["A"], d, d // self.H, self.dtype, TERMS[k], f"user {b} {k}")


@pytest.mark.parametrize("self_term", [False, True])
@pytest.mark.parametrize("dtype,B,C,d,H,S", [
    ("f32", 1, 1, 64, 1, 1), ("f32", 3, 70, 64, 2, 33), ("f32", 2, 130, 30, 3, 100), ("bf16", 2, 65, 15, 5, 17),
    ("bf16", 1, 3000, 48, 1, 20), ("f32", 1, 1500, 128, 2, 300), ("bf16", 5, 33, 192, 4, 512)])
def test_candidate_gradients(dtype, B, C, d, H, S, self_term):
    p = Candidates(11, B, C, d, H, S, dtype, self_term)
    p.check(p.run())


@pytest.mark.parametrize("B,C,d,H,S", [
    (3, 63, 64, 1, 1), (2, 65, 48, 1, 16), (1, 700, 64, 2, 63), (600, 70, 32, 2, 112), (5, 128, 33, 1, 127), (300, 200, 64, 1, 128),
    (2, 129, 64, 4, 129), (1, 1, 7, 7, 65)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_candidate_gradients_around_128_summaries(dtype, B, C, d, H, S):
    p = Candidates(16, B, C, d, H, S, dtype, self_term=B % 2 == 1)
    a = p.run()
    p.check(a, users=sorted({0, B // 2, B - 1}))
    b = p.run(ws=p.ws.fill_(255))
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("self_term", [False, True])
@pytest.mark.parametrize("B,C,d,H,S", [
    (1, 1, 32, 1, 1), (2, 100, 128, 4, 256), (3, 31, 64, 2, 100), (2, 64, 128, 4, 64), (1, 5000, 128, 4, 256),
    (4, 33, 256, 8, 512), (70, 129, 128, 4, 300), (1, 2049, 96, 3, 31), (2, 513, 64, 2, 511)])
def test_candidate_gradients_of_heads_of_width_32(B, C, d, H, S, self_term):
    p = Candidates(12, B, C, d, H, S, "bf16", self_term)
    p.check(p.run(), users=sorted({0, B // 2, B - 1}))


@pytest.mark.parametrize("dtype,d,H,S", [("bf16", 128, 4, 64), ("f32", 64, 2, 24)])
@pytest.mark.parametrize("std,scale,shift", [(30.0, 0.0, False), (1.0, 4.0, False), (0.0, 0.0, False), (1.0, 0.0, True)])
def test_candidate_gradients_of_large_scores_and_unaligned_tensors(dtype, d, H, S, std, scale, shift):
    p = Candidates(13, 3, 77, d, H, S, dtype, scale=scale, std=std)
    p.check(p.run(shift=shift))


@pytest.mark.parametrize("dtype,d,H,S", [("bf16", 128, 4, 256), ("f32", 64, 2, 24), ("bf16", 128, 4, 90)])
def test_candidates_that_are_not_finite_keep_to_their_user(dtype, d, H, S):
    p = Candidates(14, 3, 70, d, H, S, dtype)
    clean = p.run()
    p.T[1, 5, 2] = np.nan
    p.T[1, 69, 0] = np.inf
    dirty = p.run()
    for b in (0, 2):
        assert torch.equal(clean["dT"][b], dirty["dT"][b]) and torch.equal(clean["dY"][b], dirty["dY"][b])
    keep = [i for i in range(70) if i not in (5, 69)]
    assert torch.equal(clean["dT"][1][keep], dirty["dT"][1][keep])       # candidates do not see each other
    assert bool(torch.isnan(dirty["dT"][1, 5]).any())


def test_candidate_gradients_repeat_and_ignore_the_workspace():
    p = Candidates(15, 2, 4000, 128, 4, 256, "bf16", True)
    a = p.run()
    b = p.run(ws=p.ws.fill_(255))
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("seed", range(12))
def test_random_gradients(seed):
    g = np.random.default_rng(100 + seed)
    dtype = "bf16" if g.random() < 0.7 else "f32"
    H = int(g.integers(1, 6))
    dh = int(g.choice([32, 32, 32, 16, 64, int(g.integers(1, 65))]))
    S, self_term = int(g.choice([int(g.integers(1, 513)), 64, 256])), bool(g.random() < 0.4)
    lens = [int(x) for x in g.integers(0, 200, size=int(g.integers(1, 9)))] + [int(g.integers(1, 1500))]
    p = History(seed, lens, H * dh, H, S, dtype, bool(g.random() < 0.5), self_term)
    p.check(p.run(int(g.choice([0, 0, 64, 96])), host=bool(g.random() < 0.5)))
    c = Candidates(seed, int(g.integers(1, 6)), int(g.integers(1, 400)), H * dh, H, S, dtype, self_term)
    c.check(c.run())


def test_calls_on_two_streams_with_a_workspace_each():
    jobs = [History(31, [900, 40, 0, 2000], 128, 4, 96, "bf16", True, True), History(32, [500, 700], 64, 1, 30, "f32")]
    once = [j.run() for j in jobs]
    spaces = [j.ws for j in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    args = []
    for j, first in zip(jobs, once):
        out = {k: torch.full_like(t, float("nan")) for k, t in first.items()}
        args.append(([dev(j.X, j.dtype), torch.from_numpy(j.off).cuda(), *(dev(a, j.dtype) for a in (j.Q, j.Wk, j.Wv, j.dO))], out))
    torch.cuda.synchronize()
    for _ in range(5):
        for j, s, ws, (given, out) in zip(jobs, streams, spaces, args):
            with torch.cuda.stream(s):
                V.vista_summarize_backward(*given, out["dQ"], out["dK"], out["dV"], H=j.H, workspace=ws,
                                           d_self_keys=out.get("dKs"), d_self_values=out.get("dVs"))
    torch.cuda.synchronize()
    for first, (_, out) in zip(once, args):
        assert all(torch.equal(first[k], out[k]) for k in first)


# ------------------------------------------------------------------------------------------------ differences of the forward calls
def test_gradients_against_differences_of_the_forward_calls():
    """fp32: the change of sum(out * d_out) along a direction, from the forward entry points themselves.  A central difference of
    step h is off by h^2 / 6 of the third derivative (here of order one times the sum's size) and by the outputs' fp32 errors over
    h: with h = 2^-6 some 1e-4 and 1e-5 of the sum of absolute terms."""
    h, d, H, S = 2.0 ** -6, 64, 2, 24
    p = History(21, [200, 33, 1], d, H, S, "f32")
    out = p.run()
    g = np.random.default_rng(22)
    step = g.normal(size=p.Q.shape).astype(np.float32)
    step /= np.linalg.norm(step)

    def forward(q):
        y = torch.empty(p.dO.shape, device="cuda")
        V.vista_summarize(dev(p.X, "f32"), torch.from_numpy(p.off).cuda(), dev(q, "f32"), dev(p.Wk, "f32"), dev(p.Wv, "f32"), y, H=H)
        return (host64(y) * p.dO).sum(), (np.abs(host64(y)) * np.abs(p.dO)).sum()

    (up, size), (down, _) = forward(p.Q + h * step), forward(p.Q - h * step)
    want = (host64(out["dQ"]).sum(0) * step).sum()
    assert abs((up - down) / (2 * h) - want) <= 2e-4 * size
    c = Candidates(23, 2, 40, d, H, S, "f32", True)
    got = c.run()
    for k, name in (("T", "dT"), ("Y", "dY")):
        step = g.normal(size=getattr(c, k).shape).astype(np.float32)
        step /= np.linalg.norm(step)

        def attend(x):
            y = torch.empty(c.T.shape, device="cuda")
            V.vista_target_attend(dev(x if k == "T" else c.T, "f32"), dev(x if k == "Y" else c.Y, "f32"), y, H=H, self_term=True)
            return (host64(y) * c.dO).sum(), (np.abs(host64(y)) * np.abs(c.dO)).sum()

        (up, size), (down, _) = attend(getattr(c, k) + h * step), attend(getattr(c, k) - h * step)
        assert abs((up - down) / (2 * h) - (host64(got[name]) * step).sum()) <= 2e-4 * size
