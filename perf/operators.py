"""The training operators of this framework as calls to measure: gradients of both attention stages, layer norm and
its gradients, in plain elementary torch operations and through the public entry points.

    own               False: `run` computes the plain form; True: it calls the framework
    listed()          the cases by name
    draw(rng)         one more case of the same ranges
    prepare(case, s)  what a training program holds before the call, from the seed alone
    run(state)        one pass
    work(case)        bytes and flops the pass cannot do without
    exact(case, s)    what `run` returns, from the definitions in 64 bits (torch's automatic differentiation)

Shapes are those of the package's five workloads and of the ranges around them.  The plain forms hold everything in
32 bits, whatever the storage type, and round once at the end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------- the cases

def _history(users, items, d, H, S, dtype="bf16", spread=1.0, empty=0, self_term=False, per_user=False, host_offsets=True):
    return {"path": "history", "users": users, "items": items, "spread": spread, "empty": empty, "d": d, "H": H, "S": S,
            "dtype": dtype, "self_term": self_term, "per_user": per_user, "host_offsets": host_offsets}


def _candidates(users, C, d, H, S, dtype="bf16", self_term=False):
    return {"path": "candidates", "users": users, "C": C, "d": d, "H": H, "S": S, "dtype": dtype, "self_term": self_term}


def _norm(direction, rows, d, dtype="bf16", affine=True):
    return {"path": "norm_" + direction, "rows": rows, "d": d, "dtype": dtype, "affine": affine}


def listed():
    return [
        # the tiny configuration: fp32, one head of 64; a unit test or a notebook's first step, all latency
        {"name": "history_tiny_fp32", **_history(1, 1024, 64, 1, 16, dtype="f32")},
        # one ordinary user: the online refresh of a single history, offsets on the device only
        {"name": "history_one_user", **_history(1, 7001, 128, 4, 256, host_offsets=False)},
        # the jagged batch (lognormal lengths around 8k), the workload a training step is quoted on
        {"name": "history_jagged", **_history(64, 768597, 128, 4, 256)},
        # a narrower model, a seed count that is no power of two, users without history, seeds that see themselves
        {"name": "history_odd", **_history(48, 300007, 64, 2, 100, empty=3, self_term=True)},
        # second layer of a stack: queries of each user's own, the widest seeds
        {"name": "history_stacked", **_history(16, 200003, 256, 8, 512, spread=0.5, per_user=True)},
        # two requests' worth of candidates: latency
        {"name": "candidates_small", **_candidates(2, 100, 128, 4, 256)},
        # ragged sizes in fp32, candidates that also see themselves
        {"name": "candidates_ragged_fp32", **_candidates(75, 333, 64, 1, 100, dtype="f32", self_term=True)},
        # a ranking batch: 1024 users, 512 candidates each
        {"name": "candidates_batch", **_candidates(1024, 512, 128, 4, 256)},
        # item embeddings of the jagged batch on their way into the first layer
        {"name": "norm_history", **_norm("forward", 768597, 128)},
        # a handful of summaries between two layers, fp32: latency
        {"name": "norm_small_fp32", **_norm("forward", 333, 512, dtype="f32")},
        # gradients over the same jagged batch, those of the weight and the bias among them
        {"name": "norm_backward_history", **_norm("backward", 768597, 128)},
        # and over the summaries of 64 users, odd rows, fp32
        {"name": "norm_backward_fp32", **_norm("backward", 16381, 256, dtype="f32")},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    path = rng.choice(["history", "history", "history", "history_f32", "candidates", "candidates", "candidates_f32", "norm_forward",
                       "norm_backward"])
    d, H = rng.choice([(128, 4), (128, 4), (256, 8), (64, 2)])
    self_term = rng.random() < 0.25
    if path == "history":
        S = rng.choice([64, 128, 256, 512, rng.randint(1, 512)])
        users = _log(rng, 1, 128)
        most = int(min(1_500_000, 2.9e11 / (4 * d * d + 10 * S * d)))         # no more work than the largest listed case's
        return _history(users, _log(rng, 300, most), d, H, S, spread=rng.choice([0.0, 0.5, 1.0]),
                        empty=rng.randint(0, users // 4), self_term=self_term, per_user=rng.random() < 0.3,
                        host_offsets=rng.random() < 0.75)
    if path == "history_f32":
        users = _log(rng, 1, 16)
        return _history(users, _log(rng, 100, 60_000), 64, rng.choice([1, 2, 4]), rng.randint(1, 128), dtype="f32",
                        empty=rng.randint(0, users // 4), self_term=self_term, per_user=rng.random() < 0.3)
    if path.startswith("candidates"):
        f32 = path.endswith("f32")
        users = _log(rng, 1, 128 if f32 else 1024)
        if f32:
            C = _log(rng, 1, max(2, min(8192, 40_000 // users)))
            return _candidates(users, C, 64, rng.choice([1, 2, 4]), rng.randint(1, 256), "f32", self_term)
        S = rng.choice([64, 128, 256, 512, rng.randint(1, 512)])
        most = min(500_000, 2.0e11 / (12 * S * d))
        return _candidates(users, _log(rng, 1, max(2, min(8192, int(most / users)))), d, H, S, self_term=self_term)
    d = rng.choice([64, 128, 256, 512, rng.randint(16, 1024)])
    return _norm(path[5:], _log(rng, 1, 98_000_000 // d), d, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.8)


# ------------------------------------------------------------------------------- a pass

def _offsets(case, seed):
    """Users' first rows: lognormal shares of exactly `items` rows; `empty` users, every second one, have none."""
    g = np.random.default_rng(seed)
    share = np.exp(case["spread"] * g.standard_normal(case["users"]))
    share[1:2 * case["empty"]:2] = 0.0                       # users without history, never the first
    cut = np.floor(np.cumsum(share) / share.sum() * case["items"]).astype(np.int64)
    cut[np.flatnonzero(share)[-1]:] = case["items"]
    return np.concatenate([np.zeros(1, dtype=np.int64), cut])


def prepare(case, seed):
    dt, d = DTYPES[case["dtype"]], case["d"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        t = torch.empty(shape, device="cuda", dtype=dt).normal_(generator=g)
        return t.mul_(std) if std != 1.0 else t

    def empty(*shape):
        return torch.empty(shape, device="cuda", dtype=dt)

    st = {"case": case, "ws": None}
    if case["path"] == "history":
        B, N, S = case["users"], case["items"], case["S"]
        off = torch.from_numpy(_offsets(case, seed))
        st["off"], st["off_list"] = off.cuda(), off.tolist()
        st["off_host"] = off if case["host_offsets"] else None
        st["X"] = normal(N, d)
        st["Q"] = normal(B, S, d) if case["per_user"] else normal(S, d)
        st["Wk"], st["Wv"] = normal(d, d, std=d ** -0.5), normal(d, d, std=d ** -0.5)
        st["dO"] = normal(B, S, d, std=1e-2)                 # a loss averaged over a batch
        st["dQ"], st["dK"], st["dV"] = empty(B, S, d), empty(N, d), empty(N, d)
        st["dKs"], st["dVs"] = (empty(B, S, d), empty(B, S, d)) if case["self_term"] else (None, None)
    elif case["path"] == "candidates":
        B, C, S = case["users"], case["C"], case["S"]
        st["T"], st["Y"], st["dO"] = normal(B, C, d), normal(B, S, d), normal(B, C, d, std=1e-2)
        st["dT"], st["dY"] = empty(B, C, d), empty(B, S, d)
    else:
        rows = case["rows"]
        st["X"] = normal(rows, d)
        st["w"], st["b"] = ((1 + 0.1 * normal(d).float()).to(dt), normal(d, std=0.1)) if case["affine"] else (None, None)
        if case["path"] == "norm_forward":
            st["Z"] = empty(rows, d)
        else:
            st["dZ"], st["dX"] = normal(rows, d, std=1e-2), empty(rows, d)
            st["dw"], st["db"] = (empty(d), empty(d)) if case["affine"] else (None, None)
    return st


def run(st):
    if own:
        return _run_own(st)
    return {"history": _plain_history, "candidates": _plain_candidates, "norm_forward": _plain_norm,
            "norm_backward": _plain_norm_backward}[st["case"]["path"]](st)


def _run_own(st):
    from paper_2510_22049_amd import binding as V
    case = st["case"]
    if case["path"] == "history":
        st["ws"] = V.vista_summarize_backward(st["X"], st["off"], st["Q"], st["Wk"], st["Wv"], st["dO"], st["dQ"], st["dK"],
                                              st["dV"], H=case["H"], offsets_host=st["off_host"], workspace=st["ws"],
                                              d_self_keys=st["dKs"], d_self_values=st["dVs"])
        return {k: st[k] for k in ("dQ", "dK", "dV", "dKs", "dVs") if st[k] is not None}
    if case["path"] == "candidates":
        st["ws"] = V.vista_target_attend_backward(st["T"], st["Y"], st["dO"], st["dT"], st["dY"], H=case["H"],
                                                  self_term=case["self_term"], workspace=st["ws"])
        return {"dT": st["dT"], "dY": st["dY"]}
    if case["path"] == "norm_forward":
        V.vista_layer_norm(st["X"], st["w"], st["b"], st["Z"])
        return {"Z": st["Z"]}
    st["ws"] = V.vista_layer_norm_backward(st["X"], st["w"], st["dZ"], st["dX"], st["dw"], st["db"], workspace=st["ws"])
    return {k: st[k] for k in ("dX", "dw", "db") if st[k] is not None}


# ------------------------------------------------------------------------------- plain forms

def _heads(t, H):
    """[n, d] -> [H, n, d / H] in 32 bits."""
    return t.float().reshape(t.shape[0], H, -1).transpose(0, 1).contiguous()


def _rows(t):
    """[H, n, d / H] -> [n, d]."""
    return t.transpose(0, 1).reshape(t.shape[1], -1)


def _softmax_gradient(s, dp):
    """Probabilities of the scores' last axis and the scores' gradient from the probabilities'."""
    p = (s - s.amax(-1, keepdim=True)).exp_()
    p = p.div_(p.sum(-1, keepdim=True))
    return p, dp.sub_((p * dp).sum(-1, keepdim=True)).mul_(p)


def _plain_user(x, q, do, wk, wv, H, self_term):
    """Gradients of one user's summaries: [dQ, dK, dV] and with the self term [dKs, dVs]."""
    scale = (q.shape[1] // H) ** -0.5
    if not x.shape[0]:
        zero = torch.zeros_like(q, dtype=torch.float32)
        return [zero, x.float(), x.float()] + ([zero, zero] if self_term else [])
    q, do = _heads(q, H), _heads(do, H)
    k, v = _heads(x.float() @ wk, H), _heads(x.float() @ wv, H)
    s, dp = torch.bmm(q, k.transpose(1, 2)).mul_(scale), torch.bmm(do, v.transpose(1, 2))
    if self_term:
        ks, vs = torch.matmul(_rows(q), wk), torch.matmul(_rows(q), wv)
        ks, vs = _heads(ks, H), _heads(vs, H)
        s = torch.cat([s, (q * ks).sum(-1, keepdim=True) * scale], -1)
        dp = torch.cat([dp, (do * vs).sum(-1, keepdim=True)], -1)
    p, ds = _softmax_gradient(s, dp)
    n = x.shape[0]
    dq = torch.bmm(ds[..., :n], k).mul_(scale)
    dk, dv = torch.bmm(ds[..., :n].transpose(1, 2), q).mul_(scale), torch.bmm(p[..., :n].transpose(1, 2), do)
    if not self_term:
        return [_rows(dq), _rows(dk), _rows(dv)]
    own_ds, own_p = ds[..., n:] * scale, p[..., n:]
    return [_rows(dq + own_ds * ks), _rows(dk), _rows(dv), _rows(own_ds * q), _rows(own_p * do)]


def _plain_history(st):
    case, off, dt = st["case"], st["off_list"], st["X"].dtype
    wk, wv = st["Wk"].float(), st["Wv"].float()
    q_of = (lambda b: st["Q"][b]) if case["per_user"] else (lambda b: st["Q"])

    def user(b):
        # rounded at once, so that no more than one user is held in 32 bits
        return [t.to(dt) for t in _plain_user(st["X"][off[b]:off[b + 1]], q_of(b), st["dO"][b], wk, wv, case["H"], case["self_term"])]

    got = [user(b) for b in range(case["users"])]
    out = {"dQ": torch.stack([g[0] for g in got]), "dK": torch.cat([g[1] for g in got]), "dV": torch.cat([g[2] for g in got])}
    if case["self_term"]:
        out |= {"dKs": torch.stack([g[3] for g in got]), "dVs": torch.stack([g[4] for g in got])}
    return out


def _plain_candidates(st):
    case = st["case"]
    B, C, d = st["T"].shape
    H, S, dh = case["H"], case["S"], d // case["H"]
    scale = dh ** -0.5

    def heads(t):
        return t.float().reshape(B, -1, H, dh).transpose(1, 2).reshape(B * H, -1, dh)

    def rows(t):
        return t.reshape(B, H, -1, dh).transpose(1, 2).reshape(B, -1, d).to(st["T"].dtype)

    q, y, do = heads(st["T"]), heads(st["Y"]), heads(st["dO"])
    s, dp = torch.bmm(q, y.transpose(1, 2)).mul_(scale), torch.bmm(do, y.transpose(1, 2))
    if case["self_term"]:
        s = torch.cat([s, (q * q).sum(-1, keepdim=True) * scale], -1)
        dp = torch.cat([dp, (do * q).sum(-1, keepdim=True)], -1)
    p, ds = _softmax_gradient(s, dp)
    ds.mul_(scale)
    dq = torch.bmm(ds[..., :S], y)
    dy = torch.bmm(ds[..., :S].transpose(1, 2), q) + torch.bmm(p[..., :S].transpose(1, 2), do)
    if case["self_term"]:
        dq = dq + 2 * ds[..., S:] * q + p[..., S:] * do
    return {"dT": rows(dq), "dY": rows(dy)}


def _normalised(x):
    x = x.float()
    x = x - x.mean(-1, keepdim=True)
    r = ((x * x).mean(-1, keepdim=True) + 1e-6).rsqrt()
    return x * r, r


def _plain_norm(st):
    z = _normalised(st["X"])[0]
    return {"Z": (z * st["w"].float() + st["b"].float() if st["w"] is not None else z).to(st["X"].dtype)}


def _plain_norm_backward(st):
    dt = st["X"].dtype
    (z, r), dz = _normalised(st["X"]), st["dZ"].float()
    g = dz * st["w"].float() if st["w"] is not None else dz
    dx = r * (g - g.mean(-1, keepdim=True) - z * (g * z).mean(-1, keepdim=True))
    if st["w"] is None:
        return {"dX": dx.to(dt)}
    return {"dX": dx.to(dt), "dw": (dz * z).sum(0).to(dt), "db": dz.sum(0).to(dt)}


# ------------------------------------------------------------------------------- work

def work(case):
    """Each input read once, each output written once, every product of the definition once, 2 flops a term: the projections of
    the items, scores, the probabilities' gradients and the products of the gradients (three; four where keys are values too)."""
    e, d = (2 if case["dtype"] == "bf16" else 4), case["d"]
    if case["path"] == "history":
        B, N, S = case["users"], case["items"], case["S"]
        own_rows = 4 if case["self_term"] else 0
        rows = (2 + own_rows // 2) * B * S + (B * S if case["per_user"] else S)     # d_out, dQ, own gradients; queries
        return {"bytes": float(e * d * (3 * N + rows + 2 * d) + 8 * (B + 1)),
                "flops": float(4 * d * d * N + 10 * S * d * N + (own_rows and 4 * d * d * B * S))}
    if case["path"] == "candidates":
        B, C, S = case["users"], case["C"], case["S"]
        return {"bytes": float(e * d * B * (3 * C + 2 * S)), "flops": float(12 * S * d * B * C)}
    n = case["rows"] * d
    backward = case["path"] == "norm_backward"
    return {"bytes": float(e * ((3 if backward else 2) * n + (3 if backward else 2) * d * case["affine"])),
            "flops": float((14 if backward else 8) * n)}


# ------------------------------------------------------------------------------- the definitions in 64 bits

def _attend64(q, k, v, H, own_k=None, own_v=None):
    """RowSoftmax(q k^T / sqrt(d / H)) v for every head, as written; own_k, own_v: one more key and value for each row."""
    n, d = q.shape
    outs = []
    for h in range(H):
        c = slice(h * (d // H), (h + 1) * (d // H))
        s = q[:, c] @ k[:, c].T
        if own_k is not None:
            s = torch.cat([s, (q[:, c] * own_k[:, c]).sum(1, keepdim=True)], 1)
        p = torch.softmax(s / math.sqrt(d // H), 1)
        o = p[:, :k.shape[0]] @ v[:, c]
        outs.append(o if own_k is None else o + p[:, k.shape[0]:] * own_v[:, c])
    return torch.cat(outs, 1)


def _leaf(t):
    return t.detach().double().requires_grad_(True)


def exact(case, seed):
    st = prepare(case, seed)
    if case["path"] == "history":
        off, H, wk, wv = st["off_list"], case["H"], st["Wk"].double(), st["Wv"].double()
        got = {k: torch.zeros(st[k].shape, dtype=torch.float64, device="cuda") for k in ("dQ", "dK", "dV", "dKs", "dVs") if st[k] is not None}
        for b in range(case["users"]):
            if off[b] == off[b + 1]:
                continue
            r, d = slice(off[b], off[b + 1]), case["d"]
            x, q0 = st["X"][r].double(), (st["Q"][b] if case["per_user"] else st["Q"]).double()
            k0, v0 = x @ wk, x @ wv
            for h in range(H):                               # a head at a time: a million items fit
                c = slice(h * (d // H), (h + 1) * (d // H))
                at = [_leaf(q0[:, c]), _leaf(k0[:, c]), _leaf(v0[:, c])]
                if case["self_term"]:
                    at += [_leaf((q0 @ wk)[:, c]), _leaf((q0 @ wv)[:, c])]
                o = _attend64(at[0], at[1], at[2], 1, *at[3:])
                g = torch.autograd.grad(o, at, st["dO"][b][:, c].double())
                got["dQ"][b, :, c], got["dK"][r, c], got["dV"][r, c] = g[:3]
                if case["self_term"]:
                    got["dKs"][b, :, c], got["dVs"][b, :, c] = g[3:]
                del o, g, at
        return got
    if case["path"] == "candidates":
        got = {"dT": torch.empty(st["T"].shape, dtype=torch.float64, device="cuda"),
               "dY": torch.empty(st["Y"].shape, dtype=torch.float64, device="cuda")}
        for b in range(case["users"]):
            t, y = _leaf(st["T"][b]), _leaf(st["Y"][b])
            o = _attend64(t, y, y, case["H"], *((t, t) if case["self_term"] else ()))
            got["dT"][b], got["dY"][b] = torch.autograd.grad(o, [t, y], st["dO"][b].double())
        return got
    x = _leaf(st["X"])
    wb = [_leaf(st["w"]), _leaf(st["b"])] if case["affine"] else []
    mean = x.sum(-1, keepdim=True) / case["d"]
    z = (x - mean) / torch.sqrt(((x - mean) ** 2).sum(-1, keepdim=True) / case["d"] + 1e-6)
    z = z * wb[0] + wb[1] if wb else z
    if case["path"] == "norm_forward":
        return {"Z": z.detach()}
    g = torch.autograd.grad(z, [x] + wb, st["dZ"].double())
    return dict(zip(("dX", "dw", "db"), g))
