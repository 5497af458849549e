"""Host-only checks of the training entry points: everything that is wrong with a call is found before the first launch,
by the library's codes and, for shapes a pointer does not carry, by the binding."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2510_22049_amd import binding as V
from tests.test_launch_limits_host import STUB

ONE = C.c_void_p(256)                  # never dereferenced


def desc(**kw):
    base = dict(B=2, S=16, d=64, H=1, dtype=V.VISTA_F32, total_items=100)
    base.update(kw)
    return V.summarize_desc(**base)


def summarize_backward(d, **kw):
    names = ("x", "off", "off_host", "q", "wk", "wv", "do", "dq", "dk", "dv", "dks", "dvs", "ws")
    args = [kw.get(n, None if n == "off_host" else ONE) for n in names]
    return V.lib().vista_summarize_backward(C.byref(d) if d is not None else None, *args, kw.get("bytes", 1 << 40), None)


def need(d):
    return V.lib().vista_summarize_backward_workspace_bytes(C.byref(d))


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), V.VISTA_ERR_SHAPE), (dict(d=66, H=4), V.VISTA_ERR_SHAPE), (dict(segment_items=40), V.VISTA_ERR_SHAPE),
    (dict(total_items=-1), V.VISTA_ERR_SHAPE), (dict(scale=-1.0), V.VISTA_ERR_SHAPE), (dict(scale=float("nan")), V.VISTA_ERR_SHAPE),
    (dict(S=513), V.VISTA_ERR_UNSUPPORTED), (dict(d=512, H=4), V.VISTA_ERR_UNSUPPORTED), (dict(dtype=7), V.VISTA_ERR_UNSUPPORTED),
    (dict(attn=V.VISTA_ATTN_SILU), V.VISTA_ERR_UNSUPPORTED), (dict(attn=V.VISTA_ATTN_QLA), V.VISTA_ERR_UNSUPPORTED),
    (dict(total_items=1 << 40, segment_items=32), V.VISTA_ERR_UNSUPPORTED)])
def test_summarize_backward_rejects_bad_descriptors(kw, code):
    assert summarize_backward(desc(**kw)) == code
    if "segment_items" not in kw or kw["segment_items"] == 40:
        assert need(desc(**kw)) == 0


def test_summarize_backward_rejects_null_bad_offsets_and_small_workspace():
    d = desc()
    assert summarize_backward(None) == V.VISTA_ERR_NULL
    for name in ("x", "off", "q", "wk", "wv", "do", "dq", "dk", "dv"):
        assert summarize_backward(d, **{name: None}) == V.VISTA_ERR_NULL
    for bad in ([1, 50, 100], [0, 60, 50], [0, 50, 99]):
        off = np.array(bad, dtype=np.int64)
        assert summarize_backward(d, off_host=off.ctypes.data) == V.VISTA_ERR_OFFSETS
    assert summarize_backward(d, bytes=need(d) - 1) == V.VISTA_ERR_WORKSPACE
    assert summarize_backward(d, ws=None) == V.VISTA_ERR_WORKSPACE
    assert summarize_backward(d, ws=C.c_void_p(264)) == V.VISTA_ERR_WORKSPACE
    s = desc(self_term=True)
    assert need(s) > need(d) > 0
    for name in ("dks", "dvs"):
        assert summarize_backward(s, **{name: None}) == V.VISTA_ERR_NULL


def attend_backward(a, null=None, ws=ONE, size=1 << 40):
    args = [None if i == null else ONE for i in range(5)]
    return V.lib().vista_target_attend_backward(C.byref(a) if a is not None else None, *args, ws, size, None)


def test_target_attend_backward_rejects_bad_arguments():
    make = lambda **kw: V.AttendDesc(**{**dict(B=2, C=4, S=8, d=64, H=1, dtype=V.VISTA_F32, scale=0.0, flags=0), **kw})
    size = lambda a: V.lib().vista_target_attend_backward_workspace_bytes(C.byref(a))
    for kw, code in ((dict(B=0), 2), (dict(C=0), 2), (dict(S=0), 2), (dict(H=3), 2), (dict(scale=-1.0), 2), (dict(flags=2), 2),
                     (dict(S=513), 4), (dict(d=128), 4), (dict(dtype=5), 4)):
        assert attend_backward(make(**kw)) == code and size(make(**kw)) == 0
    a = make()
    assert attend_backward(None) == V.VISTA_ERR_NULL
    for i in range(5):
        assert attend_backward(a, null=i) == V.VISTA_ERR_NULL
    assert size(a) > 0
    for ws, n in ((None, 1 << 40), (C.c_void_p(128), 1 << 40), (ONE, size(a) - 1)):
        assert attend_backward(a, ws=ws, size=n) == V.VISTA_ERR_WORKSPACE


def test_layer_norm_rejects_bad_arguments():
    L = V.lib()
    make = lambda **kw: V.NormDesc(**{**dict(rows=4, d=64, dtype=V.VISTA_BF16, eps=0.0), **kw})
    size = lambda n: L.vista_layer_norm_backward_workspace_bytes(C.byref(n))
    forward = lambda n, x=ONE, y=ONE: L.vista_layer_norm(C.byref(n), x, ONE, ONE, y, None)
    backward = lambda n, x=ONE, dy=ONE, dx=ONE, dw=ONE, db=ONE, ws=ONE, nbytes=1 << 30: L.vista_layer_norm_backward(
        C.byref(n), x, ONE, dy, dx, dw, db, ws, nbytes, None)
    for kw, code in ((dict(rows=-1), 2), (dict(d=0), 2), (dict(eps=-1.0), 2), (dict(eps=float("inf")), 2), (dict(d=1025), 4),
                     (dict(dtype=3), 4)):
        assert forward(make(**kw)) == code and backward(make(**kw)) == code and size(make(**kw)) == 0
    n = make()
    assert L.vista_layer_norm(None, ONE, ONE, ONE, ONE, None) == V.VISTA_ERR_NULL
    for kw in (dict(x=None), dict(y=None)):
        assert forward(n, **kw) == V.VISTA_ERR_NULL
    for kw in (dict(x=None), dict(dy=None), dict(dx=None)):
        assert backward(n, **kw) == V.VISTA_ERR_NULL
    for kw in (dict(ws=None), dict(ws=C.c_void_p(128)), dict(nbytes=size(n) - 1), dict(dw=None, ws=None), dict(db=None, ws=None)):
        assert backward(n, **kw) == V.VISTA_ERR_WORKSPACE
    assert forward(make(rows=0), x=None, y=None) == V.VISTA_OK                     # nothing to do
    assert backward(make(rows=0), x=None, dy=None, dx=None, dw=None, db=None, ws=None) == V.VISTA_OK


def test_binding_checks_what_pointers_do_not_carry():
    """Shapes, types and devices that do not belong together, on CPU tensors: the check comes before the library."""
    B, S, N, d = 2, 3, 5, 8
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)
    off = torch.tensor([0, 2, 5])
    good = dict(history_emb=t(N, d), offsets=off, virtual_queries=t(S, d), W_k=t(d, d), W_v=t(d, d), d_out=t(B, S, d),
                d_queries=t(B, S, d), d_keys=t(N, d), d_values=t(N, d))
    call = lambda **kw: V.vista_summarize_backward(**{**good, **kw}, H=2)
    for kw in (dict(W_k=t(d, d + 1)), dict(d_out=t(B, S + 1, d)), dict(d_keys=t(N - 1, d)), dict(d_values=t(N, d // 2)),
               dict(d_queries=t(S, d)), dict(virtual_queries=t(B + 1, S, d)), dict(history_emb=t(N, 2, d // 2))):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(d_out=t(B, S, d, dtype=torch.bfloat16)), dict(offsets=off.int()), dict(offsets=off[:1])):
        with pytest.raises(TypeError):
            call(**kw)
    with pytest.raises(ValueError):
        call(d_self_keys=t(B, S, d))
    with pytest.raises(ValueError):
        call(offsets_host=torch.tensor([0, 5]))
    with pytest.raises(ValueError, match="device memory"):
        call()
    c = dict(candidates=t(B, 4, d), summaries=t(B, S, d), d_out=t(B, 4, d), d_candidates=t(B, 4, d), d_summaries=t(B, S, d))
    for kw in (dict(d_out=t(B, 5, d)), dict(summaries=t(B + 1, S, d)), dict(d_summaries=t(B, S, d + 1)), dict(candidates=t(4, d))):
        with pytest.raises(ValueError):
            V.vista_target_attend_backward(**{**c, **kw}, H=2)
    with pytest.raises(TypeError):
        V.vista_target_attend_backward(**{**c, "d_out": t(B, 4, d, dtype=torch.bfloat16)}, H=2)
    for w, b, y in ((t(d + 1), None, t(N, d)), (None, t(1), t(N, d)), (None, None, t(N, d + 1))):
        with pytest.raises(ValueError):
            V.vista_layer_norm(t(N, d), w, b, y)
    with pytest.raises(ValueError):
        V.vista_layer_norm_backward(t(N, d), None, t(N, d), t(N, d), t(d - 1), None)
    with pytest.raises(TypeError):
        V.vista_layer_norm_backward(t(N, d), None, t(N, d), t(N, d), t(d, dtype=torch.bfloat16), None)


# ---------------------------------------------------------------- launches of large calls keep to the runtime's limits
CALL = r"""
import ctypes as C, json, sys
stub = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
from paper_2510_22049_amd import binding as V
entry, kw = sys.argv[2], json.loads(sys.argv[3])
p, L = C.c_void_p(1 << 20), V.lib()
if entry == "summarize":
    st = L.vista_summarize_backward(C.byref(V.summarize_desc(**kw)), p, p, None, *[p] * 10, 1 << 60, None)
elif entry == "attend":
    st = L.vista_target_attend_backward(C.byref(V.AttendDesc(**kw)), *[p] * 6, 1 << 60, None)
else:
    st = L.vista_layer_norm_backward(C.byref(V.NormDesc(**kw)), *[p] * 7, 1 << 60, None)
    st += L.vista_layer_norm(C.byref(V.NormDesc(**kw)), *[p] * 4, None)
print(json.dumps([st, C.c_int.in_dll(stub, "launches").value, C.c_int.in_dll(stub, "refused").value]))
"""


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    import subprocess
    folder = tmp_path_factory.mktemp("stub")
    (folder / "stub.c").write_text(STUB)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(folder / "stub.so"), str(folder / "stub.c")], check=True)
    return str(folder / "stub.so")


@pytest.mark.parametrize("entry,kw", [
    ("summarize", dict(B=1 << 17, S=256, d=128, H=4, dtype=0, total_items=1 << 20)),
    ("summarize", dict(B=3, S=512, d=64, H=1, dtype=0, total_items=1 << 36)),
    ("summarize", dict(B=1 << 17, S=256, d=128, H=4, dtype=1, total_items=1 << 20, self_term=True)),
    ("summarize", dict(B=8, S=512, d=256, H=8, dtype=1, total_items=1 << 32)),
    ("summarize", dict(B=1, S=1, d=512, H=512, dtype=1, total_items=1 << 30)),
    ("attend", dict(B=1 << 20, C=1 << 12, S=16, d=16, H=1, dtype=1)),
    ("attend", dict(B=1 << 20, C=1 << 14, S=512, d=128, H=4, dtype=1)),
    ("attend", dict(B=1, C=1 << 30, S=512, d=64, H=1, dtype=0)),
    ("norm", dict(rows=1 << 40, d=1024, dtype=1)), ("norm", dict(rows=1 << 40, d=1, dtype=0))])
def test_large_calls_keep_to_the_launch_limits(stub, entry, kw):
    import json
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CALL, stub, entry, json.dumps(kw)], cwd=root, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    status, launches, refused = json.loads(r.stdout.strip().splitlines()[-1])
    assert (status, refused) == (0, 0) and launches >= 1
