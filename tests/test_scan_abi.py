"""The gated linear recurrence on the host: what its entry points refuse, its
sizes, and the 64-bit reference of its GPU tests against the definition and
differences."""
import ctypes

import numpy as np
import pytest

import layer_ref as R
from paper_2607_19378_amd import hyenand as H

FAKE = 1 << 40  # never dereferenced: every call below is refused
GAP = 1 << 36


def call(fn, ptrs, tail):
    return getattr(H.lib(), fn)(*[ctypes.c_void_p(p) if p else None for p in ptrs], *tail)


def pointers(n, **at):
    p = [FAKE + i * GAP for i in range(n)]
    for i, x in at.items():
        p[int(i[1:])] = x
    return p


FORWARD = ("x1", "x2", "v", "log_a", "D", "h0", "lengths", "y", "h_last", "states")
BACKWARD = ("x1", "x2", "v", "log_a", "D", "lengths", "states", "gy", "gh_last", "gx1", "gx2", "gv", "glog_a", "gD", "gh0")
STEP = ("x1", "x2", "v", "log_a", "D", "slots", "state", "y")
OPTIONAL = {"h0", "lengths", "h_last", "states", "gh_last", "gh0", "slots"}


def kinds(B=2, C=3, L=700, dtype=0, ws=FAKE + 60 * GAP, ws_bytes=1 << 20, slots=9):
    return {"hyenand_scan": (FORWARD, (B, C, L, dtype, ctypes.c_void_p(ws), ws_bytes, None)),
            "hyenand_scan_backward": (BACKWARD, (B, C, L, dtype, ctypes.c_void_p(ws), ws_bytes, None)),
            "hyenand_scan_step": (STEP, (B, C, slots, dtype, None))}


@pytest.mark.parametrize("fn", list(kinds()))
def test_missing_and_unaligned_buffers(fn):
    for dtype, es in ((0, 4), (1, 2)):
        names, tail = kinds(dtype=dtype)[fn]
        for i, name in enumerate(names):
            if not (name in OPTIONAL and not (fn.endswith("backward") and name == "states")):
                assert call(fn, pointers(len(names), **{f"_{i}": 0}), tail) == H.ERR_INVALID_ARGUMENT
                assert f"{name} is NULL".encode() in H.lib().hyenand_last_error()
            assert call(fn, pointers(len(names), **{f"_{i}": FAKE + i * GAP + 1}), tail) == H.ERR_INVALID_ARGUMENT
            assert f"{name} is not".encode() in H.lib().hyenand_last_error()


@pytest.mark.parametrize("fn", list(kinds()))
def test_overlapping_outputs(fn):
    names, tail = kinds()[fn]
    outs = {"hyenand_scan": ("y", "h_last", "states"), "hyenand_scan_step": ("state", "y"),
            "hyenand_scan_backward": ("gx1", "gx2", "gv", "glog_a", "gD", "gh0")}[fn]
    for out in outs:
        for i, name in enumerate(names):
            if name == out or (out, name) == ("h_last", "h0"):
                continue
            p = pointers(len(names), **{f"_{names.index(out)}": FAKE + i * GAP})
            assert call(fn, p, tail) == H.ERR_INVALID_ARGUMENT, (out, name)
            assert b"overlaps" in H.lib().hyenand_last_error()
    if fn == "hyenand_scan":  # h_last may be h0, not a part of it
        p = pointers(len(names), _8=FAKE + 5 * GAP + 4)
        assert call(fn, p, tail) == H.ERR_INVALID_ARGUMENT
        assert b"h_last overlaps h0" in H.lib().hyenand_last_error()


@pytest.mark.parametrize("fn", list(kinds()))
def test_shapes_and_types(fn):
    for kw, status in ((dict(B=0), H.ERR_INVALID_ARGUMENT), (dict(C=0), H.ERR_INVALID_ARGUMENT), (dict(dtype=2), H.ERR_INVALID_ARGUMENT),
                       (dict(B=-1), H.ERR_INVALID_ARGUMENT), (dict(B=1 << 14, C=1 << 12), H.ERR_UNSUPPORTED),
                       (dict(B=1 << 62, C=1 << 62), H.ERR_UNSUPPORTED)):
        names, tail = kinds(**kw)[fn]
        assert call(fn, pointers(len(names)), tail) == status, kw
    if fn != "hyenand_scan_step":
        for L, status in ((0, H.ERR_INVALID_ARGUMENT), (-5, H.ERR_INVALID_ARGUMENT), ((1 << 40) + 1, H.ERR_UNSUPPORTED), (1 << 62, H.ERR_UNSUPPORTED)):
            names, tail = kinds(L=L)[fn]
            assert call(fn, pointers(len(names)), tail) == status, L


def test_step_pool():
    names, tail = kinds(B=4, slots=3)["hyenand_scan_step"]
    assert call("hyenand_scan_step", pointers(8, _5=0), tail) == H.ERR_INVALID_ARGUMENT  # a state for each row, without slots
    names, tail = kinds(slots=0)["hyenand_scan_step"]
    assert call("hyenand_scan_step", pointers(8), tail) == H.ERR_INVALID_ARGUMENT
    names, tail = kinds(B=65536, C=1)["hyenand_scan_step"]
    assert call("hyenand_scan_step", pointers(8), tail) == H.ERR_UNSUPPORTED


def test_workspace():
    assert H.scan_workspace_size((8, 512, 4096), "bf16") == 0
    need = H.scan_workspace_size((1, 4, 1 << 17), "f32")
    assert need > 0
    for fn, size in (("hyenand_scan", need), ("hyenand_scan_backward", H.scan_backward_workspace_size((1, 4, 1 << 17), "f32"))):
        names, tail = kinds(B=1, C=4, L=1 << 17, ws_bytes=size - 1)[fn]
        assert call(fn, pointers(len(names)), tail) == H.ERR_WORKSPACE_TOO_SMALL
        names, tail = kinds(B=1, C=4, L=1 << 17, ws=FAKE + 60 * GAP + 8)[fn]
        assert call(fn, pointers(len(names)), tail) == H.ERR_INVALID_ARGUMENT
        i = names.index("y" if fn == "hyenand_scan" else "gv")
        names, tail = kinds(B=1, C=4, L=1 << 17, ws=FAKE + i * GAP)[fn]
        assert call(fn, pointers(len(names)), tail) == H.ERR_INVALID_ARGUMENT
        assert b"workspace" in H.lib().hyenand_last_error()
    for fn in ("hyenand_scan_workspace_size", "hyenand_scan_backward_workspace_size"):
        assert getattr(H.lib(), fn)(1, 4, 8, 0, None) == H.ERR_INVALID_ARGUMENT
        out = ctypes.c_size_t(7)
        assert getattr(H.lib(), fn)(1, 4, 0, 0, ctypes.byref(out)) == H.ERR_INVALID_ARGUMENT and out.value == 7


def test_binding_refuses_host_tensors_and_other_shapes():
    import torch
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError):
        H.scan(x, x, x, x, torch.zeros(3))
    with pytest.raises(ValueError):
        H.scan_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], x[:, :, 0], torch.zeros(3), torch.zeros(2, 3))
    with pytest.raises(ValueError):
        H.scan(x.to(torch.float16), x, x, x, torch.zeros(3))


def _case(seed, L=9):
    rng = np.random.default_rng(seed)
    a = [rng.standard_normal((2, 3, L)) for _ in range(3)] + [-rng.uniform(0, 1.5, (2, 3, L))]
    return a + [rng.standard_normal(3)], rng.standard_normal((2, 3)), rng.standard_normal((2, 3, L)), rng.standard_normal((2, 3))


def test_reference_is_the_definition():
    """h_t as the sum over earlier positions of the decays between, times u; a start cuts the sum."""
    (x1, x2, v, la, D), h0, _, _ = _case(1)
    la[0, 1, 4] = -np.inf
    la[1, 2, 6] = -90.0
    out = R.scan(x1, x2, v, la, D, h0, lengths=[7, 9])
    for b in range(2):
        for c in range(3):
            for t in range(9):
                if b == 0 and t >= 7:
                    assert out["y"][b, c, t] == 0
                    continue
                h, alive = 0.0, 1.0
                for i in range(t, -1, -1):
                    h += alive * x1[b, c, i] * v[b, c, i]
                    alive *= 0.0 if la[b, c, i] < -87 else np.exp(la[b, c, i])
                h += alive * h0[b, c]
                assert abs(out["y"][b, c, t] - x2[b, c, t] * (h + D[c] * x1[b, c, t] * v[b, c, t])) < 1e-12


def test_reference_gradients_are_differences():
    args, h0, gy, gh = _case(2)
    lengths = [6, 9]

    def loss(a, h):
        o = R.scan(*a, h, lengths)
        return (o["y"] * gy).sum() + (o["h_last"] * gh).sum()

    g = R.scan(*args, h0, lengths, gy, gh)
    rng = np.random.default_rng(3)
    for i, name in enumerate(("gx1", "gx2", "gv", "glog_a", "gD", "gh0")):
        d = rng.standard_normal(g[name].shape)
        up, down = [x.copy() for x in args], [x.copy() for x in args]
        hu, hd = h0.copy(), h0.copy()
        if name == "gh0":
            hu, hd = h0 + 1e-5 * d, h0 - 1e-5 * d
        else:
            up[i], down[i] = args[i] + 1e-5 * d, args[i] - 1e-5 * d
        num = (loss(up, hu) - loss(down, hd)) / 2e-5
        assert abs(num - (g[name] * d).sum()) < 1e-7 * max(1, abs(num)), name
