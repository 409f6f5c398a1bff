"""The norms around a block on the host: what their entry points refuse, their
sizes, the generator's published outputs, and the 64-bit reference against
differences."""
import ctypes
import math

import numpy as np
import pytest

import layer_ref as R
from paper_2607_19378_amd import hyenand as H

FAKE = 1 << 40  # never dereferenced: every call below is refused
GAP = 1 << 36
FORWARD = ("x", "z", "gate", "w_post", "scale", "w_pre", "rng", "x_out", "n")
BACKWARD = ("x_out", "z", "gate", "w_post", "scale", "w_pre", "rng", "gx_out", "gn", "gx", "gz", "ggate", "gw_post", "gscale", "gw_pre")


def call(names, B=2, C=3, P=40, dtype=0, eps=(0.0, 0.0), p=0.5, ws=FAKE + 60 * GAP, ws_bytes=1 << 20, **at):
    ptr = {n: FAKE + i * GAP for i, n in enumerate(names)}
    ptr.update(at)
    v = [ctypes.c_void_p(ptr[n]) if ptr[n] else None for n in names]
    head, rest = v[:6], v[6:]
    if names is FORWARD:
        return H.lib().hyenand_block_norm(*head, *eps, p, *rest, B, C, P, dtype, None)
    return H.lib().hyenand_block_norm_backward(*head, *eps, p, *rest, B, C, P, dtype, ctypes.c_void_p(ws), ws_bytes, None)


def said():
    return H.lib().hyenand_last_error().decode()


@pytest.mark.parametrize("names", [FORWARD, BACKWARD])
def test_unaligned_and_overlapping(names):
    for dtype in (0, 1):
        for i, n in enumerate(names):
            assert call(names, dtype=dtype, **{n: FAKE + i * GAP + 1}) == H.ERR_INVALID_ARGUMENT
            assert f"{n} is not" in said()
    for out in (FORWARD[7:] if names is FORWARD else BACKWARD[9:]):
        for i, n in enumerate(names):
            if n != out:
                assert call(names, **{out: FAKE + i * GAP}) == H.ERR_INVALID_ARGUMENT, (out, n)
                assert "overlaps" in said()


def test_missing_parts():
    for n in ("x", "w_post", "rng", "x_out"):
        assert call(FORWARD, **{n: 0}) == H.ERR_INVALID_ARGUMENT, n
    for n in ("w_pre", "n", "z"):  # one without the other
        assert call(FORWARD, **{n: 0}) == H.ERR_INVALID_ARGUMENT, n
    none = dict(z=0, gate=0, w_post=0, scale=0, x_out=0)
    assert call(FORWARD, **none) == H.ERR_INVALID_ARGUMENT  # dropout of nothing
    assert call(FORWARD, p=0.0, **none, w_pre=0, n=0) == H.ERR_INVALID_ARGUMENT
    for n in ("gate", "w_post", "scale"):
        assert call(FORWARD, p=0.0, **{**none, n: FAKE + 50 * GAP}) == H.ERR_INVALID_ARGUMENT, n
    for n in ("x_out", "z", "gate", "w_post", "scale", "w_pre", "rng", "gn", "gx", "gz", "ggate", "gw_post", "gscale", "gw_pre"):
        assert call(BACKWARD, **{n: 0}) == H.ERR_INVALID_ARGUMENT, n
    assert call(BACKWARD, gx_out=0, gn=0, w_pre=0, gw_pre=0) == H.ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("names", [FORWARD, BACKWARD])
def test_numbers(names):
    for p in (-0.1, 1.0, 2.0, math.nan, math.inf):
        assert call(names, p=p) == H.ERR_INVALID_ARGUMENT and "dropout_p" in said()
    for eps in ((-1e-6, 0.0), (0.0, math.nan), (math.inf, 0.0)):
        assert call(names, eps=eps) == H.ERR_INVALID_ARGUMENT and "eps" in said()
    for kw, st in ((dict(B=0), 1), (dict(C=-1), 1), (dict(P=0), 1), (dict(dtype=2), 1), (dict(C=1 << 26), 2), (dict(P=1 << 41), 2)):
        assert call(names, **kw) == st, kw


def test_workspace():
    need = H.block_norm_backward_workspace_size((2, 3, 40), "f32")
    assert need > 0
    assert call(BACKWARD, ws_bytes=need - 1) == H.ERR_WORKSPACE_TOO_SMALL
    assert call(BACKWARD, ws=FAKE + 60 * GAP + 8) == H.ERR_INVALID_ARGUMENT
    assert call(BACKWARD, ws=FAKE + 10 * GAP) == H.ERR_INVALID_ARGUMENT and "workspace" in said()
    assert H.lib().hyenand_block_norm_backward_workspace_size(1, 4, 8, 0, None) == H.ERR_INVALID_ARGUMENT


def test_binding_refuses():
    import torch
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError):
        H.block_norm(x, w_pre=torch.zeros(3))
    with pytest.raises(ValueError):
        H.block_norm(torch.zeros(3), w_pre=torch.zeros(3))


def test_generator_published_outputs():
    """The known answers that the generator's authors give for Philox4x32-10."""
    ones = 0xFFFFFFFF
    assert R.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert R.philox((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert R.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [
        0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_reference_gradients_are_differences():
    rng = np.random.default_rng(4)
    B, C, P = 2, 5, 9
    a = {n: rng.standard_normal((B, C, P)) for n in ("x", "z", "gate")}
    a.update({n: rng.standard_normal(C) for n in ("w_post", "scale", "w_pre")})
    gx, gn = rng.standard_normal((B, C, P)), rng.standard_normal((B, C, P))
    keep = R.keep_factors(B, C, P, 0.3, 1, 2)
    order = ("x", "z", "gate", "w_post", "scale", "w_pre")
    for without in ((), ("gate",), ("scale",), ("gate", "scale")):
        arg = {n: None if n in without else a[n] for n in order}

        def loss(w):
            o, n = R.block_norm(*[w[k] for k in order], keep=keep)
            return (o * gx).sum() + (n * gn).sum()

        x_out, _ = R.block_norm(*[arg[k] for k in order], keep=keep)
        g = R.block_norm_backward(x_out, *[arg[k] for k in order[1:]], gx, gn, keep=keep)
        for name in order:
            key = "gx" if name == "x" else "g" + name
            assert (key in g) == (name not in without)
            if name in without:
                continue
            d = rng.standard_normal(a[name].shape)
            num = (loss({**arg, name: arg[name] + 1e-5 * d}) - loss({**arg, name: arg[name] - 1e-5 * d})) / 2e-5
            assert abs(num - (g[key][0] * d).sum()) < 1e-7 * max(1, abs(num)), name
