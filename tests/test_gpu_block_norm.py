"""The norms before and behind a block (hyenand_block_norm and its backward)
against a plain 64-bit reference.

Tolerance of a value: fp32 roundings relative to the magnitudes of its terms,
and half a step of the storage type.  Roundings on the way, at most: 4 of a
gate, the sum of squares over a thread's channels (16, or C / 1024 where a
thread has more), 6 lanes and 16 wavefronts, of which a root keeps half, 4 of
the root, the quotient and the weights: 8 + (16 + C / 1024 + 22) / 2 below.
Gradients go through two such norms."""
import numpy as np
import pytest

import layer_ref as R
from paper_2607_19378_amd import workloads as W

from gpu_util import from_device, log, to_device

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
SEED, OFFSET = -0x123456789ABCDEF, 0x1F00000003
NAMES = ("x", "z", "gate", "w_post", "scale", "w_pre", "gx_out", "gn")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make(B, C, P, dtype, seed):
    rng = np.random.default_rng(seed)
    a = {n: rng.standard_normal((B, C, P)) for n in ("x", "z", "gate", "gx_out", "gn")}
    a["gate"] *= 3
    a["w_post"], a["w_pre"], a["scale"] = 1 + 0.2 * rng.standard_normal(C), 1 + 0.2 * rng.standard_normal(C), 0.5 * rng.standard_normal(C)
    store = {n: W.quantise(x, dtype) for n, x in a.items()}
    return store, {n: W.storage_to_f64(x, dtype) for n, x in store.items()}


def roundings(C):
    return 8 + (16 + C / 1024 + 22) / 2


def close(tag, got, ref, mag, units, dtype):
    assert got.shape == ref.shape, tag
    tol = units * 2.0 ** -23 * mag + HALF[dtype] * np.abs(ref) + 1e-37
    worst = float(np.max(np.abs(got - ref) / tol))
    log(f"[norm] {tag}: worst error / tolerance = {worst:.3f}")
    assert np.all(np.isfinite(got)) and worst <= 1.0, tag


def run_case(B, C, P, dtype, without=(), p=0.0, eps=(1e-6, 1e-5), grid=None, seed=0):
    """Forward and backward with everything but the tensors named in `without`."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    store, val = make(B, C, P, dtype, seed + 7 * C + P)
    shape = (B, C) + (grid or (P,))
    dev = {n: None if n in without else to_device(store[n].reshape(shape) if store[n].ndim > 1 else store[n], dtype) for n in NAMES}
    val = {n: None if n in without else val[n] for n in NAMES}
    rng = torch.tensor([SEED, OFFSET], device="cuda") if p else None
    keep = R.keep_factors(B, C, P, p, SEED, OFFSET) if p else None
    log(f"[norm] B={B} C={C} P={P} {dtype} without={without} p={p}")
    head = [dev[n] for n in NAMES[:6]]
    x_out, n = H.block_norm(*head, *eps, p, rng)
    torch.cuda.synchronize()
    rx, rn = R.block_norm(*[val[k] for k in NAMES[:6]], *eps, keep)
    units = roundings(C)
    flat = lambda t: from_device(t).reshape(B, C, P)  # noqa: E731
    if val["z"] is None:
        assert x_out is dev["x"]
        mag = np.abs(rx)
    else:
        mag = np.abs(val["x"]) + np.abs(rx - val["x"])
        close("x_out", flat(x_out), rx, mag, units, dtype)
    if val["w_pre"] is None:
        assert n is None
    else:
        q = R.inverse_rms(rx, eps[1])
        rms_mag = np.sqrt((mag * mag).mean(1, keepdims=True)) * q
        close("n", flat(n), rn, np.abs(val["w_pre"])[None, :, None] * q * (mag + np.abs(rx) * rms_mag), units, dtype)
    # the backward goes by what the forward stored
    stored = flat(x_out)
    kw = {k: val[k] for k in NAMES[1:]}
    if kw["gn"] is None:
        kw["w_pre"] = None
    ref = R.block_norm_backward(stored, **kw, eps_post=eps[0], eps_pre=eps[1], keep=keep)
    got = H.block_norm_backward(x_out, *[dev[k] for k in NAMES[1:6]], dev["gx_out"], dev["gn"], *eps, p, rng)
    torch.cuda.synchronize()
    for name, t in zip(("gx", "gz", "ggate", "gw_post", "gscale", "gw_pre"), got):
        assert (t is None) == (name not in ref), name
        if t is None:
            continue
        if t.dim() > 1:
            close(name, flat(t), *ref[name], 2 * units, dtype)
        else:  # 8 points a lane of every 1024th tile, the lanes, the rest in 64 bits
            close(name, from_device(t), *ref[name], 2 * units + 8 * (1 + B * P / 8 / 1024) + 3, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [1, 2, 7, 8, 9, 31, 33, 64, 65, 196, 1000])
@pytest.mark.parametrize("C", [3, 100, 384])
def test_points(C, P, dtype):
    run_case(2, C, P, dtype)


# channels: one, the edges of a wavefront, more than a thread's registers hold at a full tile, and than at any
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 16, 63, 64, 65, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8200])
def test_channels(C, dtype):
    run_case(1, C, 37, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C", [(1, 1), (5, 1024), (33, 1000), (3, 4096), (2, 16384), (2, 17000), (700, 1000), (1200, 900), (2100, 250)])
def test_tokens(B, C, dtype):
    run_case(B, C, 1, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,P", [(1, 2, 70001), (70, 5, 999), (1500, 20, 1), (1300, 17, 9), (1100, 4100, 1), (1100, 2100, 5)])
def test_many_tiles(B, C, P, dtype):
    """More tiles than the backward has workgroups: each adds up the weights' sums of several."""
    run_case(B, C, P, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("without", [("gate",), ("scale",), ("gate", "scale"), ("z", "gate", "w_post", "scale"), ("w_pre", "gn"),
                                     ("gate", "w_pre", "gn"), ("gx_out",), ("gn",), ("z", "gate", "w_post", "scale", "gx_out")])
@pytest.mark.parametrize("C,P", [(100, 33), (24, 1), (5000, 9), (17000, 1)])
def test_parts(C, P, without, dtype):
    run_case(2, C, P, dtype, without)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,P,p", [(2, 30, 77, 0.1), (3, 100, 8, 0.5), (2, 200, 1, 0.3), (1, 9, 515, 0.999), (1, 5000, 9, 0.25), (1, 17000, 1, 0.1)])
def test_dropout(B, C, P, p, dtype):
    run_case(B, C, P, dtype, p=p)


def test_dropout_rate_and_seeds():
    """The share of dropped points, and masks that differ by seed and by offset and by nothing else."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    x = torch.zeros(4, 64, 4096, device="cuda")
    z, one = torch.ones_like(x), torch.ones(64, device="cuda")

    def kept(seed, offset, p):
        return H.block_norm(x, z, None, one, None, None, dropout_p=p, rng=torch.tensor([seed, offset], device="cuda"))[0] != 0

    n = x.numel()
    for p in (0.1, 0.5, 0.9):
        m = kept(3, 4, p)
        share = 1 - float(m.double().mean())
        assert abs(share - p) < 6 * (p * (1 - p) / n) ** 0.5 + 2.0 ** -17, (p, share)
        assert torch.equal(m, kept(3, 4, p))
    for other in ((4, 4), (3, 5), (3 + (1 << 40), 4), (3, 4 + (1 << 40))):
        agree = float((kept(3, 4, 0.5) == kept(*other, 0.5)).double().mean())
        assert abs(agree - 0.5) < 6 * 0.5 / n ** 0.5, other
    assert torch.equal(kept(3, 4, 1e-7), torch.ones_like(m))  # rounds to no dropout
    assert torch.all(H.block_norm(x, z, None, one, None, None, dropout_p=0.99999, rng=torch.tensor([1, 2], device="cuda"))[0].isfinite())


@pytest.mark.parametrize("grid", [(14, 14), (4, 6, 5), (33,)])
def test_grids(grid):
    run_case(2, 12, int(np.prod(grid)), "f32", grid=grid)


def test_zeros_without_eps_and_extreme_gates():
    import torch
    from paper_2607_19378_amd import hyenand as H
    for C, P in ((8, 1), (8, 20), (5000, 9)):
        x = torch.randn(2, C, P, device="cuda")
        x[1] = 0
        z, one = torch.zeros_like(x), torch.ones(C, device="cuda")
        x_out, n = H.block_norm(x, z, None, one, one, one, 0.0, 0.0)
        assert torch.equal(x_out, x) and torch.all(n[1] == 0) and torch.isfinite(n).all()
        g = H.block_norm_backward(x_out, z, None, one, one, one, x, x, 0.0, 0.0)
        assert all(torch.isfinite(t).all() for t in g if t is not None) and torch.all(g[1] == 0) and torch.equal(g[0][1], x[1])
        # gates of any size: sigmoid is 0 or 1, its slope 0
        gate = torch.full_like(x, 200.0)
        gate[:, ::2] = -200.0
        gate[:, 1] = float("inf")
        gate[:, 2] = -float("inf")
        z = torch.randn_like(x)
        x_out, n = H.block_norm(x, z, gate, one, one, one)
        ref = H.block_norm(x, z * (gate > 0), None, one, one, one)
        assert torch.equal(x_out, ref[0]) and torch.equal(n, ref[1])
        g = H.block_norm_backward(x_out, z, gate, one, one, one, x, x)
        assert all(torch.isfinite(t).all() for t in g) and torch.all(g[2] == 0) and torch.all(g[1][:, ::2] == 0)


def test_views_at_any_alignment_and_nothing_behind_them():
    import torch
    from paper_2607_19378_amd import hyenand as H
    for dt in (torch.float32, torch.bfloat16):
        for B, C, P in ((2, 7, 37), (3, 50, 1), (1, 600, 130), (1, 5000, 9)):
            size = B * C * P

            def place(shape):
                k = int(np.prod(shape))
                whole = torch.full((k + 16,), 7.0, device="cuda", dtype=dt)
                return whole, whole[3:3 + k].view(shape)

            x, z, gate, a, b = (torch.randn(size + 1, device="cuda").to(dt)[1:].view(B, C, P) for _ in range(5))
            w = [torch.randn(C + 1, device="cuda").to(dt)[1:] for _ in range(3)]
            log(f"[norm] views {dt} {(B, C, P)}")
            want = H.block_norm(x, z, gate, *w)
            grads = H.block_norm_backward(want[0], z, gate, *w, a, b)
            outs = [place((B, C, P)) for _ in range(2)]
            H.PreparedBlockNorm(outs[0][1], outs[1][1], x, z, gate, *w)()
            gouts = [place((B, C, P)) for _ in range(3)] + [place((C,)) for _ in range(3)]
            H.PreparedBlockNormBackward(*[t for _, t in gouts], want[0], z, gate, *w, a, b)()
            torch.cuda.synchronize()
            for (whole, t), ref in zip(outs + gouts, want + grads):
                assert torch.equal(t, ref) and torch.all(whole[:3] == 7) and torch.all(whole[3 + t.numel():] == 7)


def test_a_block_in_training():
    """Norm, recurrent mixer, norms and dropout, and all gradients of the chain, against differences of it in 64 bits."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    B, C, L, p = 2, 6, 45, 0.2
    rng = np.random.default_rng(8)
    a = {n: rng.standard_normal((B, C, L)) for n in ("x", "x2", "v", "gate", "gx", "gn")}
    a["log_a"] = -rng.uniform(0, 0.5, (B, C, L))
    for n in ("D", "w1", "w_post", "scale", "w2"):
        a[n] = rng.standard_normal(C)
    a = {n: x.astype(np.float32) for n, x in a.items()}
    val = {n: x.astype(np.float64) for n, x in a.items()}
    t = {n: torch.from_numpy(x).cuda() for n, x in a.items()}
    keep, seed = R.keep_factors(B, C, L, p, 5, 6), torch.tensor([5, 6], device="cuda")

    _, n1 = H.block_norm(t["x"], w_pre=t["w1"])
    y, _, states = H.scan(n1, t["x2"], t["v"], t["log_a"], t["D"], return_states=True)
    x_out, n2 = H.block_norm(t["x"], y, t["gate"], t["w_post"], t["scale"], t["w2"], dropout_p=p, rng=seed)
    gx, gy, ggate, gw_post, gscale, gw2 = H.block_norm_backward(x_out, y, t["gate"], t["w_post"], t["scale"], t["w2"],
                                                                t["gx"], t["gn"], dropout_p=p, rng=seed)
    gn1, gx2, gv, gla, gD = H.scan_backward(n1, t["x2"], t["v"], t["log_a"], t["D"], states, gy)
    gx, _, _, _, _, gw1 = H.block_norm_backward(t["x"], None, None, None, None, t["w1"], gx, gn1)
    torch.cuda.synchronize()

    def loss(w):
        _, m = R.block_norm(w["x"], w_pre=w["w1"])
        s = R.scan(m, w["x2"], w["v"], w["log_a"], w["D"])["y"]
        o, q = R.block_norm(w["x"], s, w["gate"], w["w_post"], w["scale"], w["w2"], keep=keep)
        return (o * val["gx"]).sum() + (q * val["gn"]).sum()

    got = dict(x=gx, x2=gx2, v=gv, gate=ggate, log_a=gla, D=gD, w1=gw1, w_post=gw_post, scale=gscale, w2=gw2)
    for name, g in got.items():
        d = rng.standard_normal(val[name].shape)
        num = (loss({**val, name: val[name] + 1e-5 * d}) - loss({**val, name: val[name] - 1e-5 * d})) / 2e-5
        mine = float((from_device(g) * d).sum())
        # fp32 through the chain: 2^-23 times some hundred roundings of terms of the size of the gradients' norm
        assert abs(mine - num) <= 3e-5 * float(np.linalg.norm(from_device(g)) * np.linalg.norm(d)) + 1e-6, name


def test_captured_and_replayed():
    """One graph with forward and backward: a changed seed draws anew in the next replay."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    for B, C, P in ((2, 24, 300), (64, 20, 1), (1, 5000, 9)):
        x, z, gate, a, b = (torch.randn(B, C, P, device="cuda") for _ in range(5))
        w = [torch.randn(C, device="cuda") for _ in range(3)]
        rng = torch.tensor([1, 2], device="cuda")
        H.block_norm_backward(*[H.block_norm(x, z, gate, *w, dropout_p=0.5, rng=rng)[0], z, gate, *w, a, b], dropout_p=0.5, rng=rng)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        log(f"[norm] graph {(B, C, P)}")
        with torch.cuda.graph(graph):
            out = H.block_norm(x, z, gate, *w, dropout_p=0.5, rng=rng)
            grads = H.block_norm_backward(out[0], z, gate, *w, a, b, dropout_p=0.5, rng=rng)
        seen = []
        for i in range(4):
            rng.copy_(torch.tensor([1, 10 + i], device="cuda"))
            z.copy_(torch.randn(B, C, P, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            eager = H.block_norm(x, z, gate, *w, dropout_p=0.5, rng=rng)
            ge = H.block_norm_backward(eager[0], z, gate, *w, a, b, dropout_p=0.5, rng=rng)
            torch.cuda.synchronize()
            for s, t in zip(out + grads, eager + ge):
                assert torch.equal(s, t), i
            seen.append((out[0] == x).clone())
        assert not torch.equal(seen[0], seen[1])


def test_side_stream():
    import torch
    from paper_2607_19378_amd import hyenand as H
    x, z, gate, a, b = (torch.randn(2, 300, 500, device="cuda") for _ in range(5))
    w = [torch.randn(300, device="cuda") for _ in range(3)]
    want = H.block_norm(x, z, gate, *w)
    gw = H.block_norm_backward(want[0], z, gate, *w, a, b)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = H.block_norm(x, z, gate, *w, stream=s)
    gg = H.block_norm_backward(got[0], z, gate, *w, a, b, stream=s)
    s.synchronize()
    for p, q in zip(want + gw, got + gg):
        assert torch.equal(p, q)


def test_offsets_beyond_32_bits():
    """Points behind 2^31 elements: what their own values give alone, with the same draws of the generator."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    C, P = 3, (1 << 30) + 77
    x = torch.randn(1, 1, P, device="cuda", dtype=torch.bfloat16).expand(1, C, P).contiguous()
    one = torch.ones(C, device="cuda", dtype=torch.bfloat16)
    log("[norm] more than 2^31 elements")
    x_out, n = H.block_norm(x, x, None, one, one, one)
    g = H.block_norm_backward(x_out, x, None, one, one, one, None, x)
    torch.cuda.synchronize()
    tail = x[:, :, P - 100001:].contiguous()
    xt, nt = H.block_norm(tail, tail, None, one, one, one)
    gt = H.block_norm_backward(xt, tail, None, one, one, one, None, tail)
    torch.cuda.synchronize()
    for s, t in ((x_out, xt), (n, nt)):
        assert torch.equal(s[:, :, P - 100001:], t)
    # The gradients of the two calls may be summed in different orders.  All channels of a point are alike, so that with
    # q = 1 / |x_out| and r = 1 / |z| the terms of gx, q gn and its mean along the unit vector, are q |gn| each, those of
    # gz r times the two of gx each: each call is off by the roundings of the other tests relative to these magnitudes.
    # Where a draw is 0 itself (1 / 0 times 0 is no bound) all terms are 0, and so are both calls'.
    units = 2 * 2 * roundings(C) * 2.0 ** -23
    q, r = xt.double().abs().reciprocal(), tail.double().abs().reciprocal()
    mag = 2 * q * tail.double().abs()
    for s, t, m in ((g[0], gt[0], mag), (g[1], gt[1], 2 * r * mag)):
        s = s[:, :, P - 100001:]
        assert torch.all((s == t) & (tail == 0) | ((s.double() - t.double()).abs() <= units * m))


def test_samples_beyond_32_bits():
    """A sample of less than 4 GB behind more than 2^31 elements: what it gives alone."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    B, C, P = 5, 512, (1 << 20) + 8
    x = torch.randn(1, C, P, device="cuda", dtype=torch.bfloat16).expand(B, C, P).contiguous()
    w = [torch.randn(C, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
    log("[norm] samples beyond 2^31 elements")
    x_out, n = H.block_norm(x, x, x, *w)
    g = H.block_norm_backward(x_out, x, x, *w, x, x)
    torch.cuda.synchronize()
    for t in (x_out, n) + g[:3]:
        assert torch.equal(t[0], t[B - 1])
    one = H.block_norm(x[:1].contiguous(), x[:1].contiguous(), x[:1].contiguous(), *w)
    assert torch.equal(one[0][0], x_out[B - 1]) and torch.equal(one[1][0], n[B - 1])


@pytest.mark.parametrize("B,P", [((1 << 26) - 4, 1), (1, 1 << 29), (1, 1 << 30)])
def test_weights_of_very_many_points(B, P):
    """One channel, every point's term of each weight's gradient 1 + 2^-11, in tiles of one point, tiles in registers and
    two sweeps.  The sum goes through fp32 over 64 tiles of 4 points (half a step each) at most, then through 64 bits."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    one, term = 1.0, 1 + 2.0 ** -11
    x = torch.full((B, 1, P), one, device="cuda")
    g = torch.full((B, 1, P), term, device="cuda")
    w = torch.ones(1, device="cuda")
    log(f"[norm] weights of {B} x {P} points")
    # a single channel's norms are signs: gx = gx_out, and all three sums are those of the terms
    grads = H.block_norm_backward(x, x, None, w, w, w, g, g, 0.0, 0.0)
    torch.cuda.synchronize()
    ref = term * B * P
    for t in grads[3:]:
        assert abs(float(t) - ref) <= (64 * 4 + 1) * 2.0 ** -24 * ref, float(t) / ref - 1


@pytest.mark.parametrize("C,P", [(100, 33), (24, 1), (5000, 9), (17000, 1)])
def test_stream_without_its_norm(C, P):
    """Without gn the gradients do not depend on x_out, whatever stands there."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    x, z, gate, g = (torch.randn(2, C, P, device="cuda") for _ in range(4))
    w, s = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    wild = x.clone()
    wild[0, 1], wild[1, 2], wild[1, 3] = float("inf"), float("nan"), 3e38
    want = H.block_norm_backward(x, z, gate, w, s, None, g, None)
    got = H.block_norm_backward(wild, z, gate, w, s, None, g, None)
    torch.cuda.synchronize()
    assert torch.equal(want[0], g)
    for name, a, b in zip(("gx", "gz", "ggate", "gw_post", "gscale"), got, want):
        assert torch.isfinite(b).all() and torch.equal(a, b), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,P", [(8, 1), (8, 20), (200, 77), (5000, 9), (17000, 1)])
def test_gates_whose_smaller_part_is_zero(C, P, dtype):
    """Gates of 100 and more (sigmoid 1, its rest 0) are none, gates of -100 and less close the branch, and an absent gate
    is an open one: forward and backward, bit for bit."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x, z, a, b = (torch.randn(2, C, P, device="cuda").to(dt) for _ in range(4))
    w = [torch.randn(C, device="cuda").to(dt) for _ in range(3)]
    gate = torch.full((2, C, P), 200.0, device="cuda", dtype=dt)
    gate[:, ::3], gate[:, 1::3] = 100.0, float("inf")
    closed = gate.clone()
    closed[:, 2::4], closed[:, 3::8] = -200.0, -float("inf")
    for g, zz in ((gate, z), (closed, torch.where(closed > 0, z, 0.0))):
        got, want = H.block_norm(x, z, g, *w), H.block_norm(x, zz, None, *w)
        gg, gw = H.block_norm_backward(got[0], z, g, *w, a, b), H.block_norm_backward(want[0], zz, None, *w, a, b)
        torch.cuda.synchronize()
        for s, t in list(zip(got, want)) + [(gg[0], gw[0])] + list(zip(gg[3:], gw[3:])):
            assert torch.equal(s, t)
        assert torch.equal(gg[1], torch.where(g > 0, gw[1], 0.0)) and torch.all(gg[2] == 0)
        assert torch.all(zz[:, 0] == z[:, 0]) and bool((gw[1] != 0).any())
