"""The gated linear recurrence (hyenand_scan, its backward and its step) against
a plain 64-bit reference, on every way that a call's rows are spread.

Tolerance of a point: the fp32 roundings on a contribution's way (layer_ref.
scan_roundings) relative to the sum of the magnitudes of its terms, and half a
step of the storage type for each stored value."""
import numpy as np
import pytest

import layer_ref as R
from paper_2607_19378_amd import workloads as W

from gpu_util import from_device, log, to_device

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
NAMES = ("x1", "x2", "v", "log_a")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make(B, C, L, dtype, seed, packed=False, lengths=False, memory=(4, 4096)):
    """Storage arrays of a call and their 64-bit values."""
    rng = np.random.default_rng(seed)
    a = {n: rng.standard_normal((B, C, L)) for n in ("x1", "x2", "v", "gy")}
    rate = np.exp(-rng.uniform(np.log(memory[0]), np.log(memory[1]), (1, C, 1)))
    a["log_a"] = -rate * np.exp(rng.uniform(-2, 2, (B, C, L)))
    if packed:
        a["log_a"][rng.uniform(size=(B, C, L)) < 0.02] = -np.inf
    a["D"] = rng.standard_normal(C)
    with np.errstate(invalid="ignore"):
        store = {n: W.quantise(x, dtype) for n, x in a.items()}
    if packed and dtype == "bf16":  # -inf as bf16 bits
        store["log_a"][np.isneginf(a["log_a"])] = 0xFF80
    val = {n: W.storage_to_f64(x, dtype) for n, x in store.items()}
    state = dict(h0=rng.standard_normal((B, C)).astype(np.float32), gh_last=rng.standard_normal((B, C)).astype(np.float32))
    n = rng.integers(0, L + 1, B) if lengths else None
    if n is not None and B > 2:
        n[0], n[1] = 0, L
    return store, val, state, n


def on_gpu(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def close(tag, got, ref, mag, roundings, dtype):
    assert got.shape == ref.shape
    tol = roundings * 2.0 ** -23 * mag + HALF[dtype] * np.abs(ref) + 1e-37
    off = np.abs(got - ref)
    worst = float(np.max(off / tol)) if off.size else 0.0
    log(f"[scan] {tag}: worst error / tolerance = {worst:.3f}")
    assert np.all(np.isfinite(got)) and worst <= 1.0, tag


def run_case(B, C, L, dtype, seed, packed, lengths, carry, memory=(4, 4096)):
    import torch
    from paper_2607_19378_amd import hyenand as H
    store, val, state, n = make(B, C, L, dtype, seed, packed, lengths, memory)
    if n is not None:  # what stands behind a sample's end is not looked at
        bad = np.uint16(0x7FC0) if dtype == "bf16" else np.float32(np.nan)
        for i, end in enumerate(n):
            for name in NAMES + ("gy",):
                store[name][i, :, end:] = bad
    dev = {k: to_device(x, dtype) for k, x in store.items()}
    h0, gh_last = (on_gpu(state[k]) if carry else None for k in ("h0", "gh_last"))
    lens = None if n is None else on_gpu(n.astype(np.int64))
    mix = [dev[k] for k in NAMES] + [dev["D"]]
    log(f"[scan] B={B} C={C} L={L} {dtype} packed={packed} lengths={lengths} carry={carry}")
    y, last, states = H.scan(*mix, h0=h0, lengths=lens, return_last=True, return_states=True)
    g = H.scan_backward(*mix, states, dev["gy"], lengths=lens, gh_last=gh_last, return_gh0=True)
    torch.cuda.synchronize()
    kw = dict(h0=state["h0"] if carry else None, lengths=n, gy=val["gy"], gh_last=state["gh_last"] if carry else None)
    args = [val[k] for k in NAMES] + [val["D"]]
    ref, mag = R.scan(*args, **kw), R.scan_magnitudes(*args, **kw)
    r = R.scan_roundings(L)
    close("y", from_device(y), ref["y"], mag["y"], r, dtype)
    close("h_last", from_device(last), ref["h_last"], mag["h_last"], r, "f32")
    close("states", from_device(states), ref["states"], mag["states"], r, "f32")
    for name, t in zip(("gx1", "gx2", "gv", "glog_a"), g):
        # the gradient of a log decay is a product of two such sums
        close(name, from_device(t), ref[name], mag[name], 2 * r if name == "glog_a" else r, dtype)
    close("gD", from_device(g[4]), ref["gD"], mag["gD"], 8, dtype)  # products and a sum in lanes, the rest in 64 bits
    close("gh0", from_device(g[5]), ref["gh0"], mag["gh0"], r, "f32")


# lanes per row 1, 2, 4, ... 32, each with a last lane that is full, short and alone
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 127, 129, 196, 255, 256])
def test_short_rows(L, dtype):
    run_case(3, 37, L, dtype, L, packed=L % 2 == 1, lengths=True, carry=True)


# four wavefronts a row, from five tiles on eight, with tiles that end inside, at and behind a block
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [257, 511, 512, 513, 1025, 1501, 2048, 2049, 4095, 8192, 8193, 9001])
def test_long_rows(L, dtype):
    run_case(2, 3, L, dtype, L, packed=False, lengths=L % 2 == 1, carry=True)


@pytest.mark.parametrize("L", [700, 2500])
def test_packed_rows(L):
    run_case(2, 5, L, "f32", L, packed=True, lengths=False, carry=False)


# four wavefronts a row, and eight below 1024 rows
@pytest.mark.parametrize("B,C,L", [(4, 515, 600), (3, 700, 1300), (2, 300, 2700), (1, 513, 4100)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows(B, C, L, dtype):
    run_case(B, C, L, dtype, C, packed=True, lengths=True, carry=True)


# the longest row of one piece, then rows split into segments: the last one shorter, and a sample that ends in each
@pytest.mark.parametrize("B,C,L", [(1, 1, 16384), (1, 3, 40000), (5, 2, 33333), (2, 50, 17001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_split_rows(B, C, L, dtype):
    run_case(B, C, L, dtype, C, packed=False, lengths=B > 1, carry=True)


def test_long_memory():
    """Decays that forget almost nothing over the whole row, through every level of the joins."""
    run_case(1, 4, 50000, "f32", 11, packed=False, lengths=False, carry=True, memory=(20000, 40000))


def test_starts_stop_infinities_and_nans():
    """A sequence that starts takes nothing over: -inf, the types' lowest values and anything below -87."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    for dt in (torch.float32, torch.bfloat16):
        for L in (40, 700, 20000):
            g = torch.Generator(device="cuda").manual_seed(L)
            x1, x2, v = (torch.randn(2, 4, L, generator=g, device="cuda").to(dt) for _ in range(3))
            la = (-0.01 * torch.rand(2, 4, L, generator=g, device="cuda")).to(dt)
            D = torch.randn(4, generator=g, device="cuda").to(dt)
            gy = torch.randn(2, 4, L, generator=g, device="cuda").to(dt)
            cut = L // 2 + 3
            for c, mark in enumerate((-float("inf"), torch.finfo(dt).min, -88.0, -1000.0)):
                la[:, c, cut] = mark
            args = (x1, x2, v, la, D)
            log(f"[scan] starts {dt} L={L}")
            y, last, st = H.scan(*args, return_last=True, return_states=True)
            grads = H.scan_backward(*args, st, gy)
            bad = x1.clone()
            bad[:, :, cut - 1] = float("inf")
            bad[0, :, 0] = float("nan")
            wild = la.clone()  # and the decays themselves
            wild[0, :, cut // 2] = float("nan")
            wild[1, :, cut // 3] = float("inf")
            yb, lastb, stb = H.scan(bad, x2, v, wild, D, return_last=True, return_states=True)
            gb = H.scan_backward(bad, x2, v, wild, D, stb, gy)
            late = gy.clone()  # and nothing of the later sequence's gradient reaches the earlier one
            late[:, :, cut:] = float("nan")
            after = la.clone()
            after[0, :, cut + 1:] = float("nan")
            after[1, :, -1] = float("inf")
            gl = H.scan_backward(x1, x2, v, after, D, st, late)
            torch.cuda.synchronize()
            assert torch.equal(yb[:, :, cut:], y[:, :, cut:]) and torch.equal(lastb, last)
            assert not torch.isfinite(yb[:, :, cut - 1]).any()
            for i in range(4):
                assert torch.equal(gb[i][:, :, cut:], grads[i][:, :, cut:]), i
                assert torch.equal(gl[i][:, :, :cut], grads[i][:, :, :cut]), i
            assert torch.all(gl[3][:, :, cut] == 0) and torch.all(grads[3][:, :, cut] == 0)


def test_nan_reaches_everything_behind_it():
    import torch
    from paper_2607_19378_amd import hyenand as H
    for L in (33, 1200, 20000):
        x = torch.ones(1, 2, L, device="cuda")
        la = torch.full_like(x, -0.5)
        x1 = x.clone()
        x1[0, 0, 9] = float("nan")
        y, _, _ = H.scan(x1, x, x, la, torch.zeros(2, device="cuda"))
        assert torch.isnan(y[0, 0, 9:]).all() and torch.isfinite(y[0, 0, :9]).all() and torch.isfinite(y[0, 1]).all()


def test_lengths_out_of_range_and_state_in_place():
    import torch
    from paper_2607_19378_amd import hyenand as H
    for L in (20, 3000, 20000):
        g = torch.Generator(device="cuda").manual_seed(L)
        x1, x2, v = (torch.randn(3, 5, L, generator=g, device="cuda") for _ in range(3))
        la = -0.01 * torch.rand(3, 5, L, generator=g, device="cuda")
        D, h0 = torch.randn(5, generator=g, device="cuda"), torch.randn(3, 5, generator=g, device="cuda")
        log(f"[scan] lengths out of range L={L}")
        a = H.scan(x1, x2, v, la, D, h0=h0, lengths=torch.tensor([-4, L + 9, 7], device="cuda"), return_last=True)
        b = H.scan(x1, x2, v, la, D, h0=h0, lengths=torch.tensor([0, L, 7], device="cuda"), return_last=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert torch.equal(a[1][0], h0[0]) and torch.all(a[0][0] == 0) and torch.all(a[0][2, :, 7:] == 0)
        state, y = h0.clone(), torch.empty_like(x1)
        H.PreparedScan(y, x1, x2, v, la, D, h0=state, lengths=torch.tensor([0, L, 7], device="cuda"), h_last=state)()
        assert torch.equal(y, b[0]) and torch.equal(state, b[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_follow_the_scan(dtype):
    """Chunks and single steps on kept states give what one call gives (fp32 roundings of the state apart)."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    B, C, L = 3, 300, 21
    store, val, state, _ = make(B, C, L, dtype, 5, packed=True)
    dev = {k: to_device(x, dtype) for k, x in store.items()}
    mix = [dev[k] for k in NAMES]
    y, last, _ = H.scan(*mix, dev["D"], h0=on_gpu(state["h0"]), return_last=True)
    h = on_gpu(state["h0"])
    ys = [H.scan_step(*[t[:, :, i].contiguous() for t in mix], dev["D"], h) for i in range(L)]
    args = [val[k] for k in NAMES] + [val["D"]]
    ref, mag = R.scan(*args, h0=state["h0"]), R.scan_magnitudes(*args, h0=state["h0"])
    close("steps y", from_device(torch.stack(ys, 2)), ref["y"], mag["y"], 2.0 * L + 4, dtype)
    close("steps state", from_device(h), ref["h_last"], mag["h_last"], 2.0 * L + 4, "f32")
    h2 = on_gpu(state["h0"])
    first = H.scan(*[t[:, :, :9].contiguous() for t in mix], dev["D"], h0=h2, return_last=True)
    second = H.scan(*[t[:, :, 9:].contiguous() for t in mix], dev["D"], h0=first[1], return_last=True)
    close("chunks", from_device(torch.cat([first[0], second[0]], 2)), ref["y"], mag["y"], R.scan_roundings(L), dtype)
    close("chunks state", from_device(second[1]), ref["h_last"], mag["h_last"], R.scan_roundings(L), "f32")


def test_slots():
    """Idle rows, states that no row names, and rows that name the same state: positions in the order of the batch."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    for B, C in ((6, 5), (40, 513), (700, 3)):
        g = torch.Generator(device="cuda").manual_seed(B)
        x1, x2, v = (torch.randn(B, C, generator=g, device="cuda") for _ in range(3))
        la, D = -torch.rand(B, C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
        N = B // 2 + 3
        slots = torch.randint(-1, N + 1, (B,), generator=g, device="cuda")  # some idle (-1, N), many the same
        slots[1], slots[4], slots[5] = slots[0], -(1 << 40), 1 << 40
        pool = torch.randn(N + 2, C, generator=g, device="cuda")
        start = pool.clone()
        log(f"[scan] slots B={B} C={C}")
        y = H.scan_step(x1, x2, v, la, D, pool[1:-1], slots)
        torch.cuda.synchronize()
        ref, yr = start[1:-1].double().cpu(), torch.zeros(B, C, dtype=torch.float64)
        ins = [t.double().cpu() for t in (x1, x2, v, la, D)]
        for b, s in enumerate(slots.tolist()):
            if 0 <= s < N:
                u = ins[0][b] * ins[2][b]
                ref[s] = torch.exp(ins[3][b]) * ref[s] + u
                yr[b] = ins[1][b] * (ref[s] + ins[4] * u)
        assert torch.equal(pool[0], start[0]) and torch.equal(pool[-1], start[-1])
        named = set(s for s in slots.tolist() if 0 <= s < N)
        for s in set(range(N)) - named:
            assert torch.equal(pool[1 + s], start[1 + s])
        # at most B steps on one state, decays and sums of magnitudes below 10 * B
        assert torch.allclose(pool[1:-1].double().cpu(), ref, rtol=0, atol=2e-5) and torch.allclose(y.double().cpu(), yr, rtol=1e-5, atol=2e-4)
        assert torch.all(y[4:6] == 0)


@pytest.mark.parametrize("L", [64, 3000])
def test_constant_decay_is_the_long_convolution(L):
    """With one decay along a row the recurrence is hyenand_fftconv with k_t = exp(t log_a)."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    g = torch.Generator(device="cuda").manual_seed(L)
    x1, x2, v = (torch.randn(2, 6, L, generator=g, device="cuda") for _ in range(3))
    D, rate = torch.randn(6, generator=g, device="cuda"), -torch.rand(2, 6, 1, generator=g, device="cuda") / 4 - 0.01
    y, _, _ = H.scan(x1, x2, v, rate.expand(2, 6, L).contiguous(), D)
    k = torch.exp(rate.double() * torch.arange(L, device="cuda")).float()
    ref = H.fftconv(x1, x2, v, k, D)
    err = float((y - ref).norm() / ref.norm())
    assert err <= 1e-5, err  # the convolution's own tolerance


def test_views_at_any_alignment_and_nothing_behind_them():
    """Outputs in the middle of larger buffers, at element alignment: nothing else is written."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    for dt in (torch.float32, torch.bfloat16):
        for B, C, L in ((2, 3, 37), (1, 5, 1501), (1, 2, 20001), (700, 3, 515)):
            g = torch.Generator(device="cuda").manual_seed(L)
            n = B * C * L

            def place(shape, dtype=dt, off=3):
                size = int(np.prod(shape))
                whole = torch.full((size + 16,), 7.0, device="cuda", dtype=dtype)
                return whole, whole[off:off + size].view(shape)

            ins = [torch.randn(n + 1, generator=g, device="cuda").to(dt)[1:].view(B, C, L) for _ in range(4)]
            la = (-torch.rand(n + 1, generator=g, device="cuda")).to(dt)[1:].view(B, C, L)
            D = torch.randn(C, generator=g, device="cuda").to(dt)
            x1, x2, v, gy = ins
            log(f"[scan] views {dt} {(B, C, L)}")
            y0, last0, st0 = H.scan(x1, x2, v, la, D, return_last=True, return_states=True)
            g0 = H.scan_backward(x1, x2, v, la, D, st0, gy, return_gh0=True)
            outs = [place((B, C, L)), place((B, C), torch.float32), place(H.scan_states_shape((B, C, L)), torch.float32)]
            H.PreparedScan(outs[0][1], x1, x2, v, la, D, h_last=outs[1][1], states=outs[2][1])()
            grads = [place((B, C, L)) for _ in range(4)] + [place((C,)), place((B, C), torch.float32)]
            H.PreparedScanBackward(*[t for _, t in grads], x1, x2, v, la, D, outs[2][1], gy)()
            torch.cuda.synchronize()
            for (whole, t), want in zip(outs + grads, (y0, last0, st0) + g0):
                assert torch.equal(t, want)
                assert torch.all(whole[:3] == 7) and torch.all(whole[3 + t.numel():] == 7)


def test_long_linked_rows_are_their_chunks():
    """More segments than one look takes in, in both orders of the rows: what calls on 16384 positions at a time give,
    whose states are handed on (fp32 roundings of the joins apart)."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    for R, L in ((2, 300001), (70, 300001)):
        g = torch.Generator(device="cuda").manual_seed(R)
        x1, x2, v, gy = (torch.randn(1, R, L, generator=g, device="cuda") for _ in range(4))
        la = -0.002 * torch.rand(1, R, L, generator=g, device="cuda")
        D, h0 = torch.randn(R, generator=g, device="cuda"), torch.randn(1, R, generator=g, device="cuda")
        gh = torch.randn(1, R, generator=g, device="cuda")
        log(f"[scan] linked rows {(R, L)}")
        y, last, st = H.scan(x1, x2, v, la, D, h0=h0, return_last=True, return_states=True)
        grads = H.scan_backward(x1, x2, v, la, D, st, gy, gh_last=gh, return_gh0=True)
        h, parts = h0, []
        for a in range(0, L, 16384):
            cut = [t[:, :, a:a + 16384].contiguous() for t in (x1, x2, v, la)]
            yc, h, sc = H.scan(*cut, D, h0=h, return_last=True, return_states=True)
            parts.append((cut, yc, sc))
        c, back = gh, []
        for i, a in reversed(list(enumerate(range(0, L, 16384)))):
            *gc, c = H.scan_backward(*parts[i][0], D, parts[i][2], gy[:, :, a:a + 16384].contiguous(), gh_last=c, return_gh0=True)
            back.insert(0, gc)
        torch.cuda.synchronize()
        for got, want in [(y, torch.cat([p[1] for p in parts], 2)), (last, h), (grads[5], c)] + [
                (grads[i], torch.cat([b[i] for b in back], 2)) for i in range(4)]:
            assert float((got - want).norm() / want.norm()) < 2e-6  # some sixteen roundings of 2^-24 against each other


def test_two_streams_at_once():
    """Split calls that run at the same time, each on its own workspace."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    x1, x2, v, gy = (torch.randn(1, 40, 60000, device="cuda") for _ in range(4))
    la, D = -torch.rand(1, 40, 60000, device="cuda") / 100, torch.randn(40, device="cuda")
    want = H.scan(x1, x2, v, la, D, return_states=True)
    gw = H.scan_backward(x1, x2, v, la, D, want[2], gy)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(5):
                f = H.scan(x1, x2, v, la, D, return_states=True)
                b = H.scan_backward(x1, x2, v, la, D, f[2], gy)
            got.append((f[0], f[2]) + b)
    torch.cuda.synchronize()
    for one in got:
        for p, q in zip(one, (want[0], want[2]) + gw):
            assert torch.equal(p, q)


def test_captured_and_replayed():
    """Forward, backward and steps in one graph, replayed with other work between: each replay as the eager calls."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    for B, C, L in ((2, 8, 100), (1, 3, 20000)):
        g = torch.Generator(device="cuda").manual_seed(L)
        x1, x2, v, gy = (torch.randn(B, C, L, generator=g, device="cuda") for _ in range(4))
        la, D = -torch.rand(B, C, L, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
        state0 = torch.randn(B, C, generator=g, device="cuda")
        state = state0.clone()
        tok = [t[:, :, 0].contiguous() for t in (x1, x2, v, la)]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        log(f"[scan] graph {(B, C, L)}")
        with torch.cuda.stream(s):
            H.scan(x1, x2, v, la, D)  # loads the code before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, last, st = H.scan(x1, x2, v, la, D, return_last=True, return_states=True)
            grads = H.scan_backward(x1, x2, v, la, D, st, gy)
            H.scan_step(*tok, D, state)
            H.scan_step(*tok, D, state)
        for i in range(4):
            for t in (x1, v, gy):
                t.copy_(torch.randn(B, C, L, generator=g, device="cuda"))
            state.copy_(state0)
            graph.replay()
            torch.cuda.synchronize()
            ye, laste, ste = H.scan(x1, x2, v, la, D, return_last=True, return_states=True)
            ge = H.scan_backward(x1, x2, v, la, D, ste, gy)
            se = state0.clone()
            H.scan_step(*tok, D, se)
            H.scan_step(*tok, D, se)
            torch.cuda.synchronize()
            for a, b in zip((y, last, st, state) + grads, (ye, laste, ste, se) + ge):
                assert torch.equal(a, b), i


def test_side_stream_and_repeats():
    import torch
    from paper_2607_19378_amd import hyenand as H
    x1, x2, v, gy = (torch.randn(1, 7, 33000, device="cuda") for _ in range(4))
    la, D = -torch.rand(1, 7, 33000, device="cuda") / 100, torch.randn(7, device="cuda")
    want = H.scan(x1, x2, v, la, D, return_states=True)
    gw = H.scan_backward(x1, x2, v, la, D, want[2], gy)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = H.scan(x1, x2, v, la, D, return_states=True, stream=s)
    gg = H.scan_backward(x1, x2, v, la, D, got[2], gy, stream=s)
    s.synchronize()
    for a, b in zip((want[0], want[2]) + gw, (got[0], got[2]) + gg):
        assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    """Rows that begin and end behind 2^31 elements give what they give alone."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    L = (1 << 29) + 4099
    C = 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1, C, L, generator=g, device="cuda", dtype=torch.bfloat16)
    la = torch.full((1, C, L), -0.001, device="cuda", dtype=torch.bfloat16)
    D = torch.ones(C, device="cuda", dtype=torch.bfloat16)
    log("[scan] more than 2^31 elements")
    y, last, st = H.scan(x, x, x, la, D, return_last=True, return_states=True)
    one = x[:, C - 1:].clone()
    y1, last1, st1 = H.scan(one, one, one, la[:, :1].clone(), D[:1].clone(), return_last=True, return_states=True)
    torch.cuda.synchronize()
    tail = slice(L - (1 << 20), L)
    # one row alone may be split elsewhere: the roundings of its sums differ
    assert torch.allclose(last[:, C - 1:], last1, rtol=1e-4)
    assert float((y[:, C - 1:, tail].float() - y1[:, :, tail].float()).norm() / y1[:, :, tail].float().norm()) < 4e-3
    g1 = H.scan_backward(x, x, x, la, D, st, x, return_gh0=True)
    g2 = H.scan_backward(one, one, one, la[:, :1].clone(), D[:1].clone(), st1, one, return_gh0=True)
    torch.cuda.synchronize()
    for i in range(4):
        a, b = g1[i][:, C - 1:, tail].float(), g2[i][:, :, tail].float()
        assert float((a - b).norm() / b.norm()) < 4e-3, i


def test_many_channels():
    """More channels than a launch has workgroups for, of one position and two samples: gD is a sum of two products."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    B, C = 2, (1 << 24) + 3
    log("[scan] 2^24 channels")
    x1, x2, v, la, gy = (torch.randn(B, C, 1, device="cuda") for _ in range(5))
    D = torch.randn(C, device="cuda")
    y, _, states = H.scan(x1, x2, v, la, D, return_states=True)
    gx1, gx2, gv, gla, gD = H.scan_backward(x1, x2, v, la, D, states, gy)[:5]
    u, gz = x1.double() * v, gy.double() * x2
    # one product of three factors and a sum of two terms: four roundings of 2^-24 of the terms' magnitudes
    for got, ref, mag in ((gD, (gz * u).sum((0, 2)), (gz * u).abs().sum((0, 2))),
                          (gx1, gz * v * (1 + D.double()[:, None]), (gz * v).abs() * (1 + D.double().abs()[:, None])),
                          (gx2, gy * u * (1 + D.double()[:, None]), (gy * u).abs() * (1 + D.double().abs()[:, None]))):
        assert torch.all((got.double() - ref).abs() <= 6 * 2.0 ** -24 * mag + 1e-37)
    assert torch.all(gla == 0)


def test_one_row_of_very_many_segments():
    """A row of 2^33 positions: what its parts give from the states kept before them, and a sum over the whole of it."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    L, part, edge = (1 << 33) + 4099, 1 << 17, 1 << 14
    if torch.cuda.mem_get_info()[0] < 160e9:
        pytest.skip("needs 160 GB of GPU memory")
    log("[scan] a row of 2^33 positions")
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(1, 1, L, generator=g, device="cuda", dtype=torch.bfloat16)
    la, D = torch.full_like(x, -0.01), torch.ones(1, device="cuda", dtype=torch.bfloat16)
    y, last, st = H.scan(x, x, x, la, D, return_last=True, return_states=True)
    grads = H.scan_backward(x, x, x, la, D, st, x)
    torch.cuda.synchronize()
    total = sum(float(x[..., i:i + (1 << 28)].double().pow(4).sum()) for i in range(0, L, 1 << 28))
    # x2 is x and gy is x: gz u = x^4; half a step of bf16, and eight products and sums a lane before 64 bits
    assert abs(float(grads[4]) - total) <= (2.0 ** -8 + 16 * 2.0 ** -24) * total
    for a in (0, 1 << 20, 1 << 31, (1 << 32) - (1 << 16), (1 << 33) - (1 << 18), L - part):
        a = a // 512 * 512
        cut = slice(a, L if L - a < part + 512 else a + part)  # the last one to the end
        one, decay = x[..., cut].contiguous(), la[..., cut].contiguous()
        yc, lc, sc = H.scan(one, one, one, decay, D, h0=st[..., a // 512].contiguous(), return_last=True, return_states=True)
        gc = H.scan_backward(one, one, one, decay, D, sc, one)
        torch.cuda.synchronize()
        # the part's sums are joined elsewhere: fp32 roundings, and a step of bf16 where they cross a border
        assert torch.allclose(sc, st[..., a // 512:a // 512 + sc.shape[-1]], rtol=1e-4, atol=1e-4)
        assert float((yc.float() - y[..., cut].float()).norm() / yc.float().norm()) < 4e-3
        # what comes from behind the part has decayed by exp(-163) before its last 2^14 positions
        inner = slice(0, one.shape[-1] if cut.stop == L else one.shape[-1] - edge)
        for p, q in zip(gc[:4], grads[:4]):
            p, q = p[..., inner].float(), q[..., cut][..., inner].float()
            assert float((p - q).norm() / p.norm()) < 4e-3
    assert torch.allclose(last, lc, rtol=1e-4)


@pytest.mark.parametrize("B,C,N", [(2047, 3, 1), (2049, 300, 2), (5000, 5, 7), (5000, 2, 3000), (65535, 3, 1)])
def test_slots_named_many_times(B, C, N):
    """Rows of one state all over a batch, next to each other and far apart: each state is a sequence of the recurrence, and
    the largest batch on one state takes no second of the GPU's time."""
    import torch
    from paper_2607_19378_amd import hyenand as H
    rng = np.random.default_rng(B + N)
    x1, x2, v = (rng.standard_normal((B, C)).astype(np.float32) for _ in range(3))
    la, D = -rng.uniform(0.5, 1, (B, C)).astype(np.float32), rng.standard_normal(C).astype(np.float32)
    slots, state = rng.integers(0, N, B), rng.standard_normal((N, C)).astype(np.float32)
    if N > 2:
        slots[slots == 1] = N + 4  # idle rows among the others
    dev = [on_gpu(t) for t in (x1, x2, v, la, D, state)]
    pool, where = dev[5], on_gpu(slots)
    log(f"[scan] slots named many times B={B} C={C} N={N}")
    H.scan_step(*dev[:5], pool.clone(), where)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    y = H.scan_step(*dev[:5], pool, where)
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) < 1000
    y, pool = from_device(y), from_device(pool)
    assert np.all(y[slots >= N] == 0)
    for s in range(N):
        rows = np.flatnonzero(slots == s)
        if rows.size == 0:
            assert np.array_equal(pool[s], state[s])
            continue
        args = [np.ascontiguousarray(t[rows].T)[None].astype(np.float64) for t in (x1, x2, v, la)] + [D.astype(np.float64)]
        ref, mag = R.scan(*args, h0=state[s:s + 1]), R.scan_magnitudes(*args, h0=state[s:s + 1])
        # two roundings and an exponential's a step, each older one by exp(-1/2) less: 3 / (1 - exp(-1/2)), and four of y
        tol = (3 / (1 - np.exp(-0.5)) + 4) * 2.0 ** -23
        assert np.all(np.abs(y[rows].T - ref["y"][0]) <= tol * mag["y"][0] + 1e-37), s
        assert np.all(np.abs(pool[s] - ref["h_last"][0]) <= tol * mag["h_last"][0] + 1e-37), s
