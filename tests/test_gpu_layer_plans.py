"""The recurrence and the norms on every way that a call is spread over the chip (layer_plans), against the plain 64-bit
references, with the tolerances of test_gpu_scan and test_gpu_block_norm."""
import numpy as np
import pytest

import layer_plans as plans
import layer_ref as R
import test_gpu_block_norm as N
import test_gpu_scan as S

from gpu_util import from_device, log, to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [s for s, _, _ in plans.SCAN])
def test_recurrence(shape, dtype):
    B, C, L = shape
    S.run_case(B, C, L, dtype, L, packed=B == 2, lengths=B > 2, carry=True)


@pytest.mark.parametrize("shape", [(3, 1400, 1100), (2, 600, 2600)])
def test_recurrence_of_ragged_samples(shape):
    """A sample that ends at once, one that ends at the last position and one between, with starts."""
    S.run_case(*shape, "f32", 3, packed=True, lengths=True, carry=True)


# everything; no gate; what is looked up as the kernel runs: no next norm, no branch, no gradient of the stream
VARIANTS = [((), 0.0), ((), 0.2), (("gate",), 0.0), (("gate", "scale"), 0.2), (("w_pre", "gn"), 0.3),
            (("z", "gate", "w_post", "scale"), 0.0), (("gx_out",), 0.4)]


def check_norm(store, val, B, C, P, dtype, without, p, eps=(1e-6, 1e-5)):
    import torch
    from paper_2607_19378_amd import hyenand as H
    log(f"[norm] plans B={B} C={C} P={P} {dtype} without={without} p={p}")
    dev = {n: None if n in without else to_device(x, dtype) for n, x in store.items()}
    val = {n: None if n in without else x for n, x in val.items()}
    rng = torch.tensor([N.SEED, N.OFFSET], device="cuda") if p else None
    keep = plans.keep_factors(B, C, P, p, N.SEED, N.OFFSET) if p else None
    head, units = N.NAMES[:6], N.roundings(C)
    x_out, n = H.block_norm(*[dev[k] for k in head], *eps, p, rng)
    rx, rn = R.block_norm(*[val[k] for k in head], *eps, keep)
    mag = np.abs(rx) if val["z"] is None else np.abs(val["x"]) + np.abs(rx - val["x"])
    if val["z"] is not None:
        N.close("x_out", from_device(x_out), rx, mag, units, dtype)
    if val["w_pre"] is not None:
        q = R.inverse_rms(rx, eps[1])
        rms_mag = np.sqrt((mag * mag).mean(1, keepdims=True)) * q
        N.close("n", from_device(n), rn, np.abs(val["w_pre"])[None, :, None] * q * (mag + np.abs(rx) * rms_mag), units, dtype)
    kw = {k: val[k] for k in N.NAMES[1:]}
    ref = R.block_norm_backward(from_device(x_out), **kw, eps_post=eps[0], eps_pre=eps[1], keep=keep)
    got = H.block_norm_backward(x_out, *[dev[k] for k in N.NAMES[1:6]], dev["gx_out"], dev["gn"], *eps, p, rng)
    for name, t in zip(("gx", "gz", "ggate", "gw_post", "gscale", "gw_pre"), got):
        assert (t is None) == (name not in ref), name
        if t is not None:  # sums of weights: 8 points a lane of every 1024th tile, the lanes, the rest in 64 bits
            more = 0 if t.dim() > 1 else 8 * (1 + B * P / 8 / 1024) + 3
            N.close(name, from_device(t), *ref[name], 2 * units + more, dtype)


@pytest.mark.parametrize("shape,dtype", [(s, t) for s, t, _, _ in plans.NORM])
def test_norms(shape, dtype):
    store, val = N.make(*shape, dtype, sum(shape))
    for without, p in VARIANTS[:5 if np.prod(shape) > 1 << 20 else 7]:
        check_norm(store, val, *shape, dtype, without, p)
