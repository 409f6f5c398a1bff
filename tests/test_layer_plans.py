"""The GPU tests of the recurrence and the norms reach the plans that they are meant for: a rule that moves fails here,
without a GPU."""
import re

import numpy as np
import pytest

import layer_plans as plans
import layer_ref as R


@pytest.mark.parametrize("shape,waves,split", plans.SCAN)
def test_recurrence(shape, waves, split):
    B, C, L = shape
    lanes, w, nseg = plans.scan_plan(B * C, L)
    assert (lanes, w, nseg > 1) == (64, waves, split)
    assert -(-L // 512) > w  # more than one turn of the wavefronts, or more than one segment


@pytest.mark.parametrize("shape,dtype,forward,backward", plans.NORM)
def test_norms(shape, dtype, forward, backward):
    f, b = (plans.norm_plan(*shape, dtype, way) for way in (False, True))
    assert (f[2], b[2]) == (forward, backward)
    points = 8 if dtype == "bf16" else 4
    assert f[0] == b[0] == (points if shape[2] >= points else 1)


def test_norms_reach_every_kind():
    """Channels a thread, points a lane, whole and ragged rows: all that a dense set of shapes asks for are listed."""
    def kinds(shapes):
        return {(dtype, way, p[0] > 1, p[2], p[0] > 1 and p[2] > 0 and s[2] % p[0] > 0)
                for s, dtype in shapes for way in (False, True) for p in [plans.norm_plan(*s, dtype, way)]}

    dense = [((B, C, P), dtype) for dtype in ("f32", "bf16") for B in (1, 64, 3000) for P in (1, 2, 3, 5, 7, 8, 9, 40, 513, 4096)
             for C in [1, 9, 60] + [2 ** i + d for i in range(6, 15) for d in (-3, 0, 3)]]
    mine = {k[1:] for k in kinds([(s, dtype) for s, dtype, _, _ in plans.NORM])}
    assert {k[1:] for k in kinds(dense)} == mine


def test_masks_of_whole_tensors():
    """The masks in arrays are those of the reference, drawn one after another."""
    for B, C, P in ((2, 3, 1), (1, 5, 7), (2, 2, 29)):
        assert np.array_equal(plans.keep_factors(B, C, P, 0.3, -5, 1 << 40), R.keep_factors(B, C, P, 0.3, -5, 1 << 40))


def test_long_rows_are_split():
    """Few rows of more than 16384 positions are split whatever their length, as long as five tensors of two bytes fit in
    288 GB and a launch has fewer than 2^32 work-items."""
    for rows in (1, 2, 3, 17, 64, 100, 191):
        for L in [16385] + [2 ** i + d for i in range(15, 41) for d in (-1, 0, 1)]:
            lanes, waves, nseg = plans.scan_plan(rows, L)
            if rows * L * 10 <= 288e9:
                assert nseg == -(-L // 4096), (rows, L)
            assert rows * nseg * 64 * waves < 1 << 32, (rows, L)


def test_every_kernel_of_the_norms_is_chosen():
    """The kernels in the library, by type, points a lane and channels a thread, are those that the listed calls choose."""
    with open(plans.H.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"1[23]norm_(forward|backward)I([ft])Li(\d)ELi(\d)ENS", f.read()))
    built = {(way == b"backward", "bf16" if t == b"t" else "f32", int(v), int(k)) for way, t, v, k in names}
    chosen = set()
    for dtype in ("f32", "bf16"):
        for way in (False, True):
            for shape in [s for s, _, _, _ in plans.NORM]:
                V, _, K, _ = plans.norm_plan(*shape, dtype, way)
                if K:
                    chosen.add((way, dtype, V, K))
    assert built == chosen


def test_wide_samples_of_one_tile_go_to_several_xcds():
    """An XCD's turn is at most 256 KB of a tensor, or one sample; small ones stay together."""
    for B, C, size, run in ((32, 1024, 2, 32), (32, 4096, 2, 32), (32, 8192, 2, 16), (64, 6000, 2, 16), (64, 2048, 4, 32),
                            (32, 4096, 4, 16), (16, 8192, 4, 8), (4, 1 << 20, 2, 1), (1, 1 << 25, 4, 1)):
        assert plans.norm_run(C * size, B, 1, 0, False) == run
        assert plans.norm_run(C * size, B, 1, 0, True) == 1
    assert plans.norm_run(1 << 24, 1 << 14, 64, 2, False) == plans.norm_run(1 << 24, 1 << 14, 64, 2, True) == 8
    assert plans.norm_run(1 << 21, 8, 8, 3, True) == 1  # every XCD has a tile
