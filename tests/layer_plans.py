"""The plans that the recurrence and the norms choose, read from the built library, and calls that reach each of them."""
import ctypes

import numpy as np

import layer_ref as R
from paper_2607_19378_amd import hyenand as H


class _ScanShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("lanes", "waves", "nseg")]


class _NormShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("V", "lp", "K", "NT")]


def scan_plan(rows, L):
    """(lanes of a row, wavefronts of a row, segments of a row) of scan_shape."""
    fn = H.lib()._ZN7hyenand10scan_shapeEll
    fn.argtypes, fn.restype = [ctypes.c_int64] * 2, _ScanShape
    s = fn(rows, L)
    return s.lanes, s.waves, s.nseg


def norm_plan(B, C, P, dtype, backward):
    """(points a lane, log2 of the lanes over points, channels a thread or 0, threads) of norm_shape."""
    fn = H.lib()._ZN7hyenand10norm_shapeElllbb
    fn.argtypes, fn.restype = [ctypes.c_int64] * 3 + [ctypes.c_bool] * 2, _NormShape
    s = fn(C, P, B, dtype == "bf16", backward)
    return s.V, s.lp, s.K, s.NT


# (B, C, L) -> wavefronts of a row, whether it is split; all of more than one turn of a row's wavefronts, the last turn
# whole, with one tile, and with all but one
SCAN = [((8, 515, 600), 1, False), ((2, 2051, 1030), 1, False), ((1, 4099, 1537), 1, False),
        ((2, 515, 2100), 4, False), ((1, 1027, 4700), 4, False), ((1, 1030, 4096), 4, False),
        ((1, 200, 4200), 8, False), ((2, 100, 8200), 8, False),
        ((1, 1, 16385), 8, True), ((1, 2, 20479), 8, True), ((1, 191, 16900), 8, True)]

# (B, C, P), dtype -> channels a thread of the forward, of the backward (0: its tile is read again); rows of a whole
# number of a lane's points, then others
NORM = [((2, 60, 96), "f32", 1, 1), ((2, 60, 97), "f32", 1, 1), ((2, 60, 96), "bf16", 1, 1), ((2, 60, 99), "bf16", 1, 1),
        ((3, 200, 76), "f32", 2, 2), ((3, 200, 77), "f32", 2, 2), ((3, 200, 80), "bf16", 2, 2), ((3, 200, 77), "bf16", 2, 2),
        ((4, 130, 4096), "f32", 4, 2), ((4, 130, 4095), "f32", 4, 2), ((2, 130, 16384), "bf16", 4, 2),
        ((2, 130, 16381), "bf16", 4, 2), ((8, 260, 1024), "f32", 4, 2), ((8, 257, 2050), "bf16", 4, 2),
        ((8, 520, 512), "f32", 4, 2), ((8, 520, 1022), "bf16", 4, 2),
        ((2, 2048, 40), "f32", 8, 0), ((2, 2048, 43), "f32", 8, 0), ((1, 4000, 40), "bf16", 8, 0), ((1, 4000, 43), "bf16", 8, 0),
        ((1, 4500, 12), "f32", 0, 0), ((1, 4500, 17), "bf16", 0, 0),
        # rows shorter than a lane's points: one point a lane
        ((5, 70, 1), "f32", 1, 1), ((5, 70, 2), "bf16", 1, 1), ((5, 70, 3), "f32", 1, 1), ((5, 70, 5), "bf16", 1, 1),
        ((5, 70, 7), "bf16", 1, 1), ((3, 3000, 1), "f32", 4, 4), ((3, 500, 3), "f32", 4, 4), ((3, 500, 6), "bf16", 4, 4),
        ((2100, 1000, 1), "bf16", 4, 4), ((2, 7000, 1), "bf16", 8, 0), ((2, 1700, 3), "f32", 8, 4), ((2, 9000, 1), "f32", 0, 0)]


def keep_factors(B, C, P, p, seed, offset):
    """layer_ref.keep_factors, all points at once."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    drop, groups = min(65535, int(np.floor(p * 65536 + 0.5))), -(-P // 8)
    seed, offset = seed % (1 << 64), offset % (1 << 64)
    i = np.arange(B * C * groups, dtype=np.uint64)
    c = [i & low, i >> half, np.full_like(i, offset & 0xFFFFFFFF), np.full_like(i, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(R._M[0]), c[2] * np.uint64(R._M[1])
        c = [(p1 >> half) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> half) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + R._W[0]) & 0xFFFFFFFF, (k[1] + R._W[1]) & 0xFFFFFFFF]
    bits = np.stack([w for x in c for w in (x & np.uint64(0xFFFF), x >> np.uint64(16))], -1)
    return (bits.reshape(B, C, groups * 8)[..., :P] >= drop) * (65536.0 / (65536 - drop))


def norm_run(sample_bytes, tiles, row_tiles, lp, backward):
    """Consecutive tiles of an XCD's turn, of norm_log_run."""
    fn = H.lib()._ZN7hyenand12norm_log_runElllib
    fn.argtypes, fn.restype = [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_bool], ctypes.c_uint32
    return 1 << fn(sample_bytes, tiles, row_tiles, lp, backward)
