"""The plans that the recurrence chooses, read from the built library, and calls that reach each of them."""
import ctypes

from paper_2607_19378_amd import hyenand as H


class _ScanShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("lanes", "waves", "nseg")]


def scan_plan(rows, L):
    """(lanes of a row, wavefronts of a row, segments of a row) of scan_shape."""
    fn = H.lib()._ZN7hyenand10scan_shapeEll
    fn.argtypes, fn.restype = [ctypes.c_int64] * 2, _ScanShape
    s = fn(rows, L)
    return s.lanes, s.waves, s.nseg


# (B, C, L) -> wavefronts of a row, whether it is split; all of more than one turn of a row's wavefronts, the last turn
# whole, with one tile, and with all but one
SCAN = [((8, 515, 600), 1, False), ((2, 2051, 1030), 1, False), ((1, 4099, 1537), 1, False),
        ((2, 515, 2100), 4, False), ((1, 1027, 4700), 4, False), ((1, 1030, 4096), 4, False),
        ((1, 200, 4200), 8, False), ((2, 100, 8200), 8, False),
        ((1, 1, 16385), 8, True), ((1, 2, 20479), 8, True), ((1, 191, 16900), 8, True)]
