"""The division in three steps by a block's scale (the reciprocal y rounded; q = x y rounded; r = q d - x, exact; q - r y rounded once) for
divisors that are no quotient of a bf16 maximum: the scales of normed and rotated queries and keys can have any significand."""
import ctypes as C

import numpy as np


def test_quotients_at_the_borders_between_codes():
    """Against the division itself: divisors all over the significands, those of all ones and of zeros among them, numerators within six
    units of every border between two E4M3 numbers (odd multiples of a sixteenth of a power of two, up to 31)."""
    f32, f64 = np.float32, np.float64
    d = (np.concatenate([np.arange(0, 1 << 23, 4099), np.arange(64), (1 << 23) - 1 - np.arange(64)]).astype(np.uint32) | np.uint32(0x3F800000)).view(f32)[:, None, None]
    x = ((np.arange(1, 32, 2).astype(f32)[None, :, None] * d).view(np.uint32).astype(np.int64) + np.arange(-6, 7)[None, None, :]).astype(np.uint32).view(f32)
    y = (f32(1) / d).astype(f32)
    q = (x * y).astype(f32)
    r = (q.astype(f64) * d.astype(f64) - x.astype(f64)).astype(f32)          # 48 bits less a close number of 24: exact
    got = (q.astype(f64) - r.astype(f64) * y.astype(f64)).astype(f32)
    want = (x / d).astype(f32)
    # the emulation rounds twice: what it has otherwise goes through a true multiply-add
    fmaf = C.CDLL("libm.so.6").fmaf
    fmaf.restype, fmaf.argtypes = C.c_float, [C.c_float] * 3
    other = np.argwhere(got != want)
    assert len(other) < 100
    for i, j, k in other:
        assert fmaf(-float(r[i, j, k]), float(y[i, 0, 0]), float(q[i, j, k])) == want[i, j, k], (d[i, 0, 0], x[i, j, k])
