"""Facts of arithmetic that the sampling kernel's bins rest on."""
from decimal import Decimal, localcontext

import numpy as np

SPAN, BINS = 48, 4096


def test_no_float_lies_at_a_bin_edge():
    """Min-p, a float, keeps whole bins but one: its logarithm is further from every edge (but 1's, which is exact) than the
    roundings of a token's place on the scale (2^-50 of up to 4096 bins) and of its own."""
    nearest = 1.0
    with localcontext() as ctx:
        ctx.prec = 30
        for n in range(1, BINS):
            edge = Decimal(-n * SPAN) / BINS
            f = np.float32(float(edge.exp()))
            for g in (np.nextafter(f, np.float32(0)), f, np.nextafter(f, np.float32(2))):
                nearest = min(nearest, float(abs(Decimal(float(g)).ln() - edge)) * BINS / SPAN)
    assert 1.7e-10 < nearest < 1.8e-10 and nearest > 40 * 2.0 ** -50 * BINS
