"""Further arguments of the calls between layers that are refused before anything touches a device (no GPU)."""
import pytest

from paper_2410_03348_amd import binding as dol

F32, BF16 = 0, 1


def at(k, rows, cols, dtype=F32, ld=None):
    return dtype, rows, cols, cols if ld is None else ld, 4096 * k


def test_residual_norm_backward_from_h_refuses():
    h, u, gh, gy, gx, gu = (at(k, 8, 16) for k in range(1, 7))
    ok = [h, u, 1, None, None, 1.0, None, 4096, 4096, gh, gy, gx, gu, None, None, None, None, 0, 0]
    for k, value, why in ((0, None, "h is NULL"), (0, at(1, 7, 16), "h is 7 x 16"), (0, at(1, 8, 16, BF16), "h is of another type"), (7, None, "rstd_u"), (8, None, "rstd_h"),
                          (11, gu, "the same"), (13, 4096, "workspace"), (1, None, "u is NULL")):
        a = list(ok)
        a[k] = value
        with pytest.raises(dol.DolError, match=why):
            dol._native.residual_norm_backward_from_h(*a)
