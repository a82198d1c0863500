"""Further arguments of the calls between layers that are refused before anything touches a device (no GPU)."""
import pytest

from paper_2410_03348_amd import binding as dol

F32, BF16 = 0, 1


def at(k, rows, cols, dtype=F32, ld=None, more=0):
    """A matrix at the k-th block of memory (of 2^16 bytes), `more` bytes behind its beginning."""
    return dtype, rows, cols, cols if ld is None else ld, 65536 * k + more


def test_residual_norm_backward_from_h_refuses():
    h, u, gh, gy, gx, gu = (at(k, 8, 16) for k in range(1, 7))
    ok = [h, u, 1, None, None, 1.0, None, 65536 * 7, 65536 * 8, gh, gy, gx, gu, None, None, None, None, 0, 0]
    for k, value, why in ((0, None, "h is NULL"), (0, at(1, 7, 16), "h is 7 x 16"), (0, at(1, 8, 16, BF16), "h is of another type"), (7, None, "rstd_u"), (8, None, "rstd_h"),
                          (11, gu, "the same"), (13, 65536 * 9, "workspace"), (1, None, "u is NULL")):
        a = list(ok)
        a[k] = value
        with pytest.raises(dol.DolError, match=why):
            dol._native.residual_norm_backward_from_h(*a)


def over(m, ld=None, more=0):
    """The same matrix with other distances of its rows, or from another byte on."""
    return m[0], m[1], m[2], m[3] if ld is None else ld, m[4] + more


# rows of 40 numbers of 4 bytes
SHIFTS = [dict(more=4), dict(more=-4), dict(more=160), dict(more=160 * 7), dict(more=-160 * 7 - 156), dict(ld=41), dict(ld=80), dict(more=80, ld=80)]
APART = [dict(more=160 * 8), dict(more=-160 * 8), dict(more=4096)]


def refused(call, args, k, value, why):
    a = list(args)
    a[k] = value
    with pytest.raises(dol.DolError, match=why):
        call(*a)


@pytest.mark.parametrize("shift", SHIFTS)
def test_linear_refuses_results_over_parts_of_operands(shift):
    x, w, r, y, z = at(1, 8, 40), at(2, 40, 40), at(3, 8, 40), at(4, 8, 40), at(5, 8, 40)
    bias = 65536 * 6
    args = [x, w, bias, 2, r, y, z, None, None, 0, 0]
    for m in (x, z, w):
        refused(dol._native.linear, args, 5, over((F32, 8, 40, 40, m[4]), **shift), "y is x|z is x")
    for m in (x, r, w):
        refused(dol._native.linear, args, 6, over((F32, 8, 40, 40, m[4]), **shift), "z is x")
    refused(dol._native.linear, args, 5, over(r, **shift), "y lies over the residual")
    for k in (5, 6):
        refused(dol._native.linear, args, k, at(6, 8, 40, more=-1276), "y is x|z is x")          # the last number over the first of the bias
    g, gx, gw = at(7, 8, 40), at(8, 8, 40), at(9, 40, 40)
    back = [x, w, 2, z, None, g, gx, gw, bias, None, 0, 0]
    for m in (x, w, z, g):
        refused(dol._native.linear_backward, back, 6, over((F32, 8, 40, 40, m[4]), **shift), "grad_x or grad_weight is x")
        refused(dol._native.linear_backward, back, 8, m[4] + 4, "grad_bias lies over")
    for m in (w, x):
        refused(dol._native.linear_backward, back, 7, over((F32, 40, 40, 40, m[4]), **shift), "grad_x or grad_weight is x")
    refused(dol._native.linear_backward, back, 6, over((F32, 8, 40, 40, gw[4]), **shift), "lie over each other")
    for k in (6, 7):
        refused(dol._native.linear_backward, back, 8, back[k][4] + 8, "lie over each other")


def test_linear_refuses_rests_over_operands():
    x, w, r, y, z = (at(k, 8, 40, BF16) for k in range(1, 6))
    w = at(2, 40, 40, BF16)
    for m in (x, w, r, y, z):
        for more in (0, 2, -638):
            refused(dol._native.linear, [x, w, None, 2, r, y, z, None, None, 0, 0], 7, m[4] + more, "is x|z_rest lies over")
    for m in (at(6, 8, 40, BF16), at(7, 40, 40, BF16)):
        back = [x, w, 2, z, m[4] + 2, y, at(6, 8, 40, BF16), at(7, 40, 40, BF16), None, None, 0, 0]
        refused(dol._native.linear_backward, back, 0, x, "grad_x or grad_weight")


@pytest.mark.parametrize("shift", SHIFTS)
def test_residual_norm_refuses_results_over_parts_of_operands(shift):
    x, u, gate, h, y = (at(k, 8, 40) for k in range(1, 6))
    vec = [65536 * k for k in range(6, 10)]
    args = [x, u, 1, vec[0], gate, 1.0, vec[1], 1e-6, h, y, vec[2], vec[3], 0]
    call = dol._native.residual_norm
    for k in (8, 9):
        for m in (x, u):
            refused(call, args, k, over(m, **shift), "not each row over its own")
        refused(call, args, k, over(gate, **shift), "the same")
        for v in vec:
            refused(call, args, k, over(at(0, 8, 40), more=v - 1276), "vector of the call")
    refused(call, args, 8, over(y, **shift), "the same")
    for k in (10, 11):
        for m in (x, u, gate):
            refused(call, args, k, m[4] + 4, "rstd_u or rstd_h lies over")
    refused(call, args, 11, vec[2] + 28, "rstd_u and rstd_h lie over")
    gh, gy, gx, gu, gg = (at(k, 8, 40) for k in range(11, 16))
    sums = [65536 * 16, 65536 * 17]
    back = [x, u, 1, vec[0], gate, 1.0, vec[1], vec[2], vec[3], gh, gy, gx, gu, sums[0], gg, sums[1], None, 0, 0]
    for call in (dol._native.residual_norm_backward, dol._native.residual_norm_backward_from_h):
        for k in (11, 12):
            for m in (x, u, gh, gy):
                refused(call, back, k, over(m, **shift), "not each row over its own")
            refused(call, back, k, over(gate, **shift), "the same")
            for v in vec + sums:
                refused(call, back, k, over(at(0, 8, 40), more=v - 1276), "vector of the call")
        refused(call, back, 11, over(gu, **shift), "the same")
        for m in (x, u, gate, gh, gy, gx, gu):
            refused(call, back, 14, over(m, **shift), "grad_gate is")
        refused(call, back, 15, sums[0] + 156, "lie over each other")
        for k in (13, 15):
            for m in (x, u, gate, gh, gy):
                refused(call, back, k, m[4] + 4, "grad_gamma_u or grad_gamma_y lies over")


@pytest.mark.parametrize("shift", APART)
def test_results_beside_operands_are_taken(shift):
    """What lies behind or before an operand, or in its place; refused only for want of a workspace."""
    x, u, gate = (at(k, 8, 40) for k in range(1, 4))
    gh, gy, gx, gu, gg = (at(k, 8, 40) for k in range(11, 16))
    for call in (dol._native.residual_norm_backward, dol._native.residual_norm_backward_from_h):
        back = [x, u, 1, None, gate, 1.0, None, 65536 * 20, 65536 * 21, gh, gy, gx, gu, None, gg, None, None, 0, 0]
        for k in (11, 12):
            for m in (x, u, gh, gy):
                refused(call, back, k, m, "workspace")
                refused(call, back, k, over(m, **shift), "workspace")
    x, w, r = at(1, 300, 40), at(10, 40, 40), at(20, 300, 40)
    for y in (r, over(r, more=160 * 300), over(r, more=-160 * 300)):
        refused(dol._native.linear, [x, w, None, 2, r, y, at(30, 300, 40), None, None, 0, 0], 3, 2, "workspace")


@pytest.mark.parametrize("dtype,size", [(F32, 4), (BF16, 2)])
def test_columns_of_one_buffer_side_by_side_are_taken(dtype, size):
    """x, what is added and the results as columns 0 .. 39, 40 .. 79 and so on of rows of 240 numbers; refused where they share a column."""
    def cols(k, rows=300, first=0):
        return dtype, rows, 40, 240, 65536 + (40 * k + first) * size

    w = at(200, 40, 40, dtype)
    args = [cols(0), w, None, 2, cols(1), cols(2), cols(3), None, None, 0, 0]
    refused(dol._native.linear, args, 3, 2, "workspace")
    refused(dol._native.linear, args, 5, cols(2, first=1), "y is x")
    refused(dol._native.linear, args, 5, cols(0, first=39), "y is x")
    refused(dol._native.linear, args, 6, cols(5, first=1), "z is x")             # around the row's end into the next one's first column
    refused(dol._native.linear, args, 6, (dtype, 300, 40, 480, cols(1, first=39)[4]), "is x")
    refused(dol._native.linear, args, 6, (dtype, 300, 40, 480, cols(4)[4]), "workspace")
    back = [cols(0), cols(1), 1, None, None, 1.0, None, 65536 * 200, 65536 * 210, cols(2), cols(3), cols(4), cols(5), None, None, None, None, 0, 0]
    refused(dol._native.residual_norm_backward, back, 2, 1, "workspace")
    refused(dol._native.residual_norm_backward, back, 11, cols(2), "workspace")
    refused(dol._native.residual_norm_backward, back, 11, cols(2, first=1), "not each row over its own")
    refused(dol._native.residual_norm_backward, back, 11, cols(4, first=1), "the same")


def test_one_row_has_no_distance():
    r, y = at(3, 1, 40, ld=40), at(3, 1, 40, ld=90)
    gh, gx, gu = at(4, 1, 40), at(4, 1, 40, ld=1000), at(5, 1, 40)
    refused(dol._native.residual_norm_backward, [r, y, 1, None, None, 1.0, None, 65536 * 20, 65536 * 21, gh, gh, gx, gu, None, None, None, None, 0, 0], 2, 1, "workspace")
