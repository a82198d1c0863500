"""Arguments of the calls between layers and of clipping that are refused before anything touches a device (no GPU)."""
import ctypes as C

import pytest

from paper_2410_03348_amd import binding as dol

F32, BF16 = 0, 1


def tensor_list(count, dtype=(), size=(), data=()):
    h = C.c_void_p()
    n = max(count, 1)
    return dol._lib.dol_tensor_list_create(count, (C.c_int32 * n)(*dtype), (C.c_int64 * n)(*size), (C.c_void_p * n)(*data), C.byref(h)), h


@pytest.mark.parametrize("count,dtype,size,data,status,why", [
    (-1, (), (), (), 1, "negative"), (1, (7,), (3,), (4096,), 1, "type"), (1, (F32,), (-1,), (4096,), 2, "elements"), (1, (F32,), (3,), (None,), 1, "NULL"),
    (1, (F32,), (3,), (4098,), 1, "aligned"), (2, (F32, BF16), (3, 3), (4096, 4097), 1, "aligned"),
    (2, (F32, F32), (1 << 62, 1 << 62), (4096, 4096), 5, "more than"), (2, (F32, F32), ((1 << 63) - 1, 1 << 44), (4096, 4096), 5, "more than")])
def test_tensor_list_refusals(count, dtype, size, data, status, why):
    st, h = tensor_list(count, dtype, size, data)
    assert st == status and h.value is None and why in dol.last_error()


def test_tensor_list_arrays_and_handle():
    assert dol._lib.dol_tensor_list_create(1, None, None, None, C.byref(C.c_void_p())) == 1
    assert dol._lib.dol_tensor_list_create(0, None, None, None, None) == 1
    dol._lib.dol_tensor_list_destroy(None)


def test_clip_refuses_no_list():
    for call in (lambda: dol._native.grad_norm_workspace(None), lambda: dol._native.grad_norm(None, 4096, 4096, 0, 0),
                 lambda: dol._native.clip_grads(None, None, 1.0, 0.0, 4096, 4096, 4096, 0, 0)):
        with pytest.raises(dol.DolError, match="NULL"):
            call()


def test_host_tensors_are_refused_in_lists():
    torch = pytest.importorskip("torch")
    with pytest.raises(AssertionError):
        dol.TensorList([torch.zeros(3)])


def matrix(rows, cols, dtype=F32, ld=None, data=4096):
    return dtype, rows, cols, cols if ld is None else ld, data


@pytest.mark.parametrize("u,gate,why", [
    (None, None, "NULL"), (matrix(8, 16, 7), None, "type"), (matrix(8, 0), None, "columns"), (matrix(8, (1 << 24) + 1), None, "EUNSUPPORTED"),
    (matrix(8, 16, ld=15), None, "ESHAPE"), (matrix(8, 16), matrix(3, 16), "divide"), (matrix(8, 16), matrix(0, 16), "divide"),
    (matrix(8, 16), matrix(16, 16), "divide"), (matrix(8, 16), matrix(4, 15), "columns"), (matrix(8, 16), matrix(4, 16, BF16), "type"),
    (matrix(-1, 16), None, "ESHAPE")])
def test_residual_norm_refusals(u, gate, why):
    with pytest.raises(dol.DolError, match=why):
        dol._native.residual_norm_workspace(u, gate)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,gates,cols", [(1, 1, 1), (64, 0, 32), (64, 8, 4096), (1 << 20, 1 << 19, 8), (1 << 20, 1 << 10, 512), (100, 50, 40000), (1 << 20, 1 << 20, 32),
                                             ((1 << 31) - 1, 1, 4), (1 << 30, 1 << 25, 4)])
def test_residual_norm_workspace(rows, gates, cols, dtype):
    """Sums over rows leave a part to a workgroup: no more than the tensors themselves but for small ones, and as much as a row's sums where rows are read twice."""
    n = dol._native.residual_norm_workspace(matrix(rows, cols, dtype), matrix(gates, cols, dtype) if gates else None)
    assert 0 < n and n % 256 == 0 and n <= max(3 * 1024 * (cols + 64) * 4, 3 * rows * cols * 4 + rows * 8) + 4096
    assert dol._native.residual_norm_workspace(matrix(0, cols, dtype), None) == 0


@pytest.mark.parametrize("x,w,why", [
    (matrix(8, 16), matrix(20, 15), "ESHAPE"), (matrix(8, 16), matrix(20, 16, BF16), "types"), (matrix(8, 16), matrix(0, 16), "one out"),
    (matrix(8, 0), matrix(4, 0), "one out"), (matrix(8, 16, 7), matrix(4, 16), "type"), (matrix((1 << 22) + 1, 16), matrix(4, 16), "more than"),
    (matrix(8, (1 << 20) + 1), matrix(4, (1 << 20) + 1), "more than"), (matrix(8, 16, ld=15), matrix(4, 16), "ESHAPE"), (None, matrix(4, 16), "NULL")])
@pytest.mark.parametrize("backward", [0, 1])
def test_linear_refusals(x, w, why, backward):
    with pytest.raises(dol.DolError, match=why):
        dol._native.linear_workspace(x, w, backward)
    assert dol._native.linear_kernel(x, w, backward) == ""


def test_linear_refuses_unknown_activation_functions():
    for act in (-1, 4):
        with pytest.raises(dol.DolError, match="activation"):
            dol._native.linear(matrix(8, 16), matrix(4, 16), None, act, None, matrix(8, 4), None, None, None, 0, 0)
        with pytest.raises(dol.DolError, match="activation"):
            dol._native.linear_backward(matrix(8, 16), matrix(4, 16), act, None, None, matrix(8, 4), matrix(8, 16), None, None, None, 0, 0)


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width,out", [(0, 1, 1), (1, 1, 1), (1, 4096, 16384), (64, 1568, 128), (1000, 777, 1501), (8192, 4096, 4096), (1 << 22, 3, 2), (7, 1 << 20, 1), (1, 8, 1 << 22)])
def test_linear_workspace(rows, width, out, dtype, backward):
    n = dol._native.linear_workspace(matrix(rows, width, dtype), matrix(out, width, dtype), backward)
    assert 0 <= n < 1 << 36 and n % 256 == 0
    assert n == dol._native.linear_workspace(matrix(rows, width, dtype), matrix(out, width, dtype), backward)


def at(k, rows, cols):
    return matrix(rows, cols, data=4096 * k)


def test_linear_refuses_results_on_operands():
    x, w, r, y, z = at(1, 8, 4), at(2, 4, 4), at(3, 8, 4), at(4, 8, 4), at(5, 8, 4)
    for y_, z_ in ((x, z), (at(2, 8, 4), z), (z, z), (y, x), (y, at(2, 8, 4)), (y, r)):
        with pytest.raises(dol.DolError, match="y is x|z is x"):
            dol._native.linear(x, w, None, 2, r, y_, z_, None, None, 0, 0)
    g, gw = at(4, 8, 4), at(6, 4, 4)
    for gx_, gw_ in ((x, gw), (at(2, 8, 4), gw), (z, gw), (y, gw), (at(7, 8, 4), w), (at(7, 8, 4), at(1, 4, 4)), (at(6, 8, 4), gw)):
        with pytest.raises(dol.DolError, match="grad_x"):
            dol._native.linear_backward(x, w, 2, z, None, g, gx_, gw_, None, None, 0, 0)


def test_residual_norm_refuses_results_on_each_other_and_on_gates():
    x, u, gate, h, y = (at(k, 8, 16) for k in range(1, 6))
    for h_, y_ in ((h, h), (gate, y), (h, gate)):
        with pytest.raises(dol.DolError, match="the same"):
            dol._native.residual_norm(x, u, 0, None, gate, 1.0, None, 1e-6, h_, y_, None, None, 0)
    gx, gu, gg = (at(k, 8, 16) for k in range(6, 9))
    for gx_, gu_, gg_ in ((gx, gx, gg), (gate, gu, gg), (gx, gate, gg), (gx, gu, gate), (gx, gu, gx), (gx, gu, x), (gx, gu, h)):
        with pytest.raises(dol.DolError, match="the same|grad_gate is"):
            dol._native.residual_norm_backward(x, u, 0, None, gate, 1.0, None, None, 4096, h, y, gx_, gu_, None, gg_, None, None, 0, 0)
