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
