"""Arguments of the training calls that are refused before anything touches a device, and the sizes of their workspaces (no GPU)."""
import pytest

from paper_2410_03348_amd import binding as dol

F32, BF16 = 0, 1


def matrix(rows, cols, dtype=F32, ld=None, data=4096):
    return dtype, rows, cols, cols if ld is None else ld, data


def acts(batch, points, channels, dtype=F32, data=4096):
    return dtype, batch, points, channels, points * channels, channels, data


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width,classes", [(0, 1, 1), (1, 1, 1), (64, 128, 10), (100, 100, 1000), (8192, 1024, 65535), (1 << 22, 3, 2), (7, 1 << 20, 1)])
def test_cross_entropy_workspace(rows, width, classes, dtype, backward):
    n = dol._native.cross_entropy_workspace(matrix(rows, width, dtype), matrix(classes, width, dtype), backward)
    assert 0 <= n < 1 << 38 and n % 256 == 0
    assert n == dol._native.cross_entropy_workspace(matrix(rows, width, dtype), matrix(classes, width, dtype), backward)


@pytest.mark.parametrize("x,w,why", [
    (matrix(8, 16), matrix(20, 15), "ESHAPE"), (matrix(8, 16), matrix(20, 16, BF16), "types"), (matrix(8, 16), matrix(0, 16), "classes"),
    (matrix(8, 0), matrix(4, 0), "classes"), (matrix(8, 16, 7), matrix(4, 16), "type"), (matrix((1 << 22) + 1, 16), matrix(4, 16), "more than"),
    (matrix(8, 16, ld=15), matrix(4, 16), "ESHAPE"), (None, matrix(4, 16), "NULL")])
def test_cross_entropy_refusals(x, w, why):
    with pytest.raises(dol.DolError, match=why):
        dol._native.cross_entropy_workspace(x, w, 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_newton_schulz_workspace(dtype):
    small, large = (dol._native.newton_schulz_workspace(matrix(r, c, dtype), 1) for r, c in ((10, 128), (1000, 777)))
    assert small == 0 < large
    assert dol._native.newton_schulz_workspace(matrix(777, 1000, dtype), 1) == large
    assert dol._native.newton_schulz_workspace(matrix(1000, 777, dtype), 4) > 3 * large


@pytest.mark.parametrize("g,batch,why", [(matrix(8, 16, 9), 1, "type"), (matrix(-1, 16), 1, "ESHAPE"), (matrix(8, 16), -1, "batch"), (None, 1, "NULL"),
                                         (matrix((1 << 20) + 1, 100), 1, "EUNSUPPORTED")])
def test_newton_schulz_refusals(g, batch, why):
    with pytest.raises(dol.DolError, match=why):
        dol._native.newton_schulz_workspace(g, batch)


@pytest.mark.parametrize("x,groups,why", [(acts(2, 10, 12), 5, "groups"), (acts(2, 10, 12), 0, "groups"), (acts(2, 10, 12, 5), 4, "type"), (None, 1, "NULL"),
                                          (acts(-1, 10, 12), 4, "ESHAPE")])
def test_group_norm_refusals(x, groups, why):
    with pytest.raises(dol.DolError, match=why):
        dol._native.group_norm_workspace(x, groups, 0)


def test_group_norm_workspace():
    assert dol._native.group_norm_workspace(acts(64, 784, 32), 8, 0) == 0               # a slab of a sample at a time
    assert dol._native.group_norm_workspace(acts(64, 784, 32), 8, 1) >= 2 * 64 * 32 * 4
    assert dol._native.group_norm_workspace(acts(16, 65536, 128, BF16), 32, 0) > 0
    assert dol._native.group_norm_workspace(acts(0, 10, 12), 4, 1) >= 0


def test_tuples_of_another_shape_and_numbers_past_32_bits():
    with pytest.raises(TypeError):
        dol._native.cross_entropy_workspace((0, 1, 2), matrix(4, 16), 0)
    with pytest.raises(OverflowError):
        dol._native.cross_entropy_workspace(matrix(1 << 32, 16), matrix(4, 16), 0)
    with pytest.raises(TypeError):
        dol._native.cross_entropy_workspace(matrix(8, 16), matrix(4, 16))


def test_host_tensors_are_refused():
    torch = pytest.importorskip("torch")
    for call in (dol._native.matrix, dol._native.activations):
        with pytest.raises(AssertionError):
            call(torch.zeros(2, 3, 4))
    with pytest.raises(AssertionError):
        dol._native.values(torch.zeros(3), torch.float32, 3)
    assert dol._native.matrix(None) is None and dol._native.values(None, torch.float32, 3) is None
    with pytest.raises(AttributeError):
        dol._native.matrix(3)


def test_a_workspace_is_taken_on_the_stream_of_the_call(monkeypatch):
    """The allocator hands out again, without waiting, what the same stream has freed: memory for a call on another stream than the current one
    has to come from that stream's own."""
    torch = pytest.importorskip("torch")
    import contextlib

    class Side:
        cuda_stream = 8192

    class External(Side):
        def __init__(self, handle, device=None):
            self.handle = handle

    current, taken, empty = [None], [], torch.empty

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def recorded(n, dtype, device):
        taken.append(current[-1])
        return empty(n, dtype=dtype)

    monkeypatch.setattr(torch.cuda, "Stream", Side)
    monkeypatch.setattr(torch.cuda, "ExternalStream", External)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", recorded)
    monkeypatch.setattr(dol, "_current", lambda: 0)
    side = Side()
    dol._workspace(None, 512, "cuda", side)
    dol._workspace(None, 512, "cuda", 4096)
    dol._workspace(None, 512, "cuda", None)
    assert taken[0] is side and taken[1].handle == 4096 and taken[2] is None
    assert dol._workspace(None, 0, "cuda", side) == (None, 0, None) and len(taken) == 3
    monkeypatch.setattr(dol, "_current", lambda: 8192)
    dol._workspace(None, 512, "cuda", side)                 # (the current one by name: no need to enter it)
    dol._workspace(None, 512, "cuda", 4096)
    assert taken[3] is None and taken[4].handle == 4096


@pytest.mark.parametrize("points", [2 ** 31 - 1, 2 ** 31 - 8, 2 ** 31 - 16, 2 ** 31 - 17])
@pytest.mark.parametrize("backward", [0, 1])
def test_group_norm_of_as_many_points_as_32_bits_count(points, backward):
    """Far more than a slab holds: such a group is shared out over its points, eight workgroups to each of 256 units, a float2 from each."""
    assert dol._native.group_norm_workspace(acts(1, points, 1), 1, backward) >= 8 * 256 * 8


def test_plain_numbers_past_32_bits():
    """Not cut to the 32 bits of the C call, where they would name another size."""
    big, null = 1 << 32, None
    for call in (lambda: dol._native.group_norm_workspace(acts(2, 10, 12), big + 4, 1), lambda: dol._native.newton_schulz_workspace(matrix(100, 200), big + 1),
                 lambda: dol._native.group_norm(acts(2, 10, 12), big + 4, null, null, 1e-5, 0, acts(2, 10, 12), null, null, null, 0, 0),
                 lambda: dol._native.newton_schulz(matrix(10, 20), 0, matrix(10, 20), 0, 0, big + 5, 1.0, 0.0, 0.0, 0.0, null, 0, 0),
                 lambda: dol._native.group_norm_backward(acts(0, 10, 12), -big + 4, null, null, 0, null, null, acts(0, 10, 12), acts(0, 10, 12), null, null, null, 0, 0)):
        with pytest.raises(OverflowError):
            call()


def test_layouts_with_samples_side_by_side():
    """[points][batch][channels] in memory is as good as [batch][points][channels]; one element less to a point and samples overlap."""
    for b, p, c, ld_batch, ld_point in ((3, 10, 12, 12, 36), (3, 10, 12, 13, 40), (2, 2, 4, 4, 8), (2, 2, 4, 8, 4)):
        assert dol._native.group_norm_workspace((F32, b, p, c, ld_batch, ld_point, 4096), 2, 1) > 0
    for b, p, c, ld_batch, ld_point in ((3, 10, 12, 12, 35), (3, 10, 12, 11, 40), (3, 10, 12, 0, 12), (2, 2, 4, 4, 4), (3, 10, 12, 119, 12)):
        with pytest.raises(dol.DolError, match="overlap"):
            dol._native.group_norm_workspace((F32, b, p, c, ld_batch, ld_point, 4096), 2, 1)


def test_names_of_kernels():
    """What the calls will launch, without a device; nothing for what they refuse."""
    k = dol._native.cross_entropy_kernel
    assert k(matrix(64, 128), matrix(10, 128), 0) == k(matrix(64, 128), matrix(10, 128), 1) == "xent_few_kernel"
    assert k(matrix(8192, 1024, BF16), matrix(65535, 1024, BF16), 0) == "xent_sums_kernel 256x256x64"
    assert k(matrix(8192, 1024, BF16), matrix(65535, 1024, BF16), 1) == "xent_dlogits_kernel 256x256x64, xent_products_kernel 256x256x64"
    assert k(matrix(8, 16), matrix(20, 15), 0) == k(matrix(0, 16), matrix(20, 16), 1) == k(None, matrix(4, 16), 0) == ""
    k = dol._native.newton_schulz_kernel
    assert k(matrix(10, 128), 1) == "ns_small_kernel"
    assert k(matrix(1000, 777), 1) == k(matrix(777, 1000), 1) == "ns_symmetric_kernel 64x64, ns_apply_kernel 64x64"
    assert k(matrix(4096, 4096, BF16), 1) == "ns_symmetric_kernel 256x256, ns_apply_kernel 256x256"
    assert k(matrix(10, 128), 0) == k(None, 1) == k(matrix(10, 128), -1) == ""
    with pytest.raises(TypeError):
        k(matrix(10, 128))


@pytest.mark.parametrize("backward", [0, 1])
def test_group_norm_of_more_slabs_than_a_launch_has_threads_for(backward):
    """65 535 samples of 4 093 groups, a wavefront to each: more than 2^32 threads.  The shared-out form needs space for its parts."""
    parts = 65535 * 8 * 4093 * 8
    assert dol._native.group_norm_workspace(acts(65535, 1, 8 * 4093, BF16), 4093, backward) >= parts
    # with fewer samples the slabs' own: nothing forward, two sums of a channel and sample backward
    assert dol._native.group_norm_workspace(acts(4000, 1, 8 * 4093, BF16), 4093, backward) == 8 * 4000 * 8 * 4093 * backward
