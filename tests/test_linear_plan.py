"""The sizes of the GPU tests of the linear operator's tiles take the kernels that they are
there for (CPU only)."""
import pytest

import linear_plan as lp


@pytest.fixture(scope="module")
def tables():
    t = lp.costs()
    assert [len(t[n]) for n in ("kStream16", "kStream32", "kChecked")] == [3, 3, 2]
    return t


@pytest.mark.parametrize("size,half,single", lp.FORWARD)
def test_forward(tables, size, half, single):
    assert (lp.kernels(tables, *size, 2)[0], lp.kernels(tables, *size, 4)[0]) == (half, single)


@pytest.mark.parametrize("size,half,single", lp.BACKWARD)
def test_backward(tables, size, half, single):
    for formed in (False, True):
        assert (lp.kernels(tables, *size, 2, formed)[1:], lp.kernels(tables, *size, 4, formed)[1:]) == (half, single)


def test_every_kernel_is_taken():
    """Streamed and checked ones of each tile, whole and in parts."""
    tiles = lambda names: {n.strip("/+") for n in names}
    for i in (1, 2):
        assert {"s64", "s128", "s256", "e64", "e128", "e256", "c128"} <= tiles(f[i] for f in lp.FORWARD)
        assert {"s64", "s128", "s256", "c128"} <= tiles(f[i][0] for f in lp.BACKWARD)
        assert {"s64", "s128", "s256", "c64"} <= tiles(f[i][1] for f in lp.BACKWARD)


@pytest.mark.parametrize("size,dtype,parts", [
    ((1, 4096, 4096), 2, False), ((16, 4096, 4096), 2, False), ((32, 1024, 1024), 2, False),
    ((32, 32, 32), 0, False), ((32, 256, 256), 0, False), ((1, 4096, 4096), 0, False), ((1, 8, 1 << 18), 2, False),
    ((1, 8192, 64), 2, True), ((32, 4096, 4096), 2, True), ((16, 8192, 256), 0, True),
    ((32, 8192, 64), 0, True), ((32, 8192, 8192), 0, True), ((17, 8192, 33), 0, True)])
def test_few_rows(size, dtype, parts):
    """Up to 32 rows take one pass over the weight (no workspace) where that is the faster
    one, and tiles in parts where the reduction axis is long beside the rest."""
    import ctypes

    import paper_2607_10071_amd as fb
    from paper_2607_10071_amd import block

    M, K, N = size
    n = ctypes.c_uint64()
    args = block._PACK_LINEAR.pack(M, K, K, N, N, N, K, N, dtype, dtype, 0, 1.0)
    assert fb._packed_call("flashblock_linear_workspace_size", "PP")(args, ctypes.byref(n)) == 0
    assert (n.value > 0) == parts
