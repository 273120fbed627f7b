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
