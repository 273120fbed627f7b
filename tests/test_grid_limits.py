"""Calls whose grid would hold 2^32 threads or more are refused (CPU only: HIP launches such
a grid modulo 2^32 without an error, so that most of the output would not be written)."""
import numpy as np
import pytest

import paper_2607_10071_amd as fb

Z = np.linspace(-3, 3, 4, dtype=np.float32)


def grid(X, Y):
    return fb.BevGrid(-50.0, 100.0 / X, X, -50.0, 100.0 / Y, Y)


def first_refused(launch):
    """The least power of two of rows of 2^14 cells that `launch` refuses, and the
    threads of the last grid that it takes."""
    threads = 0
    for k in range(8, 22):
        try:
            info = launch(grid(1 << k, 1 << 14))
        except fb.FlashBevError as e:
            assert e.status == fb.STATUS["ERR_UNSUPPORTED"]
            return 1 << k, threads
        threads = info["workgroups"] * info["threads"]
        assert threads < 1 << 32
    raise AssertionError("never refused")


@pytest.mark.parametrize("C", [1, 16, 80])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sampling(C, dtype):
    """The grid that is twice the last one taken would not fit."""
    shape, img = (1, 6, 16, 44, C), (256, 704)
    for launch in (lambda g: fb.launch_info(shape, dtype, Z, g, img),
                   lambda g: fb.backward_launch_info(shape, dtype, Z, g, img)):
        _, threads = first_refused(launch)
        assert threads * 2 >= 1 << 32


@pytest.mark.parametrize("P", [4, 8])
def test_sca(P):
    levels = ((16, 44), (8, 22))
    shape = (1, 6, sum(h * w for h, w in levels), 32)
    _, threads = first_refused(lambda g: fb.sca_launch_info(shape, "f32", 4, levels, Z, g, (256, 704), P))
    assert threads * 2 >= 1 << 32
