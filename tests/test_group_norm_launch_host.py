"""The launches of the group norm's plans (host code; no GPU needed)."""
import ctypes

import pytest

from paper_2104_02621_amd import capscaps as cc


def launch(images, positions, width, groups, types, forward):
    norm = cc.GroupNormArgs(images, positions, width, groups, *types, cc.ACT_SILU, 1e-5)
    out = (ctypes.c_longlong * 3)()
    fn = cc._load().capscaps_testing_group_norm_launch
    fn.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
    assert fn(ctypes.addressof(norm), forward, ctypes.addressof(out)) == 1
    return tuple(out)


def check(images, positions, width, groups, types):
    kinds = []
    for forward in (0, 1):
        blocks, threads, resident = launch(images, positions, width, groups, types, forward)
        assert 1 <= blocks and 64 <= threads <= 1024 and blocks * threads < 1 << 32, (images, positions, width, groups, forward)
        kinds.append(resident)
    return kinds


TYPES = [(cc.FP32, cc.FP32), (cc.BF16, cc.BF16), (cc.FP32, cc.FP16)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("positions", [1, 3, 93, 1024])
def test_no_launch_passes_the_limit_of_threads(positions, types):
    """Workgroups times threads stay below 2^32, however many images there are."""
    resident = 0
    for images in (1, (1 << 22) - 1, 1 << 22, 6200000, 1 << 30):
        for width in [*range(1, 2300), *range(2301, 8400, 7), 4096, 4104, 8192]:
            resident += check(images, positions, width, 1, types)[1]
    assert resident > 0


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("groups", [3, 32, 1 << 10, 3 << 20, 64 * 16777213, 1 << 28])
def test_nor_do_launches_for_many_groups(groups, types):
    for columns in (1, 3, 4, 27, 64, 513, 1024):
        if groups * columns <= 1 << 30:
            for images in (1, 1000, 1 << 20):
                for positions in (1, 40, 300, 4000):
                    check(images, positions, groups * columns, groups, types)
