"""Group norm's sizes, checked without a GPU through the workspace function, which makes the same choices as the calls."""
import ctypes

import pytest

import paper_2304_04237_b200 as sa
from paper_2304_04237_b200 import binding


@pytest.fixture(scope="module")
def lib():
    from paper_2304_04237_b200 import build
    build.build()
    return binding.load()


def workspace(lib, *sizes):
    n = ctypes.c_size_t()
    return lib.slide_attn_group_norm_workspace(*sizes, ctypes.byref(n)), n.value


# B, H, W, C, groups, dtype: images that one CTA cannot keep in registers, few and so many that each is one chunk
@pytest.mark.parametrize("shape", [(296, 56, 56, 96, 32, 1), (297, 56, 56, 96, 32, 1), (300, 20, 20, 96, 8, 1), (400, 14, 14, 96, 32, 0), (160, 4, 4, 4096, 32, 1),
                                   (4096, 1, 337, 96, 32, 1), (1000, 128, 128, 8, 1, 0)], ids=str)
def test_large_images_need_room_for_their_sums_however_many_there_are(lib, shape):
    status, size = workspace(lib, *shape, 0)
    assert status == sa.OK and size >= 8 * shape[0] * shape[4]


@pytest.mark.parametrize("shape", [(2, 1, 336, 96, 32, 1), (4096, 1, 336, 96, 32, 1), (4096, 13, 13, 64, 8, 1), (100000, 1, 1, 64, 1, 0), (160, 2, 4, 4096, 32, 1)], ids=str)
def test_small_images_need_none(lib, shape):
    assert workspace(lib, *shape, 0) == (sa.OK, 0)


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("dtype,most", [(0, 2048), (1, 4096)])
def test_channels_past_the_limit_are_refused_whatever_their_bytes_come_to(lib, dtype, most, backward):
    """2^29 channels and more: their bytes pass 31 and 32 bits, to nothing, to two columns or to a negative number."""
    for C in [most + 8, 2 * most] + [2 ** p + more for p in (20, 27, 28, 29, 30) for more in (0, 8, 16, 512)] + [2 ** 31 - 8]:
        for groups in (1, 8):
            assert workspace(lib, 1, 1, 1, C, groups, dtype, backward)[0] == sa.ERR_UNSUPPORTED, C
    assert workspace(lib, 1, 1, 1, most, 1, dtype, backward)[0] == sa.OK


@pytest.mark.parametrize("C", [2 ** 29, 2 ** 30, 2 ** 30 + 8])
def test_calls_of_such_channels_are_refused(lib, C):
    x, y, mean, rstd, dx, room = (i << 40 for i in range(1, 7))          # addresses that nothing reads
    for dtype in (0, 1):
        assert lib.slide_attn_group_norm_forward(x, None, None, y, mean, rstd, 1, 1, 1, C, 1, 1e-5, 0, dtype, room, 1 << 40, None) == sa.ERR_UNSUPPORTED
        assert lib.slide_attn_group_norm_backward(x, None, None, mean, rstd, y, dx, None, None, 1, 1, 1, C, 1, 0, dtype, room, 1 << 40, None) == sa.ERR_UNSUPPORTED
