"""Sizes that the operators on point features ask for, over the stated limits, without a GPU."""
import ctypes as C

import pytest

from paper_1912_02984_amd import cagq

BLOCKS = 256 * 3  # workgroups whose partial sums of the bias's gradient the reduction reads


def _workspace(g, a, b, backward):
    n = C.c_size_t()
    assert cagq.lib().cagq_group_attention_workspace(C.byref(g), C.byref(a), C.byref(b), backward, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("H,Hkv,D,nb", [(32, 32, 128, 32), (128, 128, 256, 64), (128, 32, 256, 64), (8, 8, 32, 32),
                                        (128, 1, 8, 64), (97, 97, 33, 17)])
def test_workspace_of_a_bias_gradient(dtype, H, Hkv, D, nb):
    """(lse, delta) of each center and head, and one table of all heads for each workgroup of a row of the launch:
    heads that take several passes do not multiply it. At most one more float for each center and head."""
    for B, N, M, K in ((4, 81920, 8192, 32), (1, 50, 7, 3), (2, 30000, 90, 1000)):
        g = cagq.GroupsC(B, N, M, K, 0x100000, 0x110000, None, 0, 0x120000, 0x130000)
        a = cagq.AttnC(dtype, H, Hkv, D, 0.25, 0.0, 0, 0, 0)
        b = cagq.BiasC(0x150000, 0x160000, 0x170000, nb)
        least, most = B * M * H * 8, B * M * H * 12 + 512
        got = _workspace(g, a, b, 1)
        assert least < got <= most + BLOCKS * (3 * nb + 1) * H * 4
        assert (got - least) >= 4 * (3 * nb + 1) * H
