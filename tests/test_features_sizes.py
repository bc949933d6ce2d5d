"""Sizes that the operators on point features ask for, over the stated limits, without a GPU."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

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


@pytest.mark.parametrize("H,Hkv,D", [(2, 2, 0), (2, 0, 8), (0, 0, 0)])
def test_rows_of_nothing_are_refused(H, Hkv, D):
    """By the binding, as heads that do not fit: before a scale is made of the width."""
    groups = SimpleNamespace(B=1, N=5, M=3, device=torch.device("cpu"))
    q, k = torch.zeros(1, 3, H, D), torch.zeros(1, 5, Hkv, D)
    with pytest.raises(ValueError, match="heads"):
        cagq._attn(groups, q, k, k, None, None, 0.0)
