"""Operators on point features where values that are not finite stand in places that do not count, and at the
ends of the stated ranges (bounds: tests/features_ref.py)."""
import numpy as np
import pytest
import torch

from paper_1912_02984_amd import cagq
from tests import features_ref as F
from tests.test_gpu_features import _attend, _bias, _dev, _features

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")

# How lists share waves: groups that share a wave's slots and points walked in a row; a list per slot at the
# centers and long lists at the points; ragged ones of both kinds; a workgroup to a list.
WAYS = [dict(N=400, M=300, K=20), dict(N=20, M=600, K=2), dict(N=300, M=200, lens=[0, 1, 17, 40]),
        dict(N=24, M=700, lens=[0, 1, 2, 5]), dict(N=500, M=6, lens=[700, 3, 141])]


def _groups(rng, N, M, K=0, lens=None, masked=0.1):
    return F.rand_groups(rng, 2, N, M, K, lens=lens, masked=masked)


def _odd(t, where):
    """t with NaN, infinity and -infinity in turn at the rows ``where`` says."""
    t = t.clone()
    flat = t.reshape(-1, t.shape[-1])
    rows = torch.nonzero(torch.as_tensor(where).reshape(-1)).reshape(-1)
    for i, x in enumerate((NAN, INF, -INF)):
        flat[rows[i::3]] = x
    return t


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("cap", [0.0, 9.0, 100.0])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_pairs_masked_by_the_bias(dt, cap, way):
    """A pair whose bias is -infinity contributes nothing, whatever k and v hold: not to the outputs, nor to any
    gradient. Points far away on one axis are masked for all heads, on another for the first head alone."""
    rng = np.random.default_rng(101 + way)
    c = _groups(rng, **WAYS[way])
    c.points[:, ::3, 0] -= 100.0
    c.points[:, 1::4, 1] -= 100.0
    for H, Hkv, D in ((4, 4, 16), (8, 2, 16), (3, 3, 24)):
        q, k, v, dout = (_features(rng, (2, n, h, D), dt) for n, h in ((c.M, H), (c.N, Hkv), (c.N, Hkv), (c.M, H)))
        table, edges, _ = F.rand_bias(rng, H, 6, False)
        edges[:2, 0] = -50.0
        table[0, 0] = -np.inf
        table[1, 0, 0] = -np.inf
        bias = (table, edges, None)
        u, _ = c.places(edges)
        dead = np.isinf(table[0][u[:, 0]] + table[1][u[:, 1]])  # [pairs][H]
        live = np.zeros((2 * c.N, Hkv), bool)
        np.logical_or.at(live, c.pt, ~dead.reshape(-1, Hkv, H // Hkv).all(2))
        held = np.zeros(2 * c.N, bool)
        held[c.pt] = True
        assert (held[:, None] & ~live).any() and live.any()
        zero = torch.from_numpy(~live).reshape(2, c.N, Hkv)
        k, v = (torch.where(zero[..., None], torch.zeros((), dtype=dt), t) for t in (k, v))
        want = F.attention(c, q, k, v, bias, None, cap, dout)
        F.check(_attend(c, q, _odd(k, zero), _odd(v, zero), bias, None, cap, dout), want, f"{dt} {cap} {way} {H}")


@pytest.mark.parametrize("dt,D", [(BF16, 24), (F16, 48), (F32, 12), (F32, 20), (BF16, 40), (BF16, 16)])
@pytest.mark.parametrize("cap", [0.0, 9.0, 100.0])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_a_point_in_no_group(dt, D, cap, way):
    """The first point of each cloud is in no group, and what its features hold reaches nothing; also where a head
    takes more lanes than it has channels for, and where lists end inside a round."""
    rng = np.random.default_rng(131 + way)
    c = _groups(rng, **WAYS[way])
    c.idx[c.idx == 0] = -1
    c = F.Case(2, c.N, c.M, c.idx, n_valid=c.n_valid, off=c.off, rng=rng)
    for H, Hkv in ((3, 3), (4, 2)):
        q, k, v, dout = (_features(rng, (2, n, h, D), dt) for n, h in ((c.M, H), (c.N, Hkv), (c.N, Hkv), (c.M, H)))
        bias = F.rand_bias(rng, H, 5, True)
        want = F.attention(c, q, k, v, bias, None, cap, dout)
        for x in (NAN, INF):
            k[:, 0], v[:, 0] = x, x
            F.check(_attend(c, q, k, v, bias, None, cap, dout), want, f"{dt} {D} {cap} {way} {H} {x}")
