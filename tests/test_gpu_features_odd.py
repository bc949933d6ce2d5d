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


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("cap", [0.0, 9.0, 100.0])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_groups_of_nothing(dt, cap, way):
    """Padded centers: groups without a slot, and with masked slots alone. What their q and dout hold reaches
    nothing; their own rows of out and dq are zeros."""
    rng = np.random.default_rng(151 + way)
    c = _groups(rng, **WAYS[way])
    H, Hkv, D = 4, 2, 24
    some = np.zeros(2 * c.M, bool)
    some[c.row] = True
    none = rng.random(2 * c.M) < 0.3
    none[:2] = True
    idx = c.idx.reshape(2 * c.M, -1) if c.off is None else c.idx
    if c.off is None:
        idx[none] = -1
    else:
        idx[np.isin(np.repeat(np.arange(2 * c.M), np.diff(c.off)), np.flatnonzero(none))] = c.N
    c = F.Case(2, c.N, c.M, c.idx, n_valid=c.n_valid, off=c.off, rng=rng)
    none |= ~some
    q, k, v, dout = (_features(rng, (2, n, h, D), dt) for n, h in ((c.M, H), (c.N, Hkv), (c.N, Hkv), (c.M, H)))
    bias = F.rand_bias(rng, H, 5, True)
    want = F.attention(c, q, k, v, bias, None, cap, dout)
    rows = torch.from_numpy(none).reshape(2, c.M, 1).expand(2, c.M, H)
    got = _attend(c, _odd(q, rows), k, v, bias, None, cap, _odd(dout, rows))
    F.check(got, want, f"{dt} {cap} {way}")
    assert (got["dq"].cpu()[rows] == 0).all() and (got["out"].cpu()[rows] == 0).all()


@pytest.mark.parametrize("dt", [F32, BF16])
def test_a_score_at_its_cap(dt):
    """An infinite q under a cap: every score is the cap or its negative, the weights are finite, and the
    tanh is flat there, so that nothing comes back to q. Lists that end inside a round. (At most 9 entries, a score's
    weight off by less than 30 steps of 2^-24, values below 5, a point in at most 40 lists.)"""
    rng = np.random.default_rng(171)
    c = _groups(rng, 60, 50, lens=[1, 2, 5, 9], masked=0.0)
    q, k, v, dout = (_features(rng, (2, n, 2, 16), dt) for n in (50, 60, 60, 50))
    k = k.abs() + 0.5
    none = (None, None, None)
    big = torch.where(torch.arange(16) == 3, 1e30, 0.0).to(dt).expand(q.shape).contiguous()
    want = F.attention(c, big, k, v, none, None, 3.0, dout)
    got = _attend(c, torch.where(big > 0, INF, 0.0).to(dt), k, v, none, None, 3.0, dout)
    zero = lambda t: torch.zeros_like(t, dtype=torch.float64)  # noqa: E731
    u = torch.full((), 2.0 ** -16, dtype=torch.float64)
    F.check({n: got[n] for n in ("out", "dv", "dq")}, {
        "out": (want["out"][0], F.half_step(dt) * want["out"][0].abs() + u),
        "dv": (want["dv"][0], F.half_step(dt) * want["dv"][0].abs() + 64 * u),
        "dq": (zero(q), u)}, str(dt))


@pytest.mark.parametrize("dt,H,Hkv,D", [(BF16, 128, 1, 8), (F16, 124, 1, 3), (F32, 128, 1, 4), (F32, 126, 1, 1),
                                        (BF16, 128, 2, 8), (F16, 128, 128, 8)])
@pytest.mark.parametrize("N,M,K", [(60, 9, 12), (3, 40, 30)])
def test_most_heads_and_buckets(dt, H, Hkv, D, N, M, K):
    """The gradient's table at its largest, where points are walked in a row and where a wave takes a point's list."""
    rng = np.random.default_rng(H + D + N)
    c = F.rand_groups(rng, 2, N, M, K, masked=0.1)
    q, k, v, dout = (_features(rng, (2, n, h, D), dt) for n, h in ((M, H), (N, Hkv), (N, Hkv), (M, H)))
    bias = F.rand_bias(rng, H, 64, True)
    want = F.attention(c, q, k, v, bias, None, 0.0, dout)
    F.check(_attend(c, q, k, v, bias, None, 0.0, dout), want, f"{dt} {H} {D} {N}")


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("cap", [0.0, 9.0])
@pytest.mark.parametrize("mask", [float(np.finfo(np.float32).min), -1e30, -1e9, -65504.0, 1e9])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_groups_all_of_one_far_score(dt, cap, mask, way):
    """Groups whose slots all have the same score, of the type's lowest value or another far from 0: their weights
    are alike and sum up to 1, in the gradients as well. A softmax does not change by what is added to all scores,
    so the definition without that value is the reference (their q is 0: the scores are the value itself)."""
    rng = np.random.default_rng(191 + way)
    c = _groups(rng, **WAYS[way])
    far = rng.random((2, c.M)) < 0.4
    c.centers[far] += 100.0  # every pair of these centers in the first bucket
    for H, Hkv, D in ((4, 4, 16), (2, 1, 20)):
        q, k, v, dout = (_features(rng, (2, n, h, D), dt) for n, h in ((c.M, H), (c.N, Hkv), (c.N, Hkv), (c.M, H)))
        q[torch.from_numpy(far)] = 0.0
        table, edges, _ = F.rand_bias(rng, H, 6, False)
        edges[:, 0] = -50.0
        table[:, 0] = 0.0
        want = F.attention(c, q, k, v, (table, edges, None), None, cap, dout)
        lse, bound = want["lse"]
        at = torch.from_numpy(far)[..., None].expand_as(lse) & torch.isfinite(lse)
        want["lse"] = (torch.where(at, lse + mask, lse), torch.where(at, 2 * F.U * abs(mask), bound))
        table = table.copy()
        table[0, 0] = mask
        F.check(_attend(c, q, k, v, (table, edges, None), None, cap, dout), want, f"{dt} {cap} {mask} {way} {H}")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_points_masked_by_their_distance(dt, way):
    """Padded points so far away that the distance overflows: under a negative slope their bias is -infinity, and
    they are as absent as points of masked slots, from the slope's gradient too."""
    rng = np.random.default_rng(211 + way)
    c = _groups(rng, **WAYS[way])
    gone = rng.random((2, c.N)) < 0.3
    gone[:, 1] = True
    for H, Hkv, D, nb in ((4, 4, 16, 5), (4, 2, 16, 0)):
        q, k, v, dout = (_features(rng, (2, n, h, D), dt) for n, h in ((c.M, H), (c.N, Hkv), (c.N, Hkv), (c.M, H)))
        table, edges, slope = F.rand_bias(rng, H, nb, True)
        bias = (table, edges, -np.abs(slope) - 0.1)
        idx = c.idx.copy().reshape(-1)
        dead = np.zeros(idx.size, bool)
        dead[c.slot] = gone.reshape(-1)[c.pt]
        idx[dead] = -1
        without = F.Case(2, c.N, c.M, idx.reshape(c.idx.shape), c.n_valid, c.off, c.points, c.centers)
        want = F.attention(without, q, k, v, bias, None, 0.0, dout)
        points = np.where(gone[..., None], np.float32(3e30), c.points)
        with_ = F.Case(2, c.N, c.M, c.idx, c.n_valid, c.off, points, c.centers)
        rows = torch.from_numpy(gone)[..., None].expand(2, c.N, Hkv)
        F.check(_attend(with_, q, _odd(k, rows), _odd(v, rows), bias, None, 0.0, dout), want, f"{dt} {way} {H}")


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("ragged", [False, True])
def test_relative_bias_gradient_at_a_distance_that_overflows(dt, ragged):
    """Gradients, finite and not, of slots at an infinite distance: each product once, as the sum has it."""
    rng = np.random.default_rng(231)
    H, nb = 6, 4
    c = F.rand_groups(rng, 1, 30, 9, 0 if ragged else 7, lens=[7, 9, 3])
    table, edges, slope = F.rand_bias(rng, H, nb, True)
    far = int(c.pt[10])
    points = c.points.copy()
    points[0, far] = 1e30
    c = F.Case(1, 30, 9, c.idx, c.n_valid, c.off, points, c.centers)
    hit = c.pt == far
    dbias = _features(rng, tuple(c.idx.shape) + (H,), dt)
    flat = dbias.reshape(-1, H)
    slots = torch.from_numpy(c.slot[hit])
    flat[slots] = torch.tensor([INF, 2.0, -3.0, -INF, 0.0, NAN]).to(dt)
    u, dist = c.places(edges)
    dist[hit] = np.inf
    g = flat.double().numpy()[c.slot]
    with np.errstate(invalid="ignore"):
        want_t, want_s = np.zeros((3, nb, H)), (g * dist[:, None]).sum(0)
    for a in range(3):
        np.add.at(want_t[a], u[:, a], g)
    size = np.where(np.isfinite(g), np.abs(g), 0.0)
    bound = len(g) * F.U * size.sum(0) + 1e-30
    got = cagq.relative_bias_backward(c.groups(cagq, DEV), _bias((table, edges, slope)), dbias.to(DEV))
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x))  # noqa: E731
    assert np.isnan(want_s[4:]).all() and np.array_equal(want_s[:4], [np.inf, np.inf, -np.inf, -np.inf])
    F.check(dict(dtable=got[0], dslope=got[1]), dict(dtable=(t(want_t), t(np.broadcast_to(bound, want_t.shape))),
                                                     dslope=(t(want_s), t(bound))), f"{dt} {ragged}")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("cap", [0.0, 9.0])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_masked_points_of_groups_that_are_not_finite(dt, cap, way):
    """Groups whose q or dout is not finite, and whose gradients are not: the points that the bias masks in them get
    zeros all the same, and so does the bucket that no other pair is in."""
    rng = np.random.default_rng(251 + way)
    c = _groups(rng, **WAYS[way])
    c.points[:, ::3, 0] -= 100.0
    H, Hkv, D = 4, 2, 16
    q, k, v, dout = (_features(rng, (2, n, h, D), dt) for n, h in ((c.M, H), (c.N, Hkv), (c.N, Hkv), (c.M, H)))
    rows = rng.random((2, c.M)) < 0.5
    rows[:, 0] = True
    odd = torch.from_numpy(rows)[..., None].expand(2, c.M, H)
    table, edges, slope = F.rand_bias(rng, H, 6, True)
    edges[:, 0] = -50.0
    table[0, 0] = -np.inf
    for x in ((_odd(q, odd), dout), (q, _odd(dout, odd))):
        got = _attend(c, x[0], k, v, (table, edges, slope), None, cap, x[1])
        assert not torch.isfinite(got["dk"]).all()
        assert (got["dk"][:, ::3] == 0).all() and (got["dv"][:, ::3] == 0).all() and (got["dtable"][0, 0] == 0).all()
