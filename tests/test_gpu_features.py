"""Operators on point features (group attention, its gradients, the groups
turned round, the relative position bias) against their definitions in 64 bits
(tests/features_ref.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

from paper_1912_02984_amd import cagq
from paper_1912_02984_amd import workloads as W
from tests import features_ref as F

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _features(rng, shape, dt, gain=1.0):
    return torch.from_numpy((gain * rng.normal(size=shape)).astype(np.float32)).to(dt)


def _bias(bias):
    table, edges, slope = bias
    if table is None and slope is None:
        return None
    return cagq.RelativeBias(_dev(table), _dev(edges) if table is not None else None, _dev(slope))


def _attend(c, q, k, v, bias, scale=None, cap=0.0, dout=None, **kw):
    """The library's outputs on the GPU for CPU tensors."""
    g = c.groups(cagq, DEV)
    q, k, v = (t.to(DEV) for t in (q, k, v))
    b = _bias(bias)
    out, lse = cagq.group_attention(g, q, k, v, bias=b, scale=scale, cap=cap, **kw)
    got = dict(out=out, lse=lse)
    if dout is not None:
        lists = cagq.point_lists(g)
        got.update(cagq.group_attention_backward(g, lists, q, k, v, lse, dout.to(DEV), bias=b, scale=scale, cap=cap))
    return got


def _run(c, dt, H, Hkv, D, nb, slope, cap, seed, where, scale=None, gain=1.0):
    rng = np.random.default_rng(seed)
    q, k, v = (_features(rng, s, dt, gain) for s in
               ((c.B, c.M, H, D), (c.B, c.N, Hkv, D), (c.B, c.N, Hkv, D)))
    dout = _features(rng, (c.B, c.M, H, D), dt)
    bias = F.rand_bias(rng, H, nb, slope)
    got = _attend(c, q, k, v, bias, scale, cap, dout)
    F.check(got, F.attention(c, q, k, v, bias, scale, cap, dout), where)
    return got


def test_point_lists():
    """Lists of nothing, of one, of a wave and more, of a sorted chunk and more;
    masked slots, repeats of a point in a group, both forms of groups."""
    rng = np.random.default_rng(1)
    cases = [F.rand_groups(rng, 1, 1, 1, 1), F.rand_groups(rng, 3, 50, 17, 9, masked=0.3),
             F.rand_groups(rng, 2, 7, 300, 5), F.rand_groups(rng, 1, 1, 9000, 2, n_valid=False),
             F.rand_groups(rng, 2, 3, 5000, 3, masked=0.1), F.rand_groups(rng, 1, 5000, 800, 64),
             F.rand_groups(rng, 2, 40, 65, lens=[0, 1, 64, 65, 300]), F.rand_groups(rng, 1, 9, 4, lens=[0]),
             F.rand_groups(rng, 1, 2, 20000, lens=[1, 3], masked=0.2),
             F.rand_groups(rng, 2, 2100, 33, lens=[700, 3]), F.rand_groups(rng, 70, 33, 5, 12)]
    for n, c in enumerate(cases):
        print(f"[lists] {n}: B={c.B} N={c.N} M={c.M} slots={c.idx.size}", flush=True)
        off, center = cagq.point_lists(c.groups(cagq, DEV))
        woff, wcenter = F.point_lists(c)
        assert np.array_equal(off.cpu().numpy(), woff), n
        assert np.array_equal(center.cpu().numpy(), wcenter), n


@pytest.mark.parametrize("B,N,M,K,extra", [
    (1, 1024, 128, 128, 0), (1, 1024, 5462, 3, 0), (3, 1025, 128, 128, 0), (2, 33, 4097, 4, 0),  # slots of a cloud
    (256, 10, 3, 4, 0), (257, 10, 3, 4, 0), (255, 1025, 3, 4, 0), (128, 1030, 4, 40, 0),  # clouds
    (1, 1 << 18, 9, 7, 0), (1, (1 << 18) + 1, 9, 7, 0), (2, 1 << 17, 9, 7, 0),  # points
    (1, 700, 100, 0, 0), (5, 64, 300, 0, 7), (1, 50, 1, 0, 16383), (1, 50, 1, 0, 16384), (4, 9, 2000, 0, 16384),
    (1, 5, (1 << 22) - 1, 0, 60), (1, 5, 1 << 22, 0, 60)])  # ragged: entries, centers
def test_point_lists_at_limits(B, N, M, K, extra):
    """Sizes on either side of what one workgroup takes of a cloud, and of a
    launch; every list against a stable sort of the slots that count."""
    rng = np.random.default_rng(B + N + M + K + extra)
    rows = B * M
    if K:
        idx = rng.integers(-1, N + 1, (rows, K)).astype(np.int32)
        n = rng.integers(0, K + 1, rows).astype(np.int32)
        row = np.repeat(np.arange(rows), K)
        counts = (np.arange(K) < n[:, None]).ravel()
        form = dict(n_valid=torch.from_numpy(n.reshape(B, M)).to(DEV))
        shape, flat = (B, M, K), idx.ravel()
    else:  # few of many groups have entries; `extra` more in the last, and three that no group holds
        lens = np.where(rng.random(rows) < 500 / rows, rng.integers(0, 9, rows), 0)
        if M == 1:
            lens[:] = 0
        lens[-1] += extra if M == 1 else min(extra, 16384 - int(lens.sum())) if extra > 100 else extra
        total, tail = int(lens.sum()), 0 if M == 1 else 3
        flat = rng.integers(-1, N + 1, total + tail).astype(np.int32)
        row = np.concatenate([np.repeat(np.arange(rows), lens), np.zeros(tail, np.int64)])
        counts = np.arange(total + tail) < total
        off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        form, shape = dict(off=torch.from_numpy(off).to(DEV)), flat.shape
    counts &= (flat >= 0) & (flat < N)
    point, center = (row // M * N + flat)[counts], (row % M)[counts]
    want = np.full(flat.size, -1, np.int32)
    want[:center.size] = center[np.argsort(point, kind="stable")]
    woff = np.concatenate([[0], np.cumsum(np.bincount(point, minlength=B * N))])
    pts, cen = (torch.zeros((B, m, 3), device=DEV) for m in (N, M))
    g = cagq.Groups(torch.from_numpy(flat.reshape(shape)).to(DEV), pts, cen, **form)
    o = torch.full((B * N + 1 + 2,), -7, dtype=torch.int64, device=DEV)
    c = torch.full((flat.size + 5,), -7, dtype=torch.int32, device=DEV)
    cagq.point_lists(g, off=o[:-2], center=c[:-2])
    assert np.array_equal(o[:-2].cpu().numpy(), woff)
    got = c.cpu().numpy()
    assert np.array_equal(got[:flat.size], want) and (got[flat.size:-2] == -1).all()
    assert (got[-2:] == -7).all() and (o[-2:] == -7).all()


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("H,Hkv,D", [(1, 1, 1), (3, 3, 5), (4, 4, 16), (5, 5, 24), (6, 2, 32), (8, 8, 32), (2, 1, 64),
                                     (12, 12, 7), (1, 1, 256), (9, 3, 128), (33, 33, 8), (128, 64, 2), (16, 4, 256),
                                     (128, 1, 8)])
def test_attention_shapes(dt, H, Hkv, D):
    """Heads and widths: a lane to a head, a wave to a head, several waves to a
    row, odd widths, shared heads; fixed groups with masked slots and a bias."""
    rng = np.random.default_rng(H * 1000 + D)
    c = F.rand_groups(rng, 2, 61, 37, 20, masked=0.1)
    _run(c, dt, H, Hkv, D, 5, True, 0.0, 2, f"{dt} {H} {Hkv} {D}")


@pytest.mark.parametrize("dt,cap,nb,slope", [(F32, 0.0, 0, False), (F32, 2.5, 64, True), (BF16, 30.0, 1, False),
                                             (BF16, 0.0, 0, True), (F16, 10.0, 33, False)])
@pytest.mark.parametrize("form", ["fixed", "ragged", "all slots", "one slot"])
def test_attention_forms(dt, cap, nb, slope, form):
    """Fixed and ragged groups, lengths around the wave's, empty groups, points
    in no group and in many, with every part of the score."""
    rng = np.random.default_rng(7)
    c = {"fixed": lambda: F.rand_groups(rng, 3, 200, 50, 130, masked=0.2),
         "ragged": lambda: F.rand_groups(rng, 2, 150, 12, lens=[0, 1, 2, 63, 64, 65, 127, 129, 0, 400], masked=0.1),
         "all slots": lambda: F.rand_groups(rng, 2, 90, 40, 64, n_valid=False),
         "one slot": lambda: F.rand_groups(rng, 2, 9, 40, 1)}[form]()
    _run(c, dt, 4, 2, 16, nb, slope, cap, 3, f"{form} {dt} {cap} {nb}")


@pytest.mark.parametrize("dt,H,Hkv,D,N,M", [(BF16, 2, 2, 32, 40000, 38000), (F32, 4, 2, 16, 24001, 20001),
                                            (F16, 5, 5, 24, 14000, 13001), (BF16, 1, 1, 8, 270000, 262200),
                                            (F32, 3, 1, 7, 40001, 29000), (F16, 8, 4, 16, 70000, 20000)])
def test_attention_many_short_lists(dt, H, Hkv, D, N, M):
    """So many short lists that each slot of a wave takes its own, at the centers and,
    walked through in a row, at the points: most of a few entries, many of none, one
    of hundreds."""
    rng = np.random.default_rng(N)
    for K in (3, 0):
        c = F.rand_groups(rng, 1, N, M, K, masked=0.1, lens=rng.choice([0, 1, 2, 5], M) if K == 0 else None)
        c.idx[rng.random(c.idx.shape) < 300 / c.idx.size] = 77  # one point in many groups
        c = F.Case(1, N, M, c.idx, n_valid=c.n_valid, off=c.off, rng=rng)
        _run(c, dt, H, Hkv, D, 9, True, 4.0, 5, f"{dt} {H} {Hkv} {D} {N} {M} K={K}")


@pytest.mark.parametrize("dt,H,Hkv,D,M", [(BF16, 2, 2, 32, 36000), (F32, 2, 1, 16, 50000), (F16, 8, 8, 32, 9000),
                                          (F32, 3, 3, 20, 12000)])
def test_attention_of_tangled_groups(dt, H, Hkv, D, M):
    """Many groups, some longer than a slot's lanes, the same point two and three
    times in a group and in all its slots, groups that share all their points,
    masked slots, points in no group."""
    rng = np.random.default_rng(M)
    N = 33000
    for K in (12, 0):
        c = F.rand_groups(rng, 1, N, M, K, masked=0.1, lens=rng.choice([0, 1, 3, 9, 70], M, p=[.2, .3, .3, .19, .01])
                          if K == 0 else None)
        idx = c.idx.copy()
        if K:
            idx[:, ::5, 1] = idx[:, ::5, 0]
            idx[:, ::7, 3] = idx[:, ::7, 0]
            idx[:, 1::11] = idx[:, ::11][:, :idx[:, 1::11].shape[1]]
            idx[:, 5, :] = 4  # one point in all slots
        else:
            idx[1::3] = idx[:-1:3]
        idx[(idx >= 0) & (idx < N)] //= 2  # half of the points in no group
        c = F.Case(1, N, M, idx, n_valid=c.n_valid, off=c.off, rng=rng)
        _run(c, dt, H, Hkv, D, 9, True, 4.0, 5, f"{dt} {H} {Hkv} {D} {M} K={K}")


@pytest.mark.parametrize("dt,H,Hkv,D,N,M,lens", [
    (F16, 8, 2, 64, 300, 40, 20), (F32, 4, 1, 16, 300, 40, 20),      # four query heads a lane, a list for all slots
    (BF16, 2, 2, 5, 6, 300, 40), (F32, 3, 1, 7, 6, 300, 40),         # long lists at the points, rows off 16 bytes
    (F32, 2, 1, 64, 66000, 400, 3), (F16, 4, 2, 128, 66000, 400, 3),  # several points a slot, shared heads
    (BF16, 2, 1, 8, 200, 1100, 140), (F32, 1, 1, 3, 200, 1100, 140),  # a workgroup to a list, not cut
    (F16, 1, 1, 3, 500, 3, 2000), (BF16, 4, 4, 32, 40, 900, 2),      # cut, rows off 16 bytes; a list per slot
    (F16, 3, 3, 32, 700, 500, 8), (F32, 3, 3, 32, 700, 500, 9),      # either side of that
    (F32, 2, 1, 256, 6, 300, 40), (BF16, 4, 2, 256, 6, 300, 40)])    # a row to a wave, long lists at the points
@pytest.mark.parametrize("ragged", [False, True])
def test_attention_ways_to_share_waves(dt, H, Hkv, D, N, M, lens, ragged):
    """Every way in which lists share waves, with fixed and ragged groups, with and without a bias."""
    rng = np.random.default_rng(lens)
    c = F.rand_groups(rng, 1, N, M, 0 if ragged else lens, masked=0.05, n_valid=M != 1100,
                      lens=[lens, lens + 1, lens - 1] if ragged else None)
    _run(c, dt, H, Hkv, D, 5, True, 3.0, 6, f"{dt} {H} {Hkv} {D} {N} {M} {lens} {ragged}")
    if not ragged:
        _run(c, dt, H, Hkv, D, 0, False, 0.0, 7, f"{dt} {H} {Hkv} {D} {N} {M} {lens}, no bias")


def test_attention_long_lists():
    """Few centers with long lists: the work is split along them. Lengths that leave
    later parts empty, an empty list, and one center alone."""
    rng = np.random.default_rng(11)
    for lens, M in (([5000, 0, 1, 2999, 700], 5), ([21000], 1), ([300, 4000], 2)):
        for dt, H, Hkv, D in ((F16, 8, 2, 64), (F32, 3, 3, 20)):
            c = F.rand_groups(rng, 1, 3000, M, lens=lens, masked=0.05)
            print(f"[long] {lens} {dt}", flush=True)
            _run(c, dt, H, Hkv, D, 48, False, 50.0, 5, f"{lens} {dt}")


@pytest.mark.parametrize("cap", [1e3, 3e4, 1e6, 1e30])
def test_attention_wide_caps(cap):
    """A cap far above the scores is hardly a cap: the score's error goes with the score,
    not with the cap. Scores stay below 12 in size here, and cap * tanh(x / cap) is
    within x^3 / (3 cap^2) < 6e-4 of x at the first of these caps, 7e-7 at the second."""
    rng = np.random.default_rng(3)
    c = F.rand_groups(rng, 1, 200, 60, 20)
    q, k, v, dout = (_features(rng, (1, n, 4, 16), F32, 1.4) for n in (60, 200, 200, 60))
    none = (None, None, None)
    want = F.attention(c, q, k, v, none, None, cap, dout)
    for name, (ref, bound) in F.attention(c, q, k, v, none, None, 0.0, dout).items():  # bounds without the cap
        want[name] = (want[name][0], bound)
    F.check(_attend(c, q, k, v, none, None, cap, dout), want, f"cap={cap}")


def test_attention_masks_and_infinities():
    """-infinity in the bias masks pairs, whole groups among them; the type's lowest
    values and large scores; NaN and infinity where nothing reads: behind
    n_valid, at masked slots' points and at points of masked pairs."""
    rng = np.random.default_rng(13)
    B, N, M, K, H, D = 2, 80, 30, 16, 4, 16
    for dt in (F32, BF16, F16):
        c = F.rand_groups(rng, B, N, M, K, masked=0.1)
        c.centers[:, 5] = c.centers[:, 5] + 100.0  # every pair of this center in the first bucket on all axes
        q, k, v, dout = (_features(rng, (B, n, H, D), dt) for n in (M, N, N, M))
        table, edges, _ = F.rand_bias(rng, H, 6, False)
        edges[:, 0] = -50.0
        table[0, 0] = -np.inf
        table[1, 3, 1] = -np.inf
        table[2, 4, 2] = -3.0e38
        read = np.zeros(B * N, bool)
        read[c.pt] = True
        read = read.reshape(B, N)
        k[torch.from_numpy(~read)] = float("nan")
        v[torch.from_numpy(~read)] = float("inf")
        # a point that only the masked center's groups read holds NaN as well
        alone = np.setdiff1d(c.pt[c.row % M == 5], c.pt[c.row % M != 5])
        k.reshape(-1, H, D)[torch.from_numpy(alone)] = float("nan")
        v.reshape(-1, H, D)[torch.from_numpy(alone)] = float("nan")
        q[0, 3] *= 100.0  # one weight of nearly 1
        bias = (table, edges, None)
        want = F.attention(c, q, torch.nan_to_num(k, 0.0), torch.nan_to_num(v, 0.0, posinf=0.0), bias, None, 0.0,
                           dout)
        got = _attend(c, q, k, v, bias, None, 0.0, dout)
        assert (got["out"][:, 5] == 0).all() and (got["lse"][:, 5] == -np.inf).all()
        assert not read.all() and (got["dk"].cpu()[torch.from_numpy(~read)] == 0).all()
        F.check(got, want, str(dt))


def test_attention_all_groups_empty():
    for c in (F.rand_groups(np.random.default_rng(1), 2, 5, 7, lens=[0]),
              F.Case(1, 4, 3, np.full((1, 3, 2), -1, np.int32)),
              F.Case(1, 4, 3, np.zeros((1, 3, 2), np.int32), n_valid=np.int32([[0, -5, 0]]))):
        got = _run(c, BF16, 2, 2, 8, 3, True, 1.0, 3, "empty")
        for x in ("out", "dq", "dk", "dv", "dtable", "dslope"):
            assert (got[x] == 0).all(), x
        assert (got["lse"] == -np.inf).all()


@pytest.mark.parametrize("dt", [F32, BF16])
def test_attention_strided_rows(dt):
    """q, k and v as parts of one projection, rows that are not 16-byte aligned, and
    a scale of one's own."""
    rng = np.random.default_rng(17)
    B, N, H, D = 2, 70, 3, 16
    for pad in (0, 1, 8):
        c = F.rand_groups(rng, B, N, N, 12)
        qkv = _features(rng, (B, N, 3 * H * D + pad), dt)
        q, k, v = (qkv[..., i * H * D:(i + 1) * H * D].reshape(B, N, H, D) for i in range(3))
        dout = _features(rng, (B, N, H, D), dt)
        bias = F.rand_bias(rng, H, 9, True)
        whole = qkv.to(DEV)
        parts = [whole[..., i * H * D:(i + 1) * H * D].unflatten(-1, (H, D)) for i in range(3)]
        assert all(p.data_ptr() != q_.data_ptr() for p, q_ in zip(parts, (q, k, v)))
        g, b = c.groups(cagq, DEV), _bias(bias)
        out, lse = cagq.group_attention(g, *parts, bias=b, scale=0.7)
        got = dict(out=out, lse=lse, **cagq.group_attention_backward(g, cagq.point_lists(g), *parts, lse, dout.to(DEV),
                                                                     bias=b, scale=0.7))
        F.check(got, F.attention(c, q, k, v, bias, 0.7, 0.0, dout), f"{dt} pad={pad}")


def test_attention_offsets_past_32_bits():
    """Rows far apart: the last point's features lie more than 2^32 bytes, and more
    than 2^31 elements, into their tensor."""
    rng = np.random.default_rng(19)
    N, H, D, row = 70001, 2, 16, 32768
    some = np.array([0, 1, 2, 35000, 65535, 65536, 69999, 70000])
    idx = some[rng.integers(0, len(some), (1, 5, 6))].astype(np.int32)
    c = F.Case(1, N, 5, idx, rng=rng)
    store = torch.empty(N * row, dtype=BF16, device=DEV)
    assert store.numel() > 2 ** 31
    kv = store.view(1, N, row)[..., :2 * H * D].unflatten(-1, (2, H, D))
    k, v = torch.zeros((1, N, H, D), dtype=BF16), torch.zeros((1, N, H, D), dtype=BF16)
    for i in some:
        k[0, i], v[0, i] = _features(rng, (H, D), BF16), _features(rng, (H, D), BF16)
        kv[0, i, 0], kv[0, i, 1] = k[0, i].to(DEV), v[0, i].to(DEV)
    q, dout = _features(rng, (1, 5, H, D), BF16), _features(rng, (1, 5, H, D), BF16)
    g = c.groups(cagq, DEV)
    out, lse = cagq.group_attention(g, q.to(DEV), kv[:, :, 0], kv[:, :, 1])
    got = dict(out=out, lse=lse, **cagq.group_attention_backward(g, cagq.point_lists(g), q.to(DEV), kv[:, :, 0],
                                                                 kv[:, :, 1], lse, dout.to(DEV)))
    F.check(got, F.attention(c, q, k, v, (None, None, None), None, 0.0, dout), "far rows")


def test_gradients_against_differences():
    """Central differences of the 64-bit forward. A step of 2^-10 in a third derivative
    of at most about 30 leaves 30 / 6 * 2^-20 < 5e-6; the kernel's own part is
    within the bounds of features_ref."""
    rng = np.random.default_rng(23)
    c = F.rand_groups(rng, 1, 9, 6, 5, masked=0.1)
    H, D = 2, 4
    q, k, v, dout = (_features(rng, (1, n, H, D), F32) for n in (6, 9, 9, 6))
    bias = F.rand_bias(rng, H, 4, True)
    got = _attend(c, q, k, v, bias, None, 3.0, dout)
    want = F.attention(c, q, k, v, bias, None, 3.0, dout)

    def loss(**put):
        x = dict(q=q, k=k, v=v, table=torch.from_numpy(bias[0]), slope=torch.from_numpy(bias[2]))
        x.update(put)
        o = F.attention(c, x["q"], x["k"], x["v"], (x["table"].numpy(), bias[1], x["slope"].numpy()), None, 3.0)["out"][0]
        return float((o * dout.double()).sum())

    h = 2.0 ** -10
    for name, t in (("q", q), ("k", k), ("v", v), ("table", torch.from_numpy(bias[0])),
                    ("slope", torch.from_numpy(bias[2]))):
        for e in rng.choice(t.numel(), min(t.numel(), 12), replace=False):
            step = torch.zeros(t.numel(), dtype=torch.float64)
            step[e] = h
            up, dn = (t.double() + s * step.reshape(t.shape) for s in (1, -1))
            diff = (loss(**{name: up}) - loss(**{name: dn})) / (2 * h)
            mine = float(got["d" + name].flatten()[e])
            allowed = 5e-6 + float(want["d" + name][1].flatten()[e])
            assert abs(mine - diff) <= allowed, (name, e, mine, diff)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("H,nb,slope", [(1, 1, False), (3, 0, True), (8, 32, True), (5, 64, False), (128, 64, True)])
def test_relative_bias(dt, H, nb, slope):
    rng = np.random.default_rng(29)
    for c in (F.rand_groups(rng, 2, 60, 40, 33, masked=0.1), F.rand_groups(rng, 1, 1, 1, 1, n_valid=False),
              F.rand_groups(rng, 2, 60, 15, lens=[0, 1, 64, 65, 200], masked=0.1),
              F.rand_groups(rng, 1, 5, 3, lens=[0])):
        bias = F.rand_bias(rng, H, nb, slope)
        g, b = c.groups(cagq, DEV), _bias(bias)
        dbias = _features(rng, tuple(c.idx.shape) + (H,), dt)
        got = {"bias": cagq.relative_bias(g, b, dt).reshape(-1, H)}
        dtable, dslope = cagq.relative_bias_backward(g, b, dbias.to(DEV))
        want = F.relative_bias(c, bias, dbias, dt)
        if nb:
            got["dtable"] = dtable
        if slope:
            got["dslope"] = dslope
        F.check(got, want, f"{dt} {H} {nb}")


@pytest.mark.parametrize("dt", [F32, BF16, F16])
def test_relative_bias_of_what_is_not_finite(dt):
    """Infinity and NaN in the gradient of slots that count reach their own buckets and
    heads alone, those of slots that do not count none."""
    rng = np.random.default_rng(53)
    c = F.rand_groups(rng, 2, 40, 30, 12, masked=0.1)
    H = 5
    bias = F.rand_bias(rng, H, 20, True)
    dbias = _features(rng, (2, 30, 12, H), dt)
    flat = dbias.reshape(-1, H)
    out = np.setdiff1d(np.arange(c.idx.size), c.slot)
    flat[torch.from_numpy(out)] = float("nan")
    flat[int(c.slot[3]), 1] = float("inf")
    flat[int(c.slot[50]), 4] = float("nan")
    clean = torch.where(torch.isfinite(flat), flat, 0.0).reshape(dbias.shape)
    want = F.relative_bias(c, bias, clean.to(dt), dt)
    u, _ = c.places(bias[1])
    for slot, h, x in ((3, 1, float("inf")), (50, 4, float("nan"))):
        for a in range(3):
            want["dtable"][0][a, u[slot, a], h] = x
        want["dslope"][0][h] = x
    dtable, dslope = cagq.relative_bias_backward(c.groups(cagq, DEV), _bias(bias), dbias.to(DEV))
    for got, (ref, bound) in ((dtable, want["dtable"]), (dslope, want["dslope"])):
        got = got.cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        F.check(dict(x=torch.nan_to_num(got, 0.0, 7.0)), dict(x=(torch.nan_to_num(ref, 0.0, 7.0), bound)), str(dt))


def test_relative_bias_outside_ragged_groups():
    """Entries before the first list and behind the last are no group's: 0, and not in the gradient."""
    rng = np.random.default_rng(31)
    off = np.array([7, 9, 9, 15], np.int64)
    c = F.Case(1, 20, 3, rng.integers(0, 20, 40).astype(np.int32), off=off, rng=rng)
    bias = F.rand_bias(rng, 2, 8, True)
    dbias = _features(rng, (40, 2), F32)
    g, b = c.groups(cagq, DEV), _bias(bias)
    out = torch.full((40, 2), 9.0, device=DEV)
    dtable, dslope = cagq.relative_bias_backward(g, b, dbias.to(DEV))
    F.check({"bias": cagq.relative_bias(g, b, out=out), "dtable": dtable, "dslope": dslope},
            F.relative_bias(c, bias, dbias, F32), "outside")
    o, l = cagq.group_attention(g, *(torch.ones((1, n, 2, 8), device=DEV) for n in (3, 20, 20)), bias=b)
    assert (o[0, 1] == 0).all() and (l[0, 1] == -np.inf).all() and (o[0, 0] == 1).all()


def test_results_do_not_vary():
    """The same call again, in between other work: the same bits, the gradients of
    shared points and of the bias among them."""
    rng = np.random.default_rng(37)
    c = F.rand_groups(rng, 2, 500, 700, 40)
    q, k, v, dout = (_features(rng, (2, n, 8, 16), BF16) for n in (700, 500, 500, 700))
    bias = F.rand_bias(rng, 8, 4, True)
    first = None
    for _ in range(5):
        got = {n: t.clone() for n, t in _attend(c, q, k, v, bias, None, 5.0, dout).items()}
        got["rb"], got["rs"] = cagq.relative_bias_backward(c.groups(cagq, DEV), _bias(bias),
                                                           torch.ones((2, 700, 40, 8), device=DEV) * 0.1)
        first = first or got
        for n, t in got.items():
            assert torch.equal(t, first[n]), n


def test_captured_and_replayed():
    """Forward, turned groups, gradients and bias in one graph, and in two graphs that share a
    pool; replayed with other inputs and the program's own work in between."""
    rng = np.random.default_rng(41)
    B, N, M, H, D = 2, 300, 90, 4, 16
    bias = F.rand_bias(rng, H, 12, True)
    cs = [F.rand_groups(rng, B, N, M, 20, masked=0.1) for _ in range(3)]
    feats = [[_features(rng, (B, n, H, D), BF16) for n in (M, N, N, M)] for _ in range(3)]
    g = cs[0].groups(cagq, DEV)
    q, k, v, dout = (t.to(DEV) for t in feats[0])
    b = _bias(bias)
    long = F.rand_groups(rng, 1, N, 2, lens=[2500, 1100])
    gl = long.groups(cagq, DEV)

    def step():
        out, lse = cagq.group_attention(g, q, k, v, bias=b, cap=9.0)
        grads = cagq.group_attention_backward(g, cagq.point_lists(g), q, k, v, lse, dout, bias=b, cap=9.0)
        return dict(out=out, lse=lse, **grads)

    def few():
        return cagq.group_attention(gl, q[:1, :2], k[:1], v[:1], bias=b)

    step(), few()
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        r1 = step()
    with torch.cuda.graph(g2, pool=g1.pool()):
        r2 = few()
    for i in (1, 2, 0, 1):
        g.idx.copy_(_dev(cs[i].idx))
        g.n_valid.copy_(_dev(cs[i].n_valid))
        g.points.copy_(_dev(cs[i].points))
        g.centers.copy_(_dev(cs[i].centers))
        for d, s in zip((q, k, v, dout), feats[i]):
            d.copy_(s)
        g1.replay()
        got = {n: t.clone() for n, t in r1.items()}
        g2.replay()
        two = [t.clone() for t in r2]
        torch.cuda.synchronize()
        eager, alone = step(), few()
        for n, t in got.items():
            assert torch.equal(t, eager[n]), (i, n)
        assert all(torch.equal(x, y) for x, y in zip(two, alone))
        F.check(got, F.attention(cs[i], *feats[i][:3], bias, None, 9.0, feats[i][3]), f"replay {i}")


def test_on_another_stream():
    """Calls on a stream of the caller's, two at once with workspaces of their own."""
    rng = np.random.default_rng(43)
    cs = [F.rand_groups(rng, 1, 4000, 3, lens=[3000, 900]) for _ in range(2)]
    feats = [[_features(rng, (1, n, 4, 32), F16) for n in (3, 4000, 4000, 3)] for _ in range(2)]
    bias = F.rand_bias(rng, 4, 12, True)
    b = _bias(bias)
    on = [[t.to(DEV) for t in f] for f in feats]
    gs = [c.groups(cagq, DEV) for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    res = []
    for _ in range(3):
        res = []
        for s, g, (q, k, v, dout) in zip(streams, gs, on):
            out, lse = cagq.group_attention(g, q, k, v, bias=b, stream=s)
            lists = cagq.point_lists(g, stream=s)
            res.append(dict(out=out, lse=lse, **cagq.group_attention_backward(g, lists, q, k, v, lse, dout, bias=b,
                                                                              stream=s)))
    torch.cuda.synchronize()
    for c, f, r in zip(cs, feats, res):
        F.check(r, F.attention(c, *f[:3], bias, None, 0.0, f[3]), "streams")


def test_after_the_queries():
    """As a network uses them: a grid, its centers, their nodes, attention over the nodes and
    over the whole contexts, an upsampling layer back, and all gradients."""
    w = W.get_workload("room")
    L = w.layers[0]
    B, H, D = 2, 4, 16
    rng = np.random.default_rng(47)
    P = w.points(B=B)
    N, M = P.shape[1], 300
    Pt = torch.from_numpy(P).to(DEV)
    grid = cagq.build_grid(Pt, cagq.desc_from_spec(L.grid))
    cl, _ = cagq.sample_centers(grid, M, "rvs", 3)
    nodes = cagq.query_context(grid, cl, 16, "knn", 3)
    off = cagq.context_offsets(grid, cl)
    ctx = cagq.context_list(grid, cl, off)
    coarse = cagq.build_grid(nodes["center_xyz"], cagq.make_desc(L.grid.origin, (0.4,) * 3, (16, 16, 9), 32, 1))
    up = cagq.query_points(coarse, Pt, 8, "knn", 3)
    assert cagq.get_device_status(grid) == 0 and cagq.get_device_status(coarse) == 0
    xyz = nodes["center_xyz"]
    made = [cagq.Groups(nodes["node_idx"], Pt, xyz, n_valid=nodes["n_valid"]),
            cagq.Groups(ctx, Pt, xyz, off=off),
            cagq.Groups(up["node_idx"], xyz, Pt, n_valid=up["n_valid"])]
    h = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    bias = F.rand_bias(rng, H, 8, True, 0.3)
    for n, g in enumerate(made):
        c = F.Case(B, g.N, g.M, h(g.idx), n_valid=h(g.n_valid), off=h(g.off), points=h(g.points), centers=h(g.centers))
        q, k, v, dout = (_features(rng, (B, x, H, D), BF16) for x in (g.M, g.N, g.N, g.M))
        on = [t.to(DEV) for t in (q, k, v)]
        out, lse = cagq.group_attention(g, *on, bias=_bias(bias), cap=20.0)
        grads = cagq.group_attention_backward(g, cagq.point_lists(g), *on, lse, dout.to(DEV), bias=_bias(bias), cap=20.0)
        F.check(dict(out=out, lse=lse, **grads), F.attention(c, q, k, v, bias, None, 20.0, dout), f"layer {n}")


def test_refusals():
    """What the binding refuses before any device work."""
    t = lambda *s, dt=F32: torch.zeros(s, dtype=dt, device=DEV)  # noqa: E731
    idx, P, C = t(2, 5, 4, dt=torch.int32), t(2, 9, 3), t(2, 5, 3)
    g = cagq.Groups(idx, P, C)
    bad = [lambda: cagq.Groups(idx.long(), P, C), lambda: cagq.Groups(idx, P.double(), C),
           lambda: cagq.Groups(idx, P, C[:1]), lambda: cagq.Groups(idx, P, C.cpu()),
           lambda: cagq.Groups(idx[..., :2], P, C), lambda: cagq.Groups(idx, P, C, n_valid=t(2, 5)),
           lambda: cagq.Groups(idx.flatten(), P, C), lambda: cagq.Groups(idx.flatten(), P, C, off=t(10, dt=torch.int64)),
           lambda: cagq.RelativeBias(), lambda: cagq.RelativeBias(t(3, 65, 2), t(3, 64)),
           lambda: cagq.RelativeBias(t(3, 4, 2)), lambda: cagq.RelativeBias(t(3, 4, 2), t(3, 4)),
           lambda: cagq.RelativeBias(t(3, 4, 2), t(3, 3), t(3))]
    q, k = t(2, 5, 4, 8), t(2, 9, 2, 8)
    go = lambda q=q, k=k, v=k, **kw: cagq.group_attention(g, q, k, v, **kw)  # noqa: E731
    bad += [lambda: go(q=q.double(), k=k.double(), v=k.double()), lambda: go(k=k.half()), lambda: go(k=k[:, :8]),
            lambda: go(q=t(2, 5, 3, 8)), lambda: go(q=t(2, 5, 4, 7)), lambda: go(v=t(2, 9, 4, 8)),
            lambda: go(k=t(2, 9, 8, 2).transpose(2, 3)), lambda: go(k=t(9, 2, 2, 8).transpose(0, 1)),
            lambda: go(k=t(2, 1, 2, 8).expand(2, 9, 2, 8)), lambda: go(q=q.cpu()),
            lambda: go(bias=cagq.RelativeBias(slope=t(3))), lambda: go(out=t(2, 5, 4, 8, dt=F16)),
            lambda: go(lse=t(2, 5, 4)[:, ::2]), lambda: go(cap=-1.0), lambda: go(scale=float("nan")),
            lambda: go(q=t(2, 5, 2, 257), k=t(2, 9, 2, 257), v=t(2, 9, 2, 257))]
    off, center = cagq.point_lists(g)
    out, lse = go()
    bk = lambda off=off, center=center, lse=lse, dout=out: cagq.group_attention_backward(  # noqa: E731
        g, (off, center), q, k, k, lse, dout)
    bk()
    bad += [lambda: bk(off=off[1:]), lambda: bk(center=center.long()), lambda: bk(lse=lse.half()),
            lambda: bk(dout=out.half()), lambda: cagq.point_lists(g, center=center[:-1].clone()),
            lambda: cagq.relative_bias(g, cagq.RelativeBias(slope=t(3)), dtype=torch.float64),
            lambda: cagq.relative_bias_backward(g, cagq.RelativeBias(slope=t(3)), t(2, 5, 4, 2)),
            lambda: cagq.point_lists(g, workspace=t(16, dt=torch.uint8)),
            lambda: cagq.point_lists(g, workspace=t(1 << 20)[1:])]
    for n, f in enumerate(bad):
        with pytest.raises((ValueError, cagq.CagqError)):
            f()
            print("not refused:", n)
