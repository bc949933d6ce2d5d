"""The operators on point features in 64 bits on the CPU, from their definitions in
include/cagq.h (gradients by automatic differentiation), with the bounds that
the kernels' 32-bit arithmetic allows.

Bounds. u = 2^-24 is half a step of fp32. A score is a product of D terms, a
bias of up to four and a capped value; each of its operations is off by at most
u of its operands' magnitudes, so with
    S = scale * sum |q_d k_d| + |biases| + cap
a score is off by at most (D + 16) u S (the cap's exponential and reciprocal, a
few u of the cap, are among the 16), and the exponent's own error is 2 u
(|s| + |lse|) + 4 u, from the rounded difference, the multiplication by log2 e
and the exponential. A weight p is then off by the relative
    e = 2 ((D + 20) u S + 2 u |lse| + 4 u) + n u,
the score's error counted twice (once through the sum), n the length of the
list. out is a sum of n products p v: off by (e + (n + 2) u) max |v|, and half a
step of the features' type. Gradients are sums of products p (dp - delta) x:
their magnitude A is the sum with |dp| + |delta|-like magnitudes in place of the
difference, and they are off by (2 e + (n + 2 D + 16) u) A. Below its least
normal number a type's step no longer shrinks with the value: half of its least
step (2^-25 in fp16, whose subnormal numbers are multiples of 2^-24) is allowed
as well.
"""
import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def least_half_step(dtype):
    f = torch.finfo(dtype)
    return f.smallest_normal * f.eps / 2


class Case:
    """Groups on the CPU: idx int32 [B, M, K] with n_valid or None, or idx [T] with off."""

    def __init__(self, B, N, M, idx, n_valid=None, off=None, points=None, centers=None, rng=None):
        self.B, self.N, self.M = B, N, M
        self.idx, self.n_valid, self.off = idx, n_valid, off
        rng = rng or np.random.default_rng(0)
        self.points = rng.random((B, N, 3), dtype=np.float32) if points is None else points
        self.centers = rng.random((B, M, 3), dtype=np.float32) if centers is None else centers
        slot, row = [], []
        for r in range(B * M):
            if off is None:
                K = idx.shape[2]
                n = K if n_valid is None else min(max(int(n_valid.reshape(-1)[r]), 0), K)
                s = np.arange(r * K, r * K + n)
            else:
                s = np.arange(off[r], off[r + 1])
            s = s[(idx.reshape(-1)[s] >= 0) & (idx.reshape(-1)[s] < N)]
            slot.append(s)
            row.append(np.full(len(s), r))
        self.slot = np.concatenate(slot).astype(np.int64)
        self.row = np.concatenate(row).astype(np.int64)
        self.pt = idx.reshape(-1)[self.slot].astype(np.int64) + self.row // M * N

    def groups(self, cagq, dev):
        t = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        return cagq.Groups(t(self.idx), t(self.points), t(self.centers), n_valid=t(self.n_valid), off=t(self.off))

    def places(self, edges):
        """Buckets [T][3] and distances [T] of the pairs."""
        d = self.points.reshape(-1, 3)[self.pt] - self.centers.reshape(-1, 3)[self.row]  # fp32, the definition's
        u = None
        if edges is not None:
            u = np.stack([(edges[a][None] <= d[:, a:a + 1]).sum(1) for a in range(3)], 1)
        return u, np.sqrt((d.astype(np.float64) ** 2).sum(1))


def rand_groups(rng, B, N, M, K=0, lens=None, masked=0.0, n_valid=True):
    """Random groups: K slots of which a random number counts (garbage behind), or lists of random or given lengths;
    a share of the slots masked by indexes outside [0, N)."""
    if K:
        idx = rng.integers(0, N, (B, M, K))
        nv = rng.integers(0, K + 1, (B, M)).astype(np.int32) if n_valid else None
    else:
        lens = rng.integers(0, 40, B * M) if lens is None else np.resize(np.asarray(lens), B * M)
        off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        idx = rng.integers(0, N, int(off[-1]))
    bad = rng.choice([-1, N, 2 ** 31 - 1, -2 ** 31], idx.shape)
    idx = np.where(rng.random(idx.shape) < masked, bad, idx).astype(np.int32)
    if K:
        if nv is not None:
            idx = np.where(np.arange(K) < nv[..., None], idx, -2 ** 31 + 7).astype(np.int32)
        return Case(B, N, M, idx, n_valid=nv, rng=rng)
    return Case(B, N, M, idx, off=off, rng=rng)


def rand_bias(rng, H, nb, slope, reach=1.0):
    table = edges = sl = None
    if nb:
        table = rng.normal(size=(3, nb, H)).astype(np.float32)
        edges = np.sort(rng.uniform(-reach, reach, (3, nb - 1)).astype(np.float32), 1)
    if slope:
        sl = rng.normal(size=H).astype(np.float32)
    return table, edges, sl


def attention(c: Case, q, k, v, bias, scale, cap, dout=None):
    """Outputs in 64 bits and their bounds: {name: (value, bound)}. q, k, v, dout: CPU tensors of the features' type."""
    dt = q.dtype
    table, edges, slope = bias
    B, N, M = c.B, c.N, c.M
    H, D, Hkv = q.shape[2], q.shape[3], k.shape[2]
    R = H // Hkv
    scale = D ** -0.5 if scale is None else scale
    leaf = lambda t: t.detach().double().contiguous().requires_grad_(True)  # noqa: E731
    q, k, v = leaf(q), leaf(k), leaf(v)
    row, pt = torch.from_numpy(c.row), torch.from_numpy(c.pt)
    T = len(row)
    qq, kk, vv = q.reshape(-1, H, D)[row], k.reshape(-1, Hkv, D)[pt], v.reshape(-1, Hkv, D)[pt]
    kk, vv = kk.repeat_interleave(R, 1), vv.repeat_interleave(R, 1)
    s = (qq * kk).sum(-1) * scale
    mag = (qq * kk).abs().sum(-1).detach() * abs(scale)
    if cap:
        s = cap * torch.tanh(s / cap)
        mag = mag + cap
    u, dist = c.places(edges)
    dist = torch.from_numpy(dist)[:, None]
    tt = ss = None
    if table is not None:
        tt = leaf(torch.from_numpy(table))
        for a in range(3):
            x = tt[a][torch.from_numpy(u[:, a])]
            s, mag = s + x, mag + torch.where(torch.isinf(x), 0.0, x.detach().abs())
    if slope is not None:
        ss = leaf(torch.from_numpy(slope))
        s, mag = s + ss * dist, mag + (ss * dist).detach().abs()
    dead = s == -float("inf")
    rows = B * M
    m = torch.full((rows, H), -float("inf"), dtype=torch.float64)
    m = m.scatter_reduce(0, row[:, None].expand(T, H), s.detach(), "amax") if T else m
    safe = torch.where(torch.isinf(m), 0.0, m)
    e = torch.where(dead, 0.0, torch.exp(torch.where(dead, 0.0, s) - safe[row]))
    zero = torch.zeros((rows, H), dtype=torch.float64)
    total = zero.index_add(0, row, e)
    some = total > 0
    p = e / torch.where(some, total, 1.0)[row]
    lse = torch.where(some, safe + torch.log(torch.where(some, total, 1.0)), -float("inf")).detach()
    vz = torch.where(dead[..., None], 0.0, vv)
    out = torch.zeros((rows, H, D), dtype=torch.float64).index_add(0, row, p[..., None] * vz)
    # bounds
    n = torch.zeros(rows, dtype=torch.float64).index_add(0, row, torch.ones(T, dtype=torch.float64))[:, None]
    top = lambda x: torch.zeros((rows, H), dtype=torch.float64).scatter_reduce(  # noqa: E731
        0, row[:, None].expand(T, H), x, "amax") if T else zero
    S = top(torch.where(p.detach() > 0, mag, 0.0))  # a pair of weight 0 is one in 32 bits too
    L = torch.where(some, lse.abs(), 0.0)
    es = (D + 20) * U * S + 2 * U * L + 4 * U
    ew = 2 * es + n * U
    vmax = top(vz.detach().abs().amax(-1))
    hs, hs0 = half_step(dt), least_half_step(dt) + 1e-30
    shape = lambda x, *sh: x.detach().reshape(*sh)  # noqa: E731
    res = {"out": (shape(out, B, M, H, D), hs * out.detach().abs().reshape(B, M, H, D) +
                   ((ew + (n + 2) * U) * vmax).reshape(B, M, H, 1) + hs0),
           "lse": (shape(lse, B, M, H), (es + (n + 4) * U + 2 * U * L).reshape(B, M, H))}
    if dout is None:
        return res
    g = dout.double().reshape(-1, H, D)
    (out * g).sum().backward()
    pd, gg = p.detach(), g[row]
    dp = torch.where(dead, 0.0, (gg * vz.detach()).sum(-1)).abs()
    dpm = (gg.abs() * vz.detach().abs()).sum(-1)  # magnitude of dp's products
    w = pd * (dpm + top(dpm)[row])  # of p (dp - delta)
    eg = (2 * ew + (n + 2 * D + 16) * U)[row]
    kz, qz = kk.detach().abs(), qq.detach().abs()
    lots = torch.zeros(B * N, dtype=torch.float64).index_add(0, pt, torch.ones(T, dtype=torch.float64))
    heads = lambda x: x.reshape(T, Hkv, R, D).sum(2)  # noqa: E731
    at_pt = lambda x: torch.zeros((B * N, Hkv, D), dtype=torch.float64).index_add(0, pt, heads(x))  # noqa: E731
    more = ((lots * R + 2) * U)[:, None, None]

    def of(grad, bound, sh):
        grad = grad.reshape(sh)
        return grad, hs * grad.abs() + bound.reshape(sh) + hs0

    bq = torch.zeros((rows, H, D), dtype=torch.float64).index_add(0, row, (eg * w)[..., None] * kz) * abs(scale)
    bk = at_pt((eg * w)[..., None] * qz) * abs(scale) + more * at_pt(w[..., None] * qz) * abs(scale)
    bv = at_pt((eg * pd)[..., None] * gg.abs()) + more * at_pt(pd[..., None] * gg.abs())
    res["dq"] = of(q.grad, bq, q.shape)
    res["dk"] = of(k.grad, bk, k.shape)
    res["dv"] = of(v.grad, bv, v.shape)
    if tt is not None:
        bt = torch.zeros_like(tt)
        cnt = torch.zeros(tt.shape[:2], dtype=torch.float64)
        for a in range(3):
            ua = torch.from_numpy(u[:, a])
            cnt[a].index_add_(0, ua, torch.ones(T, dtype=torch.float64))
            bt[a].index_add_(0, ua, eg * w)
            bt[a] += cnt[a][:, None] * U * torch.zeros_like(bt[a]).index_add_(0, ua, w)
        res["dtable"] = (tt.grad, bt + U * tt.grad.abs() + 1e-30)
    if ss is not None:
        wd = w * dist
        res["dslope"] = (ss.grad, (eg * wd).sum(0) + (T + 4) * U * wd.sum(0) + 1e-30)
    return res


def check(got, want, where):
    """Every value within its bound, and where the reference is not finite, the same as it. Written so that a value
    passes by a comparison that holds: a NaN makes every comparison false."""
    for name, (ref, bound) in want.items():
        x = got[name].detach().cpu().double()
        assert x.shape == ref.shape, (where, name)
        fin, bound = torch.isfinite(ref), bound.expand_as(ref)
        assert torch.isfinite(bound[fin]).all(), (where, name, "a bound that is not finite")
        same = (x == ref) | (torch.isnan(x) & torch.isnan(ref))
        assert same[~fin].all() and torch.equal(torch.isfinite(x), fin), (where, name, "not finite alike")
        off = torch.where(fin, (x - ref).abs(), 0.0)
        ok = off <= torch.where(fin, bound, 0.0)
        assert ok.all(), (where, name, int((~ok).sum()), float(off[~ok].max()), float((off / bound)[~ok].max()))


def point_lists(c: Case):
    order = np.lexsort((c.row, c.pt))
    off = np.concatenate([[0], np.cumsum(np.bincount(c.pt, minlength=c.B * c.N))]).astype(np.int64)
    center = np.full(c.idx.size, -1, np.int32)
    center[:len(order)] = (c.row % c.M)[order]
    return off, center


def relative_bias(c: Case, bias, dbias, dtype):
    """(bias, its bound), (dtable, bound), (dslope, bound) for dbias [slots][H] (a CPU tensor)."""
    table, edges, slope = bias
    u, dist = c.places(edges)
    H = (table if table is not None else slope).shape[-1]
    T = len(c.slot)
    b, mag = np.zeros((T, H)), np.zeros((T, H))
    g = dbias.double().reshape(-1, H).numpy()[c.slot]
    dt = bt = ds = bs = None
    if table is not None:
        dt, bt = np.zeros(table.shape), np.zeros(table.shape)
        for a in range(3):
            x = table[a].astype(np.float64)[u[:, a]]
            b, mag = b + x, mag + np.abs(x)
            np.add.at(dt[a], u[:, a], g)
            np.add.at(bt[a], u[:, a], np.abs(g) * T * U)
    if slope is not None:
        x = slope.astype(np.float64) * dist[:, None]
        b, mag = b + x, mag + np.abs(x)
        ds, bs = (g * dist[:, None]).sum(0), (np.abs(g) * dist[:, None]).sum(0) * (T + 8) * U
    full, bound = np.zeros((c.idx.size, H)), np.zeros((c.idx.size, H))
    full[c.slot], bound[c.slot] = b, half_step(dtype) * np.abs(b) + 8 * U * mag
    t = lambda x: None if x is None else torch.from_numpy(x)  # noqa: E731
    res = {"bias": (t(full), t(bound + least_half_step(dtype) + 1e-30))}
    if dt is not None:
        res["dtable"] = (t(dt), t(bt + 1e-30))
    if ds is not None:
        res["dslope"] = (t(ds), t(bs + 1e-30))
    return res
