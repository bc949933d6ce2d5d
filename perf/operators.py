"""The operators on point features that this library's speed is measured on: attention of each
group's center over the features of the group's points, its gradients, the groups turned round
(for each point the centers that gathered it), and the learned relative position bias alone.

With ``own`` false every operator is computed from elementary tensor operations in 32 bits; with
``own`` true by the library's public calls. Groups are what CAGQ gives: the K nearest stored points
of a center voxel's neighbourhood, or all of them as a ragged list.

Kinds of cases:

* ``forward`` - the attention of a network that answers;
* ``train``   - forward and backward, from the groups alone (the turned groups are made in the pass);
* ``lists``   - the groups turned round;
* ``bias``    - the relative position bias of every pair, and its gradient.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, kind, B, N, M, K, side, n_v, radius, centers, H, Hkv, D, dtype, cap, buckets, slope):
    return {"name": name, "kind": kind, "B": B, "N": N, "M": M, "K": K, "side": side, "n_v": n_v, "radius": radius,
            "centers": centers, "H": H, "Hkv": Hkv, "D": D, "dtype": dtype, "cap": cap, "buckets": buckets, "slope": slope}


def listed():
    return [
        # the least call: one small cloud, eight groups of eight points, where latency is everything
        _case("forward_few", "forward", 1, 1024, 8, 8, 40, 8, 1, "voxels", 4, 4, 16, "f32", 0.0, 16, False),
        # upsampling: every input point of the rooms looks up its coarse neighbours, some have none; odd head count and width
        _case("forward_upsample", "forward", 4, 2048, 8192, 16, 24, 32, 1, "points", 5, 5, 24, "f16", 20.0, 0, True),
        # the first layer of whole indoor scenes
        _case("forward_scenes", "forward", 4, 81920, 8192, 32, 168, 32, 1, "voxels", 8, 8, 32, "bf16", 30.0, 32, False),
        # a ragged batch that attends to whole contexts instead of K of their points
        _case("forward_contexts", "forward", 2, 30011, 3001, 0, 60, 32, 2, "voxels", 6, 6, 16, "bf16", 0.0, 24, True),
        # three centers with the longest contexts: work has to be split along the lists; heads share keys and values
        _case("forward_long", "forward", 1, 81920, 3, 0, 24, 64, 3, "voxels", 8, 2, 64, "f16", 50.0, 48, False),
        # training on a batch of objects, second layer, in 32 bits
        _case("train_objects", "train", 16, 1024, 128, 32, 40, 16, 1, "voxels", 4, 4, 16, "f32", 0.0, 16, True),
        # training, first layer of whole indoor scenes
        _case("train_scenes", "train", 4, 81920, 8192, 32, 168, 32, 1, "voxels", 8, 8, 32, "bf16", 30.0, 32, True),
        # training on room blocks over whole contexts, two query heads to a key head
        _case("train_contexts", "train", 8, 8192, 1024, 0, 64, 32, 1, "voxels", 8, 4, 32, "bf16", 20.0, 24, False),
        # the groups turned round: objects, and whole scenes
        _case("lists_objects", "lists", 16, 1024, 512, 32, 40, 16, 1, "voxels", 1, 1, 1, "f32", 0.0, 0, False),
        _case("lists_scenes", "lists", 4, 81920, 8192, 32, 168, 32, 1, "voxels", 1, 1, 1, "f32", 0.0, 0, False),
        # the relative position bias by itself, for scores of the user's own
        _case("bias_objects", "bias", 16, 1024, 128, 16, 40, 16, 1, "voxels", 4, 4, 1, "f32", 0.0, 16, True),
        _case("bias_scenes", "bias", 4, 81920, 8192, 32, 168, 32, 1, "voxels", 8, 8, 1, "bf16", 0.0, 32, True),
    ]


def _span(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["forward", "forward", "train", "train", "lists", "bias"])
        B, N = _span(rng, 1, 16), _span(rng, 200, 81920)
        M = _span(rng, 1, 8192)
        K = rng.choice([0, _span(rng, 1, 128), _span(rng, 8, 64)])
        if kind in ("lists", "bias"):
            K = K or _span(rng, 1, 128)  # of contexts, these outputs' sizes would go by the scene
        Hkv = _span(rng, 1, 12)
        H = Hkv * rng.choice([1, 1, 1, 2, 3])
        D = rng.choice([8, 16, 24, 32, 48, 64, 128, _span(rng, 1, 100)])
        c = _case("", kind, B, N, M, K, _span(rng, 10, 168), _span(rng, 4, 64), rng.choice([1, 1, 1, 2, 3]),
                  rng.choice(["voxels", "voxels", "points"]), H, Hkv, D if kind in ("forward", "train") else 1,
                  rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice([0.0, round(rng.uniform(5, 50), 1)]),
                  rng.choice([0, _span(rng, 2, 48), 32]), rng.random() < 0.5)
        if kind == "bias" and not c["buckets"] and not c["slope"]:
            continue
        # no dearer than the largest listed case: its pairs (contexts of surfaces, at most) and their features
        s = 2 * c["radius"] + 1
        longest = min(N, c["n_v"] * min(s ** 3, 3 * s * s), max(1, 6 * N * s * s // c["side"] ** 2) * 2)
        pairs = B * M * (min(K, longest) or longest)
        if B * N <= 4 * 81920 and B * M * s ** 3 <= 8 << 20 and pairs <= 1 << 20 and pairs * H * D <= 1 << 28 \
                and B * max(N, M) * H * D <= 84 << 20 and M <= 4 * N:
            del c["name"]
            return c


# ------------------------------------------------------------------ inputs

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _surfaces(B, N, g, dev):
    """Points on 16 axis-parallel rectangles of the unit cube per cloud, slightly noisy."""
    R = 16
    axis = torch.randint(0, 3, (B, R), generator=g, device=dev)
    lo = torch.rand((B, R, 3), generator=g, device=dev) * 0.6
    ext = 0.1 + 0.3 * torch.rand((B, R, 3), generator=g, device=dev)
    ext = ext.scatter(2, axis[..., None], 0.0)
    r = torch.randint(0, R, (B, N), generator=g, device=dev)[..., None].expand(B, N, 3)
    p = lo.gather(1, r) + torch.rand((B, N, 3), generator=g, device=dev) * ext.gather(1, r)
    p = p + 0.002 * torch.randn((B, N, 3), generator=g, device=dev)
    return p.clamp(0.0, 0.999)


def _groups(c, seed):
    """Points, centers and groups as the library's queries give them."""
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(1000003 * seed + 17)
    B, N, M, K, side = c["B"], c["N"], c["M"], c["K"], c["side"]
    V = side ** 3
    p = _surfaces(B, N, g, dev)
    cloud = torch.arange(B, device=dev)[:, None]
    strides = torch.tensor([1, side, side * side], device=dev)
    key = (((p * side).long().clamp(0, side - 1) * strides).sum(-1) + cloud * V).reshape(-1)
    key, order = torch.sort(key, stable=True)
    rank = torch.arange(B * N, device=dev) - torch.searchsorted(key, key)
    stored = rank < c["n_v"]
    key, order = key[stored], order[stored]
    occupied = torch.unique_consecutive(key)
    if c["centers"] == "voxels":  # random occupied voxels in ascending order, repeated where there are fewer than M
        lin = []
        for b in range(B):
            occ = occupied[(occupied >= b * V) & (occupied < (b + 1) * V)] - b * V
            some = torch.randperm(occ.numel(), generator=g, device=dev)[:M].sort().values
            lin.append(occ[some[torch.arange(M, device=dev) % some.numel()]])
        lin = torch.stack(lin)
        vox = torch.stack([lin % side, lin // side % side, lin // (side * side)], -1)
        near = (vox.float() + 0.5) / side
    else:  # given points, near the cloud and away from it
        near = p.gather(1, torch.randint(0, N, (B, M), generator=g, device=dev)[..., None].expand(B, M, 3))
        near = (near + torch.randn((B, M, 3), generator=g, device=dev) * (0.8 / side)).clamp(0.0, 0.999)
        vox = (near * side).long().clamp(0, side - 1)
    s = torch.arange(-c["radius"], c["radius"] + 1, device=dev)
    offs = torch.stack(torch.meshgrid(s, s, s, indexing="ij"), -1).reshape(-1, 3).flip(1)  # ascending linear ids
    cell = vox.reshape(B * M, 1, 3) + offs
    inside = ((cell >= 0) & (cell < side)).all(-1)
    lin = (cell * strides).sum(-1) + cloud.expand(B, M).reshape(-1, 1) * V
    lo, hi = torch.searchsorted(key, lin), torch.searchsorted(key, lin, right=True)
    cnt = torch.where(inside, hi - lo, 0).reshape(-1)
    cell = torch.repeat_interleave(torch.arange(cnt.numel(), device=dev), cnt)
    pos = torch.arange(cell.numel(), device=dev) - (cnt.cumsum(0) - cnt)[cell] + lo.reshape(-1)[cell]
    row, pt = cell // offs.shape[0], order[pos]
    length = cnt.reshape(B * M, -1).sum(1)
    if not K:
        off = torch.zeros(B * M + 1, dtype=torch.int64, device=dev)
        off[1:] = length.cumsum(0)
        return {"points": p, "centers": near.contiguous(), "idx": (pt % N).int(), "off": off, "n_valid": None}
    d2 = (p.reshape(-1, 3)[pt] - near.reshape(-1, 3)[row]).square().sum(-1)
    by = torch.argsort(d2, stable=True)
    by = by[torch.argsort(row[by], stable=True)]
    rank = torch.arange(by.numel(), device=dev) - (length.cumsum(0) - length)[row[by]]
    by, rank = by[rank < K], rank[rank < K]
    idx = torch.full((B * M, K), -1, dtype=torch.int64, device=dev)
    idx[row[by], rank] = pt[by] % N
    n = length.clamp(max=K)
    idx = torch.where(torch.arange(K, device=dev) < n[:, None], idx, idx[:, :1])  # further slots repeat the first
    if c["centers"] == "voxels":  # a group's center is the mean of its nodes
        xyz = p.gather(1, idx.reshape(B, M * K, 1).clamp(min=0).expand(B, M * K, 3)).reshape(B * M, K, 3)
        live = (torch.arange(K, device=dev) < n[:, None])[..., None]
        near = (torch.where(live, xyz, 0.0).sum(1) / n[:, None].clamp(min=1)).reshape(B, M, 3)
    return {"points": p, "centers": near.contiguous(), "idx": idx.int().reshape(B, M, K), "off": None,
            "n_valid": n.int().reshape(B, M)}


def prepare(case, seed):
    c = case
    st = _groups(c, seed)
    dev, dt = st["points"].device, DTYPES[c["dtype"]]
    g = torch.Generator(device=dev).manual_seed(7919 * seed + 5)
    B, N, M, H, Hkv, D = (c[x] for x in ("B", "N", "M", "H", "Hkv", "D"))

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    reach = (c["radius"] + 1.0) / c["side"]
    nb = c["buckets"]
    st["table"] = 0.5 * normal(3, nb, H) if nb else None
    st["edges"] = torch.linspace(-reach, reach, nb - 1, device=dev).repeat(3, 1).contiguous() if nb else None
    st["slope"] = -torch.exp2(-8.0 * torch.arange(1, H + 1, device=dev) / H) / reach if c["slope"] else None
    if c["kind"] in ("forward", "train"):
        st["q"] = (2.0 * normal(B, M, H, D)).to(dt)
        kv = normal(B, N, 2, Hkv, D).to(dt)  # one projection gives keys and values
        st["k"], st["v"] = kv[:, :, 0], kv[:, :, 1]
    if c["kind"] == "train":
        st["dout"] = normal(B, M, H, D).to(dt)
    if c["kind"] == "bias":
        shape = st["idx"].shape + (H,)
        st["dbias"] = normal(*shape).to(dt)
    st["case"] = dict(c)
    return st


# ------------------------------------------------------------------ the operators

def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return {"forward": _attend, "train": _train, "lists": _turn, "bias": _bias}[kind](state)


def _own(st):
    from paper_1912_02984_amd import cagq
    c = st["case"]
    groups = cagq.Groups(st["idx"], n_valid=st["n_valid"], off=st["off"], points=st["points"], centers=st["centers"])
    if c["kind"] == "lists":
        off, center = cagq.point_lists(groups)
        return {"off": off, "center": center}
    bias = None
    if c["buckets"] or c["slope"]:
        bias = cagq.RelativeBias(table=st["table"], edges=st["edges"], slope=st["slope"])
    if c["kind"] == "bias":
        b = cagq.relative_bias(groups, bias, dtype=DTYPES[c["dtype"]])
        dtable, dslope = cagq.relative_bias_backward(groups, bias, st["dbias"])
        return {"bias": b, "dtable": dtable, "dslope": dslope}
    out, lse = cagq.group_attention(groups, st["q"], st["k"], st["v"], bias=bias, cap=c["cap"])
    if c["kind"] == "forward":
        return {"out": out, "lse": lse}
    lists = cagq.point_lists(groups)
    grads = cagq.group_attention_backward(groups, lists, st["q"], st["k"], st["v"], lse, st["dout"], bias=bias, cap=c["cap"])
    return {"out": out, "lse": lse, **grads}


def _pairs(st):
    """Row (center) and point of every slot, over the batch, and which slots count (None: all)."""
    c, dev = st["case"], st["idx"].device
    B, N, M, K = c["B"], c["N"], c["M"], c["K"]
    if K:
        row = torch.arange(B * M, device=dev)[:, None].expand(B * M, K).reshape(-1)
        live = ((torch.arange(K, device=dev) < st["n_valid"].reshape(-1, 1)) & (st["idx"].reshape(-1, K) >= 0)).reshape(-1)
    else:
        row = torch.repeat_interleave(torch.arange(B * M, device=dev), st["off"].diff())
        live = None
    return row, st["idx"].reshape(-1).long().clamp(min=0) + row // M * N, live


def _over_rows(x, row, st):
    """Sums of the slots of each center."""
    c = st["case"]
    rows = c["B"] * c["M"]
    if c["K"]:
        return x.reshape(rows, c["K"], *x.shape[1:]).sum(1)
    return x.new_zeros((rows, *x.shape[1:])).index_add_(0, row, x)


def _most_of_rows(x, row, st):
    c = st["case"]
    rows = c["B"] * c["M"]
    if c["K"]:
        return x.reshape(rows, c["K"], -1).amax(1)
    return x.new_full((rows, x.shape[1]), -math.inf).scatter_reduce_(0, row[:, None].expand_as(x), x, "amax")


def _places(st, row, pt):
    """Bucket of each pair on each axis, and its distance."""
    d = st["points"].reshape(-1, 3)[pt] - st["centers"].reshape(-1, 3)[row]
    u = [torch.searchsorted(st["edges"][a], d[:, a].contiguous(), right=True) for a in range(3)] if st["table"] is not None else None
    x, y, z = d.unbind(1)
    return u, torch.sqrt((x * x + y * y) + z * z)


def _bias_of(st, u, dist):
    b = 0.0
    if u is not None:
        t = st["table"]
        b = t[0][u[0]] + t[1][u[1]] + t[2][u[2]]
    if st["slope"] is not None:
        b = b + st["slope"] * dist[:, None]
    return b


def _scores(st, row, pt, live):
    """Scores [T][H], the capped part's tanh, and the places."""
    c = st["case"]
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    q = st["q"].float().reshape(-1, Hkv, H // Hkv, D)[row]
    k = st["k"].float().reshape(-1, Hkv, 1, D)[pt]
    a = (q * k).sum(-1).reshape(-1, H) * D ** -0.5
    t = None
    if c["cap"]:
        t = torch.tanh(a / c["cap"])
        a = t * c["cap"]
    u, dist = _places(st, row, pt)
    s = a + _bias_of(st, u, dist)
    if live is not None:
        s = torch.where(live[:, None], s, -math.inf)
    return s, t, u, dist


def _softmax(st, s, row):
    m = _most_of_rows(s, row, st)
    safe = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(s - safe[row])
    total = _over_rows(p, row, st)
    lse = torch.where(total > 0, safe + torch.log(total), -math.inf)
    return p / torch.where(total > 0, total, 1.0)[row], lse


def _attend(st):
    c = st["case"]
    row, pt, live = _pairs(st)
    s, _, _, _ = _scores(st, row, pt, live)
    p, lse = _softmax(st, s, row)
    return _weigh(st, p, row, pt, lse)


def _weigh(st, p, row, pt, lse):
    c = st["case"]
    B, M, H, Hkv, D = (c[x] for x in ("B", "M", "H", "Hkv", "D"))
    v = st["v"].float().reshape(-1, Hkv, 1, D)[pt]
    o = _over_rows((p.reshape(-1, Hkv, H // Hkv, 1) * v).reshape(-1, H, D), row, st)
    return {"out": o.reshape(B, M, H, D).to(st["q"].dtype), "lse": lse.reshape(B, M, H)}


def _bias_gradient(st, ds, u, dist):
    out = {"dtable": None, "dslope": None}
    if u is not None:
        out["dtable"] = torch.stack([torch.zeros_like(st["table"][a]).index_add_(0, u[a], ds) for a in range(3)])
    if st["slope"] is not None:
        out["dslope"] = (ds * dist[:, None]).sum(0)
    return out


def _train(st):
    c = st["case"]
    B, N, M, H, Hkv, D = (c[x] for x in ("B", "N", "M", "H", "Hkv", "D"))
    R, dt = H // Hkv, st["q"].dtype
    row, pt, live = _pairs(st)
    s, t, u, dist = _scores(st, row, pt, live)
    p, lse = _softmax(st, s, row)
    out = _weigh(st, p, row, pt, lse)
    do = st["dout"].float().reshape(-1, Hkv, R, D)[row]
    dp = (do * st["v"].float().reshape(-1, Hkv, 1, D)[pt]).sum(-1).reshape(-1, H)
    ds = p * (dp - _over_rows(p * dp, row, st)[row])
    da = (ds * (1 - t * t) if t is not None else ds).reshape(-1, Hkv, R, 1) * D ** -0.5
    dv = torch.zeros((B * N, Hkv, D), device=do.device).index_add_(0, pt, (p.reshape(-1, Hkv, R, 1) * do).sum(2))
    del do
    q = st["q"].float().reshape(-1, Hkv, R, D)[row]
    dk = torch.zeros((B * N, Hkv, D), device=q.device).index_add_(0, pt, (da * q).sum(2))
    del q
    k = st["k"].float().reshape(-1, Hkv, 1, D)[pt]
    dq = _over_rows((da * k).reshape(-1, H, D), row, st)
    return {**out, "dq": dq.reshape(B, M, H, D).to(dt), "dk": dk.reshape(B, N, Hkv, D).to(dt),
            "dv": dv.reshape(B, N, Hkv, D).to(dt), **_bias_gradient(st, ds, u, dist)}


def _turn(st):
    c = st["case"]
    B, N, M = c["B"], c["N"], c["M"]
    row, pt, live = _pairs(st)
    slots = row.numel()
    if live is not None:
        row, pt = row[live], pt[live]
    key = torch.sort(pt * M + row % M).values
    off = torch.zeros(B * N + 1, dtype=torch.int64, device=pt.device)
    off[1:] = torch.bincount(pt, minlength=B * N).cumsum(0)
    center = torch.full((slots,), -1, dtype=torch.int32, device=pt.device)  # -1 behind the last list
    center[:key.numel()] = (key % M).int()
    return {"off": off, "center": center}


def _bias(st):
    row, pt, live = _pairs(st)
    u, dist = _places(st, row, pt)
    b = _bias_of(st, u, dist)
    g = st["dbias"].float().reshape(b.shape)
    if live is not None:
        b, g = torch.where(live[:, None], b, 0.0), torch.where(live[:, None], g, 0.0)
    return {"bias": b.to(st["dbias"].dtype).reshape(st["dbias"].shape), **_bias_gradient(st, g, u, dist)}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    st = _groups(c, 0)  # how many pairs there are, and how many points they touch
    row, pt, live = _pairs({**st, "case": c})
    pt = pt if live is None else pt[live]
    T, slots = pt.numel(), row.numel()
    U = torch.unique(pt).numel()
    B, N, M, H, Hkv, D = (c[x] for x in ("B", "N", "M", "H", "Hkv", "D"))
    E = 4 if c["dtype"] == "f32" else 2
    groups = 4 * T + (4 * B * M if c["K"] else 8 * (B * M + 1))
    if c["kind"] == "lists":
        return {"bytes": groups + 4 * T + 8 * (B * N + 1), "flops": 0}
    places = 12 * (U + B * M) if c["buckets"] or c["slope"] else 0
    if c["kind"] == "bias":
        return {"bytes": groups + places + (slots + T) * H * E, "flops": 2 * T * (10 + 4 * H)}
    rows, pts = B * M * H * D * E, Hkv * D * E
    forward = groups + places + 2 * rows + 2 * U * pts + 4 * B * M * H
    if c["kind"] == "forward":
        return {"bytes": forward, "flops": 4 * T * H * D}
    return {"bytes": forward + 2 * rows + 2 * B * N * pts, "flops": 14 * T * H * D}


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """The definition, center by center (in chunks of padded lists), gradients by differentiation."""
    st = prepare(case, seed)
    c = case
    B, N, M, K, H, Hkv, D = (c[x] for x in ("B", "N", "M", "K", "H", "Hkv", "D"))
    if c["kind"] == "lists":
        return None  # whole numbers: equal or not
    dev = st["points"].device
    idx = st["idx"].reshape(-1).long()
    if K:
        first, length = torch.arange(B * M, device=dev) * K, st["n_valid"].reshape(-1).long()
    else:
        first, length = st["off"][:-1], st["off"].diff()
    leaf = {}
    for n in ("q", "k", "v", "table", "slope"):
        if st.get(n) is not None:
            leaf[n] = st[n].double().contiguous().requires_grad_(c["kind"] != "forward")
    points, centers = st["points"].reshape(-1, 3), st["centers"].reshape(-1, 3)
    bias_out = torch.zeros((idx.numel(), H), dtype=torch.float64, device=dev)
    outs, lses = [], []
    order = torch.argsort(length)  # lists of like lengths together
    width = length[order].tolist()
    at = 0
    while at < B * M:
        n, most = 1, 1 << 25
        while at + n < B * M and n < 1 << 16 and 2 * n * max(1, width[min(at + 2 * n, B * M) - 1]) * H * D < most:
            n *= 2
        n = min(n, B * M - at)
        rows = order[at:at + n]
        L = max(1, width[at + n - 1])
        slot = first[rows, None] + torch.arange(L, device=dev)
        live = torch.arange(L, device=dev) < length[rows, None]
        slot = torch.where(live, slot, 0)
        i = idx[slot] if idx.numel() else torch.zeros_like(slot)
        live = live & (i >= 0)
        flat = torch.where(live, i, 0) + (rows // M)[:, None] * N
        d = points[flat] - centers[rows][:, None]  # 32 bits: the definition's own rounding
        b = torch.zeros((n, L, H), dtype=torch.float64, device=dev)
        if "table" in leaf:
            for a in range(3):
                u = (st["edges"][a] <= d[..., a, None]).sum(-1)
                b = b + leaf["table"][a][u]
        if "slope" in leaf:
            b = b + leaf["slope"] * d.double().norm(dim=-1, keepdim=True)
        if c["kind"] == "bias":
            b = torch.where(live[..., None], b, 0.0)
            g = torch.where(live[..., None], st["dbias"].reshape(-1, H)[slot].double(), 0.0)
            (b * g).sum().backward()
            bias_out[slot[live]] = b.detach()[live]
        else:
            kk = leaf["k"].reshape(-1, Hkv, D)[flat].repeat_interleave(H // Hkv, 2)
            vv = leaf["v"].reshape(-1, Hkv, D)[flat].repeat_interleave(H // Hkv, 2)
            s = (leaf["q"].reshape(-1, 1, H, D)[rows] * kk).sum(-1) / math.sqrt(D)
            s = c["cap"] * torch.tanh(s / c["cap"]) if c["cap"] else s
            s = torch.where(live[..., None], s + b, -math.inf)
            some = live.any(1)[:, None]
            lse = torch.where(some, torch.logsumexp(torch.where(some[..., None], s, 0.0), 1), -math.inf)
            w = torch.where(live[..., None], torch.exp(s - torch.where(some, lse, 0.0)[:, None]), 0.0)
            o = (w[..., None] * vv).sum(1)
            if c["kind"] == "train":
                (o * st["dout"].reshape(-1, H, D)[rows].double()).sum().backward()
            outs.append(o.detach())
            lses.append(lse.detach())
        at += n
    back = torch.argsort(order)
    grads = {"d" + n: leaf[n].grad if n in leaf else None for n in ("q", "k", "v", "table", "slope")}
    if c["kind"] == "bias":
        return {"bias": bias_out.reshape(st["dbias"].shape), "dtable": grads["dtable"], "dslope": grads["dslope"]}
    res = {"out": torch.cat(outs)[back].reshape(B, M, H, D), "lse": torch.cat(lses)[back].reshape(B, M, H)}
    return res if c["kind"] == "forward" else {**res, **grads}
