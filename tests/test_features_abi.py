"""The entry points on point features without a GPU: their refusals, before any
HIP call (pointers are never read), and their workspace sizes."""
import ctypes as C

import pytest

from paper_1912_02984_amd import cagq

INV, CAP, SMALL = cagq.ERR_INVALID_ARG, cagq.ERR_CAPACITY, cagq.ERR_WORKSPACE_TOO_SMALL
P = C.c_void_p(0x300000)
BIG = 1 << 40


def _groups(**kw):
    g = cagq.GroupsC(2, 100, 10, 8, 0x100000, 0x110000, None, 0, 0x120000, 0x130000)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _ragged(**kw):
    return _groups(**{**dict(K=0, n_valid=None, off=0x140000, idx_len=500), **kw})


def _attn(**kw):
    a = cagq.AttnC(1, 4, 2, 16, 0.25, 0.0, 0, 0, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _bias(table=0x150000, edges=0x160000, slope=None, buckets=8):
    return cagq.BiasC(table, edges, slope, buckets)


BAD_GROUPS = [
    dict(B=0), dict(N=0), dict(M=0), dict(K=-1), dict(B=65536, N=65536), dict(B=65536, M=65536), dict(idx=None),
    dict(idx=0x100002), dict(n_valid=0x110001), dict(off=0x140000), dict(idx_len=3), dict(B=1 << 15, M=1 << 15, K=1 << 20),
    dict(K=0), dict(K=0, n_valid=None, off=None, idx_len=5), dict(K=0, n_valid=None, off=0x140004, idx_len=5),
    dict(K=0, n_valid=None, off=0x140000, idx_len=-1), dict(K=0, n_valid=None, off=0x140000, idx_len=BIG + 1),
    dict(K=0, off=0x140000, idx_len=5),
]


@pytest.mark.parametrize("bad", BAD_GROUPS)
def test_bad_groups_are_refused(bad):
    L, g, a, b = cagq.lib(), _groups(**bad), _attn(), _bias()
    r = C.byref
    assert L.cagq_group_attention(r(g), r(a), None, P, P, P, P, P, P, BIG, None) == INV
    assert L.cagq_point_lists(r(g), P, P, BIG, P, BIG, None) == INV
    assert L.cagq_group_attention_backward(r(g), r(a), None, P, P, BIG, P, P, P, P, P, P, P, P, None, None, P, BIG,
                                           None) == INV
    assert L.cagq_relative_bias(r(g), r(b), 4, 0, P, None) == INV
    assert L.cagq_relative_bias_backward(r(g), r(b), 4, 0, P, P, None, P, BIG, None) == INV


@pytest.mark.parametrize("bad", [
    dict(dtype=-1), dict(dtype=3), dict(H=0), dict(H=129, Hkv=129), dict(Hkv=0), dict(Hkv=3), dict(Hkv=8), dict(D=0),
    dict(D=257), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")),
    dict(cap=float("inf")), dict(cap=3e38), dict(cap=1e-39), dict(cap=1e-30, scale=1e9), dict(q_row=63), dict(k_row=31), dict(v_row=-32), dict(k_row=1 << 32)])
def test_bad_attention_shapes_are_refused(bad):
    L, g, a = cagq.lib(), _groups(), _attn(**bad)
    r, n = C.byref, C.c_size_t()
    assert L.cagq_group_attention(r(g), r(a), None, P, P, P, P, P, P, BIG, None) == INV
    assert L.cagq_group_attention_backward(r(g), r(a), None, P, P, BIG, P, P, P, P, P, P, P, P, None, None, P, BIG,
                                           None) == INV
    assert L.cagq_group_attention_workspace(r(g), r(a), None, 0, r(n)) == INV


@pytest.mark.parametrize("bad", [
    dict(buckets=65), dict(buckets=-1), dict(buckets=0), dict(table=None), dict(edges=None), dict(table=0x150001),
    dict(edges=0x160002), dict(slope=0x170002)])
def test_bad_biases_are_refused(bad):
    L, g, a, b = cagq.lib(), _groups(), _attn(), _bias(**bad)
    r = C.byref
    assert L.cagq_group_attention(r(g), r(a), r(b), P, P, P, P, P, P, BIG, None) == INV
    assert L.cagq_group_attention_backward(r(g), r(a), r(b), P, P, BIG, P, P, P, P, P, P, P, P, None, None, P, BIG,
                                           None) == INV
    assert L.cagq_relative_bias(r(g), r(b), 4, 0, P, None) == INV


def test_pointers_that_are_missing_or_not_aligned():
    L, g, a, b = cagq.lib(), _groups(), _attn(), _bias()
    r, odd = C.byref, C.c_void_p(0x300001)
    for i in range(5):
        for p in (None, odd):
            args = [P, P, P, P, P]
            args[i] = p
            if i == 4 and p is None:
                continue  # lse may be missing
            assert L.cagq_group_attention(r(g), r(a), None, *args, P, BIG, None) == INV, (i, p)
    for i in (0, 3, 4, 5, 6, 7, 8, 9, 10):  # pt_off, (pt_center, capacity,) q, k, v, lse, dout, dq, dk, dv
        for p in (None, odd):
            args = [P, P, 160, P, P, P, P, P, P, P, P]
            args[i] = p
            assert L.cagq_group_attention_backward(r(g), r(a), None, *args, None, None, P, BIG, None) == INV, (i, p)
    back = lambda off=P, center=P, cap=160, dt=None, ds=None, bias=None: L.cagq_group_attention_backward(  # noqa: E731
        r(g), r(a), bias, off, center, cap, P, P, P, P, P, P, P, P, dt, ds, P, BIG, None)
    assert back(center=None) == INV and back(cap=-1) == INV and back(center=odd) == INV
    assert back(dt=P) == INV and back(ds=P) == INV  # the gradient of a part that is not there
    assert back(dt=P, ds=P, bias=r(b)) == INV and back(dt=odd, bias=r(b)) == INV
    # a bias needs the places
    for miss in ("points", "centers"):
        h = _groups(**{miss: None})
        assert L.cagq_group_attention(r(h), r(a), r(b), P, P, P, P, P, P, BIG, None) == INV
        assert L.cagq_relative_bias(r(h), r(b), 4, 0, P, None) == INV
    assert L.cagq_point_lists(r(g), None, P, BIG, P, BIG, None) == INV
    assert L.cagq_point_lists(r(g), odd, P, BIG, P, BIG, None) == INV
    assert L.cagq_point_lists(r(g), P, None, 160, P, BIG, None) == INV
    assert L.cagq_point_lists(r(g), P, P, 159, P, BIG, None) == CAP
    assert L.cagq_point_lists(r(_ragged()), P, P, 499, P, BIG, None) == CAP
    for H, dt, out in ((0, 0, P), (129, 0, P), (4, 3, P), (4, 0, None), (4, 1, odd)):
        assert L.cagq_relative_bias(r(g), r(b), H, dt, out, None) == INV
    assert L.cagq_relative_bias(r(g), None, 4, 0, P, None) == INV
    assert L.cagq_relative_bias_backward(r(g), r(b), 4, 0, P, None, None, P, BIG, None) == INV
    assert L.cagq_relative_bias_backward(r(g), r(b), 4, 0, None, P, None, P, BIG, None) == INV
    assert L.cagq_relative_bias_backward(r(g), r(b), 4, 0, P, P, P, P, BIG, None) == INV  # no slope
    for f in (L.cagq_group_attention,):
        assert f(None, r(a), None, P, P, P, P, P, P, BIG, None) == INV
        assert f(r(g), None, None, P, P, P, P, P, P, BIG, None) == INV


def test_workspaces():
    L, a, b = cagq.lib(), _attn(), _bias()
    r, n = C.byref, C.c_size_t()
    assert L.cagq_group_attention_workspace(r(_groups()), r(a), None, 0, r(n)) == 0 and n.value == 0
    assert L.cagq_group_attention_workspace(r(_groups()), r(a), None, 2, r(n)) == INV
    assert L.cagq_group_attention_workspace(r(_groups()), r(a), None, 0, None) == INV
    cases = []
    long = _ragged(B=1, M=2, idx_len=20000)  # few long lists: parts
    assert L.cagq_group_attention_workspace(r(long), r(a), None, 0, r(n)) == 0 and n.value > 0
    cases.append((n.value, lambda ws, s: L.cagq_group_attention(r(long), r(a), None, P, P, P, P, P, ws, s, None)))
    assert L.cagq_group_attention_workspace(r(_groups()), r(a), r(b), 1, r(n)) == 0
    cases.append((n.value, lambda ws, s: L.cagq_group_attention_backward(
        r(_groups()), r(a), r(b), P, P, 160, P, P, P, P, P, P, P, P, P, None, ws, s, None)))
    assert L.cagq_point_lists_workspace(r(_groups()), r(n)) == 0
    cases.append((n.value, lambda ws, s: L.cagq_point_lists(r(_groups()), P, P, 160, ws, s, None)))
    assert L.cagq_relative_bias_workspace(r(_groups()), r(b), 4, r(n)) == 0
    cases.append((n.value, lambda ws, s: L.cagq_relative_bias_backward(r(_groups()), r(b), 4, 0, P, P, None, ws, s,
                                                                       None)))
    for need, call in cases:
        assert need > 0
        assert call(P, need - 1) == SMALL
        assert call(None, need) == INV
        assert call(C.c_void_p(0x300080), need) == INV
