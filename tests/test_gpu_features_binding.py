"""The binding of the operators on point features: devices, streams and records."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_1912_02984_amd import cagq
from tests import features_ref as F
from tests.test_gpu_features import _bias, _dev

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _made(seed=1):
    rng = np.random.default_rng(seed)
    c = F.rand_groups(rng, 2, 40, 9, 6)
    g, b = c.groups(cagq, DEV), _bias(F.rand_bias(rng, 2, 5, True))
    q, k, v, dout = (_dev(rng.normal(size=(2, n, 2, 8)).astype(np.float32)) for n in (9, 40, 40, 9))
    return SimpleNamespace(rng=rng, g=g, b=b, q=q, k=k, v=v, dout=dout)


def _calls(m):
    """Every entry point on the groups m.g with the bias m.b, as functions of the stream."""
    out, lse = cagq.group_attention(m.g, m.q, m.k, m.v, bias=m.b)
    lists = cagq.point_lists(m.g)
    dbias = torch.ones((2, 9, 6, 2), device=DEV)
    return [lambda s: cagq.group_attention(m.g, m.q, m.k, m.v, bias=m.b, stream=s),
            lambda s: cagq.point_lists(m.g, stream=s),
            lambda s: cagq.group_attention_backward(m.g, lists, m.q, m.k, m.v, lse, m.dout, bias=m.b, stream=s),
            lambda s: cagq.relative_bias(m.g, m.b, stream=s),
            lambda s: cagq.relative_bias_backward(m.g, m.b, dbias, stream=s)]


def test_calls_with_another_device_current_are_refused(monkeypatch):
    """Groups of one device, made while it was the current one, in a call while another is."""
    m = _made()
    calls, here = _calls(m), torch.cuda.current_stream()
    monkeypatch.setattr(cagq, "_cur_device", lambda: 1)
    for stream in (here, None):
        for n, f in enumerate(calls):
            with pytest.raises(ValueError, match="current device"):
                f(stream)
                print("not refused:", n, stream)


def test_streams_of_another_device_are_refused():
    for f in _calls(_made()):
        with pytest.raises(ValueError, match="stream"):
            f(SimpleNamespace(cuda_stream=0, device_index=1, device=torch.device("cuda:1")))


def test_a_bias_follows_what_is_learned():
    """A learned table and slope that are given other storage after the record was made: the calls read what they
    hold now (the old storage is kept here), and refuse what no longer fits."""
    m = _made(2)
    keep, calls = [], _calls(m)

    def flat(x):
        x = list(x.values()) if isinstance(x, dict) else [x] if torch.is_tensor(x) else list(x)
        return [t for t in x if t is not None]

    def swap(t, value):
        keep.append(t.data)
        t.data = value

    b = m.b
    first = flat(calls[0](None))
    for t, value in ((b.table, b.table * 2 + 1), (b.slope, b.slope - 1)):
        swap(t, value)
        m.b = cagq.RelativeBias(b.table.clone(), b.edges, b.slope.clone())
        want = [flat(f(None)) for f in _calls(m)]
        m.b = b
        got = [flat(f(None)) for f in _calls(m)]
        for x, y in zip(got, want):
            assert len(x) == len(y) and all(torch.equal(s, t) for s, t in zip(x, y))
    assert not torch.equal(got[0][0], first[0])
    calls = _calls(m)
    del calls[1]  # the lists take no bias
    for t, value in ((b.table, b.table[:, :, :1].contiguous()), (b.table, b.table.cpu()), (b.slope, b.slope.repeat(2))):
        old = t.data
        swap(t, value)
        for f in calls:
            with pytest.raises(ValueError):
                f(None)
        t.data = old
        calls[0](None)
