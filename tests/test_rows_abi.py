"""Host checks of the operators whose rows choose their own weights: every bad argument is refused before any GPU call."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2508_04405_amd as fq
import rows_reference as ref
from paper_2508_04405_amd.binding import _Routing

P16 = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1008)          # 8-byte aligned only
OFF = ctypes.c_void_p(0x1002)          # not even 4
BIG = 1 << 40
EINVAL, ESHAPE, EALIGN, EWORKSPACE = -1, -2, -3, -5


def test_group_rows_refusals():
    f = fq.load().flexq_group_rows
    size = fq.load().flexq_group_rows_workspace_bytes
    assert size(1, 1) > 0 and size(1 << 20, 512) > 0 and size(1 << 20, 512) < 1 << 20
    assert size(0, 1) == 0 and size(1, 0) == 0 and size(1, 513) == 0
    ok = dict(ids=P16, rows=2000, count=8, order=P16, offsets=P16, ws=P16, wsb=BIG)

    def call(**kw):
        a = dict(ok, **kw)
        return f(a["ids"], a["rows"], a["count"], a["order"], a["offsets"], a["ws"], a["wsb"], None)

    for kw in (dict(ids=None), dict(order=None), dict(offsets=None), dict(rows=0), dict(rows=-1), dict(count=0)):
        assert call(**kw) == EINVAL, kw
    assert call(count=513) == ESHAPE and call(rows=(1 << 28) + 1) == ESHAPE and size((1 << 28) + 1, 8) == 0
    for kw in (dict(ids=OFF), dict(order=OFF), dict(offsets=OFF), dict(ws=ODD)):
        assert call(**kw) == EALIGN, kw
    assert call(ws=None) == EWORKSPACE and call(wsb=size(2000, 8) - 1) == EWORKSPACE


def test_route_refusals():
    f = fq.load().flexq_route
    size = fq.load().flexq_route_workspace_bytes
    assert size(1, 8, 2) > 0 and size(0, 8, 2) == 0 and size(1, 513, 2) == 0 and size(1, 8, 9) == 0 and size(1, 64, 17) == 0
    fine = dict(k=2, score=0, groups=4, top_groups=2, group_top=2, renormalise=1, scale=1.0, bias=None)
    ok = dict(logits=P16, half=0, M=100, E=8, experts=P16, weights=P16, order=P16, offsets=P16, ws=P16, wsb=BIG)

    def call(routing=None, **kw):
        a = dict(ok, **kw)
        r = _Routing(**dict(fine, **(routing or {})))
        return f(a["logits"], a["half"], a["M"], a["E"], ctypes.byref(r), a["experts"], a["weights"], a["order"], a["offsets"],
                 a["ws"], a["wsb"], None)

    for kw in (dict(logits=None), dict(experts=None), dict(weights=None), dict(M=0), dict(E=0), dict(half=2), dict(order=None),
               dict(offsets=None)):
        assert call(**kw) == EINVAL, kw
    assert f(P16, 0, 100, 8, None, P16, P16, P16, P16, P16, BIG, None) == EINVAL
    for r in (dict(k=0), dict(k=9), dict(score=2), dict(groups=0), dict(groups=3), dict(groups=16), dict(top_groups=0),
              dict(top_groups=5), dict(group_top=0), dict(group_top=3), dict(k=5), dict(scale=0.0), dict(scale=-1.0),
              dict(scale=float("inf")), dict(scale=float("nan"))):
        assert call(r) == EINVAL, r
    assert call(dict(k=17, groups=1, top_groups=1), E=64) == EINVAL
    assert call(dict(groups=128, top_groups=4), E=256) == EINVAL           # at most 64 groups
    assert call(dict(groups=1, top_groups=1), E=513) == ESHAPE
    assert call(dict(groups=1, top_groups=1, k=16), E=64, M=1 << 27) == ESHAPE and size(1 << 27, 64, 16) == 0
    for kw in (dict(logits=ODD), dict(experts=OFF), dict(weights=OFF), dict(order=OFF), dict(offsets=OFF), dict(ws=ODD)):
        assert call(**kw) == EALIGN, kw
    assert call(dict(bias=0x1002)) == EALIGN
    assert call(ws=None) == EWORKSPACE and call(wsb=16) == EWORKSPACE
    assert call(M=33, ws=None) == EWORKSPACE                               # from there on two launches


def test_expert_linear_refusals():
    f = fq.load().flexq_expert_linear
    ok = dict(packed=P16, E=4, group=0, xq=P16, sx=P16, rows=10, order=P16, offsets=P16, slots=20, k=2, scatter=0, N=64, K=256, y=P16)

    def call(**kw):
        return f(*(dict(ok, **kw)[n] for n in ok), None)

    for kw in (dict(packed=None), dict(xq=None), dict(sx=None), dict(order=None), dict(offsets=None), dict(y=None), dict(E=0),
               dict(rows=0), dict(slots=0), dict(k=-1), dict(k=17, rows=1, slots=17), dict(scatter=2), dict(group=64), dict(N=0),
               dict(K=0), dict(slots=21), dict(k=0), dict(k=3)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(E=513), dict(N=40), dict(K=200), dict(K=65536 + 128), dict(rows=1 << 20, slots=1 << 20, k=1, K=65536),
               dict(N=131072, K=65536)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(packed=ODD), dict(xq=ODD), dict(y=ODD), dict(order=OFF), dict(offsets=OFF)):
        assert call(**kw) == EALIGN, kw


def test_combine_refusals():
    f = fq.load().flexq_expert_combine
    ok = dict(y=P16, experts=P16, weights=P16, add=None, M=4, k=2, N=64, out=P16)

    def call(**kw):
        return f(*(dict(ok, **kw)[n] for n in ok), None)

    for kw in (dict(y=None), dict(experts=None), dict(weights=None), dict(out=None), dict(M=0), dict(k=0), dict(k=17), dict(N=0)):
        assert call(**kw) == EINVAL, kw
    assert call(N=40) == ESHAPE
    for kw in (dict(y=ODD), dict(out=ODD), dict(add=ODD), dict(experts=OFF), dict(weights=OFF)):
        assert call(**kw) == EALIGN, kw


def test_adapters_refusals():
    f = fq.load().flexq_adapters
    size = fq.load().flexq_adapters_workspace_bytes
    assert size(1, 1, 16, 128) > 0 and size(0, 1, 16, 128) == 0 and size(1, 1, 24, 128) == 0 and size(1, 1, 16, 100) == 0
    assert size(1, 513, 16, 128) == 0 and size(1, 1, 272, 128) == 0
    ok = dict(a=P16, b=P16, scale=P16, L=4, R=16, x=P16, order=P16, offsets=P16, M=10, N=64, K=256, y=P16, out=P16, ws=P16, wsb=BIG)

    def call(**kw):
        return f(*(dict(ok, **kw)[n] for n in ok), None)

    for kw in (dict(a=None), dict(b=None), dict(scale=None), dict(x=None), dict(order=None), dict(offsets=None), dict(y=None),
               dict(out=None), dict(L=0), dict(R=0), dict(M=0), dict(N=0), dict(K=0)):
        assert call(**kw) == EINVAL, kw
    assert call(M=1 << 24, N=1 << 30) == ESHAPE                            # more workgroups than a launch has
    for kw in (dict(L=513), dict(R=8), dict(R=24), dict(R=272), dict(N=40), dict(K=200), dict(K=65536 + 128), dict(M=(1 << 24) + 1)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(a=ODD), dict(b=ODD), dict(x=ODD), dict(y=ODD), dict(out=ODD), dict(scale=OFF), dict(order=OFF),
               dict(offsets=OFF), dict(ws=ODD)):
        assert call(**kw) == EALIGN, kw
    assert call(ws=None) == EWORKSPACE and call(wsb=size(10, 4, 16, 256) - 1) == EWORKSPACE


def test_the_binding_refuses_tensors_the_kernels_would_misread():
    """Wrong types, shapes, strides, and tensors that are not on the current device."""
    z = torch.zeros
    with pytest.raises(fq.FlexQError):
        fq.group_rows(z(4, dtype=torch.int32), 2)                           # on the CPU
    with pytest.raises(fq.FlexQError):
        fq.route_experts(z((4, 8), dtype=torch.bfloat16), 2)
    with pytest.raises(fq.FlexQError):
        fq.route_experts(z((4, 8)), 2, score="other")
    with pytest.raises(fq.FlexQError):
        fq.expert_linear(z((2, 100), dtype=torch.uint8), 33, 128, z((4, 128), dtype=torch.int8), z(4), z(4), z(3))
    with pytest.raises(fq.FlexQError):
        fq.adapters(z((1, 16, 128), dtype=torch.float16), z((1, 64, 16), dtype=torch.float16), z(1), z((2, 128)), z(2), z(2), z((2, 64)))


def test_plain_forms():
    """The oracle's own corner cases, by hand."""
    order, offsets = ref.group_rows(np.array([2, -1, 0, 2, 7, 0]), 3)
    assert order.tolist() == [2, 5, 0, 3, 1, 4] and offsets.tolist() == [0, 2, 2, 4]
    l = np.array([[0.0, 0.0, 1.0, -np.inf], [-np.inf] * 4, [np.nan, 3.0, 3.0, 2.0]])
    experts, weights = ref.route(l, 2, "softmax")
    assert experts.tolist() == [[2, 0], [-1, -1], [1, 2]]
    assert np.allclose(weights[0], [np.e / (1 + np.e), 1 / (1 + np.e)]) and not weights[1].any() and np.allclose(weights[2], 0.5)
    experts, _ = ref.route(np.array([[5.0, -9.0, 3.0, 3.0]]), 1, "sigmoid", groups=2, top_groups=1, group_top=2)
    assert experts.tolist() == [[2]]                                        # the pair is worth more than the best alone
    experts, _ = ref.route(np.array([[1.0, 0.0]]), 1, "sigmoid", bias=np.array([0.0, 0.3]))
    assert experts.tolist() == [[1]]
