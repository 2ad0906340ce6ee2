"""Host checks of a block's attention: every bad argument is refused before any GPU call."""
import ctypes

import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2508_04405_amd as fq
from paper_2508_04405_amd.binding import _Cache, _Sequences

P16 = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1008)          # 8-byte aligned only
OFF = ctypes.c_void_p(0x1002)          # not even 4
BIG = 1 << 40
INF, NAN = float("inf"), float("nan")
EINVAL, ESHAPE, EALIGN, EWORKSPACE = -1, -2, -3, -5


def caller(f, fine):
    return lambda **kw: f(*(dict(fine, **kw)[n] for n in fine), None)


def test_rotate_refusals():
    call = caller(fq.load().flexq_rotate_heads, dict(
        x=P16, xs=1536, M=4, heads=8, kv=2, D=128, positions=P16, freq=P16, rot=128, interleaved=0, gq=None, gk=None, eps=1e-5,
        out=ctypes.c_void_p(0x2000), os=1280))
    for kw in (dict(x=None), dict(positions=None), dict(freq=None), dict(out=None), dict(M=0), dict(M=-1), dict(heads=0), dict(kv=0),
               dict(interleaved=2), dict(gq=P16, eps=0.0), dict(gk=P16, eps=NAN), dict(gk=P16, eps=INF), dict(out=P16)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(D=96), dict(D=256), dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(xs=1272), dict(os=1272), dict(xs=1540),
               dict(os=1284), dict(heads=600), dict(M=2**31 - 1), dict(heads=2**31 - 1)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(x=ODD), dict(out=ODD), dict(gq=ODD), dict(gk=ODD), dict(positions=OFF), dict(freq=OFF)):
        assert call(**kw) == EALIGN, kw


def test_prompt_refusals():
    call = caller(fq.load().flexq_prompt_attention, dict(
        q=P16, qs=1024, k=P16, ks=256, v=P16, vs=256, starts=P16, S=2, M=10, heads=8, kv=2, D=128, scale=0.1, out=P16, os=1024))
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(starts=None), dict(out=None), dict(S=0), dict(M=0), dict(heads=0),
               dict(kv=0), dict(kv=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=INF), dict(scale=NAN), dict(scale=1e5)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(D=80), dict(D=32), dict(qs=1016), dict(ks=248), dict(vs=248), dict(os=1016), dict(qs=1028), dict(ks=260), dict(vs=260),
               dict(os=1028), dict(heads=1024), dict(ks=1 << 24), dict(vs=1 << 24), dict(S=(1 << 20) + 1), dict(M=1 << 29),
               dict(M=1 << 27, kv=8)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(out=ODD), dict(starts=OFF)):
        assert call(**kw) == EALIGN, kw


def test_cache_sizes():
    lib = fq.load()
    page, recent = lib.flexq_cache_page_bytes, lib.flexq_cache_recent_bytes
    assert page(1, 64, 16) == 2304
    for kv, D, p in ((1, 64, 16), (8, 128, 64), (40, 128, 1024), (3, 64, 32)):
        exact = p // 16 * kv * (32 * D + 4)
        assert exact <= page(kv, D, p) < exact + 256 and page(kv, D, p) % 256 == 0
        assert recent(kv, D) == kv * 32 * D * 2 * 2
    for bad in ((0, 64, 16), (1, 96, 16), (1, 64, 8), (1, 64, 48), (1, 64, 2048), (1, 64, 0), (1024, 128, 16), (1, 64, -16)):
        assert page(*bad) == 0, bad
    assert recent(0, 64) == 0 and recent(1, 32) == 0 and recent(1024, 128) == 0
    size = lib.flexq_cache_attention_workspace_bytes
    assert size(1, 1, 8, 8, 128) > 0 and size(1 << 20, 64, 64, 8, 64) > 0
    for bad in ((0, 1, 8, 8, 128), (1, 0, 8, 8, 128), (1, 1, 0, 8, 128), (1, 1, 8, 0, 128), (1, 1, 8, 3, 128), (1, 1, 8, 8, 96),
                (1, 1, 1024, 8, 128)):
        assert size(*bad) == 0, bad


CACHE = dict(kv_heads=2, head_dim=128, page=64, pages=10, slots=3, codes=0x1000, recent=0x1000)
SEQS = dict(count=3, max_pages=4, starts=0x1000, lengths=0x1000, table=0x1000, slots=None)
BAD_CACHE = [(dict(kv_heads=0), EINVAL), (dict(pages=0), EINVAL), (dict(slots=0), EINVAL), (dict(codes=None), EINVAL),
             (dict(recent=None), EINVAL), (dict(head_dim=96), ESHAPE), (dict(page=24), ESHAPE), (dict(page=2048), ESHAPE),
             (dict(kv_heads=1024), ESHAPE), (dict(codes=0x1008), EALIGN), (dict(recent=0x1008), EALIGN)]
BAD_SEQS = [(dict(count=0), EINVAL), (dict(max_pages=0), EINVAL), (dict(starts=None), EINVAL), (dict(lengths=None), EINVAL),
            (dict(table=None), EINVAL), (dict(count=(1 << 20) + 1), ESHAPE), (dict(max_pages=(1 << 24) + 1), ESHAPE),
            (dict(starts=0x1002), EALIGN), (dict(lengths=0x1002), EALIGN), (dict(table=0x1002), EALIGN), (dict(slots=0x1002), EALIGN)]


def check_structs(run):
    for kw, status in BAD_CACHE:
        assert run(dict(CACHE, **kw), SEQS) == status, kw
    for kw, status in BAD_SEQS:
        assert run(CACHE, dict(SEQS, **kw)) == status, kw


@pytest.mark.parametrize("name", ["flexq_cache_append", "flexq_cache_read"])
def test_append_and_read_refusals(name):
    f = getattr(fq.load(), name)

    def call(cache=CACHE, seqs=SEQS, M=20, k=P16, ks=256, v=P16, vs=264):
        return f(ctypes.byref(_Cache(**cache)), ctypes.byref(_Sequences(**seqs)), M, k, ks, v, vs, None)

    check_structs(lambda c, s: call(c, s))
    assert f(None, ctypes.byref(_Sequences(**SEQS)), 20, P16, 256, P16, 256, None) == EINVAL
    assert f(ctypes.byref(_Cache(**CACHE)), None, 20, P16, 256, P16, 256, None) == EINVAL
    for kw in (dict(M=0), dict(k=None), dict(v=None)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(ks=248), dict(vs=248), dict(ks=260), dict(vs=260), dict(M=(1 << 28) + 1), dict(M=1 << 28)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(k=ODD), dict(v=ODD)):
        assert call(**kw) == EALIGN, kw


def test_cached_attention_refusals():
    f = fq.load().flexq_cache_attention
    size = fq.load().flexq_cache_attention_workspace_bytes

    def call(cache=CACHE, seqs=SEQS, M=20, heads=8, q=P16, qs=1024, scale=0.1, out=P16, os=1024, ws=P16, wsb=BIG):
        return f(ctypes.byref(_Cache(**cache)), ctypes.byref(_Sequences(**seqs)), M, heads, q, qs, scale, out, os, ws, wsb, None)

    check_structs(lambda c, s: call(c, s))
    for kw in (dict(M=0), dict(heads=0), dict(heads=7), dict(q=None), dict(out=None), dict(scale=0.0), dict(scale=-0.5), dict(scale=NAN),
               dict(scale=1e6)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(qs=1016), dict(os=1016), dict(qs=1028), dict(os=1028), dict(heads=1024), dict(M=1 << 28, heads=8)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(q=ODD), dict(out=ODD), dict(ws=ODD)):
        assert call(**kw) == EALIGN, kw
    assert call(ws=None) == EWORKSPACE and call(wsb=size(20, 3, 8, 2, 128) - 1) == EWORKSPACE


def test_the_binding_refuses_tensors_the_kernels_would_misread():
    z, h = torch.zeros, torch.float16
    i = torch.int32
    for call in (lambda: fq.rotate_heads(z((2, 256), dtype=h), 1, 1, 128, z(2, dtype=i), z(64)),                 # on the CPU
                 lambda: fq.prompt_attention(z((2, 128), dtype=h), z((2, 128), dtype=h), z((2, 128), dtype=h), 1, 1, z(2, dtype=i)),
                 lambda: fq.Sequences(z(2, dtype=i), z(1, dtype=i), z((1, 4), dtype=i)),
                 lambda: fq.Cache(4, 24, 1, 64, 1, device="cpu"), lambda: fq.Cache(0, 16, 1, 64, 1, device="cpu")):
        with pytest.raises(fq.FlexQError):
            call()


def test_plain_forms():
    """The oracle's own corner cases, by hand."""
    y, _ = ref.attend(np.ones((2, 4)), np.zeros((3, 4)), np.arange(12.0).reshape(3, 4), 0, 1.0)
    assert np.allclose(y, [[0, 1, 2, 3], [2, 3, 4, 5]])
    y, off = ref.attend(np.ones((2, 4)), np.zeros((3, 4)), np.ones((3, 4)), -1, 1.0)
    assert not y[0].any() and not off[0].any() and np.allclose(y[1], 1.0)
    x = np.array([[1.0, 0, 0, 2.0] + [0] * 12]).astype(np.float16)
    y, _ = ref.rotate(x, 1, 0, 16, np.array([1]), np.full(8, np.pi / 2, np.float32), interleaved=True)
    assert np.allclose(y[0, :4], [0, 1, -2, 0], atol=1e-6)
    y, _ = ref.rotate(x, 1, 0, 16, np.array([1]), np.full(8, np.pi / 2, np.float32))
    assert np.allclose(y[0, [0, 8, 3, 11]], [0, 1, 0, 2], atol=1e-6)
    rows = np.zeros((17, 2), np.float16)
    rows[3], rows[16] = [127, -63.6], [0.3, 0.3]
    s = ref.stored(rows, 1)
    assert s[3].tolist() == [127, -64] and np.allclose(s[16], rows[16].astype(float))
