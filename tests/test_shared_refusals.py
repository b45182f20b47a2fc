"""Host validation of the attention over a shared prefix and its workspace contract (CPU only: nothing is enqueued)."""
import ctypes

import pytest
import torch

from paper_2607_22586_amd import binding as bd
from test_abi import FAKE, lib  # noqa: F401
from test_cache_refusals import ODD, ST, pages

BAD4 = ctypes.c_void_p(0x10002)


def shape(B=6, Hq=4, Hkv=1, T=200, d=64):
    return bd.Shape(B, Hq, Hkv, T, 0, d)


def call(lib, s=None, p=None, q=FAKE, qs=ST, q_counts=None, lens=FAKE, shared=FAKE, table=FAKE, groups=2, shared_T=100,
         n=8, causal=1, out=FAKE, os=ST, ws=FAKE, nbytes=1 << 40):
    ref = ctypes.byref
    return lib.mmshiftkv_shared_attention(ref(s or shape()), ref(p or pages()), q, ref(qs), q_counts, lens, shared, table,
                                          groups, shared_T, n, causal, out, ref(os), ws, nbytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(s=shape(B=0)), bd.MMSKV_EINVAL), (dict(s=shape(Hq=3, Hkv=2)), bd.MMSKV_EINVAL),
    (dict(s=shape(T=0)), bd.MMSKV_EINVAL), (dict(s=shape(d=96)), bd.MMSKV_EUNSUPPORTED),
    (dict(p=pages(k=None)), bd.MMSKV_EINVAL), (dict(p=pages(page=8)), bd.MMSKV_EUNSUPPORTED),
    (dict(p=pages(k_scale=None)), bd.MMSKV_EINVAL), (dict(q=None), bd.MMSKV_EINVAL), (dict(q=ODD), bd.MMSKV_EINVAL),
    (dict(qs=bd.Strides(0, 0, 3)), bd.MMSKV_EINVAL), (dict(q_counts=BAD4), bd.MMSKV_EINVAL),
    (dict(lens=None), bd.MMSKV_EINVAL), (dict(lens=BAD4), bd.MMSKV_EINVAL), (dict(shared=None), bd.MMSKV_EINVAL),
    (dict(shared=BAD4), bd.MMSKV_EINVAL), (dict(table=None), bd.MMSKV_EINVAL), (dict(table=BAD4), bd.MMSKV_EINVAL),
    (dict(groups=0), bd.MMSKV_EINVAL), (dict(groups=4), bd.MMSKV_EINVAL), (dict(groups=12), bd.MMSKV_EINVAL),
    (dict(shared_T=0), bd.MMSKV_EINVAL), (dict(n=0), bd.MMSKV_EINVAL), (dict(causal=3), bd.MMSKV_EINVAL),
    (dict(out=None), bd.MMSKV_EINVAL), (dict(out=ODD), bd.MMSKV_EINVAL),
    (dict(os=bd.Strides(64, 64, 0)), bd.MMSKV_EINVAL), (dict(n=1 << 19), bd.MMSKV_EUNSUPPORTED),
    (dict(s=shape(B=65535, Hq=129, Hkv=129), groups=1), bd.MMSKV_EUNSUPPORTED),
    (dict(s=shape(B=60000, Hq=140, Hkv=70), groups=60000, n=1), bd.MMSKV_EUNSUPPORTED),
    (dict(s=shape(B=60000, Hq=28, Hkv=1), groups=60000, n=41), bd.MMSKV_EUNSUPPORTED),
    (dict(ws=None), bd.MMSKV_EWORKSPACE), (dict(ws=ODD), bd.MMSKV_EWORKSPACE)])
def test_refusals(lib, bad, code):  # noqa: F811
    assert call(lib, **bad) == code


def test_workspace(lib):  # noqa: F811
    size = lambda B, T, n, G, Hq=28, Hkv=4, d=128: lib.mmshiftkv_shared_attention_workspace(  # noqa: E731
        ctypes.byref(bd.Shape(B, Hq, Hkv, T, 0, d)), G, n)
    need = lib.mmshiftkv_shared_attention_workspace(ctypes.byref(shape()), 2, 8)
    assert need > 0 and call(lib, nbytes=need - 1) == bd.MMSKV_EWORKSPACE
    grow = [1, 2, 3, 5, 8, 15, 16, 17, 33, 64, 100, 129, 255, 257, 512, 1000, 4096, 16384, 32768]
    for each in (1, 4, 31):
        for f in (lambda x: size(each * x, 5000, 1, x), lambda x: size(each * 2, x, 3, 2), lambda x: size(each, 32 * 999, x, 1)):
            got = [f(x) for x in grow if x * each < 60000]
            assert got == sorted(got) and got[0] > 0
    assert size(6, 100, 1, 4) == size(6, 100, 0, 2) == size(6, 100, 1, 0) == 0


def test_binding_checks():
    q, lens = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16), torch.zeros((2, 1), dtype=torch.int32)
    cache = bd.PagedCache.empty(2, 1, 40, 64, page=16, device="cpu")
    with pytest.raises(ValueError):                # host tensors
        bd.shared_attention(q, cache, lens, lens[:1].contiguous())
