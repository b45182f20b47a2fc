"""Host validation of the table of shared rows (CPU only: nothing is enqueued)."""
import ctypes

import pytest
import torch

from paper_2607_22586_amd import binding as bd
from test_abi import FAKE, lib  # noqa: F401
from test_cache_refusals import pages

BAD4 = ctypes.c_void_p(0x10002)


def shape(B=6, Hkv=1, d=64):
    return bd.Shape(B, 0, Hkv, 0, 0, d)


def call(lib, s=None, p=None, lens=FAKE, shared=FAKE, groups=2, out=FAKE):
    return lib.mmshiftkv_shared_table(ctypes.byref(s or shape()), ctypes.byref(p or pages()), lens, shared, groups, out,
                                      None)


@pytest.mark.parametrize("bad,code", [
    (dict(s=shape(B=0)), bd.MMSKV_EINVAL), (dict(s=shape(B=70000)), bd.MMSKV_EINVAL),
    (dict(s=shape(Hkv=0)), bd.MMSKV_EINVAL), (dict(s=shape(d=0)), bd.MMSKV_EINVAL),
    (dict(s=shape(d=96)), bd.MMSKV_EUNSUPPORTED), (dict(p=pages(table=None)), bd.MMSKV_EINVAL),
    (dict(p=pages(page=24)), bd.MMSKV_EUNSUPPORTED), (dict(lens=None), bd.MMSKV_EINVAL), (dict(lens=BAD4), bd.MMSKV_EINVAL),
    (dict(shared=None), bd.MMSKV_EINVAL), (dict(shared=BAD4), bd.MMSKV_EINVAL), (dict(out=None), bd.MMSKV_EINVAL),
    (dict(out=BAD4), bd.MMSKV_EINVAL), (dict(groups=0), bd.MMSKV_EINVAL), (dict(groups=4), bd.MMSKV_EINVAL),
    (dict(groups=12), bd.MMSKV_EINVAL)])
def test_refusals(lib, bad, code):  # noqa: F811
    assert call(lib, **bad) == code


def test_binding_checks():
    cache = bd.PagedCache.empty(4, 2, 40, 64, page=16, device="cpu")
    lens = torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(ValueError):                # host tensors
        bd.shared_table(cache, lens, lens[:2].contiguous())
