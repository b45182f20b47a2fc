"""Host validation of the calls that change a cache's pages (CPU only: nothing is enqueued)."""
import ctypes

import pytest
import torch

from paper_2607_22586_amd import binding as bd
from test_abi import FAKE, lib  # noqa: F401
from test_cache_refusals import ODD, pages

BAD4 = ctypes.c_void_p(0x10002)


def shape(B=2, Hkv=3, d=64):
    return bd.Shape(B, 0, Hkv, 0, 0, d)


def hold(lib, s=None, p=None, refs=FAKE, rows=FAKE, missing=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.mmshiftkv_cache_hold(ctypes.byref(s or shape()), ctypes.byref(p or pages()), refs, rows, missing, ws,
                                    nbytes, None)


def fork(lib, s=None, p=None, refs=FAKE, src=FAKE, lens=FAKE, missing=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.mmshiftkv_cache_fork(ctypes.byref(s or shape()), ctypes.byref(p or pages()), refs, src, lens, missing,
                                    ws, nbytes, None)


def compact(lib, s=None, p=None, refs=FAKE, lens=FAKE, idx=FAKE, counts=FAKE, n=5, missing=FAKE, ws=FAKE,
            nbytes=1 << 40):
    return lib.mmshiftkv_cache_compact(ctypes.byref(s or shape()), ctypes.byref(p or pages()), refs, lens, idx, counts,
                                       n, missing, ws, nbytes, None)


@pytest.mark.parametrize("call", [hold, fork, compact])
@pytest.mark.parametrize("bad,code", [
    (dict(s=shape(B=0)), bd.MMSKV_EINVAL), (dict(s=shape(B=70000)), bd.MMSKV_EINVAL),
    (dict(s=shape(Hkv=0)), bd.MMSKV_EINVAL), (dict(s=shape(d=0)), bd.MMSKV_EINVAL),
    (dict(s=shape(d=96)), bd.MMSKV_EUNSUPPORTED), (dict(p=pages(k=None)), bd.MMSKV_EINVAL),
    (dict(p=pages(table=None)), bd.MMSKV_EINVAL), (dict(p=pages(v_scale=None)), bd.MMSKV_EINVAL),
    (dict(p=pages(page=24)), bd.MMSKV_EUNSUPPORTED), (dict(p=pages(dtype=bd.MMSKV_F32)), bd.MMSKV_EUNSUPPORTED),
    (dict(refs=None), bd.MMSKV_EINVAL), (dict(refs=BAD4), bd.MMSKV_EINVAL), (dict(missing=None), bd.MMSKV_EINVAL),
    (dict(missing=BAD4), bd.MMSKV_EINVAL), (dict(ws=None), bd.MMSKV_EWORKSPACE), (dict(ws=ODD), bd.MMSKV_EWORKSPACE),
    (dict(s=shape(B=65535), p=pages(max_pages=1 << 13, page=16)), bd.MMSKV_EUNSUPPORTED)])
def test_common_refusals(lib, call, bad, code):  # noqa: F811
    assert call(lib, **bad) == code


@pytest.mark.parametrize("call,bad", [
    (hold, dict(rows=None)), (hold, dict(rows=BAD4)), (fork, dict(src=None)), (fork, dict(src=BAD4)),
    (fork, dict(lens=None)), (fork, dict(lens=BAD4)), (compact, dict(lens=None)), (compact, dict(lens=BAD4)),
    (compact, dict(idx=None)), (compact, dict(idx=BAD4)), (compact, dict(counts=None)), (compact, dict(counts=BAD4)),
    (compact, dict(n=0)), (compact, dict(n=-1))])
def test_own_refusals(lib, call, bad):  # noqa: F811
    assert call(lib, **bad) == bd.MMSKV_EINVAL


def test_limits_and_workspace(lib):  # noqa: F811
    assert compact(lib, n=(1 << 27) + 1) == bd.MMSKV_EUNSUPPORTED
    size = lambda B, Hkv, n, m: lib.mmshiftkv_cache_book_workspace(ctypes.byref(shape(B, Hkv)), n, m)  # noqa: E731
    need = size(2, 3, 10, 4)
    assert need > 0
    for call in (hold, fork, compact):
        assert call(lib, nbytes=need - 1) == bd.MMSKV_EWORKSPACE
    grow = (1, 2, 3, 10, 63, 64, 65, 1000, 4096, 60000)
    for f in (lambda x: size(x, 2, 100, 9), lambda x: size(2, x, 100, 9), lambda x: size(2, 2, x, 9),
              lambda x: size(2, 2, 100, x)):
        got = [f(x) for x in grow]
        assert got == sorted(got) and got[0] > 0
    assert size(0, 1, 1, 1) == size(1, 0, 1, 1) == size(1, 1, 0, 1) == size(1, 1, 1, 0) == size(65535, 1, 1, 1 << 13) == 0


def test_binding_checks():
    lens = torch.zeros((2, 3), dtype=torch.int32)
    cache = bd.PagedCache.pool(2, 3, 7, 4, 64, torch.int8, 16, "cpu")
    assert tuple(cache.k.shape) == (7, 3, 16, 64) and int(cache.table.max()) == -1 and int(cache.refs.sum()) == 0
    own = bd.PagedCache.empty(2, 3, 40, 64, page=16, device="cpu")
    assert own.refs.tolist() == [1] * 6 and own.k_scale is None
    with pytest.raises(ValueError):                # host tensors
        bd.cache_hold(cache, lens)
    for bad in (lens.long(), lens[:, :2], lens[:1], lens.t().contiguous().t()):
        with pytest.raises(ValueError):
            bd.cache_hold(cache, bad)
        with pytest.raises(ValueError):
            bd.cache_fork(cache, torch.zeros(2, dtype=torch.int32), bad)
        with pytest.raises(ValueError):
            bd.cache_compact(cache, bad, torch.zeros((2, 3, 5), dtype=torch.int32), lens)
    with pytest.raises(ValueError):
        bd.cache_fork(cache, torch.zeros(3, dtype=torch.int32), lens)
    with pytest.raises(ValueError):
        bd.cache_compact(cache, lens, torch.zeros((2, 2, 5), dtype=torch.int32), lens)
    bare = bd.PagedCache(cache.k, cache.v, cache.k_scale, cache.v_scale, cache.table)
    with pytest.raises(ValueError):                # pages that are not counted
        bd.cache_hold(bare, lens)
