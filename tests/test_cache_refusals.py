"""Host validation of the paged-cache calls, their workspace contract and the
binding's checks (CPU only: every call is rejected before anything is enqueued)."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2607_22586_amd import binding as bd
from test_abi import FAKE, lib  # noqa: F401

ODD = ctypes.c_void_p(0x10008)
ST = bd.Strides(1024 * 64, 1024 * 64, 64)


def pages(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, table=FAKE, n_pages=10, page=64, max_pages=4,
             dtype=bd.MMSKV_E4M3)
    a.update(kw)
    return bd.Pages(*[a[f[0]] for f in bd.Pages._fields_])


def shape(B=1, Hq=4, Hkv=1, T=1024, d=64):
    return bd.Shape(B, Hq, Hkv, T, 0, d)


def write(lib, s=None, p=None, k=FAKE, v=FAKE, dtype=1, ks=ST, vs=ST, idx=None, n=8):
    return lib.mmshiftkv_cache_write(ctypes.byref(s or shape()), ctypes.byref(p or pages()), k, v, dtype,
                                     ctypes.byref(ks), ctypes.byref(vs), idx, FAKE, FAKE, n, None)


def read(lib, s=None, p=None, lens=FAKE, dtype=1, k=FAKE, v=FAKE, ks=ST, vs=ST):
    return lib.mmshiftkv_cache_read(ctypes.byref(s or shape()), ctypes.byref(p or pages()), lens, dtype, k,
                                    ctypes.byref(ks), v, ctypes.byref(vs), None)


def attend(lib, s=None, p=None, q=FAKE, qs=ST, lens=FAKE, n=8, causal=1, out=FAKE, os=ST, ws=FAKE, nbytes=1 << 40):
    return lib.mmshiftkv_chunk_attention(ctypes.byref(s or shape()), ctypes.byref(p or pages()), q, ctypes.byref(qs),
                                         None, lens, n, causal, out, ctypes.byref(os), ws, nbytes, None)


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("bad,code", [
    (dict(k=None), bd.MMSKV_EINVAL), (dict(v=None), bd.MMSKV_EINVAL), (dict(table=None), bd.MMSKV_EINVAL),
    (dict(k=ODD), bd.MMSKV_EINVAL), (dict(v=ODD), bd.MMSKV_EINVAL), (dict(k_scale=None), bd.MMSKV_EINVAL),
    (dict(v_scale=None), bd.MMSKV_EINVAL), (dict(dtype=bd.MMSKV_I8, v_scale=None), bd.MMSKV_EINVAL),
    (dict(n_pages=0), bd.MMSKV_EINVAL), (dict(max_pages=0), bd.MMSKV_EINVAL), (dict(page=0), bd.MMSKV_EINVAL),
    (dict(page=8), bd.MMSKV_EUNSUPPORTED), (dict(page=48), bd.MMSKV_EUNSUPPORTED),
    (dict(page=2048), bd.MMSKV_EUNSUPPORTED), (dict(max_pages=1 << 25), bd.MMSKV_EUNSUPPORTED),
    (dict(dtype=bd.MMSKV_F32), bd.MMSKV_EUNSUPPORTED), (dict(dtype=4), bd.MMSKV_EINVAL),
    (dict(dtype=-1), bd.MMSKV_EINVAL)])
def test_pages_rejected(lib, call, bad, code):  # noqa: F811
    assert call(lib, p=pages(**bad)) == code


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("bad,code", [
    (dict(B=0), bd.MMSKV_EINVAL), (dict(B=70000), bd.MMSKV_EINVAL), (dict(Hkv=0), bd.MMSKV_EINVAL),
    (dict(T=0), bd.MMSKV_EINVAL), (dict(d=0), bd.MMSKV_EINVAL), (dict(d=96), bd.MMSKV_EUNSUPPORTED),
    (dict(d=256), bd.MMSKV_EUNSUPPORTED)])
def test_shapes_rejected(lib, call, bad, code):  # noqa: F811
    assert call(lib, s=shape(**bad)) == code


def test_write_rejects(lib):  # noqa: F811
    assert write(lib, k=None) == bd.MMSKV_EINVAL
    assert write(lib, v=None) == bd.MMSKV_EINVAL
    assert write(lib, k=ODD) == bd.MMSKV_EINVAL
    assert write(lib, dtype=bd.MMSKV_E4M3) == bd.MMSKV_EINVAL
    assert write(lib, ks=bd.Strides(0, 0, 3)) == bd.MMSKV_EINVAL
    assert write(lib, vs=bd.Strides(-64, 64, 64)) == bd.MMSKV_EINVAL
    assert write(lib, n=0) == bd.MMSKV_EINVAL
    assert write(lib, n=1025) == bd.MMSKV_EINVAL                      # more rows than tokens
    assert write(lib, idx=ctypes.c_void_p(0x10002), n=2000) == bd.MMSKV_EINVAL
    assert write(lib, idx=FAKE, n=(1 << 27) + 1) == bd.MMSKV_EUNSUPPORTED
    # scales are not asked for where none are kept (the call stops at its source)
    assert write(lib, p=pages(dtype=bd.MMSKV_BF16, k_scale=None, v_scale=None), k=None) == bd.MMSKV_EINVAL


def test_read_rejects(lib):  # noqa: F811
    assert read(lib, lens=None) == bd.MMSKV_EINVAL
    assert read(lib, k=None) == bd.MMSKV_EINVAL
    assert read(lib, v=ODD) == bd.MMSKV_EINVAL
    assert read(lib, dtype=bd.MMSKV_I8) == bd.MMSKV_EINVAL
    assert read(lib, ks=bd.Strides(0, 0, 3)) == bd.MMSKV_EINVAL
    assert read(lib, vs=bd.Strides(64, 64, 0)) == bd.MMSKV_EINVAL     # rows over each other
    assert read(lib, s=shape(B=2), ks=bd.Strides(0, 64, 64)) == bd.MMSKV_EINVAL
    assert read(lib, s=shape(T=(1 << 27) + 1)) == bd.MMSKV_EUNSUPPORTED


def test_attention_rejects(lib):  # noqa: F811
    need = lib.mmshiftkv_chunk_attention_workspace(ctypes.byref(shape()), 8)
    assert need > 0
    assert attend(lib, q=None) == bd.MMSKV_EINVAL
    assert attend(lib, q=ODD) == bd.MMSKV_EINVAL
    assert attend(lib, qs=bd.Strides(0, 0, 3)) == bd.MMSKV_EINVAL
    assert attend(lib, lens=None) == bd.MMSKV_EINVAL
    assert attend(lib, out=None) == bd.MMSKV_EINVAL
    assert attend(lib, os=bd.Strides(64, 64, 0)) == bd.MMSKV_EINVAL
    assert attend(lib, os=bd.Strides(64, 0, 64)) == bd.MMSKV_EINVAL
    assert attend(lib, n=0) == bd.MMSKV_EINVAL
    assert attend(lib, n=1 << 21) == bd.MMSKV_EUNSUPPORTED
    assert attend(lib, s=shape(B=65535, Hq=129, Hkv=129)) == bd.MMSKV_EUNSUPPORTED
    assert attend(lib, causal=2) == bd.MMSKV_EINVAL
    assert attend(lib, s=shape(Hq=5, Hkv=2)) == bd.MMSKV_EINVAL
    assert attend(lib, ws=None) == bd.MMSKV_EWORKSPACE
    assert attend(lib, ws=ODD) == bd.MMSKV_EWORKSPACE
    assert attend(lib, nbytes=need - 1) == bd.MMSKV_EWORKSPACE


def test_attention_workspace_never_falls(lib):  # noqa: F811
    """A workspace for the largest B, T and n serves smaller ones."""
    size = lambda B, T, n, Hq=28, Hkv=4, d=128: lib.mmshiftkv_chunk_attention_workspace(  # noqa: E731
        ctypes.byref(bd.Shape(B, Hq, Hkv, T, 0, d)), n)
    grow = [1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 64, 100, 127, 129, 250, 255, 256, 257, 511, 513, 1000, 2047, 4096,
            5000, 16384, 16385, 32768, 100000]
    for other in (1, 2, 7, 64, 500):
        for f in (lambda x: size(x, 50 * other, 1), lambda x: size(x, 50 * other, other),
                  lambda x: size(1, x, other), lambda x: size(other, x, 1), lambda x: size(1, 32 * other, x),
                  lambda x: size(other, 30000, x)):
            got = [f(x) for x in grow if x < 60000]
            assert got == sorted(got) and got[0] > 0
    assert size(1, 100, 0) == 0 and size(1, 100, 1, d=96) == 0 and size(1, 100, 1, Hq=27) == 0


def test_binding_checks():
    f = torch.zeros((1, 1, 4, 64))
    cache = bd.PagedCache.empty(1, 1, 10, 64, device="cpu")
    with pytest.raises(ValueError):                # host tensors
        bd.cache_write(cache, f, f)
    with pytest.raises(ValueError):
        bd.cache_read(cache, torch.zeros((1, 1), dtype=torch.int32), 4)
    with pytest.raises(ValueError):
        bd.chunk_attention(f.bfloat16(), cache, torch.zeros((1, 1), dtype=torch.int32))
    assert tuple(cache.table.shape) == (1, 1) and cache.k_scale is None
    eight = bd.PagedCache.empty(2, 3, 100, 128, torch.int8, 32, "cpu")
    assert tuple(eight.k.shape) == (8, 3, 32, 128) and tuple(eight.k_scale.shape) == (8, 3, 32)
    with pytest.raises(TypeError):
        bd.PagedCache(f, f, None, None, cache.table).c_pages()
    with pytest.raises(ValueError):
        bd.PagedCache(eight.k, eight.v, None, eight.v_scale, eight.table).c_pages()
    with pytest.raises(ValueError):
        bd.PagedCache(eight.k, eight.v, eight.k_scale, eight.v_scale, eight.table.long()).c_pages()


def test_bench_lists_the_paged_mode():
    bench = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "bench.py")
    r = subprocess.run([sys.executable, bench, "--help"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "--paged" in r.stdout
    r = subprocess.run([sys.executable, bench, "--paged", "fp4"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 2 and r.stdout.strip() == ""
