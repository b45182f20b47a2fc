"""Host validation of the attention of whole prompts (CPU only: nothing is enqueued)."""
import ctypes

import pytest
import torch

from paper_2607_22586_amd import binding as bd
from test_abi import FAKE, lib  # noqa: F401
from test_cache_refusals import ODD, ST

BAD4 = ctypes.c_void_p(0x10002)


def call(lib, B=1, Hq=4, Hkv=2, T=100, d=64, q=FAKE, k=FAKE, v=FAKE, out=FAKE, qs=ST, ks=ST, vs=ST, os=ST, starts=FAKE,
         n_seq=3, causal=1, lse=None):
    ref = ctypes.byref
    return lib.mmshiftkv_prompt_attention(ref(bd.Shape(B, Hq, Hkv, T, 0, d)), q, ref(qs), k, ref(ks), v, ref(vs), starts,
                                          n_seq, causal, out, ref(os), lse, None)


@pytest.mark.parametrize("bad,code", [
    (dict(B=0, starts=None), bd.MMSKV_EINVAL), (dict(Hq=3), bd.MMSKV_EINVAL), (dict(T=0), bd.MMSKV_EINVAL),
    (dict(d=0), bd.MMSKV_EINVAL), (dict(d=96), bd.MMSKV_EUNSUPPORTED), (dict(d=256), bd.MMSKV_EUNSUPPORTED),
    (dict(q=None), bd.MMSKV_EINVAL), (dict(k=None), bd.MMSKV_EINVAL), (dict(v=None), bd.MMSKV_EINVAL),
    (dict(out=None), bd.MMSKV_EINVAL), (dict(q=ODD), bd.MMSKV_EINVAL), (dict(k=ODD), bd.MMSKV_EINVAL),
    (dict(v=ODD), bd.MMSKV_EINVAL), (dict(out=ODD), bd.MMSKV_EINVAL), (dict(qs=bd.Strides(0, 0, 3)), bd.MMSKV_EINVAL),
    (dict(ks=bd.Strides(0, 4, 64)), bd.MMSKV_EINVAL), (dict(vs=bd.Strides(0, -64, 64)), bd.MMSKV_EINVAL),
    (dict(os=bd.Strides(64, 0, 64)), bd.MMSKV_EINVAL), (dict(os=bd.Strides(64, 64, 0)), bd.MMSKV_EINVAL),
    (dict(causal=2), bd.MMSKV_EINVAL), (dict(B=2), bd.MMSKV_EINVAL), (dict(n_seq=0), bd.MMSKV_EINVAL),
    (dict(starts=BAD4), bd.MMSKV_EINVAL), (dict(lse=BAD4), bd.MMSKV_EINVAL),
    (dict(T=1 << 22), bd.MMSKV_EUNSUPPORTED), (dict(ks=bd.Strides(0, 0, 1 << 28)), bd.MMSKV_EUNSUPPORTED),
    (dict(vs=bd.Strides(0, 0, 1 << 30)), bd.MMSKV_EUNSUPPORTED),
    (dict(B=1000, T=1 << 20, Hq=2, starts=None), bd.MMSKV_EUNSUPPORTED), (dict(B=65535, Hq=129, Hkv=129, starts=None), bd.MMSKV_EUNSUPPORTED)])
def test_refusals(lib, bad, code):  # noqa: F811
    assert call(lib, **bad) == code


def test_binding_checks():
    q, k = torch.zeros((1, 4, 10, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 10, 64), dtype=torch.bfloat16)
    cuts = torch.tensor([0, 10], dtype=torch.int32)
    for bad in (dict(), dict(starts=cuts)):        # host tensors
        with pytest.raises(ValueError):
            bd.prompt_attention(q, k, k, **bad)
    with pytest.raises(ValueError):
        bd.prompt_attention(q, k, k[:, :, :9])
