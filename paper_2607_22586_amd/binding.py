"""ctypes binding of libmmshiftkv (C ABI in include/mmshiftkv.h).

Argument marshalling only: every step runs in the library's HIP kernels on
the GPU.  Tensors are torch tensors on a ROCm device; the library enqueues on
the current torch stream of that device.  If the shared library is missing
or cannot be loaded, every call raises -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmmshiftkv.so")

MMSKV_OK, MMSKV_EINVAL, MMSKV_EUNSUPPORTED, MMSKV_EWORKSPACE, MMSKV_EHIP, MMSKV_ESCRATCH = 0, -1, -2, -3, -4, -5
NOALLOC_SCRATCH_BYTES = 32 << 20
MMSKV_F32, MMSKV_BF16, MMSKV_E4M3, MMSKV_I8 = 0, 1, 2, 3
MMSKV_VOTE, MMSKV_MASS = 0, 1

EXPORTED = ("mmshiftkv_build_proxies", "mmshiftkv_score_workspace", "mmshiftkv_score",
            "mmshiftkv_score_lse", "mmshiftkv_score_lse_blocks", "mmshiftkv_score_lse_merge",
            "mmshiftkv_score_mass", "mmshiftkv_select_workspace",
            "mmshiftkv_select_topk", "mmshiftkv_select_tau", "mmshiftkv_select_vote", "mmshiftkv_select_pick",
            "mmshiftkv_gather_kv", "mmshiftkv_status_string",
            "mmshiftkv_version", "mmshiftkv_hidden_stats_workspace", "mmshiftkv_hidden_stats",
            "mmshiftkv_hidden_proxies", "mmshiftkv_project_proxies", "mmshiftkv_decode_workspace",
            "mmshiftkv_decode_check", "mmshiftkv_window_rows", "mmshiftkv_shape_scores",
            "mmshiftkv_score_noalloc", "mmshiftkv_cache_write", "mmshiftkv_cache_read",
            "mmshiftkv_chunk_attention_workspace", "mmshiftkv_chunk_attention",
            "mmshiftkv_cache_book_workspace", "mmshiftkv_cache_hold", "mmshiftkv_cache_fork",
            "mmshiftkv_cache_compact", "mmshiftkv_prompt_attention", "mmshiftkv_shared_attention_workspace",
            "mmshiftkv_shared_attention", "mmshiftkv_shared_table")


class Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("T", ctypes.c_int32), ("W", ctypes.c_int32), ("d", ctypes.c_int32)]


class HShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("D", ctypes.c_int32)]


class Strides(ctypes.Structure):
    _fields_ = [("sb", ctypes.c_int64), ("sh", ctypes.c_int64), ("st", ctypes.c_int64)]


class Params(ctypes.Structure):
    _fields_ = [("P", ctypes.c_int32), ("G", ctypes.c_int32), ("gamma", ctypes.c_double),
                ("tau", ctypes.c_double), ("lambda_", ctypes.c_double),
                ("std_ddof", ctypes.c_int32), ("layer", ctypes.c_int32),
                ("seed", ctypes.c_uint64), ("mode", ctypes.c_int32), ("keep_last", ctypes.c_int32)]


class Pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("table", ctypes.c_void_p), ("n_pages", ctypes.c_int32),
                ("page", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class MMShiftKVError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__("%s failed: %s (%d)" % (fn, status_string(status), status))
        self.status = status


_lib = None


def load_library(path: str | None = None):
    """Load libmmshiftkv.so (raises if it is missing: there is no fallback)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError("libmmshiftkv.so is not built (%s); run __graft_entry__.build() or "
                           "python -m paper_2607_22586_amd.build" % p)
    lib = ctypes.CDLL(p)
    V, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    PS, PP, PT = ctypes.POINTER(Shape), ctypes.POINTER(Params), ctypes.POINTER(Strides)
    lib.mmshiftkv_build_proxies.argtypes = [PS, PP, V, I32, PT, V, V, V, V, V, V, V, V]
    lib.mmshiftkv_score_workspace.argtypes = [PS, PP]
    lib.mmshiftkv_score_workspace.restype = SZ
    lib.mmshiftkv_score.argtypes = [PS, PP, V, V, V, I32, PT, V, V, V, V, SZ, V]
    lib.mmshiftkv_score_lse.argtypes = [PS, PP, V, V, V, I32, PT, V, SZ, V]
    lib.mmshiftkv_score_lse_blocks.argtypes = [PS, PP, V, V, V, I32, PT, V, SZ, V]
    lib.mmshiftkv_score_lse_merge.argtypes = [PS, PP, V, V, V, I32, PT, V, SZ, V]
    lib.mmshiftkv_score_mass.argtypes = [PS, PP, V, V, V, I32, PT, V, V, V, V, SZ, V]
    lib.mmshiftkv_score_noalloc.argtypes = [PS, PP, V, V, V, I32, PT, V, V, V, V]
    lib.mmshiftkv_select_workspace.argtypes = [PS, PP]
    lib.mmshiftkv_select_workspace.restype = SZ
    lib.mmshiftkv_select_topk.argtypes = [PS, PP, V, V, V, V, I32, I32, V, V, V, V, SZ, V]
    lib.mmshiftkv_select_tau.argtypes = [PS, PP, V, V, SZ, V]
    lib.mmshiftkv_select_vote.argtypes = [PS, PP, V, V, V, V, SZ, V]
    lib.mmshiftkv_select_pick.argtypes = [PS, PP, V, I32, I32, V, V, V, SZ, V]
    lib.mmshiftkv_gather_kv.argtypes = [PS, V, V, I32, PT, PT, V, V, I32, V, V, V]
    PH = ctypes.POINTER(HShape)
    lib.mmshiftkv_hidden_stats_workspace.argtypes = [PH]
    lib.mmshiftkv_hidden_stats_workspace.restype = SZ
    lib.mmshiftkv_hidden_stats.argtypes = [PH, I32, V, I32, I64, I64, V, V, SZ, V]
    lib.mmshiftkv_hidden_proxies.argtypes = [PH, PP, V, V, V]
    lib.mmshiftkv_project_proxies.argtypes = [PH, I32, I32, I32, V, V, V, V, V, V]
    lib.mmshiftkv_decode_workspace.argtypes = [PS, I32]
    lib.mmshiftkv_decode_workspace.restype = SZ
    lib.mmshiftkv_decode_check.argtypes = [PS, I32, V, V, I32, PT, V, V, I32, V, V, V, V, V, SZ, V]
    lib.mmshiftkv_window_rows.argtypes = [PS, I32, V, I32, PT, V, V, V]
    lib.mmshiftkv_shape_scores.argtypes = [PS, I32, I32, I32, I32, V, V, V]
    PG = ctypes.POINTER(Pages)
    lib.mmshiftkv_cache_write.argtypes = [PS, PG, V, V, I32, PT, PT, V, V, V, I32, V]
    lib.mmshiftkv_cache_read.argtypes = [PS, PG, V, I32, V, PT, V, PT, V]
    lib.mmshiftkv_chunk_attention_workspace.argtypes = [PS, I32]
    lib.mmshiftkv_chunk_attention_workspace.restype = SZ
    lib.mmshiftkv_chunk_attention.argtypes = [PS, PG, V, PT, V, V, I32, I32, V, PT, V, SZ, V]
    lib.mmshiftkv_shared_attention_workspace.argtypes = [PS, I32, I32]
    lib.mmshiftkv_shared_attention_workspace.restype = SZ
    lib.mmshiftkv_shared_attention.argtypes = [PS, PG, V, PT, V, V, V, V, I32, I32, I32, I32, V, PT, V, SZ, V]
    lib.mmshiftkv_shared_table.argtypes = [PS, PG, V, V, I32, V, V]
    lib.mmshiftkv_prompt_attention.argtypes = [PS, V, PT, V, PT, V, PT, V, I32, I32, V, PT, V, V]
    lib.mmshiftkv_cache_book_workspace.argtypes = [PS, I32, I32]
    lib.mmshiftkv_cache_book_workspace.restype = SZ
    lib.mmshiftkv_cache_hold.argtypes = [PS, PG, V, V, V, V, SZ, V]
    lib.mmshiftkv_cache_fork.argtypes = [PS, PG, V, V, V, V, V, SZ, V]
    lib.mmshiftkv_cache_compact.argtypes = [PS, PG, V, V, V, V, I32, V, V, SZ, V]
    lib.mmshiftkv_status_string.argtypes = [ctypes.c_int]
    lib.mmshiftkv_status_string.restype = ctypes.c_char_p
    lib.mmshiftkv_version.restype = ctypes.c_int
    for name in ("mmshiftkv_build_proxies", "mmshiftkv_score", "mmshiftkv_score_lse",
                 "mmshiftkv_score_lse_blocks", "mmshiftkv_score_lse_merge",
                 "mmshiftkv_score_mass", "mmshiftkv_select_topk", "mmshiftkv_select_tau",
                 "mmshiftkv_select_vote", "mmshiftkv_select_pick", "mmshiftkv_gather_kv",
                 "mmshiftkv_hidden_stats", "mmshiftkv_hidden_proxies", "mmshiftkv_project_proxies",
                 "mmshiftkv_decode_check", "mmshiftkv_window_rows", "mmshiftkv_shape_scores",
                 "mmshiftkv_score_noalloc", "mmshiftkv_cache_write", "mmshiftkv_cache_read",
                 "mmshiftkv_chunk_attention", "mmshiftkv_cache_hold", "mmshiftkv_cache_fork",
                 "mmshiftkv_cache_compact", "mmshiftkv_prompt_attention", "mmshiftkv_shared_attention",
                 "mmshiftkv_shared_table"):
        getattr(lib, name).restype = ctypes.c_int
    if path is None:
        _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().mmshiftkv_status_string(int(status)).decode()


def _check(fn: str, rc: int):
    if rc != MMSKV_OK:
        raise MMShiftKVError(fn, rc)


@dataclass
class SelectionConfig:
    """Method parameters; defaults are the paper's (Sec. 4.1, Appendix B)."""
    P: int = 512
    G: int = 32
    gamma: float = 10.0
    tau: float = 0.95
    lam: float = 1.0
    std_ddof: int = 0
    layer: int = 0
    seed: int = 0
    mode: int = MMSKV_VOTE
    keep_last: bool = True

    def c_params(self) -> Params:
        return Params(int(self.P), int(self.G), float(self.gamma), float(self.tau), float(self.lam),
                      int(self.std_ddof), int(self.layer), int(self.seed) & 0xFFFFFFFFFFFFFFFF,
                      int(self.mode), int(bool(self.keep_last)))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return MMSKV_F32
    if t.dtype == torch.bfloat16:
        return MMSKV_BF16
    raise TypeError("expected float32 or bfloat16, got %s" % t.dtype)


def _dev(t: torch.Tensor) -> torch.device:
    if not t.is_cuda:
        raise ValueError("libmmshiftkv takes device tensors (got a %s tensor)" % t.device)
    return t.device


def _strides4(t: torch.Tensor) -> Strides:
    st = t.stride()
    if len(st) != 4 or st[3] != 1:
        raise ValueError("expected a [batch, head, token, d] tensor with contiguous d")
    return Strides(st[0], st[1], st[2])


def _public_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# the raw handle, without a Stream object around it (not part of torch's public
# interface: its public form where a version lacks it)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _public_stream)


def _stream(device) -> int:
    return _raw_stream(device.index)


def _p(t):
    # (the argument types of the library's functions make a pointer of it)
    return None if t is None else t.data_ptr()


class _RawGuard:
    """The device of a tensor made current around a call, and put back."""
    __slots__ = ("index", "before")

    def __init__(self, device):
        self.index = device.index

    def __enter__(self):
        self.before = torch.cuda._exchange_device(self.index)

    def __exit__(self, *exc):
        torch.cuda._maybe_exchange_device(self.before)
        return False


# (the same of the light form of torch.cuda.device)
_on = (_RawGuard if hasattr(torch.cuda, "_exchange_device") and hasattr(torch.cuda, "_maybe_exchange_device")
       else torch.cuda.device)


def _tables(rope, dev):
    """(cos, sin) as contiguous fp32 tensors on dev."""
    return [t if t.dtype == torch.float32 and t.device == dev and t.is_contiguous()
            else t.to(device=dev, dtype=torch.float32).contiguous() for t in (rope[0], rope[1])]


def _shape(B, Hq, Hkv, T, W, d) -> Shape:
    return Shape(int(B), int(Hq), int(Hkv), int(T), int(W), int(d))


# ----------------------------------------------------------------------------
# the four calls (plus the split score passes and workspace queries)
# ----------------------------------------------------------------------------
def build_proxies(q_win: torch.Tensor, cfg: SelectionConfig, T: int, Hkv: int, rope_f=None,
                  rope_l=None, with_stats: bool = False, out=None):
    """mmshiftkv_build_proxies: returns (proxies [B,Hq,P,d] bf16, q_last [B,Hq,d] bf16[, stats]).
    `out` may hold preallocated (proxies, q_last) tensors."""
    dev = _dev(q_win)
    B, Hq, W, d = q_win.shape
    shape = _shape(B, Hq, Hkv, T, W, d)
    prm = cfg.c_params()
    if out is None:
        proxies = torch.empty((B, Hq, cfg.P, d), dtype=torch.bfloat16, device=dev)
        q_last = torch.empty((B, Hq, d), dtype=torch.bfloat16, device=dev)
    else:
        proxies, q_last = out
        if (proxies.dtype != torch.bfloat16 or q_last.dtype != torch.bfloat16 or not proxies.is_contiguous()
                or not q_last.is_contiguous() or tuple(proxies.shape) != (B, Hq, cfg.P, d)
                or tuple(q_last.shape) != (B, Hq, d)):
            raise ValueError("preallocated proxies/q_last do not match")
    stats = torch.empty((B, Hq, 2, d), dtype=torch.float64, device=dev) if with_stats else None
    tabs = []
    for rp in (rope_f, rope_l):
        if rp is None:
            tabs += [None, None]
        else:
            tabs += _tables(rp, dev)
    with _on(dev):
        rc = load_library().mmshiftkv_build_proxies(
            ctypes.byref(shape), ctypes.byref(prm), _p(q_win), _dtype_code(q_win),
            ctypes.byref(_strides4(q_win)), *[_p(t) for t in tabs], _p(proxies), _p(q_last),
            _p(stats), _stream(dev))
    _check("mmshiftkv_build_proxies", rc)
    return (proxies, q_last, stats) if with_stats else (proxies, q_last)


# hidden-state form of the proxies (statistics of the prefill hidden states,
# samples in hidden space, projection by each head's W_Q)
def hidden_stats_workspace(B: int, T: int, D: int) -> int:
    return int(load_library().mmshiftkv_hidden_stats_workspace(ctypes.byref(HShape(int(B), int(T), int(D)))))


def hidden_stats(hidden: torch.Tensor, std_ddof: int = 0, out=None, workspace=None) -> torch.Tensor:
    """mmshiftkv_hidden_stats: hidden [B, T, D] (features contiguous) -> [B, 2, D] fp64."""
    dev = _dev(hidden)
    if hidden.dim() != 3 or hidden.stride(2) != 1:
        raise ValueError("expected a [batch, token, feature] tensor with contiguous features")
    B, T, D = hidden.shape
    hs = HShape(B, T, D)
    st = out if out is not None else torch.empty((B, 2, D), dtype=torch.float64, device=dev)
    if st.dtype != torch.float64 or not st.is_contiguous() or tuple(st.shape) != (B, 2, D):
        raise ValueError("preallocated stats do not match")
    ws = workspace if workspace is not None else _ws(hidden_stats_workspace(B, T, D), dev)
    with _on(dev):
        rc = load_library().mmshiftkv_hidden_stats(
            ctypes.byref(hs), int(std_ddof), _p(hidden), _dtype_code(hidden), hidden.stride(0),
            hidden.stride(1), _p(st), _p(ws), ws.numel() * ws.element_size(), _stream(dev))
    _check("mmshiftkv_hidden_stats", rc)
    return st


def hidden_proxies(stats: torch.Tensor, cfg: SelectionConfig, T: int = 1, out=None) -> torch.Tensor:
    """mmshiftkv_hidden_proxies: stats [B, 2, D] fp64 -> samples [B, P, D] bf16."""
    dev = _dev(stats)
    B, two, D = stats.shape
    if two != 2 or stats.dtype != torch.float64 or not stats.is_contiguous():
        raise ValueError("expected contiguous fp64 stats [B, 2, D]")
    hp = out if out is not None else torch.empty((B, cfg.P, D), dtype=torch.bfloat16, device=dev)
    if hp.dtype != torch.bfloat16 or not hp.is_contiguous() or tuple(hp.shape) != (B, cfg.P, D):
        raise ValueError("preallocated samples do not match")
    with _on(dev):
        rc = load_library().mmshiftkv_hidden_proxies(ctypes.byref(HShape(B, int(T), D)),
                                                     ctypes.byref(cfg.c_params()), _p(stats), _p(hp),
                                                     _stream(dev))
    _check("mmshiftkv_hidden_proxies", rc)
    return hp


def project_proxies(hp: torch.Tensor, wq: torch.Tensor, Hq: int, rope=None, out=None) -> torch.Tensor:
    """mmshiftkv_project_proxies: samples [B, P, D] bf16 and W_Q [Hq*d, D] bf16
    -> proxies [B, Hq, P, d] bf16; rope = (cos, sin) [d/2] fp32 or None."""
    dev = _dev(hp)
    B, P, D = hp.shape
    N, D2 = wq.shape
    if D2 != D or N % Hq != 0:
        raise ValueError("W_Q must be [Hq*d, D]")
    d = N // Hq
    if hp.dtype != torch.bfloat16 or wq.dtype != torch.bfloat16 or not hp.is_contiguous() \
            or not wq.is_contiguous():
        raise ValueError("samples and W_Q must be contiguous bf16")
    pr = out if out is not None else torch.empty((B, Hq, P, d), dtype=torch.bfloat16, device=dev)
    if pr.dtype != torch.bfloat16 or not pr.is_contiguous() or tuple(pr.shape) != (B, Hq, P, d):
        raise ValueError("preallocated proxies do not match")
    tabs = [None, None]
    if rope is not None:
        tabs = _tables(rope, dev)
    with _on(dev):
        rc = load_library().mmshiftkv_project_proxies(ctypes.byref(HShape(B, 1, D)), P, int(Hq), d, _p(hp),
                                                      _p(wq), _p(tabs[0]), _p(tabs[1]), _p(pr), _stream(dev))
    _check("mmshiftkv_project_proxies", rc)
    return pr


def score_workspace(B, Hq, Hkv, T, W, d, cfg: SelectionConfig) -> int:
    return int(load_library().mmshiftkv_score_workspace(ctypes.byref(_shape(B, Hq, Hkv, T, W, d)),
                                                         ctypes.byref(cfg.c_params())))


def select_workspace(B, Hq, Hkv, T, W, d, cfg: SelectionConfig) -> int:
    return int(load_library().mmshiftkv_select_workspace(ctypes.byref(_shape(B, Hq, Hkv, T, W, d)),
                                                          ctypes.byref(cfg.c_params())))


def _ws(nbytes: int, dev) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=dev)


@dataclass
class ScoreOut:
    group_mass: torch.Tensor | None    # [B, Hkv, G, T] fp32
    mass: torch.Tensor                 # [B, Hkv, T] fp32
    anchor: torch.Tensor               # [B, Hkv, T] fp32


def _score_call(which: str, proxies, q_last, k, cfg, W, out: ScoreOut | None, workspace):
    dev = _dev(k)
    B, Hkv, T, d = k.shape
    Hq = proxies.shape[1]
    if proxies.dtype != torch.bfloat16 or q_last.dtype != torch.bfloat16:
        raise TypeError("proxies and q_last are bf16")
    if not (proxies.is_contiguous() and q_last.is_contiguous()):
        raise ValueError("proxies and q_last must be contiguous")
    if tuple(proxies.shape) != (B, Hq, cfg.P, d) or tuple(q_last.shape) != (B, Hq, d):
        raise ValueError("proxies/q_last shapes do not match k")
    shape = _shape(B, Hq, Hkv, T, W, d)
    prm = cfg.c_params()
    lib = load_library()
    ws = workspace
    if ws is None:
        ws = _ws(lib.mmshiftkv_score_workspace(ctypes.byref(shape), ctypes.byref(prm)), dev)
    strides = _strides4(k)
    with _on(dev):
        if which in ("lse", "lse_blocks", "lse_merge"):
            name = "mmshiftkv_score_" + which
            rc = getattr(lib, name)(ctypes.byref(shape), ctypes.byref(prm), _p(proxies), _p(q_last),
                                    _p(k), _dtype_code(k), ctypes.byref(strides), _p(ws),
                                    ws.numel() * ws.element_size(), _stream(dev))
            _check(name, rc)
            return ws
        if out is None:
            gm = (torch.empty((B, Hkv, cfg.G, T), dtype=torch.float32, device=dev)
                  if cfg.mode == MMSKV_VOTE else None)
            out = ScoreOut(gm, torch.empty((B, Hkv, T), dtype=torch.float32, device=dev),
                           torch.empty((B, Hkv, T), dtype=torch.float32, device=dev))
        fn = lib.mmshiftkv_score if which == "full" else lib.mmshiftkv_score_mass
        rc = fn(ctypes.byref(shape), ctypes.byref(prm), _p(proxies), _p(q_last), _p(k), _dtype_code(k),
                ctypes.byref(strides), _p(out.group_mass), _p(out.mass), _p(out.anchor), _p(ws),
                ws.numel() * ws.element_size(), _stream(dev))
    _check("mmshiftkv_score" if which == "full" else "mmshiftkv_score_mass", rc)
    return out


def score(proxies, q_last, k, cfg: SelectionConfig, W: int = 1, out: ScoreOut | None = None,
          workspace: torch.Tensor | None = None) -> ScoreOut:
    """mmshiftkv_score: group masses, total mass and anchor for every (b, KV head)."""
    return _score_call("full", proxies, q_last, k, cfg, W, out, workspace)


def score_noalloc(proxies, q_last, k, cfg: SelectionConfig, out: ScoreOut, W: int = 1) -> ScoreOut:
    """mmshiftkv_score_noalloc: mmshiftkv_score with the library's per-GPU
    scratch instead of a workspace (the outputs `out` are the caller's)."""
    dev = _dev(k)
    B, Hkv, T, d = k.shape
    Hq = proxies.shape[1]
    if proxies.dtype != torch.bfloat16 or q_last.dtype != torch.bfloat16:
        raise TypeError("proxies and q_last are bf16")
    if not (proxies.is_contiguous() and q_last.is_contiguous()):
        raise ValueError("proxies and q_last must be contiguous")
    shape = _shape(B, Hq, Hkv, T, W, d)
    prm = cfg.c_params()
    with _on(dev):
        rc = load_library().mmshiftkv_score_noalloc(
            ctypes.byref(shape), ctypes.byref(prm), _p(proxies), _p(q_last), _p(k), _dtype_code(k),
            ctypes.byref(_strides4(k)), _p(out.group_mass), _p(out.mass), _p(out.anchor), _stream(dev))
    _check("mmshiftkv_score_noalloc", rc)
    return out


def score_lse(proxies, q_last, k, cfg: SelectionConfig, workspace: torch.Tensor, W: int = 1,
              stage: str | None = None):
    """mmshiftkv_score_lse: the row log-sum-exp pass (result kept in `workspace`);
    with stage "blocks" or "merge" only that half (mmshiftkv_score_lse_blocks /
    _merge), which must run in that order on one workspace."""
    if stage not in (None, "blocks", "merge"):
        raise ValueError("stage is None, 'blocks' or 'merge'")
    return _score_call("lse" if stage is None else "lse_" + stage, proxies, q_last, k, cfg, W, None, workspace)


def score_mass(proxies, q_last, k, cfg: SelectionConfig, workspace: torch.Tensor, W: int = 1,
               out: ScoreOut | None = None) -> ScoreOut:
    """mmshiftkv_score_mass: the mass pass, after score_lse on the same workspace."""
    return _score_call("mass", proxies, q_last, k, cfg, W, out, workspace)


@dataclass
class Selected:
    idx: torch.Tensor        # [B, Hkv, c_max] int32 ascending, -1 padded
    counts: torch.Tensor     # [B, Hkv] int32
    votes: torch.Tensor | None


def select_topk(s: ScoreOut, cfg: SelectionConfig, budget: int, c_max: int | None = None,
                budgets: torch.Tensor | None = None, Hq: int | None = None, W: int = 1,
                want_votes: bool = False, out: Selected | None = None,
                workspace: torch.Tensor | None = None, stage: str | None = None) -> Selected:
    """mmshiftkv_select_topk: tau-sets, votes, score and budgeted top-k; with
    stage "tau", "vote" or "pick" only that stage's call (mmshiftkv_select_tau /
    _vote / _pick), which must run in that order on one workspace."""
    dev = _dev(s.mass)
    B, Hkv, T = s.mass.shape
    Hq = Hkv if Hq is None else Hq
    c_max = int(budget if c_max is None else c_max)
    shape = _shape(B, Hq, Hkv, T, 0, 0)           # W and d are not read by the selection
    prm = cfg.c_params()
    lib = load_library()
    ws = workspace
    if ws is None:
        ws = _ws(lib.mmshiftkv_select_workspace(ctypes.byref(shape), ctypes.byref(prm)), dev)
    if out is None:
        out = Selected(torch.empty((B, Hkv, c_max), dtype=torch.int32, device=dev),
                       torch.empty((B, Hkv), dtype=torch.int32, device=dev),
                       torch.empty((B, Hkv, T), dtype=torch.uint8, device=dev) if want_votes else None)
    if budgets is not None:
        budgets = budgets.to(device=dev, dtype=torch.int32).contiguous()
    nbytes = ws.numel() * ws.element_size()
    S, Pm = ctypes.byref(shape), ctypes.byref(prm)
    with _on(dev):
        if stage is None:
            name = "mmshiftkv_select_topk"
            rc = lib.mmshiftkv_select_topk(S, Pm, _p(s.group_mass), _p(s.mass), _p(s.anchor), _p(budgets),
                                           int(budget), c_max, _p(out.idx), _p(out.counts), _p(out.votes),
                                           _p(ws), nbytes, _stream(dev))
        elif stage == "tau":
            name = "mmshiftkv_select_tau"
            rc = lib.mmshiftkv_select_tau(S, Pm, _p(s.group_mass), _p(ws), nbytes, _stream(dev))
        elif stage == "vote":
            name = "mmshiftkv_select_vote"
            rc = lib.mmshiftkv_select_vote(S, Pm, _p(s.mass), _p(s.anchor), _p(out.votes), _p(ws), nbytes,
                                           _stream(dev))
        elif stage == "pick":
            name = "mmshiftkv_select_pick"
            rc = lib.mmshiftkv_select_pick(S, Pm, _p(budgets), int(budget), c_max, _p(out.idx), _p(out.counts),
                                           _p(ws), nbytes, _stream(dev))
        else:
            raise ValueError("stage must be None, 'tau', 'vote' or 'pick'")
    _check(name, rc)
    return out


def decode_workspace(B, Hq, Hkv, T, d, n_dec) -> int:
    return int(load_library().mmshiftkv_decode_workspace(ctypes.byref(_shape(B, Hq, Hkv, T, 1, d)), int(n_dec)))


def decode_check(q_dec: torch.Tensor, k: torch.Tensor, sel: Selected, k_out: torch.Tensor, v_out: torch.Tensor,
                 workspace: torch.Tensor | None = None, out=None):
    """mmshiftkv_decode_check: (coverage [B, Hq, n_dec] fp32, out [B, Hq, n_dec, d] fp32) of the
    decode queries q_dec [B, Hq, n_dec, d] bf16 against the full cache k and the compacted
    cache (k_out, v_out) of the selection `sel`."""
    dev = _dev(k)
    B, Hq, n_dec, d = q_dec.shape
    Hkv, T = k.shape[1], k.shape[2]
    if q_dec.dtype != torch.bfloat16 or not q_dec.is_contiguous():
        raise ValueError("q_dec must be a contiguous bf16 tensor")
    if k_out.dtype != k.dtype or v_out.dtype != k.dtype or not k_out.is_contiguous() or not v_out.is_contiguous():
        raise ValueError("k_out and v_out must be contiguous and of k's dtype")
    c_max = sel.idx.shape[2]
    shape = _shape(B, Hq, Hkv, T, 1, d)
    lib = load_library()
    ws = workspace
    if ws is None:
        ws = _ws(lib.mmshiftkv_decode_workspace(ctypes.byref(shape), int(n_dec)), dev)
    if out is None:
        out = (torch.empty((B, Hq, n_dec), dtype=torch.float32, device=dev),
               torch.empty((B, Hq, n_dec, d), dtype=torch.float32, device=dev))
    with _on(dev):
        rc = lib.mmshiftkv_decode_check(ctypes.byref(shape), int(n_dec), _p(q_dec), _p(k), _dtype_code(k),
                                        ctypes.byref(_strides4(k)), _p(sel.idx), _p(sel.counts), c_max,
                                        _p(k_out), _p(v_out), _p(out[0]), _p(out[1]), _p(ws),
                                        ws.numel() * ws.element_size(), _stream(dev))
    _check("mmshiftkv_decode_check", rc)
    return out


MMSKV_SHAPE_SNAPKV, MMSKV_SHAPE_STREAMING, MMSKV_SHAPE_SINKS = 0, 1, 2


def window_rows(q_win: torch.Tensor, n: int, T: int, Hkv: int):
    """mmshiftkv_window_rows: (rows [B, Hq, n, d] bf16 scaled like proxies, q_last [B, Hq, d] bf16)."""
    dev = _dev(q_win)
    B, Hq, W, d = q_win.shape
    rows = torch.empty((B, Hq, n, d), dtype=torch.bfloat16, device=dev)
    ql = torch.empty((B, Hq, d), dtype=torch.bfloat16, device=dev)
    shape = _shape(B, Hq, Hkv, T, W, d)
    with _on(dev):
        rc = load_library().mmshiftkv_window_rows(ctypes.byref(shape), int(n), _p(q_win), _dtype_code(q_win),
                                                  ctypes.byref(_strides4(q_win)), _p(rows), _p(ql), _stream(dev))
    _check("mmshiftkv_window_rows", rc)
    return rows, ql


def shape_scores(mass: torch.Tensor | None, kind: int, B: int, Hkv: int, T: int, window: int = 0, pool: int = 1,
                 sinks: int = 0, out: torch.Tensor | None = None, device=None) -> torch.Tensor:
    """mmshiftkv_shape_scores: per-key baseline scores [B, Hkv, T] fp32."""
    dev = _dev(mass) if mass is not None else torch.device(device if device is not None else "cuda:0")
    if dev.index is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    score = out if out is not None else torch.empty((B, Hkv, T), dtype=torch.float32, device=dev)
    shape = _shape(B, 0, Hkv, T, 0, 0)            # only B, Hkv and T are read
    with _on(dev):
        rc = load_library().mmshiftkv_shape_scores(ctypes.byref(shape), int(kind), int(window), int(pool), int(sinks),
                                                   _p(mass), _p(score), _stream(dev))
    _check("mmshiftkv_shape_scores", rc)
    return score


BASELINES = ("snapkv", "streaming", "expected")


def baseline_select(name: str, q_win, k, v, budget: int, seed: int = 0, layer: int = 0, window: int = 32,
                    pool: int = 5, sinks: int = 4, P: int = 512, c_max=None):
    """A baseline selector end to end on the library's kernels: (Selected, score, mass, k_out, v_out).
    snapkv: window rows -> mass pass -> pooled scores; streaming: sinks + recency;
    expected: gamma = 1 proxies -> mass pass -> sinks; then the MASS-mode top-C and the gather."""
    B, Hkv, T, d = k.shape
    Hq, W = q_win.shape[1], q_win.shape[2]
    dev = _dev(k)
    sel_cfg = SelectionConfig(mode=MMSKV_MASS, keep_last=False, seed=seed, layer=layer)
    mass = anchor = None                         # (the anchor is not read in MASS mode)
    if name == "snapkv":
        rows, ql = window_rows(q_win, window, T, Hkv)
        cfg = SelectionConfig(P=window, G=1, mode=MMSKV_MASS, seed=seed, layer=layer)
        sc = score(rows, ql, k, cfg, W)
        mass, anchor = sc.mass, sc.anchor
        scores = shape_scores(mass, MMSKV_SHAPE_SNAPKV, B, Hkv, T, window=window, pool=pool)
    elif name == "streaming":
        scores = shape_scores(None, MMSKV_SHAPE_STREAMING, B, Hkv, T, sinks=sinks, device=dev)
    elif name == "expected":
        cfg = SelectionConfig(P=P, gamma=1.0, mode=MMSKV_MASS, seed=seed, layer=layer)
        prox, ql = build_proxies(q_win, cfg, T, Hkv)
        sc = score(prox, ql, k, cfg, W)
        mass, anchor = sc.mass, sc.anchor
        scores = shape_scores(mass, MMSKV_SHAPE_SINKS, B, Hkv, T, sinks=sinks)
    else:
        raise ValueError("unknown baseline %r" % name)
    sel = select_topk(ScoreOut(None, scores, anchor), sel_cfg, budget, c_max, None, Hq, W)
    ko, vo = gather_kv(k, v, sel)
    return sel, scores, mass, ko, vo


def gather_kv(k: torch.Tensor, v: torch.Tensor, sel: Selected, out=None):
    """mmshiftkv_gather_kv: compacted K'/V' [B, Hkv, c_max, d] in temporal order."""
    dev = _dev(k)
    B, Hkv, T, d = k.shape
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("k and v must have the same shape and dtype")
    c_max = sel.idx.shape[2]
    shape = _shape(B, 0, Hkv, T, 0, d)            # Hq and W are not read by the gather
    if out is None:
        out = (torch.empty((B, Hkv, c_max, d), dtype=k.dtype, device=dev),
               torch.empty((B, Hkv, c_max, d), dtype=k.dtype, device=dev))
    with _on(dev):
        rc = load_library().mmshiftkv_gather_kv(
            ctypes.byref(shape), _p(k), _p(v), _dtype_code(k), ctypes.byref(_strides4(k)),
            ctypes.byref(_strides4(v)), _p(sel.idx), _p(sel.counts), c_max, _p(out[0]), _p(out[1]),
            _stream(dev))
    _check("mmshiftkv_gather_kv", rc)
    return out


# ----------------------------------------------------------------------------
# paged cache: rows written (and quantised), read back and attended to
# ----------------------------------------------------------------------------
_CACHE_DTYPES = {torch.bfloat16: MMSKV_BF16, torch.float8_e4m3fn: MMSKV_E4M3, torch.int8: MMSKV_I8}


@dataclass
class PagedCache:
    """Pages of K and V rows (mmskv_pages): k and v [n_pages, Hkv, page, d] as bfloat16,
    float8_e4m3fn or int8, the 8-bit ones with fp32 scales [n_pages, Hkv, page] (else None);
    table [B, max_pages] int32, the pages of each sequence in order; refs [n_pages] int32, the
    entries of the table that name each page (only cache_hold, cache_fork and cache_compact read
    and write them; None: pages that are never given or taken)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor | None
    v_scale: torch.Tensor | None
    table: torch.Tensor
    refs: torch.Tensor | None = None

    @classmethod
    def empty(cls, B: int, Hkv: int, T: int, d: int, dtype: torch.dtype = torch.bfloat16, page: int = 64,
              device="cuda:0") -> "PagedCache":
        """A cache of its own pages for B sequences of up to T rows (the rows are not cleared)."""
        per = max(1, -(-int(T) // page))
        table = torch.arange(B * per, dtype=torch.int32, device=device).view(B, per)
        return cls(*cls._pools(B * per, Hkv, page, d, dtype, device), table, torch.ones_like(table).view(-1))

    @classmethod
    def pool(cls, B: int, Hkv: int, n_pages: int, max_pages: int, d: int, dtype: torch.dtype = torch.bfloat16,
             page: int = 64, device="cuda:0") -> "PagedCache":
        """A cache of n_pages free pages that B sequences share, up to max_pages each (cache_hold)."""
        return cls(*cls._pools(n_pages, Hkv, page, d, dtype, device),
                   torch.full((B, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device))

    @staticmethod
    def _pools(n_pages, Hkv, page, d, dtype, device):
        shape = (n_pages, Hkv, page, d)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        ks = vs = None
        if dtype != torch.bfloat16:
            ks, vs = (torch.empty(shape[:3], dtype=torch.float32, device=device) for _ in range(2))
        return k, v, ks, vs

    def c_pages(self) -> Pages:
        k, v, ks, vs, table = self.k, self.v, self.k_scale, self.v_scale, self.table
        dtype, shape, i = k.dtype, k.shape, k.get_device()
        code = _CACHE_DTYPES.get(dtype)
        if code is None:
            raise TypeError("expected bfloat16, float8_e4m3fn or int8 pages, got %s" % dtype)
        if v.dtype != dtype or v.shape != shape or len(shape) != 4 or not (k.is_contiguous() and v.is_contiguous()):
            raise ValueError("k and v pages must be contiguous [n_pages, Hkv, page, d] of one dtype")
        size = table.shape
        if table.dtype != torch.int32 or len(size) != 2 or not table.is_contiguous():
            raise ValueError("the table must be a contiguous int32 [B, max_pages] tensor")
        if v.get_device() != i or table.get_device() != i:
            raise ValueError("pages and table on different devices")
        if code == MMSKV_BF16:
            return Pages(k.data_ptr(), v.data_ptr(), None, None, table.data_ptr(), shape[0], shape[2], size[1], code)
        rows = shape[:3]
        for s in (ks, vs):
            if (s is None or s.dtype != torch.float32 or s.shape != rows or not s.is_contiguous()
                    or s.get_device() != i):
                raise ValueError("8-bit pages need contiguous fp32 scales [n_pages, Hkv, page] on their device")
        return Pages(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), table.data_ptr(), shape[0], shape[2],
                     size[1], code)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _enqueue(name: str, i: int, *args):
    """A call of the library on the current stream of device i, which is made current around it."""
    fn = getattr(load_library(), name)
    if _current_device() == i:
        rc = fn(*args, _raw_stream(i))
    else:
        with _on(torch.device("cuda", i)):
            rc = fn(*args, _raw_stream(i))
    if rc != MMSKV_OK:
        raise MMShiftKVError(name, rc)


def _same_device(t, *others) -> int:
    """The index of the device that all the tensors are on."""
    i = t.get_device()                 # (-1: host)
    for o in others:
        if o is not None and o.get_device() != i:
            raise ValueError("tensors on different devices (%s, %s)" % (t.device, o.device))
    if i < 0:
        _dev(t)
    return i


def _row_strides(t: torch.Tensor) -> Strides:
    """_strides4 with 0 for dimensions of one entry, whose stride means nothing."""
    st, n = t.stride(), t.shape
    if len(st) != 4 or st[3] != 1:
        raise ValueError("expected a [batch, head, token, d] tensor with contiguous d")
    return Strides(st[0] if n[0] > 1 else 0, st[1] if n[1] > 1 else 0, st[2] if n[2] > 1 else 0)


def _int32(t, shape, what):
    """Row numbers as the library takes them: contiguous int32 of that shape."""
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of shape %s" % (what, shape))
    return t.data_ptr()


def cache_write(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, start: torch.Tensor | None = None,
                counts: torch.Tensor | None = None, idx: torch.Tensor | None = None):
    """mmshiftkv_cache_write: rows of k, v [B, Hkv, T, d] (fp32 or bf16) into the cache, from row
    start[b, c] (None: 0) of each head on: the first counts[b, c] (None: all) tokens, or those of
    idx [B, Hkv, n] (a Selected's idx and counts: the kept tokens).  All row numbers int32."""
    i = _same_device(k, v, cache.k, start, counts, idx)
    shape = k.shape
    if v.shape != shape or v.dtype != k.dtype:
        raise ValueError("k and v must have the same shape and dtype")
    ks, vs = _row_strides(k), _row_strides(v)
    B, Hkv, T, d = shape
    pages, n = cache.c_pages(), T
    _, heads, _, row = cache.k.shape
    if heads != Hkv or row != d or cache.table.shape[0] != B:
        raise ValueError("k does not match the cache's heads, row size or sequences")
    if idx is not None:
        n = idx.shape[-1]
        idx = _int32(idx, (B, Hkv, n), "idx")
    if counts is not None:
        counts = _int32(counts, (B, Hkv), "counts")
    if start is not None:
        start = _int32(start, (B, Hkv), "start")
    ref = ctypes.byref
    _enqueue("mmshiftkv_cache_write", i, ref(Shape(B, 0, Hkv, T, 0, d)), ref(pages), k.data_ptr(), v.data_ptr(),
             _dtype_code(k), ref(ks), ref(vs), idx, counts, start, n)


def cache_read(cache: PagedCache, lens: torch.Tensor, T: int, dtype: torch.dtype = torch.bfloat16, out=None):
    """mmshiftkv_cache_read: (k, v) [B, Hkv, T, d] of the first lens[b, c] cached rows of each head
    (zeros behind them), as bfloat16 or float32; `out` may hold preallocated (k, v)."""
    i = _same_device(cache.k, lens)
    pages = cache.c_pages()
    B, T = cache.table.shape[0], int(T)
    _, Hkv, _, d = cache.k.shape
    rows = _int32(lens, (B, Hkv), "lens")
    shape = (B, Hkv, T, d)
    if out is None:
        ko, vo = out = lens.new_empty(shape, dtype=dtype), lens.new_empty(shape, dtype=dtype)
    else:
        ko, vo = out
        _same_device(lens, ko, vo)
        if ko.shape != shape or vo.shape != shape or ko.dtype != dtype or vo.dtype != dtype:
            raise ValueError("preallocated k/v do not match")
    ref = ctypes.byref
    _enqueue("mmshiftkv_cache_read", i, ref(Shape(B, 0, Hkv, T, 0, d)), ref(pages), rows, _dtype_code(ko),
             ko.data_ptr(), ref(_row_strides(ko)), vo.data_ptr(), ref(_row_strides(vo)))
    return out


def chunk_attention_workspace(B, Hq, Hkv, T, d, n) -> int:
    return int(load_library().mmshiftkv_chunk_attention_workspace(ctypes.byref(_shape(B, Hq, Hkv, T, 0, d)), int(n)))


def chunk_attention(q: torch.Tensor, cache: PagedCache, lens: torch.Tensor, q_counts: torch.Tensor | None = None,
                    T: int | None = None, causal: bool = True, workspace: torch.Tensor | None = None,
                    out: torch.Tensor | None = None) -> torch.Tensor:
    """mmshiftkv_chunk_attention: the outputs [B, Hq, n, d] bf16 of the chunk's queries q [B, Hq, n, d]
    bf16 (n = 1: a decoding step) over the first lens[b, c] cached rows of each head, the chunk's own
    among them; q_counts[b] (None: n) queries of sequence b are there.  T is an upper bound of lens
    (None: what the table can hold).  The result is laid out as q is unless `out` is given.  A chunk of
    some sequences and single tokens of others are faster as two calls: n fixes how all are worked on."""
    i = _same_device(q, cache.k, lens, q_counts, workspace, out)
    if q.dtype != torch.bfloat16:
        raise TypeError("q is bf16")
    qs = _row_strides(q)
    B, Hq, n, d = q.shape
    pages = cache.c_pages()
    _, Hkv, page, row = cache.k.shape
    if row != d or cache.table.shape[0] != B:
        raise ValueError("q does not match the cache's row size or sequences")
    rows = _int32(lens, (B, Hkv), "lens")
    if q_counts is not None:
        q_counts = _int32(q_counts, (B,), "q_counts")
    if out is None:
        out = torch.empty_like(q)
        os = _row_strides(out) if out.stride(3) == 1 else None
        if os is None:
            out = q.new_empty(q.shape)
            os = _row_strides(out)
    else:
        if out.dtype != torch.bfloat16 or out.shape != q.shape:
            raise ValueError("preallocated out does not match")
        os = _row_strides(out)
    ref = ctypes.byref
    most = cache.table.shape[1] * page
    shape = ref(Shape(B, Hq, Hkv, most if T is None else min(int(T), most), 0, d))
    ws = workspace
    if ws is None:
        ws = _ws(load_library().mmshiftkv_chunk_attention_workspace(shape, n), q.device)
    _enqueue("mmshiftkv_chunk_attention", i, shape, ref(pages), q.data_ptr(), ref(qs), q_counts, rows, n,
             1 if causal else 0, out.data_ptr(), ref(os), ws.data_ptr(), ws.numel() * ws.element_size())
    return out


def shared_attention_workspace(B, Hq, Hkv, T, d, n, groups) -> int:
    return int(load_library().mmshiftkv_shared_attention_workspace(
        ctypes.byref(_shape(B, Hq, Hkv, T, 0, d)), int(groups), int(n)))


def shared_table(cache: PagedCache, lens: torch.Tensor, shared: torch.Tensor) -> torch.Tensor:
    """mmshiftkv_shared_table: the pages [G, max_pages] int32 of the rows that G groups of sequences share
    (shared [G, Hkv] int32), each by a sequence of its group that has them, whichever have ended."""
    i = _same_device(cache.k, lens, shared)
    pages = cache.c_pages()
    _, Hkv, _, d = cache.k.shape
    B, most = cache.table.shape
    rows, G = _int32(lens, (B, Hkv), "lens"), shared.shape[0]
    prefix = _int32(shared, (G, Hkv), "shared")
    if G < 1 or B % G:
        raise ValueError("the sequences are groups of the same size: %d of %d" % (G, B))
    out = lens.new_empty((G, most))
    ref = ctypes.byref
    _enqueue("mmshiftkv_shared_table", i, ref(Shape(B, 0, Hkv, 0, 0, d)), ref(pages), rows, prefix, G, out.data_ptr())
    return out


_shared_table = shared_table                       # (where an argument has that name)


def shared_attention(q: torch.Tensor, cache: PagedCache, lens: torch.Tensor, shared: torch.Tensor,
                     shared_table: torch.Tensor | None = None, q_counts: torch.Tensor | None = None,
                     T: int | None = None, shared_T: int | None = None, causal: bool = True,
                     workspace: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """mmshiftkv_shared_attention: chunk_attention for G groups of B / G sequences that share the first
    shared[g, c] rows (shared [G, Hkv] int32), which are read once for a group.  shared_table [G, max_pages]
    int32 names their pages, which have to be held for as long as it is used: after a fork all sequences hold
    those of whole pages, the ones behind only their own (None: what shared_table finds, a short launch more,
    for groups that cache_fork has made and whose sequences end in any order).  T and shared_T are upper bounds of lens and shared (None: what the table can hold, and T)."""
    i = _same_device(q, cache.k, lens, shared, shared_table, q_counts, workspace, out)
    if q.dtype != torch.bfloat16:
        raise TypeError("q is bf16")
    qs = _row_strides(q)
    B, Hq, n, d = q.shape
    pages = cache.c_pages()
    _, Hkv, page, row = cache.k.shape
    if row != d or cache.table.shape[0] != B:
        raise ValueError("q does not match the cache's row size or sequences")
    rows = _int32(lens, (B, Hkv), "lens")
    G = shared.shape[0]
    prefix = _int32(shared, (G, Hkv), "shared")
    if G < 1 or B % G:
        raise ValueError("the sequences are groups of the same size: %d of %d" % (G, B))
    if shared_table is None:
        shared_table = cache.table if G == B else _shared_table(cache, lens, shared)
    named = _int32(shared_table, (G, cache.table.shape[1]), "shared_table")
    if q_counts is not None:
        q_counts = _int32(q_counts, (B,), "q_counts")
    if out is None:
        out = torch.empty_like(q)
        if out.stride(3) != 1:
            out = q.new_empty(q.shape)
    elif out.dtype != torch.bfloat16 or out.shape != q.shape:
        raise ValueError("preallocated out does not match")
    os = _row_strides(out)
    ref = ctypes.byref
    most = cache.table.shape[1] * page
    T = most if T is None else min(int(T), most)
    shape = ref(Shape(B, Hq, Hkv, T, 0, d))
    ws = workspace
    if ws is None:
        ws = _ws(load_library().mmshiftkv_shared_attention_workspace(shape, G, n), q.device)
    _enqueue("mmshiftkv_shared_attention", i, shape, ref(pages), q.data_ptr(), ref(qs), q_counts, rows, prefix, named, G,
             T if shared_T is None else max(1, min(int(shared_T), T)), n, 1 if causal else 0, out.data_ptr(), ref(os),
             ws.data_ptr(), ws.numel() * ws.element_size())
    return out


# ----------------------------------------------------------------------------
# whole prompts over themselves
# ----------------------------------------------------------------------------
def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor | None = None,
                     causal: bool = True, with_lse: bool = False, out: torch.Tensor | None = None,
                     lse: torch.Tensor | None = None):
    """mmshiftkv_prompt_attention: the outputs [B, Hq, T, d] bf16 of q [B, Hq, T, d] over k, v [B, Hkv, T, d]
    (bf16), each batch row a sequence; with starts [n + 1] int32 (B = 1) the T tokens are n sequences one
    behind the other, sequence s the tokens starts[s] .. starts[s + 1] - 1 (rows in none are not written).
    with_lse (or a preallocated lse [B, Hq, T] fp32): returns (out, lse), the log-sum-exp of each row's
    logits.  The result is laid out as q is unless `out` is given."""
    i = _same_device(q, k, v, starts, out, lse)
    if q.dtype != torch.bfloat16 or k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16:
        raise TypeError("q, k and v are bf16")
    qs, ks, vs = _row_strides(q), _row_strides(k), _row_strides(v)
    B, Hq, T, d = q.shape
    Hkv = k.shape[1]
    if k.shape != v.shape or k.shape != (B, Hkv, T, d):
        raise ValueError("k and v do not match q")
    n_seq, first = 0, None
    if starts is not None:
        if starts.dim() != 1 or starts.shape[0] < 2 or B != 1:
            raise ValueError("starts cut the tokens of one batch row: [n + 1] with B = 1")
        n_seq = starts.shape[0] - 1
        first = _int32(starts, (n_seq + 1,), "starts")
    if out is None:
        out = torch.empty_like(q)
        if out.stride(3) != 1:
            out = q.new_empty(q.shape)
    elif out.dtype != torch.bfloat16 or out.shape != q.shape:
        raise ValueError("preallocated out does not match")
    os = _row_strides(out)
    if lse is None:
        lse = q.new_empty((B, Hq, T), dtype=torch.float32) if with_lse else None
    elif lse.dtype != torch.float32 or lse.shape != (B, Hq, T) or not lse.is_contiguous():
        raise ValueError("preallocated lse does not match")
    ref = ctypes.byref
    _enqueue("mmshiftkv_prompt_attention", i, ref(Shape(B, Hq, Hkv, T, 0, d)), q.data_ptr(), ref(qs), k.data_ptr(),
             ref(ks), v.data_ptr(), ref(vs), first, n_seq, 1 if causal else 0, out.data_ptr(), ref(os), _p(lse))
    return out if lse is None else (out, lse)


# ----------------------------------------------------------------------------
# pages that several sequences hold
# ----------------------------------------------------------------------------
def cache_book_workspace(B, Hkv, n_pages, max_pages) -> int:
    return int(load_library().mmshiftkv_cache_book_workspace(ctypes.byref(_shape(B, 0, Hkv, 0, 0, 0)), int(n_pages),
                                                             int(max_pages)))


def _book(name: str, cache: PagedCache, missing, workspace, tensors, *args):
    """A call that changes the pages of `cache`; tensors: those of the call, args: their pointers and numbers."""
    k, refs = cache.k, cache.refs
    if refs is None:
        raise ValueError("the cache has no refs: its pages are not given or taken")
    i = _same_device(k, refs, missing, workspace, *tensors)
    pages = cache.c_pages()
    n_pages, Hkv, _, d = k.shape
    B, most = cache.table.shape
    counts = _int32(refs, (n_pages,), "refs")
    if missing is None:
        missing = refs.new_empty(B)
    lack = _int32(missing, (B,), "missing")
    ref = ctypes.byref
    shape = ref(Shape(B, 0, Hkv, 0, 0, d))
    ws = workspace
    if ws is None:
        ws = _ws(load_library().mmshiftkv_cache_book_workspace(shape, n_pages, most), k.device)
    _enqueue(name, i, shape, ref(pages), counts, *args, lack, ws.data_ptr(), ws.numel() * ws.element_size())
    return missing


def cache_hold(cache: PagedCache, rows: torch.Tensor, missing: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """mmshiftkv_cache_hold: each sequence holds the pages for max(rows[b]) rows (rows [B, Hkv] int32),
    taken from the free ones or given back.  Returns missing [B] int32: the pages that it did not get."""
    at = _int32(rows, (cache.table.shape[0], cache.k.shape[1]), "rows")
    return _book("mmshiftkv_cache_hold", cache, missing, workspace, (rows,), at)


def cache_fork(cache: PagedCache, src: torch.Tensor, lens: torch.Tensor, missing: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """mmshiftkv_cache_fork: sequence b becomes a copy of sequence src[b] (src [B] int32; b itself: it
    stays) as that was before the call, sharing the pages that are full; lens [B, Hkv] int32 follows.
    Returns missing [B] int32: the pages that it did not get (then it stays as it was)."""
    B = cache.table.shape[0]
    args = _int32(src, (B,), "src"), _int32(lens, (B, cache.k.shape[1]), "lens")
    return _book("mmshiftkv_cache_fork", cache, missing, workspace, (src, lens), *args)


def cache_compact(cache: PagedCache, lens: torch.Tensor, idx: torch.Tensor, counts: torch.Tensor,
                  missing: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """mmshiftkv_cache_compact: the first counts[b, c] of the rows idx [B, Hkv, n] become the cached rows of
    each head, on new pages, and lens [B, Hkv] follows (a Selected over the cached rows: its idx and counts;
    all counts of a sequence below 0: it stays).  All int32.  Returns missing [B] int32, as cache_fork."""
    shape = (cache.table.shape[0], cache.k.shape[1])
    n = idx.shape[-1]
    args = _int32(lens, shape, "lens"), _int32(idx, shape + (n,), "idx"), _int32(counts, shape, "counts"), n
    return _book("mmshiftkv_cache_compact", cache, missing, workspace, (lens, idx, counts), *args)


@dataclass
class LayerOut:
    proxies: torch.Tensor
    q_last: torch.Tensor
    scores: ScoreOut
    sel: Selected
    k_out: torch.Tensor
    v_out: torch.Tensor


def select_layer(q_win, k, v, budget: int, cfg: SelectionConfig | None = None, c_max=None,
                 budgets=None, rope_f=None, rope_l=None, want_votes=False) -> LayerOut:
    """All four calls for one layer (Algorithm 1), on the current stream."""
    cfg = cfg or SelectionConfig()
    B, Hkv, T, d = k.shape
    Hq, W = q_win.shape[1], q_win.shape[2]
    prox, ql = build_proxies(q_win, cfg, T, Hkv, rope_f, rope_l)
    sc = score(prox, ql, k, cfg, W)
    sel = select_topk(sc, cfg, budget, c_max, budgets, Hq, W, want_votes)
    ko, vo = gather_kv(k, v, sel)
    return LayerOut(prox, ql, sc, sel, ko, vo)
