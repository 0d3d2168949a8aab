"""MI355X-native 3D-RoPE + flash-attention forward (video-DiT attention hot path).

Thin ctypes binding over ``libvidax.so`` (C ABI declared in include/vidax.h).
This module only marshals arguments: torch provides device memory and the
current HIP stream; every step of the computation runs in the library's
kernels.  If the library has not been built the calls raise immediately --
there is no fallback implementation.
"""

from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvidax.so")

VIDAX_OK = 0
_STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported configuration", 3: "kernel launch failed",
           4: "request exceeds the fixed device scratch of an allocation-free entry point"}

EXPORTED_SYMBOLS = (
    "vidax_rope3d",
    "vidax_rope3d_transpose",
    "vidax_attn_bwd",
    "vidax_attn_bwd_workspace_floats",
    "vidax_attn_bwd_noalloc",
    "vidax_na3d_fwd",
    "vidax_qkv_proj",
    "vidax_qk_norm_rope",
    "vidax_attn_mod_fwd",
    "vidax_attn_mod_fwd_workspace_floats",
    "vidax_attn_mod_bwd",
    "vidax_attn_mod_bwd_workspace_floats",
    "vidax_block_norm_fwd",
    "vidax_block_norm_bwd",
    "vidax_block_norm_bwd_workspace_floats",
    "vidax_attn_fwd",
    "vidax_attn_fwd_naive",
    "vidax_status_string",
    "vidax_abi_version",
)


class VidaxError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} returned {status} ({_STATUS.get(status, 'unknown')})")
        self.status = status


class RopeDesc(ctypes.Structure):
    """Mirror of vidax_rope3d_desc."""

    _fields_ = [
        ("grid_t", ctypes.c_int32),
        ("grid_h", ctypes.c_int32),
        ("grid_w", ctypes.c_int32),
        ("dim_t", ctypes.c_int32),
        ("dim_h", ctypes.c_int32),
        ("dim_w", ctypes.c_int32),
        ("theta", ctypes.c_float),
        ("pair_mode", ctypes.c_int32),
        ("keys_prerotated", ctypes.c_int32),
    ]


@dataclass(frozen=True)
class Rope:
    """3D rotary convention: token grid (T, Hp, Wp), channel split, theta, pairing."""

    grid: tuple
    dims: tuple = (44, 42, 42)
    theta: float = 10000.0
    pair_mode: int = 0
    keys_prerotated: bool = False  # attention: k already rotated (rotate q only)

    def desc(self) -> RopeDesc:
        return RopeDesc(*self.grid, *self.dims, float(self.theta), int(self.pair_mode), int(self.keys_prerotated))


class ScoreDesc(ctypes.Structure):
    """Mirror of vidax_score_desc."""

    _fields_ = [("causal", ctypes.c_int32), ("cap", ctypes.c_float)] + [
        (n, ctypes.c_void_p) for n in ("slopes", "q_doc", "k_doc", "kv_valid_len", "prefix_len", "q_start")]


@dataclass(frozen=True)
class Score:
    """What attention does to its scores and which keys a query sees.

    causal: key j only up to the query's position, or j < prefix_len[b]; cap:
    scores become cap * tanh(score / cap) (0: none); slopes: float32 [H], slope *
    |position - j| is subtracted; q_doc, k_doc: int32 [B, Lq] and [B, Lk], only
    keys of the query's own document are seen (a negative id belongs to none);
    kv_valid_len, prefix_len: int32 [B]; q_start: int32 [B], the position of
    query 0 (default: Lk - Lq).  All tensors are device tensors.  Keys that hold
    anything but numbers have to lie past kv_valid_len, behind all positions and
    prefixes of a causal call, or in negative documents."""

    causal: bool = False
    cap: float = 0.0
    slopes: object = None
    q_doc: object = None
    k_doc: object = None
    kv_valid_len: object = None
    prefix_len: object = None
    q_start: object = None


class BlockMod(ctypes.Structure):
    """Mirror of vidax_block_mod."""

    _fields_ = [("p", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64)]


class BlockNormDesc(ctypes.Structure):
    """Mirror of vidax_block_norm_desc."""

    _fields_ = [
        ("stream_fp32", ctypes.c_int32),
        ("norm", ctypes.c_int32),
        ("post", ctypes.c_int32),
        ("per_token", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("alpha", ctypes.c_float),
        ("gain", ctypes.c_void_p),
        ("post_gain", ctypes.c_void_p),
        ("gate", BlockMod),
        ("scale", BlockMod),
        ("shift", BlockMod),
    ]


class BlockNormGrads(ctypes.Structure):
    """Mirror of vidax_block_norm_grads."""

    _fields_ = [(n, ctypes.c_void_p) for n in ("dgate", "dscale", "dshift", "dgain", "dpost_gain")]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded libvidax.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2609_18077_amd.build` "
                "(or __graft_entry__.build()); there is no fallback path"
            )
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
        L.vidax_rope3d.argtypes = [vp, vp, i32, i32, i32, i32, ctypes.POINTER(RopeDesc), vp]
        L.vidax_rope3d.restype = i32
        L.vidax_rope3d_transpose.argtypes = [vp, vp, i32, i32, i32, i32, ctypes.POINTER(RopeDesc), vp]
        L.vidax_rope3d_transpose.restype = i32
        L.vidax_attn_bwd.argtypes = [vp] * 10 + [ctypes.c_size_t, i32, i32, i32, i32, i32, f32, vp, vp]
        L.vidax_attn_bwd.restype = i32
        L.vidax_attn_bwd_workspace_floats.argtypes = [i32, i32, i32, i32, i32]
        L.vidax_attn_bwd_workspace_floats.restype = ctypes.c_size_t
        L.vidax_attn_bwd_noalloc.argtypes = [vp] * 9 + [i32, i32, i32, i32, i32, f32, vp, vp]
        L.vidax_attn_bwd_noalloc.restype = i32
        L.vidax_na3d_fwd.argtypes = [vp] * 5 + [i32] * 10 + [f32, vp]
        L.vidax_na3d_fwd.restype = i32
        L.vidax_qkv_proj.argtypes = [vp] * 5 + [f32] + [vp] * 3 + [i32] * 5 + [ctypes.POINTER(RopeDesc), vp]
        L.vidax_qkv_proj.restype = i32
        L.vidax_qk_norm_rope.argtypes = [vp, vp, vp, f32, i32, i32, i32, i32, ctypes.POINTER(RopeDesc), vp]
        L.vidax_qk_norm_rope.restype = i32
        L.vidax_attn_mod_fwd.argtypes = ([vp] * 5 + [i32] * 6 + [f32, ctypes.POINTER(ScoreDesc), vp, ctypes.c_size_t, vp])
        L.vidax_attn_mod_fwd.restype = i32
        L.vidax_attn_mod_fwd_workspace_floats.argtypes = [i32] * 7
        L.vidax_attn_mod_fwd_workspace_floats.restype = ctypes.c_size_t
        L.vidax_attn_mod_bwd.argtypes = ([vp] * 9 + [i32] * 6 + [f32, ctypes.POINTER(ScoreDesc), vp, ctypes.c_size_t, vp])
        L.vidax_attn_mod_bwd.restype = i32
        L.vidax_attn_mod_bwd_workspace_floats.argtypes = [i32] * 7
        L.vidax_attn_mod_bwd_workspace_floats.restype = ctypes.c_size_t
        L.vidax_block_norm_fwd.argtypes = [vp] * 4 + [i32] * 3 + [ctypes.POINTER(BlockNormDesc), vp]
        L.vidax_block_norm_fwd.restype = i32
        L.vidax_block_norm_bwd.argtypes = ([vp] * 6 + [ctypes.POINTER(BlockNormGrads), vp, ctypes.c_size_t]
                                           + [i32] * 3 + [ctypes.POINTER(BlockNormDesc), vp])
        L.vidax_block_norm_bwd.restype = i32
        L.vidax_block_norm_bwd_workspace_floats.argtypes = [i32, i32, i32]
        L.vidax_block_norm_bwd_workspace_floats.restype = ctypes.c_size_t
        for name in ("vidax_attn_fwd", "vidax_attn_fwd_naive"):
            fn = getattr(L, name)
            fn.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, f32, vp, ctypes.POINTER(RopeDesc), vp]
            fn.restype = i32
        L.vidax_status_string.argtypes = [i32]
        L.vidax_status_string.restype = ctypes.c_char_p
        L.vidax_abi_version.argtypes = []
        L.vidax_abi_version.restype = i32
        _lib = L
    return _lib


def _check(fn: str, status: int):
    if status != VIDAX_OK:
        raise VidaxError(fn, status)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _stream(stream):
    import torch

    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check_bshd(name, t):
    import torch

    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
        raise ValueError(f"{name} must be a contiguous bfloat16 [B, L, H, d] device tensor")


def rope3d(x, rope: Rope, out=None, stream=None):
    """Rotated copy of x (bf16 [B, L, H, d]); out may be x itself (in place)."""
    import torch

    _check_bshd("x", x)
    y = torch.empty_like(x) if out is None else out
    _check_bshd("out", y)
    if y.shape != x.shape:
        raise ValueError("out must have the shape of x")
    B, L, H, d = x.shape
    desc = rope.desc()
    _check("vidax_rope3d", lib().vidax_rope3d(_ptr(x), _ptr(y), B, L, H, d, ctypes.byref(desc), _stream(stream)))
    return y


def rope3d_transpose(x, rope: Rope, out=None, stream=None):
    """R^T x (every pair rotated by minus its angle); out may be x itself."""
    import torch

    _check_bshd("x", x)
    y = torch.empty_like(x) if out is None else out
    _check_bshd("out", y)
    if y.shape != x.shape:
        raise ValueError("out must have the shape of x")
    B, L, H, d = x.shape
    desc = rope.desc()
    _check("vidax_rope3d_transpose",
           lib().vidax_rope3d_transpose(_ptr(x), _ptr(y), B, L, H, d, ctypes.byref(desc), _stream(stream)))
    return y


def attn_bwd(q, k, v, o, dout, lse, scale=None, kv_valid_len=None, stream=None, noalloc=False, out=None,
             workspace=None):
    """(dq, dk, dv) of attention without rotation, from the forward's o and lse.

    noalloc=True calls vidax_attn_bwd_noalloc (D in the library's fixed
    device array instead of a workspace tensor); `out` = (dq, dk, dv) tensors
    to write into instead of new ones; `workspace` = a contiguous float32
    device tensor to use as the workspace (by default one of
    vidax_attn_bwd_workspace_floats values is allocated)."""
    import torch

    for n, t in (("q", q), ("k", k), ("v", v), ("o", o), ("dout", dout)):
        _check_bshd(n, t)
    B, Lq, H, d = q.shape
    Lk = k.shape[1]
    if k.shape != v.shape or o.shape != q.shape or dout.shape != q.shape:
        raise ValueError("shapes: q, o, dout [B, Lq, H, d]; k, v [B, Lk, H, d]")
    if lse.dtype != torch.float32 or not lse.is_cuda or not lse.is_contiguous() or lse.shape != (B, H, Lq):
        raise ValueError("lse must be a contiguous float32 [B, H, Lq] device tensor")
    if scale is None:
        scale = float(torch.tensor(1.0 / d ** 0.5, dtype=torch.float32))
    if kv_valid_len is not None:
        if kv_valid_len.dtype != torch.int32 or not kv_valid_len.is_cuda or kv_valid_len.numel() != B:
            raise ValueError("kv_valid_len must be an int32 device tensor of B elements")
        kv_valid_len = kv_valid_len.contiguous()
    if out is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    else:
        dq, dk, dv = out
        for n, t, ref in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
            _check_bshd(n, t)
            if t.shape != ref.shape:
                raise ValueError(f"{n} must have shape {tuple(ref.shape)}")
    if noalloc:
        _check("vidax_attn_bwd_noalloc",
               lib().vidax_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lse), _ptr(dq),
                                            _ptr(dk), _ptr(dv), B, H, Lq, Lk, d, float(scale), _ptr(kv_valid_len),
                                            _stream(stream)))
        return dq, dk, dv
    if workspace is None:
        n = lib().vidax_attn_bwd_workspace_floats(B, H, Lq, Lk, d)
        workspace = torch.empty((max(n, B * H * Lq),), dtype=torch.float32, device=q.device)
    elif workspace.dtype != torch.float32 or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous float32 device tensor")
    _check("vidax_attn_bwd", lib().vidax_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lse), _ptr(dq),
                                                  _ptr(dk), _ptr(dv), _ptr(workspace), workspace.numel(), B, H, Lq,
                                                  Lk, d, float(scale), _ptr(kv_valid_len), _stream(stream)))
    return dq, dk, dv


def na3d_fwd(q, k, v, grid, window=(11, 11, 11), border: str = "clip", scale=None, return_lse=False, out=None,
             stream=None):
    """3D neighbourhood attention on a token grid (T, Hp, Wp); q, k, v bf16
    [B, T*Hp*Wp, H, d].  border "clip" or "shift"."""
    import torch

    for n, t in (("q", q), ("k", k), ("v", v)):
        _check_bshd(n, t)
    if k.shape != q.shape or v.shape != q.shape:
        raise ValueError("q, k, v must have the same shape [B, L, H, d]")
    B, L, H, d = q.shape
    T, Hp, Wp = (int(x) for x in grid)
    if T * Hp * Wp != L:
        raise ValueError("grid does not match L")
    if border not in ("clip", "shift"):
        raise ValueError("border must be 'clip' or 'shift'")
    if scale is None:
        scale = float(torch.tensor(1.0 / d ** 0.5, dtype=torch.float32))
    o = torch.empty_like(q) if out is None else out
    _check_bshd("out", o)
    lse = torch.empty((B, H, L), dtype=torch.float32, device=q.device) if return_lse else None
    _check("vidax_na3d_fwd", lib().vidax_na3d_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, H, T, Hp, Wp, d,
                                                  *(int(x) for x in window), 0 if border == "clip" else 1,
                                                  float(scale), _stream(stream)))
    return (o, lse) if return_lse else o


def qkv_proj(x, w, B: int, L: int, H: int, bias=None, gain_q=None, gain_k=None, eps: float = 1e-6,
             rope: Rope | None = None, stream=None):
    """(q, k, v) bf16 [B, L, H, 128] from hidden states x (bf16 [B*L, C]) and
    the projection weight w (bf16 [3*H*128, C]); q and k RMS-normalised per
    head, gained and rotated."""
    import torch

    for n, t in (("x", x), ("w", w)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 2:
            raise ValueError(f"{n} must be a contiguous 2-D bfloat16 device tensor")
    C = x.shape[1]
    d = w.shape[0] // (3 * H) if H > 0 else 0
    if x.shape[0] != B * L or w.shape[1] != C or w.shape[0] != 3 * H * d:
        raise ValueError("x must be [B*L, C] and w [3*H*d, C]")
    for n, t, size in (("bias", bias, 3 * H * d), ("gain_q", gain_q, d), ("gain_k", gain_k, d)):
        if t is not None and (t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous()
                              or t.numel() != size):
            raise ValueError(f"{n} must be a contiguous float32 device tensor of {size} elements")
    q, k, v = (torch.empty((B, L, H, d), dtype=torch.bfloat16, device=x.device) for _ in range(3))
    desc = rope.desc() if rope is not None else None
    _check("vidax_qkv_proj", lib().vidax_qkv_proj(_ptr(x), _ptr(w), _ptr(bias), _ptr(gain_q), _ptr(gain_k),
                                                  float(eps), _ptr(q), _ptr(k), _ptr(v), B, L, H, d, C,
                                                  ctypes.byref(desc) if desc is not None else None,
                                                  _stream(stream)))
    return q, k, v


def qk_norm_rope(x, rope: Rope | None = None, gain=None, eps: float = 1e-6, out=None, stream=None):
    """Per-(token, head) RMS normalisation of x (bf16 [B, L, H, d]), channel
    gain (fp32 [d] device tensor or None), then the 3D rotation (or none);
    out may be x itself (in place)."""
    import torch

    _check_bshd("x", x)
    y = torch.empty_like(x) if out is None else out
    _check_bshd("out", y)
    if y.shape != x.shape:
        raise ValueError("out must have the shape of x")
    B, L, H, d = x.shape
    if gain is not None:
        if gain.dtype != torch.float32 or not gain.is_cuda or not gain.is_contiguous() or gain.numel() != d:
            raise ValueError("gain must be a contiguous float32 device tensor of d elements")
    desc = rope.desc() if rope is not None else None
    _check("vidax_qk_norm_rope", lib().vidax_qk_norm_rope(_ptr(x), _ptr(y), _ptr(gain), float(eps), B, L, H, d,
                                                          ctypes.byref(desc) if desc is not None else None,
                                                          _stream(stream)))
    return y


def _attn(fn_name, q, k, v, scale, kv_valid_len, rope, return_lse, out, stream):
    import torch

    for n, t in (("q", q), ("k", k), ("v", v)):
        _check_bshd(n, t)
    B, Lq, H, d = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[2] != H or k.shape[3] != d:
        raise ValueError("k and v must be [B, Lk, H, d] matching q's B, H, d")
    Lk = k.shape[1]
    if scale is None:
        scale = float(torch.tensor(1.0 / d ** 0.5, dtype=torch.float32))
    o = torch.empty_like(q) if out is None else out
    _check_bshd("out", o)
    lse = torch.empty((B, H, Lq), dtype=torch.float32, device=q.device) if return_lse else None
    if kv_valid_len is not None:
        if kv_valid_len.dtype != torch.int32 or not kv_valid_len.is_cuda or kv_valid_len.numel() != B:
            raise ValueError("kv_valid_len must be an int32 device tensor of B elements")
        kv_valid_len = kv_valid_len.contiguous()
    desc = rope.desc() if rope is not None else None
    fn = getattr(lib(), fn_name)
    st = fn(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, H, Lq, Lk, d, float(scale),
            _ptr(kv_valid_len), ctypes.byref(desc) if desc is not None else None, _stream(stream))
    _check(fn_name, st)
    return (o, lse) if return_lse else o


def attn_fwd(q, k, v, scale=None, kv_valid_len=None, rope: Rope | None = None, return_lse=False, out=None,
             stream=None):
    """softmax(scale * rope(q) rope(k)^T) v on the matrix-core kernel (bf16 in/out, fp32 accumulate)."""
    return _attn("vidax_attn_fwd", q, k, v, scale, kv_valid_len, rope, return_lse, out, stream)


def attn_fwd_naive(q, k, v, scale=None, kv_valid_len=None, rope: Rope | None = None, return_lse=False, out=None,
                   stream=None):
    """Same contract on the scalar fp32 cross-check kernel (small sizes only)."""
    return _attn("vidax_attn_fwd_naive", q, k, v, scale, kv_valid_len, rope, return_lse, out, stream)


# The calls below are short enough on the device (5 us) for the binding to count:
# torch looked up once, plain addresses instead of pointer objects, the raw stream
# instead of a Stream, device numbers instead of devices.

_torch = _raw_stream = _current_device = None


def _load_torch():
    global _torch, _raw_stream, _current_device
    import torch

    _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    _torch = torch
    return torch


def _on(stream, t):
    """Context in which `stream`, of t's device, is current: outputs and workspaces then belong to it."""
    torch = _torch or _load_torch()
    if stream.device_index != t.get_device():
        raise ValueError("stream must be of the tensors' device")
    return torch.cuda.stream(stream)


def _call(fn: str, i: int, *args):
    """fn(*args, stream) with device i current, on that device's current stream."""
    s = _raw_stream(i)
    f = getattr(_lib or lib(), fn)
    if i == _current_device():
        st = f(*args, s)
    else:
        with _torch.cuda.device(i):
            st = f(*args, s)
    if st != VIDAX_OK:
        raise VidaxError(fn, st)


@functools.lru_cache(maxsize=1024)
def _floats(fn: str, device: int, *sizes) -> int:
    """Workspace size by a function of the library (of the sizes and the device alone)."""
    with _torch.cuda.device(device):
        return getattr(lib(), fn)(*sizes)


def _addr(t):
    return None if t is None else t.data_ptr()


def _check_dense(name, t, dtype, shape, i):
    """t: contiguous, of this type and shape, on device i (-1: the CPU)."""
    if t.dtype is not dtype or t.get_device() != i or not t.is_contiguous() or t.shape != shape:
        raise ValueError(f"{name} must be a contiguous {dtype} {list(shape)} tensor on device {i}")


# ------------------------------------- attention with score modifiers ----

_SCALE_128 = 0.08838834764831845  # 1 / sqrt(128), rounded to fp32 at the call


def _score_desc(score, q, Lk):
    """Descriptor of a Score for queries q [B, Lq, H, d] against Lk keys."""
    s = score
    if s is None:
        return ScoreDesc()
    torch = _torch or _load_torch()
    i, f32, i32 = q.get_device(), torch.float32, torch.int32
    B, Lq, H, _ = q.shape
    if (s.q_doc is None) != (s.k_doc is None):
        raise ValueError("q_doc and k_doc come together")
    d = ScoreDesc(s.causal, s.cap)
    if s.slopes is not None:
        _check_dense("slopes", s.slopes, f32, (H,), i)
        d.slopes = s.slopes.data_ptr()
    if s.q_doc is not None:
        _check_dense("q_doc", s.q_doc, i32, (B, Lq), i)
        _check_dense("k_doc", s.k_doc, i32, (B, Lk), i)
        d.q_doc, d.k_doc = s.q_doc.data_ptr(), s.k_doc.data_ptr()
    if s.kv_valid_len is not None:
        _check_dense("kv_valid_len", s.kv_valid_len, i32, (B,), i)
        d.kv_valid_len = s.kv_valid_len.data_ptr()
    if s.prefix_len is not None:
        _check_dense("prefix_len", s.prefix_len, i32, (B,), i)
        d.prefix_len = s.prefix_len.data_ptr()
    if s.q_start is not None:
        _check_dense("q_start", s.q_start, i32, (B,), i)
        d.q_start = s.q_start.data_ptr()
    return d


def _check_mod_qkv(q, k, v):
    """The device number of q, k and v."""
    bf16 = (_torch or _load_torch()).bfloat16
    i, qs, ks = q.get_device(), q.shape, k.shape
    if (q.dtype is not bf16 or k.dtype is not bf16 or v.dtype is not bf16 or i < 0 or len(qs) != 4 or len(ks) != 4
            or not q.is_contiguous() or not k.is_contiguous() or not v.is_contiguous()):
        raise ValueError("q, k and v must be contiguous bfloat16 [B, L, H, d] device tensors")
    if ks != v.shape or ks[0] != qs[0] or ks[3] != qs[3]:
        raise ValueError("k and v must be [B, Lk, Hkv, d] matching q's B and d")
    if k.get_device() != i or v.get_device() != i:
        raise ValueError("q, k and v must be on one device")
    return i


def _workspace(workspace, need, i):
    """The caller's float32 workspace, checked, or a new one of `need` values (None for 0)."""
    if workspace is None:
        return _torch.empty((need,), dtype=_torch.float32, device=i) if need else None
    if workspace.dtype is not _torch.float32 or workspace.get_device() != i or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous float32 tensor on device {i}")
    return workspace


def attn_mod_fwd(q, k, v, score: Score | None = None, scale=None, return_lse=False, out=None, workspace=None,
                 stream=None):
    """Attention with score modifiers: o (and lse) of q bf16 [B, Lq, H, 128] and
    k, v bf16 [B, Lk, Hkv, 128], Hkv a divisor of H.  `workspace`: a contiguous
    float32 device tensor (by default one of vidax_attn_mod_fwd_workspace_floats
    values is allocated where the call needs one)."""
    if stream is not None:
        with _on(stream, q):
            return attn_mod_fwd(q, k, v, score, scale, return_lse, out, workspace)
    i = _check_mod_qkv(q, k, v)
    B, Lq, H, d = q.shape
    _, Lk, Hkv, _ = k.shape
    desc = _score_desc(score, q, Lk)
    if out is None:
        o = _torch.empty_like(q)
    else:
        o = out
        _check_dense("out", o, q.dtype, q.shape, i)
    lse = _torch.empty((B, H, Lq), dtype=_torch.float32, device=i) if return_lse else None
    need = 0
    if workspace is None:
        need = _floats("vidax_attn_mod_fwd_workspace_floats", i, B, H, Hkv, Lq, Lk, d, desc.k_doc is not None)
    ws = None if workspace is None and not need else _workspace(workspace, need, i)
    _call("vidax_attn_mod_fwd", i, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _addr(lse), B, H,
          Hkv, Lq, Lk, d, _SCALE_128 if scale is None else scale, ctypes.byref(desc), _addr(ws),
          0 if ws is None else ws.numel())
    return (o, lse) if return_lse else o


def attn_mod_bwd(q, k, v, o, dout, lse, score: Score | None = None, scale=None, out=None, workspace=None, stream=None):
    """(dq, dk, dv) of attn_mod_fwd from its o and lse; dk and dv are summed over
    the query heads of a K/V head.  `out` = tensors to write into; `workspace`: a
    contiguous float32 device tensor (by default one of
    vidax_attn_mod_bwd_workspace_floats values is allocated)."""
    if stream is not None:
        with _on(stream, q):
            return attn_mod_bwd(q, k, v, o, dout, lse, score, scale, out, workspace)
    i = _check_mod_qkv(q, k, v)
    torch = _torch
    B, Lq, H, d = q.shape
    _, Lk, Hkv, _ = k.shape
    _check_dense("o", o, q.dtype, q.shape, i)
    _check_dense("dout", dout, q.dtype, q.shape, i)
    _check_dense("lse", lse, torch.float32, (B, H, Lq), i)
    desc = _score_desc(score, q, Lk)
    if out is None:
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    else:
        dq, dk, dv = out
        for n, t, ref in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
            _check_dense(n, t, ref.dtype, ref.shape, i)
    need = 0
    if workspace is None:
        need = _floats("vidax_attn_mod_bwd_workspace_floats", i, B, H, Hkv, Lq, Lk, d, desc.k_doc is not None)
    ws = _workspace(workspace, need, i)
    _call("vidax_attn_mod_bwd", i, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), dout.data_ptr(),
          lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Hkv, Lq, Lk, d,
          _SCALE_128 if scale is None else scale, ctypes.byref(desc), _addr(ws), 0 if ws is None else ws.numel())
    return dq, dk, dv


# -------------------------------------------------------- block norm ----

_NORMS = {None: 0, "layer": 1, "rms": 2}


def _block_mod(name, m, t, B, L, C, i):
    """Fills the empty BlockMod m from a modulation [B, C], [B, 1, C] or [B, L, C]; True: one row a token."""
    shape, stride = t.shape, t.stride()
    if not shape or t.dtype is not _torch.float32 or t.get_device() != i or (C > 1 and stride[-1] != 1):
        raise ValueError(f"{name} must be a float32 tensor on device {i} with dense channels")
    m.p = t.data_ptr()
    if B > 1:
        m.batch_stride = stride[0]
    if shape == (B, C) or shape == (B, 1, C):
        return False
    if shape != (B, L, C):
        raise ValueError(f"{name} must be [B, C], [B, 1, C] or [B, L, C]")
    m.token_stride = stride[1]
    return True


def _block_desc(x, y, gate, scale, shift, gain, post_gain, norm, post, eps, alpha):
    """(device number, descriptor, whether the modulations are one row a token: a set)"""
    torch = _torch or _load_torch()
    i, shape, dtype = x.get_device(), x.shape, x.dtype
    wide = dtype is torch.float32
    if len(shape) != 3 or i < 0 or not (wide or dtype is torch.bfloat16) or not x.is_contiguous():
        raise ValueError("x must be a contiguous bfloat16 or float32 [B, L, C] device tensor")
    if norm not in ("layer", "rms") or post not in _NORMS:
        raise ValueError("norm must be 'layer' or 'rms', post one of them or None")
    B, L, C = shape
    if y is not None:
        _check_dense("y", y, torch.bfloat16, shape, i)
    d = BlockNormDesc(wide, _NORMS[norm], _NORMS[post], 0, eps, alpha)
    if gain is not None:
        _check_dense("gain", gain, torch.float32, (C,), i)
        d.gain = gain.data_ptr()
    if post_gain is not None:
        _check_dense("post_gain", post_gain, torch.float32, (C,), i)
        d.post_gain = post_gain.data_ptr()
    token = set()
    if gate is not None:
        token.add(_block_mod("gate", d.gate, gate, B, L, C, i))
    if scale is not None:
        token.add(_block_mod("scale", d.scale, scale, B, L, C, i))
    if shift is not None:
        token.add(_block_mod("shift", d.shift, shift, B, L, C, i))
    return i, d, token


def block_norm_fwd(x, y=None, gate=None, scale=None, shift=None, gain=None, post_gain=None, norm: str = "layer",
                   post: str | None = None, eps: float = 1e-6, alpha: float = 1.0, out=None, stream=None):
    """The step between two sublayers: (x', h) with x' = alpha x + gate post(y)
    post_gain and h = norm(x') gain (1 + scale) + shift.

    x: bf16 or fp32 [B, L, C], the residual stream; y: bf16, the sublayer's
    output, or None (no branch; x' is then x itself where alpha is 1).  gate,
    scale, shift: fp32 [B, C], [B, 1, C] or [B, L, C], rows of any strides that
    are multiples of 4 (slices of one modulation table); gain, post_gain: fp32
    [C].  norm: "layer" or "rms"; post: the norm on the branch, or None.  h is
    bf16.  `out` = (x', h) tensors to write into; x' may be x (in place)."""
    if stream is not None:
        with _on(stream, x):
            return block_norm_fwd(x, y, gate, scale, shift, gain, post_gain, norm, post, eps, alpha, out)
    i, d, _ = _block_desc(x, y, gate, scale, shift, gain, post_gain, norm, post, eps, alpha)
    torch, bf16 = _torch, _torch.bfloat16
    same = y is None and alpha == 1.0
    if out is None:
        xo = None if same else torch.empty_like(x)
        h = torch.empty_like(x) if x.dtype is bf16 else torch.empty_like(x, dtype=bf16)
    else:
        xo, h = out
        if xo is not None:
            _check_dense("out[0]", xo, x.dtype, x.shape, i)
        elif not same:
            raise ValueError("out[0] may be None only where x' is x")
        _check_dense("out[1]", h, bf16, x.shape, i)
    B, L, C = x.shape
    _call("vidax_block_norm_fwd", i, x.data_ptr(), _addr(y), _addr(xo), h.data_ptr(), B, L, C,
          ctypes.byref(d))
    return (x if xo is None else xo), h


def block_norm_bwd(dh, dx, x, y=None, gate=None, scale=None, shift=None, gain=None, post_gain=None,
                   norm: str = "layer", post: str | None = None, eps: float = 1e-6, alpha: float = 1.0, workspace=None,
                   stream=None):
    """Gradients of block_norm_fwd, as a dict: "dx", "dy" (with a branch) and
    "dgate", "dscale", "dshift", "dgain", "dpost_gain" for the operands given,
    each in its operand's shape (fp32).

    dh: gradient of h (bf16); dx: gradient of x' from what reads it later, in
    the stream's type, or None; x: the x' that the forward returned; the rest as
    for the forward (gate, scale and shift are all per sample or all per token).
    `workspace`: a contiguous float32 device tensor of at least
    vidax_block_norm_bwd_workspace_floats values (by default one is allocated)."""
    if stream is not None:
        with _on(stream, x):
            return block_norm_bwd(dh, dx, x, y, gate, scale, shift, gain, post_gain, norm, post, eps, alpha, workspace)
    i, d, token = _block_desc(x, y, gate, scale, shift, gain, post_gain, norm, post, eps, alpha)
    torch = _torch
    if len(token) > 1:
        raise ValueError("gate, scale and shift must all be per sample or all per token")
    d.per_token = int(True in token)
    B, L, C = x.shape
    _check_dense("dh", dh, torch.bfloat16, x.shape, i)
    if dx is not None:
        _check_dense("dx", dx, x.dtype, x.shape, i)
    got = {"dx": torch.empty_like(x)}
    if y is not None:
        got["dy"] = torch.empty_like(y)
    for n, t in (("dgate", gate), ("dscale", scale), ("dshift", shift), ("dgain", gain), ("dpost_gain", post_gain)):
        if t is not None:
            got[n] = torch.empty(t.shape, dtype=torch.float32, device=i)
    g = BlockNormGrads(*(got[n].data_ptr() if n in got else None for n, _ in BlockNormGrads._fields_))
    sums = (not d.per_token and len(token) > 0) or gain is not None or post_gain is not None
    need = 0
    if sums and workspace is None:
        need = _floats("vidax_block_norm_bwd_workspace_floats", i, B, L, C)
    ws = _workspace(workspace, need, i)
    _call("vidax_block_norm_bwd", i, dh.data_ptr(), _addr(dx), x.data_ptr(), _addr(y), got["dx"].data_ptr(),
          _addr(got.get("dy")), ctypes.byref(g), _addr(ws), 0 if ws is None else ws.numel(), B, L, C, ctypes.byref(d))
    return got
