"""Python binding of libpisa (piecewise sparse attention forward pass, MI355X).

Argument marshalling only: every step runs in the HIP kernels of libpisa.so.
torch supplies device memory and the stream.  Importing this package loads the
shared library and raises if it has not been built (`python -m
paper_2602_01077_amd.build`); there is no fallback path of any kind.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Optional, Tuple

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libpisa.so")

PISA_OK, PISA_INVALID_ARG, PISA_UNSUPPORTED, PISA_WORKSPACE_TOO_SMALL, PISA_HIP_ERROR = range(5)
PISA_FP32, PISA_BF16 = 0, 1
PISA_NORM_SPECTRAL, PISA_NORM_FROBENIUS, PISA_NORM_FROBENIUS_FAST = 0, 1, 2

EXPORTS = ("pisa_num_blocks", "pisa_topk_count", "pisa_workspace_bytes", "pisa_block_stats",
           "pisa_block_heterogeneity", "pisa_select", "pisa_attention", "pisa_attention_static",
           "pisa_forward_workspace_bytes", "pisa_forward", "dense_attention",
           "pisa_masked_attention_workspace_bytes", "pisa_masked_attention",
           "pisa_masked_attention_backward_workspace_bytes", "pisa_masked_attention_backward",
           "pisa_paged_append", "pisa_paged_attention_workspace_bytes", "pisa_paged_attention",
           "pisa_probe_mfma_rate", "pisa_probe_shader_clock", "pisa_last_error")


class PisaShape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class PisaStrides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("head", ctypes.c_int64), ("token", ctypes.c_int64)]


class PisaMaskedShape(ctypes.Structure):
    _fields_ = [(x, ctypes.c_int32) for x in ("batch", "heads", "kv_heads", "q_len", "kv_len", "head_dim", "dtype", "causal",
                                              "num_docs")] + \
               [("scale", ctypes.c_float), ("softcap", ctypes.c_float)] + \
               [(x, PisaStrides) for x in ("q", "k", "v", "out")]


class PisaGradStrides(ctypes.Structure):
    _fields_ = [(x, PisaStrides) for x in ("dout", "dq", "dk", "dv")]


class PisaPagedShape(ctypes.Structure):
    _fields_ = [(x, ctypes.c_int32) for x in ("seqs", "heads", "kv_heads", "head_dim", "dtype", "page_size", "num_pages",
                                              "max_pages")] + \
               [("scale", ctypes.c_float), ("softcap", ctypes.c_float)] + \
               [(x, PisaStrides) for x in ("k_pages", "v_pages")]


class PisaError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libpisa error {code}: {message}")
        self.code = code
        self.message = message


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python paper_2602_01077_amd/build.py` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    shp = ctypes.POINTER(PisaShape)
    lib.pisa_num_blocks.argtypes = [i32, i32]
    lib.pisa_num_blocks.restype = i32
    lib.pisa_topk_count.argtypes = [i32, ctypes.c_double]
    lib.pisa_topk_count.restype = i32
    lib.pisa_workspace_bytes.argtypes = [shp]
    lib.pisa_workspace_bytes.restype = sz
    lib.pisa_block_stats.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.pisa_block_stats.restype = i32
    lib.pisa_block_heterogeneity.argtypes = [shp, vp, vp, vp, vp, i32, ctypes.c_double, vp, vp, sz, vp]
    lib.pisa_block_heterogeneity.restype = i32
    lib.pisa_select.argtypes = [shp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.pisa_select.restype = i32
    lib.pisa_attention.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.pisa_attention.restype = i32
    lib.pisa_attention_static.argtypes = [shp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.pisa_attention_static.restype = i32
    lib.pisa_forward_workspace_bytes.argtypes = [shp, i32]
    lib.pisa_forward_workspace_bytes.restype = sz
    lib.pisa_forward.argtypes = [shp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.pisa_forward.restype = i32
    lib.dense_attention.argtypes = [shp, vp, vp, vp, vp, vp, vp]
    lib.dense_attention.restype = i32
    mshp, gstr, pshp = (ctypes.POINTER(x) for x in (PisaMaskedShape, PisaGradStrides, PisaPagedShape))
    lib.pisa_masked_attention_workspace_bytes.argtypes = [mshp]
    lib.pisa_masked_attention_workspace_bytes.restype = sz
    lib.pisa_masked_attention.argtypes = [mshp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.pisa_masked_attention.restype = i32
    lib.pisa_masked_attention_backward_workspace_bytes.argtypes = [mshp]
    lib.pisa_masked_attention_backward_workspace_bytes.restype = sz
    lib.pisa_masked_attention_backward.argtypes = [mshp, gstr] + [vp] * 13 + [sz, vp]
    lib.pisa_masked_attention_backward.restype = i32
    lib.pisa_paged_append.argtypes = [pshp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.pisa_paged_append.restype = i32
    lib.pisa_paged_attention_workspace_bytes.argtypes = [pshp]
    lib.pisa_paged_attention_workspace_bytes.restype = sz
    lib.pisa_paged_attention.argtypes = [pshp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.pisa_paged_attention.restype = i32
    lib.pisa_probe_mfma_rate.argtypes = [i32, vp, sz, ctypes.POINTER(ctypes.c_double), vp]
    lib.pisa_probe_mfma_rate.restype = i32
    lib.pisa_probe_shader_clock.argtypes = [ctypes.c_double, vp, ctypes.POINTER(ctypes.c_double), vp]
    lib.pisa_probe_shader_clock.restype = i32
    lib.pisa_last_error.argtypes = []
    lib.pisa_last_error.restype = ctypes.c_char_p
    return lib


_lib = _load()


def raw() -> ctypes.CDLL:
    """The ctypes handle, for tests that call the C ABI with hand-made arguments."""
    return _lib


def last_error() -> str:
    return _lib.pisa_last_error().decode()


def _check(code: int) -> None:
    if code != PISA_OK:
        raise PisaError(code, last_error())


def num_blocks(seq_len: int, block: int) -> int:
    return _lib.pisa_num_blocks(seq_len, block)


def topk_count(n_blocks: int, sparsity: float) -> int:
    return _lib.pisa_topk_count(n_blocks, float(sparsity))


def resolved_scale(head_dim: int, scale: Optional[float] = None) -> float:
    """The fp32 softmax scale the library uses (as a Python float)."""
    s = 1.0 / math.sqrt(head_dim) if scale is None or scale <= 0 else scale
    return float(torch.tensor(s, dtype=torch.float32).item())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return PISA_FP32
    if t.dtype == torch.bfloat16:
        return PISA_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def make_shape(q: torch.Tensor, block: int, scale: Optional[float] = None) -> PisaShape:
    if q.dim() != 4:
        raise ValueError("expected [batch, heads, seq_len, head_dim]")
    b, h, L, d = q.shape
    return PisaShape(b, h, L, d, block, _dtype_code(q), 0.0 if scale is None else float(scale))


def _dev(t: Optional[torch.Tensor], name: str, dtype=None, like: Optional[torch.Tensor] = None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if like is not None and (t.dtype != like.dtype or t.shape != like.shape or t.device != like.device):
        raise ValueError(f"{name} must match q in shape, dtype and device")
    return ctypes.c_void_p(t.data_ptr())


def _stream() -> int:
    """The current stream's handle.  Straight from the runtime's own table: a torch.cuda.Stream object costs 4 us a call, a
    third of what a short call takes on the host."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def workspace_bytes(shape: PisaShape) -> int:
    return int(_lib.pisa_workspace_bytes(ctypes.byref(shape)))


def alloc_workspace(shape: PisaShape, device) -> torch.Tensor:
    return torch.empty(max(1, workspace_bytes(shape)), dtype=torch.uint8, device=device)


def block_stats(q, k, v, block: int, workspace: Optional[torch.Tensor] = None):
    """pisa_block_stats.  Returns dict(qbar, kbar, vsum, hsum, qbar64, kbar64)."""
    shape = make_shape(q, block)
    b, h, L, d = q.shape
    n = num_blocks(L, block)
    dev = q.device
    out = dict(
        qbar=torch.empty(b, h, n, d, dtype=torch.float32, device=dev),
        kbar=torch.empty(b, h, n, d, dtype=torch.float32, device=dev),
        vsum=torch.empty(b, h, n, d, dtype=torch.float32, device=dev),
        hsum=torch.empty(b, h, d, d, dtype=torch.float32, device=dev),
        qbar64=torch.empty(b, h, n, d, dtype=torch.float64, device=dev),
        kbar64=torch.empty(b, h, n, d, dtype=torch.float64, device=dev),
    )
    ws = alloc_workspace(shape, dev) if workspace is None else workspace
    block_stats_into(shape, q, k, v, out, ws)
    return out


def block_stats_into(shape, q, k, v, out: dict, workspace: torch.Tensor) -> None:
    _check(_lib.pisa_block_stats(
        ctypes.byref(shape), _dev(q, "q"), _dev(k, "k", like=q), _dev(v, "v", like=q),
        _dev(out["qbar"], "qbar", torch.float32), _dev(out["kbar"], "kbar", torch.float32),
        _dev(out["vsum"], "vsum", torch.float32), _dev(out["hsum"], "hsum", torch.float32),
        _dev(out["qbar64"], "qbar64", torch.float64), _dev(out["kbar64"], "kbar64", torch.float64),
        _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream()))


def block_heterogeneity(shape: PisaShape, k, v, kbar64, norm: int = PISA_NORM_SPECTRAL, eps: float = 1e-6,
                        workspace: Optional[torch.Tensor] = None, hsum: Optional[torch.Tensor] = None
                        ) -> torch.Tensor:
    """pisa_block_heterogeneity.  Returns log(M_j + eps), fp64 [b,h,N].  hsum (fp32, from
    block_stats) lets the library take Hbar from it instead of accumulating it again in fp64."""
    b, h = k.shape[0], k.shape[1]
    n = num_blocks(shape.seq_len, shape.block)
    log_m = torch.empty(b, h, n, dtype=torch.float64, device=k.device)
    ws = alloc_workspace(shape, k.device) if workspace is None else workspace
    _check(_lib.pisa_block_heterogeneity(
        ctypes.byref(shape), _dev(k, "k"), _dev(v, "v", like=k), _dev(kbar64, "kbar64", torch.float64),
        _dev(hsum, "hsum", torch.float32), norm, float(eps), _dev(log_m, "log_m", torch.float64),
        _dev(ws, "workspace"), ws.numel() * ws.element_size(), _stream()))
    return log_m


def select(shape: PisaShape, qbar64, kbar64, k_top: int, workspace: Optional[torch.Tensor] = None,
           want_gap: bool = True, col_bias: Optional[torch.Tensor] = None
           ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """pisa_select.  Returns (idx int32 [b,h,N,k_top], kth_gap fp32 [b,h,N] or None)."""
    b, h, n, _ = qbar64.shape
    dev = qbar64.device
    idx = torch.empty(b, h, n, k_top, dtype=torch.int32, device=dev)
    gap = torch.empty(b, h, n, dtype=torch.float32, device=dev) if want_gap else None
    ws = alloc_workspace(shape, dev) if workspace is None else workspace
    select_into(shape, qbar64, kbar64, k_top, idx, gap, ws, col_bias)
    return idx, gap


def select_into(shape, qbar64, kbar64, k_top: int, idx, gap, workspace, col_bias=None) -> None:
    _check(_lib.pisa_select(
        ctypes.byref(shape), _dev(qbar64, "qbar64", torch.float64), _dev(kbar64, "kbar64", torch.float64),
        _dev(col_bias, "col_bias", torch.float64), k_top, _dev(idx, "idx", torch.int32) if k_top > 0 else None, _dev(gap, "kth_gap", torch.float32),
        _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream()))


def attention(shape: PisaShape, q, k, v, kbar, vsum, hsum, idx, k_top: int,
              out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
              want_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """pisa_attention.  Returns (out, lse or None)."""
    if workspace is None:
        workspace = alloc_workspace(shape, q.device)
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    _check(_lib.pisa_attention(
        ctypes.byref(shape), _dev(q, "q"), _dev(k, "k", like=q), _dev(v, "v", like=q),
        _dev(kbar, "kbar", torch.float32), _dev(vsum, "vsum", torch.float32),
        _dev(hsum, "hsum", torch.float32),
        _dev(idx, "idx", torch.int32) if k_top > 0 else None, k_top,
        _dev(out, "out", like=q), _dev(lse, "lse", torch.float32),
        _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(), _stream()))
    return out, lse


STATIC_SCRATCH_BYTES = 40 << 20


def attention_static(shape: PisaShape, q, k, v, kbar, vsum, hsum, idx, k_top: int,
                     out: torch.Tensor, lse: Optional[torch.Tensor] = None):
    """pisa_attention_static: pisa_attention on the library's built-in scratch array; the
    caller passes every buffer (nothing is allocated here either).  Returns (out, lse)."""
    _check(_lib.pisa_attention_static(
        ctypes.byref(shape), _dev(q, "q"), _dev(k, "k", like=q), _dev(v, "v", like=q),
        _dev(kbar, "kbar", torch.float32), _dev(vsum, "vsum", torch.float32),
        _dev(hsum, "hsum", torch.float32),
        _dev(idx, "idx", torch.int32) if k_top > 0 else None, k_top,
        _dev(out, "out", like=q), _dev(lse, "lse", torch.float32), _stream()))
    return out, lse


def dense_attention(q, k, v, block: int = 64, scale: Optional[float] = None,
                    out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                    want_lse: bool = False):
    """dense_attention.  Returns (out, lse or None)."""
    shape = make_shape(q, block, scale)
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    _check(_lib.dense_attention(
        ctypes.byref(shape), _dev(q, "q"), _dev(k, "k", like=q), _dev(v, "v", like=q),
        _dev(out, "out", like=q), _dev(lse, "lse", torch.float32), _stream()))
    return out, lse


def _on_current_device(ref: torch.Tensor, *others: Optional[torch.Tensor]) -> None:
    device = ref.get_device()
    if device < 0:
        raise ValueError("tensors must live on the GPU")
    if device != torch._C._cuda_getDevice():
        raise ValueError(f"tensors live on {ref.device}, the current device is cuda:{torch.cuda.current_device()}")
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError(f"all tensors must live on {ref.device}, got one on {t.device}")


def _plain(t: Optional[torch.Tensor], name: str, dtype, shape) -> Optional[int]:
    """Address of a dense tensor of a given type and shape."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _workspace(t: Optional[torch.Tensor], need: int, device) -> Tuple[Optional[torch.Tensor], Optional[int], int]:
    """(the tensor, which has to live until the launch, its address, its size)"""
    if t is None:
        if not need:
            return None, None, 0
        t = torch.empty(need, dtype=torch.uint8, device=device)
        return t, t.data_ptr(), need
    if not t.is_contiguous() or t.device != device:
        raise ValueError("workspace must be contiguous and on the tensors' device")
    return t, t.data_ptr(), t.numel() * t.element_size()


def _strides(size, stride, name: str) -> PisaStrides:
    """Of a [batch, heads, tokens, head_dim] view; the channels of a row have to lie together."""
    if stride[3] != 1 and size[3] > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if stride[2] == 0 and size[2] > 1:           # with batch and head strides of 0 the library would take it for a dense tensor
        raise ValueError(f"{name}: one row cannot stand for all tokens (a stride of 0)")
    return PisaStrides(stride[0], stride[1], stride[2] if size[2] > 1 else max(stride[2], size[3]))


# The structures of recent calls, by sizes, strides and options (building one anew costs as much as the launch).
@functools.lru_cache(maxsize=1024)
def _masked_plan(q_size, k_size, v_size, out_size, q_stride, k_stride, v_stride, out_stride, dtype, causal, docs, softcap, scale):
    """(shape, workspace of the forward call, of the backward call)"""
    if len(q_size) != 4 or len(k_size) != 4 or len(v_size) != 4:
        raise ValueError("expected q, k, v of shape [batch, heads, tokens, head_dim]")
    b, h, n, d = q_size
    if k_size != v_size or k_size[0] != b or k_size[3] != d:
        raise ValueError(f"k and v must be alike and match q in batch and head_dim: {tuple(q_size)}, {tuple(k_size)}, {tuple(v_size)}")
    if out_size != q_size:
        raise ValueError("out must match q in shape")
    shape = PisaMaskedShape(b, h, k_size[1], n, k_size[2], d, dtype, 1 if causal else 0, docs, scale, softcap,
                            _strides(q_size, q_stride, "q"), _strides(k_size, k_stride, "k"), _strides(v_size, v_stride, "v"),
                            _strides(out_size, out_stride, "out"))
    return shape, _lib.pisa_masked_attention_workspace_bytes(shape), _lib.pisa_masked_attention_backward_workspace_bytes(shape)


@functools.lru_cache(maxsize=1024)
def _grad_strides(q_size, k_size, dout_stride, dq_stride, dk_stride, dv_stride):
    return PisaGradStrides(_strides(q_size, dout_stride, "dout"), _strides(q_size, dq_stride, "dq"),
                           _strides(k_size, dk_stride, "dk"), _strides(k_size, dv_stride, "dv"))


def _masked_call(q, k, v, out, causal, doc_offsets, softcap, scale):
    if k.dtype != q.dtype or v.dtype != q.dtype or out.dtype != q.dtype:
        raise TypeError("q, k, v and out must have one dtype")
    docs = 0
    if doc_offsets is not None:
        if doc_offsets.dim() != 2 or doc_offsets.shape[1] < 2:
            raise ValueError("doc_offsets must have shape [batch, documents + 1], with one document at least")
        docs = doc_offsets.shape[1] - 1
    return _masked_plan(q.shape, k.shape, v.shape, out.shape, q.stride(), k.stride(), v.stride(), out.stride(), _dtype_code(q),
                        bool(causal), docs, float(softcap), 0.0 if scale is None else float(scale))


def masked_attention_workspace_bytes(q, k, v, causal: bool = False, doc_offsets: Optional[torch.Tensor] = None,
                                     backward: bool = False) -> int:
    """Bytes of workspace that masked_attention, or masked_attention_backward, needs for tensors of these shapes.  Raises what
    those would for shapes that they refuse."""
    out = torch.empty_like(q, device="meta")     # laid out as masked_attention lays out its own (q may be expanded, out never is)
    shape, forward, back = _masked_call(q, k, v, out, causal, doc_offsets, 0.0, None)
    if not back:                                 # a shape that is taken has some
        _check(_lib.pisa_masked_attention(shape, *[None] * 9, 0, None))
    return back if backward else forward


def masked_attention(q, k, v, causal: bool = False, doc_offsets: Optional[torch.Tensor] = None,
                     prefix: Optional[torch.Tensor] = None, softcap: float = 0.0, slopes: Optional[torch.Tensor] = None,
                     scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                     workspace: Optional[torch.Tensor] = None):
    """pisa_masked_attention.  q [batch, heads, q_len, d], k and v [batch, kv_heads, kv_len, d], any strides with whole
    rows of channels (a [batch, tokens, heads, d] tensor goes in as its transpose(1, 2)); doc_offsets int32
    [batch, documents + 1], prefix int32 [batch, documents] (or [batch, 1]), slopes fp32 [heads].  Returns (out, lse or None);
    `out` is laid out as q unless given.  Autograd does not see the call: what it returns has no graph, whatever q, k and v
    require, and gradients are masked_attention_backward's."""
    if out is None:
        out = torch.empty_like(q)
    shape, need, _ = _masked_call(q, k, v, out, causal, doc_offsets, softcap, scale)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    _on_current_device(q, k, v, out, lse, doc_offsets, prefix, slopes)
    keep, ws, size = _workspace(workspace, need, q.device)
    _check(_lib.pisa_masked_attention(
        shape, q.data_ptr(), k.data_ptr(), v.data_ptr(),
        _plain(doc_offsets, "doc_offsets", torch.int32, (shape.batch, shape.num_docs + 1)),
        _plain(prefix, "prefix", torch.int32, (shape.batch, shape.num_docs or 1)),
        _plain(slopes, "slopes", torch.float32, (shape.heads,)),
        out.data_ptr(), _plain(lse, "lse", torch.float32, q.shape[:3]), ws, size, _stream()))
    return out, lse


def masked_attention_backward(q, k, v, out, lse, dout, causal: bool = False, doc_offsets: Optional[torch.Tensor] = None,
                              prefix: Optional[torch.Tensor] = None, softcap: float = 0.0,
                              slopes: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                              dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                              dv: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """pisa_masked_attention_backward: gradients of masked_attention(...) with the same arguments, from its out and lse and
    the gradient dout of out.  Returns (dq, dk, dv).  out and lse have to be of these very keys (bf16 counts on it: not of calls
    over parts of them, joined)."""
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    shape, _, need = _masked_call(q, k, v, out, causal, doc_offsets, softcap, scale)
    for name, t, like in (("dout", dout, q), ("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        if t.shape != like.shape or t.dtype != like.dtype:
            raise ValueError(f"{name} must have shape {tuple(like.shape)} and dtype {like.dtype}")
    strides = _grad_strides(q.shape, k.shape, dout.stride(), dq.stride(), dk.stride(), dv.stride())
    _on_current_device(q, k, v, out, lse, dout, doc_offsets, prefix, slopes, dq, dk, dv)
    keep, ws, size = _workspace(workspace, need, q.device)
    _check(_lib.pisa_masked_attention_backward(
        shape, strides, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), _plain(lse, "lse", torch.float32, q.shape[:3]),
        dout.data_ptr(), _plain(doc_offsets, "doc_offsets", torch.int32, (shape.batch, shape.num_docs + 1)),
        _plain(prefix, "prefix", torch.int32, (shape.batch, shape.num_docs or 1)),
        _plain(slopes, "slopes", torch.float32, (shape.heads,)),
        dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws, size, _stream()))
    return dq, dk, dv


@functools.lru_cache(maxsize=1024)
def _paged_plan(k_size, v_size, k_stride, v_stride, dtype, table_size, heads, softcap, scale):
    """(shape, workspace of paged_attention)"""
    if len(k_size) != 4 or k_size != v_size:
        raise ValueError("expected k_pages and v_pages of one shape [pages, page_size, kv_heads, head_dim]")
    if len(table_size) != 2:
        raise ValueError("page_table must have shape [sequences, pages of the longest]")
    pages, page, kvh, d = k_size

    def strides(st, name):                 # as [pages, kv_heads, page_size, head_dim], the order of PisaStrides
        return _strides((pages, kvh, page, d), (st[0], st[2], st[1], st[3]), name)
    shape = PisaPagedShape(table_size[0], heads if heads else kvh, kvh, d, dtype, page, pages, table_size[1], scale, softcap,
                           strides(k_stride, "k_pages"), strides(v_stride, "v_pages"))
    return shape, _lib.pisa_paged_attention_workspace_bytes(shape)


def _paged_call(k_pages, v_pages, page_table, heads, softcap, scale):
    if v_pages.dtype != k_pages.dtype:
        raise TypeError("k_pages and v_pages must have one dtype")
    return _paged_plan(k_pages.shape, v_pages.shape, k_pages.stride(), v_pages.stride(), _dtype_code(k_pages), page_table.shape,
                       heads, float(softcap), 0.0 if scale is None else float(scale))


def paged_append(k, v, offsets, k_pages, v_pages, page_table, lengths) -> None:
    """pisa_paged_append: rows offsets[s] .. offsets[s+1]-1 of k and v [tokens, kv_heads, d] become the last cached tokens of
    sequence s, whose lengths[s] counts them already.  offsets int32 [sequences + 1], page_table int32 [sequences, pages],
    lengths int32 [sequences]; k_pages and v_pages as for paged_attention, written in place."""
    shape, _ = _paged_call(k_pages, v_pages, page_table, 0, 0.0, None)
    if k.dim() != 3:
        raise ValueError("expected k and v of shape [tokens, kv_heads, head_dim]")
    _on_current_device(k_pages, v_pages, k, v, offsets, page_table, lengths)
    tokens = k.shape[0]
    rows = (tokens, shape.kv_heads, shape.head_dim)
    _check(_lib.pisa_paged_append(
        shape, _plain(k, "k", k_pages.dtype, rows), _plain(v, "v", k_pages.dtype, rows), tokens,
        _plain(offsets, "offsets", torch.int32, (shape.seqs + 1,)), k_pages.data_ptr(), v_pages.data_ptr(),
        _plain(page_table, "page_table", torch.int32, page_table.shape),
        _plain(lengths, "lengths", torch.int32, (shape.seqs,)), _stream()))


def paged_attention_workspace_bytes(q, k_pages, v_pages, page_table) -> int:
    """Bytes of workspace that paged_attention needs for tensors of these shapes (whatever the lengths).  Raises what that would
    for shapes that it refuses."""
    shape, need = _paged_call(k_pages, v_pages, page_table, q.shape[1], 0.0, None)
    if not need:
        _check(_lib.pisa_paged_attention(shape, *[None] * 9, 0, None))
    return need


def paged_attention(q, k_pages, v_pages, page_table, lengths, softcap: float = 0.0, slopes: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                    workspace: Optional[torch.Tensor] = None):
    """pisa_paged_attention: one query row per sequence and head, q [sequences, heads, d], over a cache k_pages, v_pages
    [pages, page_size, kv_heads, d] (any strides with whole rows of channels; lengths int32 [sequences], page_table int32
    [sequences, pages]).  Returns (out, lse or None)."""
    if q.dim() != 3:
        raise ValueError("expected q of shape [sequences, heads, head_dim]")
    if q.dtype != k_pages.dtype:
        raise TypeError("q and the pages must have one dtype")
    shape, need = _paged_call(k_pages, v_pages, page_table, q.shape[1], softcap, scale)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    _on_current_device(q, k_pages, v_pages, page_table, lengths, slopes, out, lse)
    rows = (shape.seqs, shape.heads, shape.head_dim)
    keep, ws, size = _workspace(workspace, need, q.device)
    _check(_lib.pisa_paged_attention(
        shape, _plain(q, "q", q.dtype, rows), k_pages.data_ptr(), v_pages.data_ptr(),
        _plain(page_table, "page_table", torch.int32, page_table.shape), _plain(lengths, "lengths", torch.int32, (shape.seqs,)),
        _plain(slopes, "slopes", torch.float32, (shape.heads,)), _plain(out, "out", q.dtype, rows),
        _plain(lse, "lse", torch.float32, rows[:2]), ws, size, _stream()))
    return out, lse


def probe_mfma_rate(iters: int, sink: torch.Tensor) -> float:
    """pisa_probe_mfma_rate: enqueues the matrix-instruction loop; returns its flop count
    (the caller times the launch)."""
    flop = ctypes.c_double(0.0)
    _check(_lib.pisa_probe_mfma_rate(iters, _dev(sink, "sink", torch.float32), sink.numel(), ctypes.byref(flop),
                                     _stream()))
    return flop.value


def probe_shader_clock(window_ms: float, counts: torch.Tensor) -> float:
    """pisa_probe_shader_clock: enqueues the clock probe on the current stream; `counts` is an
    int64 device tensor of two entries.  Returns the wall clock's rate in Hz; once the stream
    has drained, counts[0] / counts[1] * rate is the shader clock held during the window."""
    hz = ctypes.c_double(0.0)
    _check(_lib.pisa_probe_shader_clock(float(window_ms), _dev(counts, "counts", torch.int64), ctypes.byref(hz),
                                        _stream()))
    return hz.value


def forward_workspace_bytes(shape: PisaShape, k_top: int) -> int:
    return _lib.pisa_forward_workspace_bytes(ctypes.byref(shape), k_top)


def forward(shape: PisaShape, q, k, v, k_top: int, out: Optional[torch.Tensor] = None,
            lse: Optional[torch.Tensor] = None, want_lse: bool = False,
            workspace: Optional[torch.Tensor] = None):
    """pisa_forward: statistics, selection and attention in one library call (three launches on
    the bf16 path for short sequences).  Returns (out, lse or None)."""
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.empty(forward_workspace_bytes(shape, k_top), dtype=torch.uint8, device=q.device)
    _check(_lib.pisa_forward(
        ctypes.byref(shape), _dev(q, "q"), _dev(k, "k", like=q), _dev(v, "v", like=q), k_top,
        _dev(out, "out", like=q), _dev(lse, "lse", torch.float32),
        _dev(workspace, "workspace", torch.uint8), workspace.numel(), _stream()))
    return out, lse


def forward_in_steps(q, k, v, block: int = 64, sparsity: float = 0.85, first_order: bool = True,
                 want_lse: bool = False, approximate: bool = True, covariance_aware: bool = False,
                 norm: int = PISA_NORM_SPECTRAL, eps: float = 1e-6, scale: Optional[float] = None,
                 hbar_from_stats: bool = False):
    """The whole hot path as separate library calls: block_stats -> select -> attention (the
    variants and the covariance-aware score are options of those calls; `forward` is the one-call
    form of the default configuration).

    first_order=False gives the zeroth-order variant, approximate=False plain block-sparse
    attention over the selected blocks, covariance_aware=True adds log(M_j + eps) to the
    selection score (hbar_from_stats=True: with Hbar from the statistics' fp32 hsum).  Returns dict(out, lse, idx, kth_gap, stats, k_top, log_m).
    """
    shape = make_shape(q, block, scale)
    n = num_blocks(q.shape[2], block)
    k_top = topk_count(n, sparsity)
    ws = alloc_workspace(shape, q.device)
    stats = block_stats(q, k, v, block, ws)
    log_m = block_heterogeneity(shape, k, v, stats["kbar64"], norm, eps, ws,
                                hsum=stats["hsum"] if (hbar_from_stats or norm == PISA_NORM_FROBENIUS_FAST) else None
                                ) if covariance_aware else None
    idx, gap = select(shape, stats["qbar64"], stats["kbar64"], k_top, ws, col_bias=log_m)
    out, lse = attention(shape, q, k, v, stats["kbar"] if approximate else None,
                         stats["vsum"] if approximate else None,
                         stats["hsum"] if (first_order and approximate) else None, idx, k_top,
                         want_lse=want_lse, workspace=ws)
    return dict(out=out, lse=lse, idx=idx, kth_gap=gap, stats=stats, k_top=k_top, log_m=log_m)
