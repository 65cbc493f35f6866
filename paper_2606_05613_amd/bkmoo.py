"""Python binding of libbkmoo (argument marshalling only).

Every step of the path runs in the HIP library; this module turns torch
tensors into the C ABI's pointers and sizes, allocates outputs and the
workspace with torch's caching allocator when the caller passes none, and
raises on any non-OK status.  There is no fallback: if the library is not
built, importing this module fails.

Names mirror include/bkmoo.h: workspace_size, gram, solve, combine, resolve,
resolve_noalloc, conflicts, slice_offsets, gram_reduce, resolve_path, resolve_traffic,
read_device_error, set_resolve_path, set_wait_limit, set_grid_override,
status_string; and for the layer around the resolve residual_norm_forward,
residual_norm_backward, ffn_forward, ffn_backward, set_ffn_tiles, adamw_table, adamw.

The calls take and fill tensors' memory and know nothing of autograd: outputs of inputs
that require gradients have no graph, and tensors that a call writes (adamw()'s
parameters among them) keep their autograd version.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Union

import torch  # must be imported before the library so both share one HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbkmoo.so")

F32, BF16 = 0, 1
METHODS = {"mgda": 0, "pcgrad": 1, "cagrad": 2, "mean": 3, "mgda-exact": 4, "cagrad-exact": 5}
DEVERR_OFFSETS = 0x1
DEVERR_TIMEOUT = 0x2
PATH_TWO_PASS, PATH_HYBRID, PATH_REFILL = 1, 3, 4
ACTS = {"silu": 0, "gelu": 1}
STATE_F32, STATE_F8 = 0, 1


class BkmooError(RuntimeError):
    pass


class _Hparams(ctypes.Structure):
    _fields_ = [("max_iter", ctypes.c_int32), ("cagrad_c", ctypes.c_double),
                ("pcgrad_order", ctypes.c_void_p)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("decay", ctypes.c_int32)]


class _AdamwHparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64),
                ("seed", ctypes.c_uint32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2606_05613_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, sz, vp, u32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_uint32
    vpp = ctypes.POINTER(ctypes.c_void_p)
    cint, f64 = ctypes.c_int, ctypes.c_double
    i64p = ctypes.POINTER(i64)
    sig = {
        "bkmoo_workspace_size": [i32, i64, i32, ctypes.c_int, ctypes.POINTER(sz)],
        "bkmoo_gram": [i32, vpp, ctypes.c_int, i64, i32, vp, vp, vp, sz, vp],
        "bkmoo_solve": [i32, i32, vp, ctypes.c_int, ctypes.POINTER(_Hparams), vp, vp, vp],
        "bkmoo_combine": [i32, vpp, ctypes.c_int, i64, i32, vp, vp, vp, ctypes.c_int, vp, sz, vp],
        "bkmoo_resolve": [i32, vpp, ctypes.c_int, i64, i32, vp, ctypes.c_int, ctypes.POINTER(_Hparams),
                          vp, ctypes.c_int, vp, vp, vp, vp, sz, vp],
        "bkmoo_resolve_noalloc": [i32, vpp, ctypes.c_int, i64, i32, vp, ctypes.c_int, ctypes.POINTER(_Hparams),
                                  vp, ctypes.c_int, vp, vp, vp, vp],
        "bkmoo_conflicts": [i32, i32, vp, vp, vp, vp, vp],
        "bkmoo_slice_offsets": [i32, i32, vp, vp, vp],
        "bkmoo_resolve_traffic": [i32, i64, i32, vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, i32, i32,
                                  ctypes.POINTER(ctypes.c_uint64)],
        "bkmoo_gram_reduce": [i32, i32, i32, vp, ctypes.c_int, vp, vp],
        "bkmoo_read_device_error": [vp, ctypes.POINTER(u32), vp],
        "bkmoo_set_grid_override": [i32],
        "bkmoo_resolve_path": [i32, i64, i32, ctypes.c_int, ctypes.c_int, i32, ctypes.c_int, i32,
                               ctypes.POINTER(i32)],
        "bkmoo_set_resolve_path": [i32],
        "bkmoo_set_wait_limit": [u32],
        "bkmoo_residual_norm_forward": [i64, i64, cint, vp, vp, vp, vp, vp, f64, f64, vp, vp, vp],
        "bkmoo_residual_norm_workspace_size": [i64, i64, i32, ctypes.POINTER(sz)],
        "bkmoo_residual_norm_backward": [i64, i64, cint, i32, i64p, vp, vp, vp, vp, vp, vp, vp, f64, f64,
                                         vp, vp, vp, vp, vp, i64, vp, sz, vp],
        "bkmoo_ffn_workspace_size": [i64, i64, i64, cint, i32, ctypes.POINTER(sz)],
        "bkmoo_ffn_forward": [i64, i64, i64, cint, cint, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "bkmoo_ffn_backward": [i64, i64, i64, cint, cint, i32, i64p, vp, vp, vp, vp, vp, vp, vp,
                               vp, vp, vp, vp, i64, vp, sz, vp],
        "bkmoo_set_ffn_tiles": [i32, i32, i32],
        "bkmoo_adamw_blocks": [i32, ctypes.POINTER(_Tensor), i64p],
        "bkmoo_adamw": [i32, ctypes.POINTER(_Tensor), cint, i64, vp, cint, cint, vp, vp, vp, i64, vp,
                        ctypes.POINTER(_AdamwHparams), vp, vp],
        "bkmoo_status_string": [ctypes.c_int],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_char_p if name == "bkmoo_status_string" else ctypes.c_int
    return lib


_lib = _load()

EXPORTS = ("bkmoo_workspace_size", "bkmoo_gram", "bkmoo_solve", "bkmoo_combine", "bkmoo_resolve",
           "bkmoo_resolve_noalloc",
           "bkmoo_conflicts", "bkmoo_slice_offsets", "bkmoo_gram_reduce", "bkmoo_resolve_traffic",
           "bkmoo_read_device_error", "bkmoo_set_grid_override", "bkmoo_resolve_path",
           "bkmoo_set_resolve_path", "bkmoo_set_wait_limit",
           "bkmoo_residual_norm_forward", "bkmoo_residual_norm_workspace_size", "bkmoo_residual_norm_backward",
           "bkmoo_ffn_workspace_size", "bkmoo_ffn_forward", "bkmoo_ffn_backward",
           "bkmoo_set_ffn_tiles", "bkmoo_adamw_blocks", "bkmoo_adamw", "bkmoo_status_string")


def status_string(st: int) -> str:
    return _lib.bkmoo_status_string(st).decode()


def _check(st: int, what: str):
    if st != 0:
        raise BkmooError(f"{what}: {status_string(st)} ({st})")


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype} (float32 or bfloat16)")


def _torch_dt(code: int):
    return torch.float32 if code == F32 else torch.bfloat16


def _stream_ptr(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


Grads = Union[torch.Tensor, Sequence[torch.Tensor]]


def _rows(grads: Grads):
    """K row pointers (host array), dtype code, K, N, device."""
    if isinstance(grads, torch.Tensor):
        if grads.dim() != 2:
            raise ValueError("grads must be [K, N] or a list of K 1-D tensors")
        if not grads.is_contiguous():
            raise ValueError("a [K, N] grads tensor must be contiguous")
        rows = [grads[i] for i in range(grads.shape[0])]
    else:
        rows = list(grads)
    if not rows:
        raise ValueError("no gradient rows")
    dt = _dt(rows[0])
    n = rows[0].numel()
    dev = rows[0].device
    for r in rows:
        if r.dtype != rows[0].dtype or r.numel() != n or r.device != dev or r.dim() != 1 \
                or not r.is_contiguous():
            raise ValueError("rows must be contiguous 1-D tensors of one dtype, length and device")
        if dev.type != "cuda":
            raise ValueError("gradient rows must be on a GPU")
    arr = (ctypes.c_void_p * len(rows))(*[r.data_ptr() for r in rows])
    return arr, dt, len(rows), n, dev, rows


def _gpu(t: torch.Tensor, what: str):
    """The GPU device of t; host tensors are refused (the kernels would
    dereference their pointers on the GPU)."""
    if t.device.type != "cuda":
        raise ValueError(f"{what} must be on a GPU")
    return t.device


def _tensor(t: torch.Tensor, shape, dtype, dev, what: str) -> int:
    """Pointer of a caller-supplied tensor that must match exactly."""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != dev:
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}")
    return t.data_ptr()


def _offsets(offsets: torch.Tensor, dev) -> torch.Tensor:
    if offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.device != dev \
            or not offsets.is_contiguous():
        raise ValueError("bucket_offsets must be a contiguous int64 1-D tensor on the grads' device")
    return offsets


def _hparams(max_iter: int, cagrad_c: float, pcgrad_order: Optional[torch.Tensor], K: int, B: int, dev):
    ptr = None
    if pcgrad_order is not None:
        ptr = _tensor(pcgrad_order, (B, K, K - 1), torch.int8, dev, "pcgrad_order")
    return _Hparams(int(max_iter), float(cagrad_c), ptr)


def workspace_size(K: int, N: int, B: int, dtype) -> int:
    code = dtype if isinstance(dtype, int) else (F32 if dtype in (torch.float32, "f32") else BF16)
    out = ctypes.c_size_t(0)
    _check(_lib.bkmoo_workspace_size(K, N, B, code, ctypes.byref(out)), "bkmoo_workspace_size")
    return out.value


def _workspace(ws: Optional[torch.Tensor], K, N, B, dt, dev) -> torch.Tensor:
    need = workspace_size(K, N, B, dt)
    if ws is None:
        return torch.empty(need, dtype=torch.uint8, device=dev)
    if ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the grads' device")
    return ws


def gram(grads: Grads, bucket_offsets: torch.Tensor, gram_out: Optional[torch.Tensor] = None,
         workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Per-bucket Gram matrices, fp64 [B, K, K]."""
    arr, dt, K, N, dev, _ = _rows(grads)
    offs = _offsets(bucket_offsets, dev)
    B = offs.numel() - 1
    if gram_out is None:
        gram_out = torch.empty((B, K, K), dtype=torch.float64, device=dev)
    _tensor(gram_out, (B, K, K), torch.float64, dev, "gram_out")
    ws = _workspace(workspace, K, N, B, dt, dev)
    with torch.cuda.device(dev):
        _check(_lib.bkmoo_gram(K, arr, dt, N, B, offs.data_ptr(), gram_out.data_ptr(), ws.data_ptr(),
                               ws.numel(), _stream_ptr(dev)), "bkmoo_gram")
    return gram_out


def solve(gram_in: torch.Tensor, method: str, max_iter: int = 20, cagrad_c: float = 0.5,
          pcgrad_order: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
          aux: Optional[torch.Tensor] = None):
    """Per-bucket combine weights (fp32 [B, K]) and the method's variable (fp64 [B, K])."""
    if gram_in.dtype != torch.float64 or gram_in.dim() != 3 or not gram_in.is_contiguous():
        raise ValueError("gram must be a contiguous fp64 [B, K, K] tensor")
    B, K, _ = gram_in.shape
    dev = _gpu(gram_in, "gram")
    if weights is None:
        weights = torch.empty((B, K), dtype=torch.float32, device=dev)
    if aux is None:
        aux = torch.empty((B, K), dtype=torch.float64, device=dev)
    _tensor(weights, (B, K), torch.float32, dev, "weights")
    _tensor(aux, (B, K), torch.float64, dev, "aux")
    hp = _hparams(max_iter, cagrad_c, pcgrad_order, K, B, dev)
    with torch.cuda.device(dev):
        _check(_lib.bkmoo_solve(K, B, gram_in.data_ptr(), METHODS[method], ctypes.byref(hp),
                                weights.data_ptr(), aux.data_ptr(), _stream_ptr(dev)), "bkmoo_solve")
    return weights, aux


SLICES_RANK_MAJOR, SLICES_BUCKET_MAJOR = 0, 1


def slice_offsets(bucket_offsets: torch.Tensor, T: int) -> torch.Tensor:
    """Offsets (int64 [B*T+1], bucket-major) of T contiguous slices of every
    bucket: slice t of bucket b starts at o_b + floor(t n_b / T)."""
    offs = bucket_offsets
    if offs.dtype != torch.int64 or offs.dim() != 1 or not offs.is_contiguous() or offs.device.type != "cuda":
        raise ValueError("bucket_offsets must be a contiguous int64 GPU tensor")
    B = offs.numel() - 1
    out = torch.empty(B * T + 1, dtype=torch.int64, device=offs.device)
    with torch.cuda.device(offs.device):
        _check(_lib.bkmoo_slice_offsets(B, int(T), offs.data_ptr(), out.data_ptr(), _stream_ptr(offs.device)),
               "bkmoo_slice_offsets")
    return out


def gram_reduce(partial: torch.Tensor, layout: int = SLICES_RANK_MAJOR,
                gram_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Sum per-slice partial Grams in slice order: partial fp64 [T, B, K, K]
    (rank-major) or [B, T, K, K] (bucket-major) -> [B, K, K]."""
    if partial.dtype != torch.float64 or partial.dim() != 4 or not partial.is_contiguous():
        raise ValueError("partial must be a contiguous fp64 4-d tensor")
    if layout == SLICES_RANK_MAJOR:
        T, B, K, _ = partial.shape
    else:
        B, T, K, _ = partial.shape
    dev = _gpu(partial, "partial")
    if gram_out is None:
        gram_out = torch.empty((B, K, K), dtype=torch.float64, device=dev)
    _tensor(gram_out, (B, K, K), torch.float64, dev, "gram_out")
    with torch.cuda.device(dev):
        _check(_lib.bkmoo_gram_reduce(K, B, T, partial.data_ptr(), int(layout), gram_out.data_ptr(),
                                      _stream_ptr(dev)), "bkmoo_gram_reduce")
    return gram_out


def conflicts(gram_in: torch.Tensor, cosines: bool = True, summary: bool = True,
              pairs: bool = True):
    """Per-bucket conflict diagnostics from fp64 [B, K, K] Gram matrices:
    (cosines fp64 [B, K, K], summary fp64 [B, 3] = mean / population std / min
    pairwise cosine, pairs int32 [B, 3] = argmin pair and the count of pairs
    with a negative inner product).  Outputs not asked for are None."""
    if gram_in.dtype != torch.float64 or gram_in.dim() != 3 or not gram_in.is_contiguous():
        raise ValueError("gram must be a contiguous fp64 [B, K, K] tensor")
    B, K, _ = gram_in.shape
    dev = _gpu(gram_in, "gram")
    cos = torch.empty((B, K, K), dtype=torch.float64, device=dev) if cosines else None
    summ = torch.empty((B, 3), dtype=torch.float64, device=dev) if summary else None
    prs = torch.empty((B, 3), dtype=torch.int32, device=dev) if pairs else None
    ptr = lambda t: t.data_ptr() if t is not None else None
    with torch.cuda.device(dev):
        _check(_lib.bkmoo_conflicts(K, B, gram_in.data_ptr(), ptr(cos), ptr(summ), ptr(prs),
                                    _stream_ptr(dev)), "bkmoo_conflicts")
    return cos, summ, prs


def combine(grads: Grads, bucket_offsets: torch.Tensor, weights: torch.Tensor,
            out: Optional[torch.Tensor] = None, out_dtype=None,
            workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The concatenated bucket updates, N elements of out_dtype (default: input dtype)."""
    arr, dt, K, N, dev, _ = _rows(grads)
    offs = _offsets(bucket_offsets, dev)
    B = offs.numel() - 1
    _tensor(weights, (B, K), torch.float32, dev, "weights")
    if out is None:
        out = torch.empty(N, dtype=out_dtype or _torch_dt(dt), device=dev)
    odt = _dt(out)
    _tensor(out, (N,), out.dtype, dev, "out")
    ws = _workspace(workspace, K, N, B, dt, dev)
    with torch.cuda.device(dev):
        _check(_lib.bkmoo_combine(K, arr, dt, N, B, offs.data_ptr(), weights.data_ptr(), out.data_ptr(),
                                  odt, ws.data_ptr(), ws.numel(), _stream_ptr(dev)), "bkmoo_combine")
    return out


def resolve(grads: Grads, bucket_offsets: torch.Tensor, method: str, max_iter: int = 20,
            cagrad_c: float = 0.5, pcgrad_order: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None, out_dtype=None,
            gram_out: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
            aux: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
            check_error: bool = False):
    """Gram -> solve -> combine on the current stream.  Returns `out`; gram,
    weights and aux are written to the tensors passed (if any).

    The device error word (invalid offsets, an expired wait of the hybrid
    path) lives in the workspace: pass `workspace` and read it with
    read_device_error(), or set check_error=True to wait for the call and
    raise BkmooError when the word is not zero."""
    arr, dt, K, N, dev, _ = _rows(grads)
    offs = _offsets(bucket_offsets, dev)
    B = offs.numel() - 1
    if out is None:
        out = torch.empty(N, dtype=out_dtype or _torch_dt(dt), device=dev)
    odt = _dt(out)
    _tensor(out, (N,), out.dtype, dev, "out")
    ws = _workspace(workspace, K, N, B, dt, dev)
    hp = _hparams(max_iter, cagrad_c, pcgrad_order, K, B, dev)

    def ptr(t, shape, dtype, what):
        return None if t is None else _tensor(t, shape, dtype, dev, what)

    with torch.cuda.device(dev):
        _check(_lib.bkmoo_resolve(K, arr, dt, N, B, offs.data_ptr(), METHODS[method], ctypes.byref(hp),
                                  out.data_ptr(), odt, ptr(gram_out, (B, K, K), torch.float64, "gram_out"),
                                  ptr(weights, (B, K), torch.float32, "weights"),
                                  ptr(aux, (B, K), torch.float64, "aux"),
                                  ws.data_ptr(), ws.numel(), _stream_ptr(dev)), "bkmoo_resolve")
    if check_error:
        err = read_device_error(ws)
        if err:
            what = [n for bit, n in ((DEVERR_OFFSETS, "invalid bucket offsets"),
                                     (DEVERR_TIMEOUT, "a bounded wait expired")) if err & bit]
            raise BkmooError(f"bkmoo_resolve: device error 0x{err:x} ({', '.join(what) or 'unknown'})")
    return out


def resolve_noalloc(grads: Grads, bucket_offsets: torch.Tensor, method: str, out: torch.Tensor,
                    max_iter: int = 20, cagrad_c: float = 0.5, pcgrad_order: Optional[torch.Tensor] = None,
                    gram_out: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
                    aux: Optional[torch.Tensor] = None):
    """resolve() on the library's own fixed device scratch (bkmoo_resolve_noalloc):
    nothing is allocated, so `out` must be given.  Calls that overlap on one
    device share that scratch and race.  Returns `out`."""
    arr, dt, K, N, dev, _ = _rows(grads)
    offs = _offsets(bucket_offsets, dev)
    B = offs.numel() - 1
    _tensor(out, (N,), out.dtype, dev, "out")
    hp = _hparams(max_iter, cagrad_c, pcgrad_order, K, B, dev)

    def ptr(t, shape, dtype, what):
        return None if t is None else _tensor(t, shape, dtype, dev, what)

    with torch.cuda.device(dev):
        _check(_lib.bkmoo_resolve_noalloc(K, arr, dt, N, B, offs.data_ptr(), METHODS[method], ctypes.byref(hp),
                                          out.data_ptr(), _dt(out),
                                          ptr(gram_out, (B, K, K), torch.float64, "gram_out"),
                                          ptr(weights, (B, K), torch.float32, "weights"),
                                          ptr(aux, (B, K), torch.float64, "aux"), _stream_ptr(dev)),
               "bkmoo_resolve_noalloc")
    return out


def read_device_error(workspace: torch.Tensor) -> int:
    v = ctypes.c_uint32(0)
    dev = _gpu(workspace, "workspace")
    with torch.cuda.device(dev):
        _check(_lib.bkmoo_read_device_error(workspace.data_ptr(), ctypes.byref(v), _stream_ptr(dev)),
               "bkmoo_read_device_error")
    return v.value


def set_grid_override(workgroups: int):
    _check(_lib.bkmoo_set_grid_override(int(workgroups)), "bkmoo_set_grid_override")


def resolve_path(grads: Grads, bucket_offsets_len: int, method: str = "mgda", max_iter: int = 20,
                 out_dtype=None) -> int:
    """PATH_TWO_PASS, PATH_HYBRID or PATH_REFILL: what resolve() would run for these
    grads and method (output assumed aligned like the rows)."""
    arr, dt, K, N, dev, rows = _rows(grads)
    B = bucket_offsets_len - 1
    odt = dt if out_dtype is None else _dt(torch.empty(0, dtype=out_dtype))
    phases = {r.data_ptr() % 16 for r in rows}
    out = ctypes.c_int32(0)
    _check(_lib.bkmoo_resolve_path(K, N, B, dt, odt, int(len(phases) == 1), METHODS[method],
                                   int(max_iter), ctypes.byref(out)), "bkmoo_resolve_path")
    return out.value


def resolve_traffic(K: int, bucket_offsets, dtype, path: int, out_dtype=None, method: str = "mgda",
                    max_iter: int = 20) -> int:
    """Bytes a resolve on `path` requests from memory for these offsets (a
    host int64 array-like of B+1 entries); on the hybrid path part of the
    re-read is served by the last-level cache, and on the refill path uneven
    offsets may select its tiled form, which reads everything twice."""
    import numpy as np
    offs = np.ascontiguousarray(np.asarray(bucket_offsets, dtype=np.int64))
    code = lambda d: d if isinstance(d, int) else (F32 if d in (torch.float32, "f32") else BF16)
    dt = code(dtype)
    odt = dt if out_dtype is None else code(out_dtype)
    out = ctypes.c_uint64(0)
    _check(_lib.bkmoo_resolve_traffic(K, int(offs[-1]), len(offs) - 1, offs.ctypes.data, dt, odt, METHODS[method],
                                      int(max_iter), int(path), ctypes.byref(out)), "bkmoo_resolve_traffic")
    return out.value


def set_resolve_path(path: int):
    """0 automatic, PATH_TWO_PASS, PATH_HYBRID or PATH_REFILL (process-wide)."""
    _check(_lib.bkmoo_set_resolve_path(int(path)), "bkmoo_set_resolve_path")


def set_wait_limit(polls: int):
    _check(_lib.bkmoo_set_wait_limit(int(polls)), "bkmoo_set_wait_limit")


# ----------------------------------------------------------------------------
# the layer around the resolve
# ----------------------------------------------------------------------------


def _ptr(t: Optional[torch.Tensor], shape, dtype, index: int, what: str):
    """Pointer of a contiguous tensor of this shape and type on GPU `index`; None stays None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{index}")


# the current stream's handle by device number, without a Stream object around it (2.5 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _run(fn, what: str, index: int, *args):
    """fn(*args, stream) with GPU `index`, the inputs', current."""
    stream = _raw_stream(index)
    if torch.cuda.current_device() == index:
        st = fn(*args, stream)
    else:
        with torch.cuda.device(index):
            st = fn(*args, stream)
    if st != 0:
        _check(st, what)


def _matrix(t: torch.Tensor, what: str):
    """Rows, columns, dtype code, dtype and GPU number of a 2-D GPU tensor."""
    dtype, shape = t.dtype, t.shape
    code = BF16 if dtype is torch.bfloat16 else _dt(t)
    if not t.is_cuda:
        _gpu(t, what)
    if len(shape) != 2:
        raise ValueError(f"{what} must have two dimensions")
    return shape[0], shape[1], code, dtype, t.get_device()


def _byte_workspace(ws: Optional[torch.Tensor], need: int, dev) -> torch.Tensor:
    if ws is None:
        return torch.empty(need, dtype=torch.uint8, device=dev)
    if ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the inputs' device")
    return ws


def _task_rows(task_rows: Sequence[int], M: int):
    rows = [0, M] if task_rows is None else [int(r) for r in task_rows]
    if len(rows) < 2:
        raise ValueError("task_rows holds K + 1 offsets from 0 to the number of rows")
    return (ctypes.c_int64 * len(rows))(*rows), len(rows) - 1


def _task_grads(grads, K: int, n: int, dtype, index: int):
    """Pointers and the common distance of the tasks' gradients: [K, n] tensors whose rows
    are contiguous (columns of the [K, N] gradient buffer), or None."""
    stride, shape, ptrs = None, (K, n), []
    for t, what in grads:
        if t is None:
            ptrs.append(None)
            continue
        if t.dtype is not dtype or t.shape != shape or t.get_device() != index or (n > 1 and t.stride(1) != 1):
            raise ValueError(f"{what} must be a {dtype} tensor of shape {shape} with contiguous rows on cuda:{index}")
        if K > 1:
            if stride is None:
                stride = t.stride(0)
            elif t.stride(0) != stride:
                raise ValueError("the tasks' gradients must be equally far apart in every tensor")
        ptrs.append(t.data_ptr())
    return ptrs, n if stride is None else stride


def residual_norm_forward(resid: torch.Tensor, y: torch.Tensor, weight: torch.Tensor,
                          post_weight: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                          scale: float = 1.0, eps: float = 1e-6, resid_out: Optional[torch.Tensor] = None,
                          normed: Optional[torch.Tensor] = None):
    """The norm after a block (with post_weight), its gate and residual scale, and the
    norm before the next: (resid + scale * gate * norm(y), norm of that), both [M, D].
    resid_out may be resid."""
    M, D, code, dt, gpu = _matrix(resid, "resid")
    shape, vec = resid.shape, (D,)
    if resid_out is None:
        resid_out = torch.empty_like(resid, memory_format=torch.contiguous_format)
    if normed is None:
        normed = torch.empty_like(resid, memory_format=torch.contiguous_format)
    _run(_lib.bkmoo_residual_norm_forward, "bkmoo_residual_norm_forward", gpu, M, D, code,
         _ptr(resid, shape, dt, gpu, "resid"), _ptr(y, shape, dt, gpu, "y"), _ptr(weight, vec, dt, gpu, "weight"),
         _ptr(post_weight, vec, dt, gpu, "post_weight"), _ptr(gate, vec, dt, gpu, "gate"), scale, eps,
         _ptr(resid_out, shape, dt, gpu, "resid_out"), _ptr(normed, shape, dt, gpu, "normed"))
    return resid_out, normed


def residual_norm_backward(dresid_out: Optional[torch.Tensor], dnormed: torch.Tensor, resid_out: torch.Tensor,
                           y: torch.Tensor, weight: torch.Tensor, post_weight: Optional[torch.Tensor] = None,
                           gate: Optional[torch.Tensor] = None, scale: float = 1.0, eps: float = 1e-6,
                           task_rows: Optional[Sequence[int]] = None, dweight: Optional[torch.Tensor] = None,
                           dpost_weight: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                           dresid: Optional[torch.Tensor] = None, dy: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None):
    """Gradients of residual_norm_forward: returns (dresid, dy) and writes the K tasks'
    weight gradients to dweight, dpost_weight and dgate, [K, D] with contiguous rows
    (columns of the gradient buffer).  task_rows: K + 1 offsets of the tasks' rows."""
    M, D, code, dt, gpu = _matrix(resid_out, "resid_out")
    shape, vec = resid_out.shape, (D,)
    rows, K = _task_rows(task_rows, M)
    if dweight is None:
        raise ValueError("dweight is needed")
    ptrs, stride = _task_grads(((dweight, "dweight"), (dpost_weight, "dpost_weight"), (dgate, "dgate")), K, D, dt,
                               gpu)
    if dresid is None:
        dresid = torch.empty_like(resid_out, memory_format=torch.contiguous_format)
    if dy is None:
        dy = torch.empty_like(resid_out, memory_format=torch.contiguous_format)
    need = ctypes.c_size_t(0)
    _check(_lib.bkmoo_residual_norm_workspace_size(M, D, K, ctypes.byref(need)), "bkmoo_residual_norm_workspace_size")
    ws = _byte_workspace(workspace, need.value, resid_out.device)
    args = (_ptr(dresid_out, shape, dt, gpu, "dresid_out"), _ptr(dnormed, shape, dt, gpu, "dnormed"),
            _ptr(resid_out, shape, dt, gpu, "resid_out"), _ptr(y, shape, dt, gpu, "y"),
            _ptr(weight, vec, dt, gpu, "weight"), _ptr(post_weight, vec, dt, gpu, "post_weight"),
            _ptr(gate, vec, dt, gpu, "gate"), scale, eps, _ptr(dresid, shape, dt, gpu, "dresid"),
            _ptr(dy, shape, dt, gpu, "dy"), *ptrs, stride)
    _run(_lib.bkmoo_residual_norm_backward, "bkmoo_residual_norm_backward", gpu, M, D, code, K, rows, *args,
         ws.data_ptr(), ws.numel())
    return dresid, dy


def ffn_workspace_size(M: int, D: int, F: int, dtype, backward: bool = False) -> int:
    code = dtype if isinstance(dtype, int) else (F32 if dtype in (torch.float32, "f32") else BF16)
    out = ctypes.c_size_t(0)
    _check(_lib.bkmoo_ffn_workspace_size(M, D, F, code, int(backward), ctypes.byref(out)), "bkmoo_ffn_workspace_size")
    return out.value


def ffn_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, act: str = "silu",
                save: bool = False, out: Optional[torch.Tensor] = None, gate_out: Optional[torch.Tensor] = None,
                up_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gated feed-forward block: (y, u, v) with y = (act(u) * v) w_down^T, u = x w_gate^T,
    v = x w_up^T for x [M, D], w_gate and w_up [F, D], w_down [D, F].  u and v, which
    the backward pass needs, are None unless `save` is set or they are given."""
    M, D, code, dt, gpu = _matrix(x, "x")
    if w_gate.dim() != 2:
        raise ValueError("w_gate must have two dimensions")
    F, dev = w_gate.shape[0], x.device
    md, mf, fd, df = (M, D), (M, F), (F, D), (D, F)
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    if save and gate_out is None:
        gate_out = torch.empty(mf, dtype=dt, device=dev)
    if save and up_out is None:
        up_out = torch.empty(mf, dtype=dt, device=dev)
    ws = _byte_workspace(workspace, ffn_workspace_size(M, D, F, code), dev)
    _run(_lib.bkmoo_ffn_forward, "bkmoo_ffn_forward", gpu, M, D, F, code, ACTS[act], _ptr(x, md, dt, gpu, "x"),
         _ptr(w_gate, fd, dt, gpu, "w_gate"), _ptr(w_up, fd, dt, gpu, "w_up"), _ptr(w_down, df, dt, gpu, "w_down"),
         _ptr(out, md, dt, gpu, "out"), _ptr(gate_out, mf, dt, gpu, "gate_out"), _ptr(up_out, mf, dt, gpu, "up_out"),
         ws.data_ptr(), ws.numel())
    return out, gate_out, up_out


def ffn_backward(dy: torch.Tensor, x: torch.Tensor, gate_out: torch.Tensor, up_out: torch.Tensor,
                 w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, act: str = "silu",
                 task_rows: Optional[Sequence[int]] = None, dw_gate: Optional[torch.Tensor] = None,
                 dw_up: Optional[torch.Tensor] = None, dw_down: Optional[torch.Tensor] = None,
                 dx: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradients of ffn_forward: returns dx and writes the K tasks' weight gradients to
    dw_gate, dw_up and dw_down, each [K, D * F] with contiguous rows (columns of the
    gradient buffer; a row is the flattened matrix).  task_rows: K + 1 offsets of the
    tasks' rows in the batch."""
    M, D, code, dt, gpu = _matrix(x, "x")
    if w_gate.dim() != 2:
        raise ValueError("w_gate must have two dimensions")
    F = w_gate.shape[0]
    md, mf, fd, df = (M, D), (M, F), (F, D), (D, F)
    rows, K = _task_rows(task_rows, M)
    if dw_gate is None or dw_up is None or dw_down is None:
        raise ValueError("dw_gate, dw_up and dw_down are needed")
    ptrs, stride = _task_grads(((dw_gate, "dw_gate"), (dw_up, "dw_up"), (dw_down, "dw_down")), K, D * F, dt,
                               gpu)
    if dx is None:
        dx = torch.empty_like(x, memory_format=torch.contiguous_format)
    ws = _byte_workspace(workspace, ffn_workspace_size(M, D, F, code, True), x.device)
    args = (_ptr(dy, md, dt, gpu, "dy"), _ptr(x, md, dt, gpu, "x"), _ptr(gate_out, mf, dt, gpu, "gate_out"),
            _ptr(up_out, mf, dt, gpu, "up_out"), _ptr(w_gate, fd, dt, gpu, "w_gate"),
            _ptr(w_up, fd, dt, gpu, "w_up"), _ptr(w_down, df, dt, gpu, "w_down"), _ptr(dx, md, dt, gpu, "dx"), *ptrs,
            stride)
    _run(_lib.bkmoo_ffn_backward, "bkmoo_ffn_backward", gpu, M, D, F, code, ACTS[act], K, rows, *args, ws.data_ptr(),
         ws.numel())
    return dx


def set_ffn_tiles(side: int = 0, splits: int = 0, workgroups: int = 0):
    """Force the side (64, 128, 256) of the feed-forward products' tiles, the parts of their split sums and the
    number of workgroups; 0: automatic (process-wide)."""
    _check(_lib.bkmoo_set_ffn_tiles(int(side), int(splits), int(workgroups)), "bkmoo_set_ffn_tiles")


_data_ptr = torch.Tensor.data_ptr


class AdamwTable:
    """The addresses and sizes of adamw()'s tensors, in the order of the flat gradient.
    N: their elements; blocks: their blocks of 256 elements (the scales of 8-bit moments).
    A table keeps the tensors' memory.  Where one is given other memory afterwards (p.data = ...,
    module.to(dtype), a storage's resize) adamw() refuses the table: lay out another."""

    def __init__(self, params: Sequence[torch.Tensor], decay: Optional[Sequence[bool]] = None):
        self.params = list(params)
        self.memory = [p.detach() for p in self.params]  # a tensor alone does not keep the memory it has now
        self.addresses = list(map(_data_ptr, self.params))
        if not self.params:
            raise ValueError("no tensors")
        self.dt, self.device = _dt(self.params[0]), _gpu(self.params[0], "parameters")
        for p in self.params:
            if p.dtype != self.params[0].dtype or p.device != self.device or not p.is_contiguous():
                raise ValueError("parameters must be contiguous tensors of one dtype and device")
        decay = [True] * len(self.params) if decay is None else list(decay)
        if len(decay) != len(self.params):
            raise ValueError("decay holds one entry for each tensor")
        self.array = (_Tensor * len(self.params))(*[(a, p.numel(), int(bool(d)))
                                                    for a, p, d in zip(self.addresses, self.params, decay)])
        self.N = sum(p.numel() for p in self.params)
        n = ctypes.c_int64(0)
        _check(_lib.bkmoo_adamw_blocks(len(self.params), self.array, ctypes.byref(n)), "bkmoo_adamw_blocks")
        self.blocks = n.value


def adamw_table(params: Sequence[torch.Tensor], decay: Optional[Sequence[bool]] = None) -> AdamwTable:
    """Lay out adamw()'s tensors once (decay: whether weight decay applies, for each)."""
    return AdamwTable(params, decay)


def adamw(table: AdamwTable, grad: torch.Tensor, moment1: torch.Tensor, moment2: torch.Tensor, step: int,
          lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01,
          master: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
          grad_scale: Optional[torch.Tensor] = None, seed: Optional[int] = None) -> None:
    """One AdamW step over the table's tensors, in place.  grad [N]: float32 or bfloat16, the tensors'
    gradients one after another (what resolve() returns).  moment1, moment2 [N]: float32, or
    float8_e4m3fn with scales float32 [2, blocks] (zeros to start with).  master: float32 [N] copy of
    bfloat16 parameters that takes the step.  grad_scale: float32 tensor of one element.  seed: of the
    random bits that round 8-bit moments, by default the step's number.  Every step needs another: with
    the same bits again an element is rounded at the same place again, and moments that move by
    less than the distance of two 8-bit values stay where they are."""
    dev, gpu, flat = table.device, table.device.index, (table.N,)
    # (as the table keeps the old memory, no other can have its address)
    if list(map(_data_ptr, table.params)) != table.addresses:
        raise ValueError("a parameter's memory is not where it was: lay it out again with adamw_table()")
    f8 = moment1.dtype == torch.float8_e4m3fn
    sdt = torch.float8_e4m3fn if f8 else torch.float32
    gp = _ptr(grad, flat, grad.dtype, gpu, "grad")
    m1, m2 = _ptr(moment1, flat, sdt, gpu, "moment1"), _ptr(moment2, flat, sdt, gpu, "moment2")
    if f8 != (scales is not None):
        raise ValueError("scales go with 8-bit moments")
    sc = _ptr(scales, (2, table.blocks), torch.float32, gpu, "scales")
    mp = _ptr(master, flat, torch.float32, gpu, "master")
    gs = None
    if grad_scale is not None:
        if grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or grad_scale.device != dev:
            raise ValueError(f"grad_scale must be one float32 value on {dev}")
        gs = grad_scale.data_ptr()
    hp = _AdamwHparams(lr, beta1, beta2, eps, weight_decay, step, (step if seed is None else seed) & 0xFFFFFFFF)
    _run(_lib.bkmoo_adamw, "bkmoo_adamw", gpu, len(table.params), table.array, table.dt, table.N, gp, _dt(grad),
         STATE_F8 if f8 else STATE_F32, m1, m2, sc, table.blocks if f8 else 0, mp, ctypes.byref(hp), gs)
