"""Python binding of libgroupsparse.so (argument marshalling only).

Every call goes straight to the C ABI declared in include/groupsparse.h; torch
is used for device memory and the current CUDA stream.  There is no fallback:
if the compiled library is missing or fails to load, importing this module
raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path
from typing import Optional, Sequence

import numpy as np
import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libgroupsparse.so"

GS_OK, GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED, GS_ERR_OOM, GS_ERR_CUDA, GS_ERR_DEVICE_TIMEOUT = range(6)
ALGO_AUTO, ALGO_DECODE, ALGO_PREFILL, ALGO_PREFILL_DENSE = 0, 1, 2, 3
ATTENTION_COUNTER_BYTES = 8192   # GS_ATTENTION_COUNTER_BYTES

_c_i64p = ctypes.POINTER(ctypes.c_int64)
_c_i32p = ctypes.POINTER(ctypes.c_int32)
_c_u16p = ctypes.POINTER(ctypes.c_uint16)


class _AdapterLayer(ctypes.Structure):   # gs_adapter_layer
    _fields_ = [("x", ctypes.c_void_p), ("base", ctypes.c_void_p), ("out_ptr", ctypes.c_void_p), ("A", ctypes.c_void_p),
                ("B", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("inp", ctypes.c_int64), ("out", ctypes.c_int64),
                ("n_adapters", ctypes.c_int32), ("rank", ctypes.c_int32)]


class _CacheStruct(ctypes.Structure):    # gs_paged_cache
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class _BatchStruct(ctypes.Structure):    # gs_seq_batch
    _fields_ = [("offsets", ctypes.c_void_p), ("kv_lens", ctypes.c_void_p), ("table", ctypes.c_void_p), ("n", ctypes.c_int32),
                ("table_width", ctypes.c_int32), ("tokens", ctypes.c_int64), ("max_new", ctypes.c_int32)]


def _load(path: Path = LIB_PATH) -> ctypes.CDLL:
    if not path.exists():
        raise ImportError(f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(str(path))
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    lib.gs_pack.argtypes = [vp, vp, i64, i64, i32, vp, ctypes.POINTER(vp)]
    lib.gs_pack_groups.argtypes = [vp, vp, i64, i64, i32, i32, vp, ctypes.POINTER(vp)]
    lib.gs_packed_group_shape.argtypes = [vp, _c_i32p, _c_i32p]
    lib.gs_linear.argtypes = [vp, vp, i64, vp, vp]
    lib.gs_linear_ex.argtypes = [vp, vp, i64, vp, vp, ctypes.c_int]
    lib.gs_linear_batched.argtypes = [i32, ctypes.POINTER(vp), ctypes.POINTER(vp), i64, ctypes.POINTER(vp), vp]
    lib.gs_unpack.argtypes = [vp, vp, vp]
    lib.gs_select_groups.argtypes = [vp, i64, vp, vp, vp]
    lib.gs_packed_info.argtypes = [vp, _c_i64p, _c_i64p, _c_i64p, ctypes.POINTER(ctypes.c_size_t)]
    lib.gs_packed_export.argtypes = [vp, _c_i64p, _c_i32p, _c_u16p, _c_i32p, _c_u16p]
    lib.gs_free.argtypes = [vp]
    lib.gs_free.restype = None
    lib.gs_trim.argtypes = []
    lib.gs_trim.restype = None
    lib.gs_status_string.argtypes = [ctypes.c_int]
    lib.gs_status_string.restype = ctypes.c_char_p
    lib.gs_device_status.argtypes = [vp]
    lib.gs_launch_count.argtypes = []
    lib.gs_launch_count.restype = ctypes.c_int64
    lib.gs_preserved_rates.argtypes = [i32, vp, vp, vp, i64, vp, vp, i32, vp, vp]
    lib.gs_gumbel_select.argtypes = [vp, vp, i64, ctypes.c_float, vp, vp, vp, vp]
    lib.gs_masked_linear_backward_workspace.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.gs_masked_linear_backward.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.gs_add_rms_norm.argtypes = [vp, vp, vp, i64, i64, ctypes.c_float, vp, vp, vp, vp, i32, vp]
    lib.gs_adapters_batched.argtypes = [i32, vp, vp, vp, i32, i64, vp]
    lib.gs_cache_append.argtypes = [vp, vp, vp, i64, i32, vp, i64, vp, i64, vp, vp, i64, vp, vp]
    lib.gs_paged_attention_workspace.argtypes = [vp, vp, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.gs_paged_attention.argtypes = [vp, vp, vp, i64, i32, ctypes.c_float, vp, vp, ctypes.c_size_t, vp]
    lib.gs_capture_id.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.gs_debug_fail_alloc.argtypes = [i64]
    lib.gs_debug_inject_wait.argtypes = [ctypes.c_int, ctypes.c_uint64]
    lib.gs_debug_inject_attention_wait.argtypes = [i32, ctypes.c_uint64]
    for fn in (lib.gs_pack, lib.gs_linear, lib.gs_linear_ex, lib.gs_linear_batched, lib.gs_unpack,
               lib.gs_packed_info, lib.gs_packed_export, lib.gs_device_status, lib.gs_select_groups,
               lib.gs_preserved_rates, lib.gs_debug_fail_alloc, lib.gs_debug_inject_wait, lib.gs_pack_groups,
               lib.gs_packed_group_shape, lib.gs_gumbel_select, lib.gs_masked_linear_backward_workspace,
               lib.gs_masked_linear_backward, lib.gs_add_rms_norm, lib.gs_adapters_batched, lib.gs_cache_append,
               lib.gs_paged_attention_workspace, lib.gs_paged_attention, lib.gs_capture_id,
               lib.gs_debug_inject_attention_wait):
        fn.restype = ctypes.c_int
    return lib


lib = _load()


class GroupSparseError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {lib.gs_status_string(status).decode()} (status {status})")
        self.status = status


def _check(status: int, what: str) -> None:
    if status != GS_OK:
        raise GroupSparseError(status, what)


def _stream_ptr(stream: Optional[torch.cuda.Stream] = None) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    # the current device's current stream, without a Stream object around it
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _require_cuda(t: torch.Tensor, dtype: torch.dtype, name: str) -> None:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class Packed:
    """A packed group-sparse weight (owns the library handle)."""

    def __init__(self, handle: int, out: int, inp: int, g_out: int = 1, g_in: int = 256):
        self._h = ctypes.c_void_p(handle)
        self.out = out
        self.inp = inp
        self.g_out = g_out
        self.g_in = g_in

    @property
    def handle(self) -> ctypes.c_void_p:
        if not self._h:
            raise ValueError("packed weight already freed")
        return self._h

    @property
    def G(self) -> int:
        return self.inp // self.g_in

    def info(self):
        out, inp, kept = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        nbytes = ctypes.c_size_t()
        _check(lib.gs_packed_info(self.handle, ctypes.byref(out), ctypes.byref(inp), ctypes.byref(kept),
                                  ctypes.byref(nbytes)), "gs_packed_info")
        return {"out": out.value, "in": inp.value, "kept": kept.value, "device_bytes": nbytes.value}

    @property
    def kept(self) -> int:
        return self.info()["kept"]

    def export(self):
        """Host copies of the packed layout: offsets, row_idx, tiles, win_off16, kmask16
        (square groups: offsets, row_idx = block rows, tiles [K, g, g])."""
        K = self.kept
        G = self.G
        if self.g_out > 1:
            offsets = np.zeros(G + 1, np.int64)
            rows = np.zeros(max(K, 1), np.int32)
            tiles = np.zeros((max(K, 1), self.g_out, self.g_in), np.uint16)
            _check(lib.gs_packed_export(self.handle, offsets.ctypes.data_as(_c_i64p), rows.ctypes.data_as(_c_i32p),
                                        tiles.ctypes.data_as(_c_u16p), None, None), "gs_packed_export")
            return {"offsets": offsets, "row_idx": rows[:K], "tiles": tiles[:K]}
        nw16 = (self.out + 15) // 16
        offsets = np.zeros(G + 1, np.int64)
        row_idx = np.zeros(max(K, 1), np.int32)
        tiles = np.zeros((max(K, 1), self.g_in), np.uint16)
        win = np.zeros((G, nw16 + 1), np.int32)
        km = np.zeros((G, nw16), np.uint16)
        _check(lib.gs_packed_export(self.handle, offsets.ctypes.data_as(_c_i64p), row_idx.ctypes.data_as(_c_i32p),
                                    tiles.ctypes.data_as(_c_u16p), win.ctypes.data_as(_c_i32p),
                                    km.ctypes.data_as(_c_u16p)), "gs_packed_export")
        return {"offsets": offsets, "row_idx": row_idx[:K], "tiles": tiles[:K], "win_off16": win, "kmask16": km}

    def free(self) -> None:
        if self._h:
            lib.gs_free(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def trim() -> None:
    """Give the device buffers kept from released handles back to the device (waits for it), and the
    attention's workspaces to torch's allocator."""
    _attention_ws.clear()
    _captured_ws.clear()
    lib.gs_trim()


def pack(W: torch.Tensor, mask: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> Packed:
    """Pack a bf16 weight [out, in] with a uint8/bool group mask [out, in/256] (nonzero = keep)."""
    _require_cuda(W, torch.bfloat16, "W")
    if mask.dtype == torch.bool:
        mask = mask.to(torch.uint8)
    _require_cuda(mask, torch.uint8, "mask")
    out, inp = W.shape
    if tuple(mask.shape) != (out, inp // 256):
        raise ValueError("mask must be [out, in/256]")
    h = ctypes.c_void_p()
    _check(lib.gs_pack(W.data_ptr(), mask.data_ptr(), out, inp, 256, _stream_ptr(stream), ctypes.byref(h)),
           "gs_pack")
    return Packed(h.value, out, inp)


def pack_groups(W: torch.Tensor, mask: torch.Tensor, g_out: int, g_in: int,
                stream: Optional[torch.cuda.Stream] = None) -> Packed:
    """Pack a bf16 weight [out, in] with a group mask [out/g_out, in/g_in] (nonzero = keep)
    for g_out x g_in groups: (1, 256), (1, 128) or square g x g, g in {16, 32, 64, 128}."""
    _require_cuda(W, torch.bfloat16, "W")
    if mask.dtype == torch.bool:
        mask = mask.to(torch.uint8)
    _require_cuda(mask, torch.uint8, "mask")
    out, inp = W.shape
    if out % g_out or inp % g_in or tuple(mask.shape) != (out // g_out, inp // g_in):
        raise ValueError("mask must be [out/g_out, in/g_in] and the groups must tile W")
    h = ctypes.c_void_p()
    _check(lib.gs_pack_groups(W.data_ptr(), mask.data_ptr(), out, inp, g_out, g_in, _stream_ptr(stream),
                              ctypes.byref(h)), "gs_pack_groups")
    return Packed(h.value, out, inp, g_out, g_in)


def linear_into(x: torch.Tensor, p: Packed, y: torch.Tensor, algo: int = ALGO_AUTO,
                stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    _require_cuda(x, torch.bfloat16, "x")
    _require_cuda(y, torch.bfloat16, "y")
    T = x.shape[0]
    if x.dim() != 2 or x.shape[1] != p.inp or y.shape != (T, p.out):
        raise ValueError("x must be [T, in] and y [T, out]")
    _check(lib.gs_linear_ex(x.data_ptr(), p.handle, T, y.data_ptr(), _stream_ptr(stream), algo), "gs_linear")
    return y


def linear(x: torch.Tensor, p: Packed, algo: int = ALGO_AUTO, stream: Optional[torch.cuda.Stream] = None):
    """y = x (W (.) M)^T as bf16 [T, out]."""
    y = torch.empty((x.shape[0], p.out), dtype=torch.bfloat16, device=x.device)
    return linear_into(x, p, y, algo, stream)


def linear_batched_into(xs: Sequence[torch.Tensor], ps: Sequence[Packed], ys: Sequence[torch.Tensor],
                        stream: Optional[torch.cuda.Stream] = None) -> None:
    n = len(ps)
    if not (len(xs) == len(ys) == n):
        raise ValueError("xs, ps, ys must have the same length")
    if n == 0:
        return
    T = xs[0].shape[0]
    for x, p, y in zip(xs, ps, ys):
        _require_cuda(x, torch.bfloat16, "x")
        _require_cuda(y, torch.bfloat16, "y")
        if x.shape[0] != T or x.shape[1] != p.inp or y.shape != (T, p.out):
            raise ValueError("every x must be [T, in_i] and y [T, out_i] with one T")
    arr = ctypes.c_void_p * n
    xa = arr(*[x.data_ptr() for x in xs])
    pa = arr(*[p.handle.value for p in ps])
    ya = arr(*[y.data_ptr() for y in ys])
    _check(lib.gs_linear_batched(n, xa, pa, T, ya, _stream_ptr(stream)), "gs_linear_batched")


def unpack(p: Packed, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """W_hat = W (.) M as bf16 [out, in]; pruned groups are +0.0."""
    W = torch.empty((p.out, p.inp), dtype=torch.bfloat16, device="cuda")
    _check(lib.gs_unpack(p.handle, W.data_ptr(), _stream_ptr(stream)), "gs_unpack")
    return W


def select_groups(logits: torch.Tensor, mask: Optional[torch.Tensor] = None,
                  kept: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Selector export (Sec. 2.2; App. F): mask = [sigmoid(logits) > 1/2] as uint8 0/1 of
    the logits' shape, and kept = the number of ones as an int64 [1] device tensor.
    For one layer with 1x256 groups, logits are float32 [out, in/256]."""
    _require_cuda(logits, torch.float32, "logits")
    if mask is None:
        mask = torch.empty(logits.shape, dtype=torch.uint8, device=logits.device)
    else:
        _require_cuda(mask, torch.uint8, "mask")
        if mask.numel() != logits.numel():
            raise ValueError("mask must hold one byte per logit")
    if kept is None:
        kept = torch.empty((1,), dtype=torch.int64, device=logits.device)
    else:
        _require_cuda(kept, torch.int64, "kept")
        if kept.numel() < 1:
            raise ValueError("kept must hold at least one int64")
    _check(lib.gs_select_groups(logits.data_ptr(), logits.numel(), mask.data_ptr(), kept.data_ptr(),
                                _stream_ptr(stream)), "gs_select_groups")
    return mask, kept


def pack_from_logits(W: torch.Tensor, logits: torch.Tensor,
                     stream: Optional[torch.cuda.Stream] = None) -> Packed:
    """Export a layer's selectors from its float32 logits [out, in/256] and pack W with them."""
    mask, _ = select_groups(logits, stream=stream)
    return pack(W, mask, stream)


_QKV = {"q": "q", "k": "k", "v": "v", "q_proj": "q", "k_proj": "k", "v_proj": "v"}


def preserved_report(kept: Sequence[int], shapes: Sequence[Sequence[int]],
                     names: Optional[Sequence[str]] = None, group: int = 256) -> dict:
    """Preserved rates of exported masks (App. F) from per-layer kept-group counts,
    computed by gs_preserved_rates: each layer's active over total weights, the
    global rate (1 - s of Eq. 2) and, for layers named q, k and v (or q_proj,
    k_proj, v_proj) under one dotted prefix, the mean of the three, keyed by
    that prefix.  This function only arranges the arguments."""
    if len(kept) != len(shapes) or (names is not None and len(names) != len(kept)):
        raise ValueError("kept, shapes (and names) must have the same length")
    names = list(names) if names is not None else [str(i) for i in range(len(kept))]
    n = len(kept)
    k_arr = np.ascontiguousarray(kept, dtype=np.int64)
    sh = np.asarray(shapes, dtype=np.int64).reshape(n, 2)
    d_out = np.ascontiguousarray(sh[:, 0])
    d_in = np.ascontiguousarray(sh[:, 1])
    index = {m: i for i, m in enumerate(names)}
    prefixes, triples = [], []
    for m in names:
        prefix, _, last = m.rpartition(".")
        if _QKV.get(last) != "q":
            continue
        trio = {}
        for m2 in names:
            p2, _, l2 = m2.rpartition(".")
            if p2 == prefix and l2 in _QKV:
                trio[_QKV[l2]] = index[m2]
        if len(trio) == 3:
            prefixes.append(prefix)
            triples.append((trio["q"], trio["k"], trio["v"]))
    qkv_idx = np.ascontiguousarray(np.asarray(triples, dtype=np.int32).reshape(-1, 3))
    rates = np.zeros(max(n, 1), np.float64)
    qkv_rates = np.zeros(max(len(triples), 1), np.float64)
    glob = ctypes.c_double()
    _check(lib.gs_preserved_rates(n, k_arr.ctypes.data, d_out.ctypes.data, d_in.ctypes.data, int(group),
                                  rates.ctypes.data, ctypes.byref(glob), len(triples), qkv_idx.ctypes.data,
                                  qkv_rates.ctypes.data), "gs_preserved_rates")
    return {"layers": {m: float(rates[i]) for i, m in enumerate(names)}, "global": glob.value,
            "qkv": {pf: float(qkv_rates[j]) for j, pf in enumerate(prefixes)}}


def gumbel_select(logits: torch.Tensor, noise: torch.Tensor, tau: float,
                  stream: Optional[torch.cuda.Stream] = None):
    """One Gumbel-Sigmoid sample of the selectors (Sec. 2.2): mask = [l + L > 0] (uint8),
    dsdl = d sigmoid((l + L) / tau) / dl (float32, the straight-through derivative) and the
    kept count (int64 [1]); L is the caller's logistic noise, of the logits' shape."""
    _require_cuda(logits, torch.float32, "logits")
    _require_cuda(noise, torch.float32, "noise")
    if noise.shape != logits.shape:
        raise ValueError("noise must have the logits' shape")
    mask = torch.empty(logits.shape, dtype=torch.uint8, device=logits.device)
    dsdl = torch.empty(logits.shape, dtype=torch.float32, device=logits.device)
    kept = torch.empty((1,), dtype=torch.int64, device=logits.device)
    _check(lib.gs_gumbel_select(logits.data_ptr(), noise.data_ptr(), logits.numel(), float(tau), mask.data_ptr(),
                                dsdl.data_ptr(), kept.data_ptr(), _stream_ptr(stream)), "gs_gumbel_select")
    return mask, dsdl, kept


def masked_linear_backward(x: torch.Tensor, W: torch.Tensor, p: Packed, dy: torch.Tensor, dsdl: torch.Tensor,
                           want_dx: bool = True, stream: Optional[torch.cuda.Stream] = None):
    """Straight-through backward of y = x W_hat^T (Sec. 2.2): (dlogits float32 of the
    mask's shape, dx bf16 [T, in] or None).  p is W packed with the sampled mask."""
    _require_cuda(x, torch.bfloat16, "x")
    _require_cuda(W, torch.bfloat16, "W")
    _require_cuda(dy, torch.bfloat16, "dy")
    _require_cuda(dsdl, torch.float32, "dsdl")
    T = x.shape[0]
    if tuple(W.shape) != (p.out, p.inp) or x.shape[1] != p.inp or tuple(dy.shape) != (T, p.out):
        raise ValueError("W must be [out, in], x [T, in] and dy [T, out]")
    shape = (p.out // p.g_out, p.inp // p.g_in)
    if tuple(dsdl.shape) != shape:
        raise ValueError(f"dsdl must be {shape}")
    nbytes = ctypes.c_size_t()
    _check(lib.gs_masked_linear_backward_workspace(p.handle, 1 if want_dx else 0, ctypes.byref(nbytes)),
           "gs_masked_linear_backward_workspace")
    ws = torch.empty((nbytes.value,), dtype=torch.uint8, device=x.device)
    dl = torch.empty(shape, dtype=torch.float32, device=x.device)
    dx = torch.empty((T, p.inp), dtype=torch.bfloat16, device=x.device) if want_dx else None
    _check(lib.gs_masked_linear_backward(x.data_ptr(), W.data_ptr(), p.handle, dy.data_ptr(), T, dsdl.data_ptr(),
                                         dl.data_ptr(), dx.data_ptr() if dx is not None else None,
                                         ws.data_ptr(), nbytes.value, _stream_ptr(stream)),
           "gs_masked_linear_backward")
    return dl, dx


# --------------------------------------------------------------------------
# the operators around a served block's projections
# --------------------------------------------------------------------------

def _empty(shape, dtype: torch.dtype, device, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """A new tensor that belongs to the stream the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _require_like(t: torch.Tensor, shape, name: str) -> int:
    """The address of a contiguous bf16 CUDA tensor of that shape."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
        _require_cuda(t, torch.bfloat16, name)
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _norm(x, weight, residual, eps, h, y, y8, scales, group, stream):
    """The outputs are addresses."""
    if x.dim() != 2:
        raise ValueError("x must be [T, n]")
    shape = x.shape
    T, n = shape
    _check(lib.gs_add_rms_norm(
        _require_like(x, shape, "x"), None if residual is None else _require_like(residual, shape, "residual"),
        _require_like(weight, (n,), "weight"), T, n, eps, h, y, y8, scales, group, _stream_ptr(stream)), "gs_add_rms_norm")


def _norm_sum(x, residual, h, stream):
    """h and its address."""
    if h is not None:
        return h, _require_like(h, x.shape, "h")
    if residual is None:
        return None, None
    h = torch.empty_like(x) if stream is None else _empty(x.shape, x.dtype, x.device, stream)
    return h, h.data_ptr()


def add_rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                 h: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None):
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight over the rows of x [T, n]: (y, h), both bf16.
    Without a residual, h is None unless it was given (a copy of x then).  h may be the residual's or x's own
    tensor, y x's own."""
    if y is None:   # x is checked before anything uses a tensor like it
        y = torch.empty_like(x) if stream is None else _empty(x.shape, x.dtype, x.device, stream)
        to_y = y.data_ptr()
    else:
        to_y = _require_like(y, x.shape, "y")
    h, to_h = _norm_sum(x, residual, h, stream)
    _norm(x, weight, residual, eps, to_h, to_y, None, None, 0, stream)
    return y, h


def add_rms_norm_fp8(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                     group: int = 0, h: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """add_rms_norm with y in 8 bits: (y8 e4m3 [T, n], scales float32 [T, groups], h), y = y8 * scales of the
    element's group of columns (0: one group a row; 128)."""
    if x.dim() != 2:
        raise ValueError("x must be [T, n]")
    shape, device = x.shape, x.device
    y8 = _empty(shape, torch.float8_e4m3fn, device, stream)
    scales = _empty((shape[0], -(-shape[1] // group) if group > 0 else 1), torch.float32, device, stream)
    h, to_h = _norm_sum(x, residual, h, stream)
    _norm(x, weight, residual, eps, to_h, None, y8.data_ptr(), scales.data_ptr(), group, stream)
    return y8, scales, h


class Adapters:
    """The low-rank adapters of one projection: A [n, rank, in], B [n, out, rank] (bf16) and scale [n] (float32,
    alpha / rank).  Ranks that are no multiple of 8 are padded with zeros, once, here (an infinity in x
    then gives NaN)."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor):
        for t, dt, name in ((A, torch.bfloat16, "A"), (B, torch.bfloat16, "B"), (scale, torch.float32, "scale")):
            _require_cuda(t, dt, name)
        if A.dim() != 3 or B.dim() != 3 or B.shape[0] != A.shape[0] or B.shape[2] != A.shape[1] or scale.shape != A.shape[:1]:
            raise ValueError("A must be [n, rank, in], B [n, out, rank] and scale [n]")
        pad = -A.shape[1] % 8
        if pad:
            A = torch.nn.functional.pad(A, (0, 0, 0, pad))
            B = torch.nn.functional.pad(B, (0, pad))
        self.A, self.B, self.scale = A, B, scale
        self.n, self.rank, self.inp = A.shape
        self.out = B.shape[1]
        self._c = _AdapterLayer(None, None, None, A.data_ptr(), B.data_ptr(), scale.data_ptr(), self.inp, self.out, self.n,
                                self.rank)


def adapters_batched_into(xs: Sequence[torch.Tensor], bases: Sequence[torch.Tensor], ads: Sequence[Adapters],
                          offsets: torch.Tensor, ids: torch.Tensor, outs: Sequence[torch.Tensor],
                          stream: Optional[torch.cuda.Stream] = None) -> None:
    """outs[i] = bases[i] + scale_a B_a (A_a xs[i]) for up to 8 layers of one step: sequence s has the tokens
    offsets[s] ... offsets[s + 1] - 1 (int32 [n + 1]) and the adapter a = ids[s] (int32 [n]; outside [0, n): none).
    outs[i] may be bases[i] itself, e.g. what linear_batched_into wrote."""
    n = len(ads)
    if not (len(xs) == len(bases) == len(outs) == n):
        raise ValueError("xs, bases, ads, outs must have the same length")
    if n == 0:
        return
    _require_cuda(offsets, torch.int32, "offsets")
    _require_cuda(ids, torch.int32, "ids")
    if offsets.dim() != 1 or ids.dim() != 1 or offsets.shape[0] != ids.shape[0] + 1:
        raise ValueError("offsets must be [n + 1] and ids [n]")
    T = xs[0].shape[0]
    arr = (_AdapterLayer * n)(*[ad._c for ad in ads])
    for l, x, base, ad, out in zip(arr, xs, bases, ads, outs):
        shape = (T, ad.out)
        l.x, l.base = _require_like(x, (T, ad.inp), "x"), _require_like(base, shape, "base")
        l.out_ptr = l.base if out is base else _require_like(out, shape, "out")
    _check(lib.gs_adapters_batched(n, arr, offsets.data_ptr(), ids.data_ptr(), ids.shape[0], T, _stream_ptr(stream)),
           "gs_adapters_batched")


def adapters_into(x: torch.Tensor, base: torch.Tensor, ad: Adapters, offsets: torch.Tensor, ids: torch.Tensor,
                  out: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """out = base + scale_a B_a (A_a x) for one layer (see adapters_batched_into)."""
    adapters_batched_into((x,), (base,), (ad,), offsets, ids, (out,), stream)
    return out


def linear_adapted(x: torch.Tensor, p: Packed, ad: Adapters, offsets: torch.Tensor, ids: torch.Tensor,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The packed projection with its requests' adapters: y = x (W (.) M)^T + scale_a B_a (A_a x)."""
    y = linear_into(x, p, _empty((x.shape[0], p.out), torch.bfloat16, x.device, stream), stream=stream)
    return adapters_into(x, y, ad, offsets, ids, y, stream)


class PagedCache:
    """Keys and values of one layer, bf16 [pages, kv_heads, page_size, head_dim] each."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor):
        _require_cuda(k_pages, torch.bfloat16, "k_pages")
        _require_cuda(v_pages, torch.bfloat16, "v_pages")
        if k_pages.dim() != 4 or v_pages.shape != k_pages.shape:
            raise ValueError("k_pages and v_pages must both be [pages, kv_heads, page_size, head_dim]")
        self.k_pages, self.v_pages = k_pages, v_pages
        self.pages, self.kv_heads, self.page_size, self.head_dim = k_pages.shape
        self._c = _CacheStruct(k_pages.data_ptr(), v_pages.data_ptr(), self.pages, self.page_size, self.kv_heads, self.head_dim)
        self._ref = ctypes.addressof(self._c)


# The attention's workspace, one per (device, stream) for all layers; calls leave its counters ready for the next.
# A graph has its own, of its memory pool: it may be replayed on any stream, beside calls on the one it was captured
# on and beside other graphs.  Each replay begins by zeroing the counters, so nothing is left of one that gave up.
_attention_ws: dict = {}
_captured_ws: dict = {}       # (device, stream): (capture, workspace), held while that capture may still use it
_foreign_ws: list = []        # of captures with no memory pool of torch's: in use as long as their graphs live


def _new_workspace(need: int, device) -> torch.Tensor:
    ws = torch.empty((need,), dtype=torch.uint8, device=device)
    ws[:ATTENTION_COUNTER_BYTES].zero_()
    return ws


def _graph_owned(t: torch.Tensor) -> bool:
    """Whether t lies in a graph's memory pool, which keeps the memory for the graph after t is gone."""
    if torch.cuda.get_allocator_backend() != "native":
        return False
    at = t.data_ptr()
    return any(s["address"] <= at < s["address"] + s["total_size"] and tuple(s["segment_pool_id"]) != (0, 0)
               for s in torch.cuda.memory_snapshot())


def _attention_workspace(need: int, device, stream: Optional[torch.cuda.Stream], sp: int) -> torch.Tensor:
    if stream is not None and stream != torch.cuda.current_stream():
        with torch.cuda.stream(stream):
            return _attention_workspace(need, device, None, sp)
    key = (device.index, sp)
    if torch.cuda.is_current_stream_capturing():
        capture = ctypes.c_uint64()
        _check(lib.gs_capture_id(sp, ctypes.byref(capture)), "gs_capture_id")
        of, ws = _captured_ws.get(key, (0, None))
        if of != capture.value or ws.numel() < need:
            ws = _new_workspace(need, device)
            if not _graph_owned(ws):
                _foreign_ws.append(ws)
            _captured_ws[key] = (capture.value, ws)
        return ws
    ws = _attention_ws.get(key)
    if ws is None or ws.numel() < need:
        ws = _attention_ws[key] = _new_workspace(need, device)
    return ws


class Batch:
    """One step's sequences, made once for all layers.  Sequence i brings the tokens offsets[i] ... offsets[i + 1] - 1
    (int32 [n + 1]), is kv_lens[i] tokens long with them (int32 [n]) and keeps position p in page
    table[i, p // page_size] (int32 [n, width]).  max_new: at least the most new tokens of a sequence."""

    def __init__(self, offsets: torch.Tensor, kv_lens: torch.Tensor, table: torch.Tensor, max_new: int):
        for t, name in ((offsets, "offsets"), (kv_lens, "kv_lens"), (table, "table")):
            _require_cuda(t, torch.int32, name)
        n = kv_lens.numel()
        if offsets.shape != (n + 1,) or kv_lens.dim() != 1 or table.dim() != 2 or table.shape[0] != n:
            raise ValueError("offsets must be [n + 1], kv_lens [n] and table [n, width]")
        if not 0 <= max_new < 2 ** 31:   # ctypes would keep its low 32 bits
            raise ValueError(f"max_new must be in [0, 2^31), got {max_new}")
        self.offsets, self.kv_lens, self.table, self.max_new = offsets, kv_lens, table, int(max_new)
        self._c = _BatchStruct(offsets.data_ptr(), kv_lens.data_ptr(), table.data_ptr(), n, table.shape[1], 0, self.max_new)
        self._ref = ctypes.addressof(self._c)
        self._need = {}

    def _workspace_bytes(self, cache: PagedCache, q_heads: int, tokens: int) -> int:
        key = (q_heads, cache.kv_heads, cache.head_dim, tokens)
        need = self._need.get(key)
        if need is None:
            c = ctypes.c_size_t()
            _check(lib.gs_paged_attention_workspace(cache._ref, self._ref, q_heads, ctypes.byref(c)),
                   "gs_paged_attention_workspace")
            need = self._need[key] = c.value
        return need


def _heads(t: torch.Tensor, D: int, name: str):
    """(tokens, heads, distance of two tokens) of [T, heads, D], whose heads lie side by side (a slice of a joint
    projection may be one)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != torch.bfloat16:
        raise ValueError(f"{name} must be torch.bfloat16, got {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [T, heads, {D}]")
    T, heads, d = t.shape
    token, head, one = t.stride()
    if d != D or one != 1 or (head != D and heads != 1):
        raise ValueError(f"{name} must be [T, heads, {D}] with dense heads")
    return T, heads, token if T != 1 else heads * D


def cache_append(cache: PagedCache, batch: Batch, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, q_out: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Turns q [T, q_heads, D] and k [T, kv_heads, D] by their positions' angles (cos, sin: float32 [positions, D / 2];
    channels i and i + D / 2 are a pair), writes k and v into the cache's pages and returns the turned q (q_out)."""
    D, kv = cache.head_dim, cache.kv_heads
    T, heads, qs = _heads(q, D, "q")
    Tk, hk, ks = _heads(k, D, "k")
    Tv, hv, vs = _heads(v, D, "v")
    if Tk != T or Tv != T or hk != kv or hv != kv:
        raise ValueError("k and v must be [T, kv_heads, D] with q's T")
    if cos.dtype != torch.float32 or not cos.is_cuda or not cos.is_contiguous():
        _require_cuda(cos, torch.float32, "cos")
    if sin.dtype != torch.float32 or not sin.is_cuda or not sin.is_contiguous():
        _require_cuda(sin, torch.float32, "sin")
    shape = cos.shape
    if len(shape) != 2 or shape[1] * 2 != D or sin.shape != shape:
        raise ValueError("cos and sin must be [positions, head_dim / 2]")
    if q_out is None:
        q_out = _empty(q.shape, torch.bfloat16, q.device, stream)
    to = _require_like(q_out, q.shape, "q_out")
    batch._c.tokens = T
    _check(lib.gs_cache_append(cache._ref, batch._ref, q.data_ptr(), qs, heads, k.data_ptr(), ks, v.data_ptr(), vs,
                               cos.data_ptr(), sin.data_ptr(), shape[0], to, _stream_ptr(stream)),
           "gs_cache_append")
    return q_out


def paged_attention(q: torch.Tensor, cache: PagedCache, batch: Batch, scale: Optional[float] = None,
                    out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Causal attention of a step's queries q [T, q_heads, D] over the cache (the step's own keys are in it already:
    cache_append), bf16 [T, q_heads, D].  scale: 1 / sqrt(D) if not given.  A token without visible keys gets zeros.
    Its workspace is the stream's, or the graph's where the stream is being captured."""
    D = cache.head_dim
    T, heads, qs = _heads(q, D, "q")
    if out is None:
        out = _empty(q.shape, torch.bfloat16, q.device, stream)
    to = _require_like(out, q.shape, "out")
    batch._c.tokens = T
    sp = _stream_ptr(stream)
    ws = _attention_workspace(batch._workspace_bytes(cache, heads, T), q.device, stream, sp)
    _check(lib.gs_paged_attention(cache._ref, batch._ref, q.data_ptr(), qs, heads, D ** -0.5 if scale is None else scale, to,
                                  ws.data_ptr(), ws.numel(), sp), "gs_paged_attention")
    return out


def debug_fail_alloc(nth: int) -> None:
    """Test hook: the nth device allocation the library makes from now on fails (0 disarms)."""
    _check(lib.gs_debug_fail_alloc(int(nth)), "gs_debug_fail_alloc")


def debug_inject_wait(algo: int, limit_ns: int) -> None:
    """Test hook: the next launch of that kernel family times out on a word nothing sets."""
    _check(lib.gs_debug_inject_wait(int(algo), int(limit_ns)), "gs_debug_inject_wait")


def debug_inject_attention_wait(chunk: bool, limit_ns: int) -> None:
    """Test hook: the next launch of the attention's kernel for few (or many) rows times out on a word nothing sets."""
    _check(lib.gs_debug_inject_attention_wait(int(bool(chunk)), int(limit_ns)), "gs_debug_inject_attention_wait")


def device_status(stream: Optional[torch.cuda.Stream] = None) -> int:
    status = int(lib.gs_device_status(_stream_ptr(stream)))
    if status == GS_ERR_DEVICE_TIMEOUT:
        _attention_ws.clear()      # counters of a kernel that gave up are not zero (graphs zero theirs)
    return status


def launch_count() -> int:
    return int(lib.gs_launch_count())
