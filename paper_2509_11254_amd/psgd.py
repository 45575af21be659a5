"""Thin ctypes binding over libpsgd.so (the C ABI of include/psgd.h).

Argument marshalling only: every step of the compressor runs in the library's HIP kernels.
PyTorch provides device memory (tensors whose data_ptr() is handed over) and the stream.
There is no CPU or PyTorch fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpsgd.so")

PSGD_F32, PSGD_BF16 = 0, 1
PSGD_OK = 0
PSGD_E_INVALID_ARG, PSGD_E_SHAPE, PSGD_E_ALIGN, PSGD_E_HIP, PSGD_E_NOMEM, PSGD_E_CAPTURE = -1, -2, -3, -4, -5, -6
PSGD_E_TOO_LARGE = -7
STATIC_WORKSPACE_BYTES = 64 * 1024 * 1024

EXPORTS = [
    "psgd_init", "psgd_workspace_bytes", "psgd_workspace_reset", "psgd_compress", "psgd_compress_static", "psgd_compress_refresh", "psgd_flush_residual", "psgd_refresh",
    "psgd_decompress", "psgd_decompress_msgd", "psgd_decompress_adam", "psgd_compress_project", "psgd_compress_finish", "psgd_status", "psgd_algorithmic_bytes", "psgd_kernel_bytes", "psgd_copy_bytes",
    "psgd_last_hip_error",
    "psgd_strerror", "psgd_destroy", "psgd_profile_enable", "psgd_profile_select", "psgd_profile_read",
    "psgd_head_workspace_bytes", "psgd_head_loss", "psgd_head_loss_grad", "psgd_act_store", "psgd_act_restore",
    "psgd_act_glu", "psgd_act_glu_backward", "psgd_act_wgrad_workspace_bytes", "psgd_act_wgrad",
    "psgd_head_distill_workspace_bytes", "psgd_head_distill", "psgd_head_distill_grad",
    "psgd_norm", "psgd_norm_backward_workspace_bytes", "psgd_norm_backward", "psgd_expert_sort_workspace_bytes", "psgd_expert_sort",
    "psgd_expert_rows", "psgd_expert_combine", "psgd_expert_combine_backward",
]
PSGD_SILU, PSGD_GELU = 0, 1
ACT_GROUP = 32      # columns of an activation that share a scale
PROF_TAGS = ("sweep1", "sweep2", "residual")


class LayerDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("r", C.c_int32),
                ("grad_dtype", C.c_int32)]


class Options(C.Structure):
    _fields_ = [("refresh_iters", C.c_int32), ("refresh_oversample", C.c_int32),
                ("refresh_warm_start", C.c_int32), ("seed", C.c_uint32), ("rank_tol", C.c_float),
                ("precision", C.c_int32), ("m_policy", C.c_int32), ("power_iters", C.c_int32),
                ("lazy_residual", C.c_int32), ("q_resident", C.c_int32)]


class LayerStatus(C.Structure):
    _fields_ = [("rank_deficient", C.c_int32), ("refresh_iters_next", C.c_int32), ("sigma_max", C.c_float),
                ("sigma_r", C.c_float), ("refresh_iters_no_gap", C.c_int32)]


class HeadDesc(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("d", C.c_int64), ("vocab", C.c_int64), ("ldx", C.c_int64), ("ldw", C.c_int64),
                ("lddx", C.c_int64), ("lddw", C.c_int64), ("dtype", C.c_int32), ("grad_dtype", C.c_int32),
                ("piece_tokens", C.c_int64)]


class PsgdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"psgd error {code}: {msg}")
        self.code = code


_lib = None


def load_library() -> C.CDLL:
    """Load libpsgd.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2509_11254_amd.build` "
            "(hipcc, gfx950). The compressor has no CPU fallback.")
    # PyTorch owns the device memory and the streams handed to the library, so both must talk to
    # the same HIP runtime instance: import torch first, then libpsgd.so binds to the runtime
    # (libamdhip64.so.7) that torch has already loaded instead of opening a second one.
    import torch  # noqa: F401
    lib = C.CDLL(LIB_PATH)
    vp, pp = C.c_void_p, C.POINTER(C.c_void_p)
    lib.psgd_init.argtypes = [pp, C.c_int, C.POINTER(LayerDesc), C.c_int, C.POINTER(Options)]
    lib.psgd_init.restype = C.c_int
    lib.psgd_workspace_bytes.argtypes = [vp]
    lib.psgd_workspace_bytes.restype = C.c_size_t
    lib.psgd_workspace_reset.argtypes = [vp]
    lib.psgd_workspace_reset.restype = C.c_int
    for name in ("psgd_compress", "psgd_compress_refresh", "psgd_compress_project"):
        fn = getattr(lib, name)
        fn.argtypes = [vp, vp, vp, pp, pp, pp, pp]
        fn.restype = C.c_int
    lib.psgd_compress_static.argtypes = [vp, vp, pp, pp, pp, pp]
    lib.psgd_compress_static.restype = C.c_int
    lib.psgd_compress_finish.argtypes = [vp, vp, vp, pp, pp, pp]
    lib.psgd_compress_finish.restype = C.c_int
    lib.psgd_flush_residual.argtypes = [vp, vp, vp, pp]
    lib.psgd_flush_residual.restype = C.c_int
    lib.psgd_refresh.argtypes = [vp, vp, vp, C.c_int, vp, vp, vp, vp]
    lib.psgd_refresh.restype = C.c_int
    lib.psgd_decompress.argtypes = [vp, vp, vp, pp, pp, pp, C.c_int]
    lib.psgd_decompress.restype = C.c_int
    lib.psgd_decompress_msgd.argtypes = [vp, vp, vp, pp, pp, pp, pp, C.c_float, C.c_float]
    lib.psgd_decompress_msgd.restype = C.c_int
    lib.psgd_decompress_adam.argtypes = [vp, vp, vp, pp, pp, pp, pp, pp, C.c_int, C.c_float, C.c_float, C.c_float,
                                         C.c_float, C.c_float]
    lib.psgd_decompress_adam.restype = C.c_int
    lib.psgd_status.argtypes = [vp, vp, vp, C.c_int, C.POINTER(LayerStatus)]
    lib.psgd_status.restype = C.c_int
    lib.psgd_algorithmic_bytes.argtypes = [vp]
    lib.psgd_algorithmic_bytes.restype = C.c_double
    lib.psgd_kernel_bytes.argtypes = [vp, C.c_int]
    lib.psgd_kernel_bytes.restype = C.c_double
    lib.psgd_copy_bytes.argtypes = [vp, vp, vp, C.c_size_t]
    lib.psgd_copy_bytes.restype = C.c_int
    lib.psgd_last_hip_error.argtypes = [vp]
    lib.psgd_last_hip_error.restype = C.c_int
    lib.psgd_strerror.argtypes = [C.c_int]
    lib.psgd_strerror.restype = C.c_char_p
    lib.psgd_profile_enable.argtypes = [vp, C.c_int]
    lib.psgd_profile_enable.restype = C.c_int
    lib.psgd_profile_select.argtypes = [vp, C.c_int]
    lib.psgd_profile_select.restype = C.c_int
    lib.psgd_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int), C.c_int]
    lib.psgd_profile_read.restype = C.c_int
    i, l, hd = C.c_int, C.c_int64, C.POINTER(HeadDesc)
    lib.psgd_head_workspace_bytes.argtypes = [hd, i]
    lib.psgd_head_workspace_bytes.restype = C.c_size_t
    lib.psgd_head_loss.argtypes = [hd, vp, vp, vp, vp, vp, vp]
    lib.psgd_head_loss_grad.argtypes = [hd, vp, vp, vp, vp, vp, vp, vp, vp, vp, i]
    lib.psgd_act_store.argtypes = [vp, l, l, vp, i, l, vp, l, vp]
    lib.psgd_act_restore.argtypes = [vp, l, l, vp, l, vp, vp, i, l]
    lib.psgd_act_glu.argtypes = [vp, l, l, i, i, vp, vp, l, vp, l, vp, vp, vp, vp, l]
    lib.psgd_act_glu_backward.argtypes = [vp, l, l, i, i, vp, vp, vp, vp, l, vp, l, vp, vp, l]
    lib.psgd_act_wgrad_workspace_bytes.argtypes = [l, l, l, i]
    lib.psgd_act_wgrad_workspace_bytes.restype = C.c_size_t
    lib.psgd_act_wgrad.argtypes = [vp, vp, l, l, l, vp, i, l, vp, l, vp, vp, i, l, i]
    lib.psgd_head_distill_workspace_bytes.argtypes = [hd, l, i]
    lib.psgd_head_distill_workspace_bytes.restype = C.c_size_t
    lib.psgd_head_distill.argtypes = [hd, vp, vp, vp, vp, l, vp, vp, i, l, C.c_float, vp]
    lib.psgd_head_distill_grad.argtypes = [hd, vp, vp, vp, vp, l, vp, vp, i, l, C.c_float, vp, vp, vp, vp, i]
    lib.psgd_norm.argtypes = [vp, l, l, i, vp, l, vp, l, vp, vp, i, C.c_float, vp, l, vp, l, vp]
    lib.psgd_norm_backward_workspace_bytes.argtypes = [l, l, i]
    lib.psgd_norm_backward_workspace_bytes.restype = C.c_size_t
    lib.psgd_norm_backward.argtypes = [vp, vp, l, l, i, vp, l, vp, l, vp, i, vp, vp, l, vp, l, vp, vp, i, i]
    lib.psgd_expert_sort_workspace_bytes.argtypes = [l, l, l]
    lib.psgd_expert_sort_workspace_bytes.restype = C.c_size_t
    lib.psgd_expert_sort.argtypes = [vp, vp, l, l, l, vp, vp, vp, vp]
    lib.psgd_expert_rows.argtypes = [vp, l, l, l, i, vp, l, vp, vp, l]
    lib.psgd_expert_combine.argtypes = [vp, l, l, l, i, vp, l, vp, vp, vp, l]
    lib.psgd_expert_combine_backward.argtypes = [vp, l, l, l, i, vp, l, vp, l, vp, vp, vp, l, vp]
    for name in ("psgd_head_loss", "psgd_head_loss_grad", "psgd_act_store", "psgd_act_restore", "psgd_act_glu",
                 "psgd_act_glu_backward", "psgd_act_wgrad", "psgd_head_distill", "psgd_head_distill_grad", "psgd_norm", "psgd_norm_backward", "psgd_expert_sort",
                 "psgd_expert_rows", "psgd_expert_combine", "psgd_expert_combine_backward"):
        getattr(lib, name).restype = C.c_int
    lib.psgd_destroy.argtypes = [vp]
    lib.psgd_destroy.restype = None
    _lib = lib
    return lib


def _check(lib, ctx, rc: int):
    if rc != PSGD_OK:
        msg = lib.psgd_strerror(rc).decode()
        if rc == PSGD_E_HIP and ctx:
            msg += f" (hipError {lib.psgd_last_hip_error(ctx)})"
        raise PsgdError(rc, msg)


def _ptr_table(tensors: Sequence) -> C.Array:
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = t.data_ptr()
    return arr


def _opt_table(tensors):
    """Pointer table, or a null pointer for None (where the ABI gives NULL a meaning)."""
    return _ptr_table(tensors) if tensors is not None else None


def _stream_handle(stream) -> int:
    import torch
    if stream is not None:
        return int(stream.cuda_stream)
    # the handle alone: a torch.cuda.Stream object of the current stream costs 3 us a call
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


class Compressor:
    """psgd_init + a torch-allocated workspace; methods mirror the C entry points one to one.

    layers: sequence of (rows, cols, r, grad_dtype) or (rows, cols, r, grad_dtype, ld).
    """

    def __init__(self, layers: Sequence[Sequence[int]], n_workers: int, *, refresh_iters: int = 0,
                 refresh_oversample: int = -1, refresh_warm_start: bool = True, seed: int = 0x5EED5EED,
                 rank_tol: float = 0.0, precision: int = 0, m_policy: int = 0, power_iters: int = 0,
                 lazy_residual: bool = False, q_resident: bool = False, device: str = "cuda:0",
                 allocate: bool = True):
        self.lib = load_library()
        self.n_layers = len(layers)
        self.n_workers = int(n_workers)
        descs = (LayerDesc * max(1, self.n_layers))()
        for i, l in enumerate(layers):
            descs[i].rows, descs[i].cols, descs[i].r, descs[i].grad_dtype = int(l[0]), int(l[1]), int(l[2]), int(l[3])
            descs[i].ld = int(l[4]) if len(l) > 4 else 0
        opt = Options(int(refresh_iters), int(refresh_oversample), 1 if refresh_warm_start else 0,
                      int(seed) & 0xFFFFFFFF, float(rank_tol), int(precision), int(m_policy), int(power_iters),
                      1 if lazy_residual else 0, 1 if q_resident else 0)
        self.ctx = C.c_void_p()
        rc = self.lib.psgd_init(C.byref(self.ctx), self.n_layers, descs, self.n_workers, C.byref(opt))
        _check(self.lib, None, rc)
        self.layers = [tuple(l) for l in layers]
        self.workspace_bytes = int(self.lib.psgd_workspace_bytes(self.ctx))
        self.workspace = None
        if allocate:
            import torch
            self.workspace = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=device)
            self._ws_ptr = (self.workspace.data_ptr() + 255) // 256 * 256
        self._keep = None

    def __del__(self):
        try:
            if getattr(self, "ctx", None) is not None and self.ctx:
                self.lib.psgd_destroy(self.ctx)
                self.ctx = None
        except Exception:
            pass

    @property
    def algorithmic_bytes(self) -> float:
        return float(self.lib.psgd_algorithmic_bytes(self.ctx))

    def kernel_bytes(self, tag: str) -> float:
        """Algorithmic bytes of one launch of the streaming kernel `tag` (one of PROF_TAGS) over all layers."""
        return float(self.lib.psgd_kernel_bytes(self.ctx, PROF_TAGS.index(tag)))

    def _tables(self, G, E, Q, P):
        flat_g = [g for per_layer in G for g in per_layer] if G and isinstance(G[0], (list, tuple)) else list(G)
        tabs = (_ptr_table(flat_g), _ptr_table(E), _ptr_table(Q), _ptr_table(P))
        self._keep = tabs
        return tabs

    def compress(self, G, E, Q, P, stream=None) -> None:
        """psgd_compress: G[l][i] gradients, E[l] error buffers (in place), Q[l] in/out, P[l] out."""
        tg, te, tq, tp = self._tables(G, E, Q, P)
        _check(self.lib, self.ctx, self.lib.psgd_compress(self.ctx, self._ws_ptr, _stream_handle(stream), tg, te, tq, tp))

    def compress_static(self, G, E, Q, P, stream=None) -> None:
        """psgd_compress_static: psgd_compress in the library's built-in workspace (allocates nothing)."""
        tg, te, tq, tp = self._tables(G, E, Q, P)
        _check(self.lib, self.ctx, self.lib.psgd_compress_static(self.ctx, _stream_handle(stream), tg, te, tq, tp))

    def compress_refresh(self, G, E, Q, P, stream=None) -> None:
        tg, te, tq, tp = self._tables(G, E, Q, P)
        _check(self.lib, self.ctx,
               self.lib.psgd_compress_refresh(self.ctx, self._ws_ptr, _stream_handle(stream), tg, te, tq, tp))

    def compress_project(self, G, E, Q, P, stream=None) -> None:
        """psgd_compress_project: E[l] <- M = G[l] + E[l]; P[l] <- M Q[l] (first half of a data-parallel step)."""
        tg, te, tq, tp = self._tables(G, E, Q, P)
        _check(self.lib, self.ctx,
               self.lib.psgd_compress_project(self.ctx, self._ws_ptr, _stream_handle(stream), tg, te, tq, tp))

    def compress_finish(self, E, Q, P, stream=None) -> None:
        """psgd_compress_finish: P[l] <- QR(P[l]) (the averaged P); Q[l] <- M^T P~; E[l] <- M - P~ Q[l]^T."""
        te, tq, tp = _ptr_table(E), _ptr_table(Q), _ptr_table(P)
        self._keep = (te, tq, tp)
        _check(self.lib, self.ctx,
               self.lib.psgd_compress_finish(self.ctx, self._ws_ptr, _stream_handle(stream), te, tq, tp))

    def workspace_reset(self) -> None:
        """psgd_workspace_reset: treat the workspace as new (its contents were lost or recycled)."""
        _check(self.lib, self.ctx, self.lib.psgd_workspace_reset(self.ctx))

    def flush_residual(self, E, stream=None) -> None:
        """psgd_flush_residual: settle the residual a lazy_residual compress step left owed (E[l] <- E_{t+1})."""
        te = _ptr_table(E)
        self._keep = (te,)
        _check(self.lib, self.ctx, self.lib.psgd_flush_residual(self.ctx, self._ws_ptr, _stream_handle(stream), te))

    def refresh(self, layer: int, M, P, Q, sigma=None, stream=None) -> None:
        _check(self.lib, self.ctx,
               self.lib.psgd_refresh(self.ctx, self._ws_ptr, _stream_handle(stream), int(layer), M.data_ptr(),
                                     P.data_ptr(), Q.data_ptr(), sigma.data_ptr() if sigma is not None else None))

    def decompress(self, P, Q, out, out_dtype: int = PSGD_F32, stream=None) -> None:
        """psgd_decompress: out[l] <- P[l] Q[l]^T; P = Q = None: the factors of the last compress call."""
        tp, tq, to = _opt_table(P), _opt_table(Q), _ptr_table(out)
        self._keep = (tp, tq, to)
        _check(self.lib, self.ctx,
               self.lib.psgd_decompress(self.ctx, self._ws_ptr, _stream_handle(stream), tp, tq, to, int(out_dtype)))

    def decompress_msgd(self, P, Q, mom, X, mu: float, eta: float, stream=None) -> None:
        """psgd_decompress_msgd: mom[l] <- mu mom[l] + P[l] Q[l]^T, X[l] <- X[l] - eta mom[l] (in place)."""
        tp, tq, tm, tx = _opt_table(P), _opt_table(Q), _ptr_table(mom), _ptr_table(X)
        self._keep = (tp, tq, tm, tx)
        _check(self.lib, self.ctx,
               self.lib.psgd_decompress_msgd(self.ctx, self._ws_ptr, _stream_handle(stream), tp, tq, tm, tx,
                                             C.c_float(mu), C.c_float(eta)))

    def decompress_adam(self, P, Q, m1, m2, X, step: int, eta: float, beta1: float = 0.9, beta2: float = 0.999,
                        eps: float = 1e-8, weight_decay: float = 0.0, stream=None) -> None:
        """psgd_decompress_adam: Adam / AdamW moments m1[l], m2[l] and weights X[l] from P[l] Q[l]^T (in place)."""
        tp, tq, t1, t2, tx = _opt_table(P), _opt_table(Q), _ptr_table(m1), _ptr_table(m2), _ptr_table(X)
        self._keep = (tp, tq, t1, t2, tx)
        _check(self.lib, self.ctx,
               self.lib.psgd_decompress_adam(self.ctx, self._ws_ptr, _stream_handle(stream), tp, tq, t1, t2, tx,
                                             int(step), C.c_float(eta), C.c_float(beta1), C.c_float(beta2),
                                             C.c_float(eps), C.c_float(weight_decay)))

    def profile_enable(self, max_records: int) -> None:
        _check(self.lib, self.ctx, self.lib.psgd_profile_enable(self.ctx, int(max_records)))

    def profile_select(self, tags: Sequence[str]) -> None:
        """Time only the launches with these tags (each timed launch costs two event records on the stream)."""
        mask = 0
        for t in tags:
            mask |= 1 << PROF_TAGS.index(t)
        _check(self.lib, self.ctx, self.lib.psgd_profile_select(self.ctx, mask))

    def profile_read(self) -> dict:
        """{tag: (total_ms, count)} of the event pairs recorded since the last read."""
        n = len(PROF_TAGS)
        ms, cnt = (C.c_double * n)(), (C.c_int * n)()
        _check(self.lib, self.ctx, self.lib.psgd_profile_read(self.ctx, ms, cnt, n))
        return {PROF_TAGS[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}

    def status(self, layer: int, stream=None) -> LayerStatus:
        st = LayerStatus()
        _check(self.lib, self.ctx,
               self.lib.psgd_status(self.ctx, self._ws_ptr, _stream_handle(stream), int(layer), C.byref(st)))
        return st


def copy_bytes(dst, src, n_bytes: int, stream=None) -> None:
    lib = load_library()
    rc = lib.psgd_copy_bytes(_stream_handle(stream), dst.data_ptr(), src.data_ptr(), int(n_bytes))
    _check(lib, None, rc)


# ---- the training step around the compressor ---------------------------------------------------------------------------

_dtype_codes: dict = {}


def _dtype_code(t) -> int:
    code = _dtype_codes.get(t.dtype)
    if code is None:
        import torch
        _dtype_codes.update({torch.float32: PSGD_F32, torch.bfloat16: PSGD_BF16})
        code = _dtype_codes.get(t.dtype)
        if code is None:
            raise ValueError("float32 or bfloat16 expected, got %s" % t.dtype)
    return code


def _matrix(name: str, t, rows: int, cols: int, dtype: Optional[int] = None) -> int:
    """Checks a rows x cols matrix on the GPU with adjacent columns; its leading dimension."""
    strides = t.stride()            # (asked once: each question costs 0.1 to 0.2 us)
    if t.shape != (rows, cols) or not t.is_cuda or (cols > 1 and strides[1] != 1):
        raise ValueError("%s: a %d x %d matrix on the GPU with adjacent columns expected, got %s with strides %s on %s"
                         % (name, rows, cols, tuple(t.shape), strides, t.device))
    if dtype is not None and _dtype_code(t) != dtype:
        raise ValueError("%s: wrong element type %s" % (name, t.dtype))
    # (with one row the stride says nothing)
    ld = strides[0] if rows > 1 else (cols + 7) // 8 * 8
    if ld < cols:
        raise ValueError("%s: rows that lie over each other (%d elements apart, %d columns)" % (name, ld, cols))
    # (a row of whole eights ends there itself; calls on small matrices take as long as these questions)
    if cols & 7 and rows and t.storage_offset() + (rows - 1) * ld + (cols + 7) // 8 * 8 > t.untyped_storage().nbytes() // t.element_size():
        raise ValueError("%s: the last row ends before the next multiple of 8 columns, up to which rows may be read" % name)
    return ld


def _stream_for(stream, *tensors) -> int:
    """Handle of the stream that a call goes to (None: the current one), on whose device all its tensors are."""
    import torch
    device = torch.cuda.current_device() if stream is None else stream.device.index
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("a tensor on %s for a call on a stream of cuda:%d" % (t.device, device))
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else int(stream.cuda_stream)


def _vector(name: str, t, n: int, dtype):
    if t.dtype != dtype or t.shape != (n,) or not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s: %d contiguous elements of %s on the GPU expected" % (name, n, dtype))
    return t


def _work_area(n_bytes: int, device):
    import torch
    buf = torch.empty(n_bytes + 256, dtype=torch.uint8, device=device)
    return buf, (buf.data_ptr() + 255) // 256 * 256


def _ptr(t):
    return t.data_ptr() if t is not None else None


class HeadLoss:
    """Softmax cross entropy of X W^T against labels without logits in memory, and its gradients: psgd_head_loss and
    psgd_head_loss_grad with a torch-allocated workspace, for one set of sizes and types.

    A token whose label lies outside [0, vocab) does not count.  grad=False: losses alone (a smaller workspace).  Calls on streams
    that do not wait for each other need an object each: they would share the workspace.
    """

    def __init__(self, tokens: int, d: int, vocab: int, dtype: int = PSGD_BF16, grad_dtype: Optional[int] = None, *,
                 grad: bool = True, piece_tokens: int = 0, device: str = "cuda"):
        self.lib = load_library()
        self.desc = HeadDesc(int(tokens), int(d), int(vocab), 0, 0, 0, 0, int(dtype),
                             int(dtype if grad_dtype is None else grad_dtype), int(piece_tokens))
        self.grad = bool(grad)
        sizes = [int(self.lib.psgd_head_workspace_bytes(C.byref(self.desc), g)) for g in ([0, 1] if grad else [0])]
        if min(sizes) == 0:
            raise PsgdError(PSGD_E_INVALID_ARG, "sizes or types of the head")
        self.workspace_bytes = max(sizes)
        self.workspace, self._ws_ptr = _work_area(self.workspace_bytes, device)

    def _inputs(self, X, W, labels, loss):
        import torch
        d = self.desc
        d.ldx, d.ldw = _matrix("X", X, d.tokens, d.d, d.dtype), _matrix("W", W, d.vocab, d.d, d.dtype)
        _vector("labels", labels, d.tokens, torch.int64)
        _vector("loss", loss, d.tokens, torch.float32)

    def loss(self, X, W, labels, loss, stream=None) -> None:
        """loss[t] <- lse_t - logit of the label, 0 for tokens that do not count."""
        self._inputs(X, W, labels, loss)
        _check(self.lib, None, self.lib.psgd_head_loss(
            C.byref(self.desc), self._ws_ptr, _stream_for(stream, self.workspace, X, W, labels, loss), X.data_ptr(), W.data_ptr(),
            labels.data_ptr(), loss.data_ptr()))

    def loss_grad(self, X, W, labels, loss, dX, dW, weight=None, accumulate: bool = False, stream=None) -> None:
        """loss as above; dX <- gradient of sum_t weight[t] loss[t] (weight None: the mean over the tokens that count), and
        dW <- (accumulate: +=) its gradient.  dX may be X itself; otherwise results overlap nothing."""
        import torch
        if not self.grad:
            raise ValueError("this HeadLoss has no workspace for gradients (grad=False)")
        self._inputs(X, W, labels, loss)
        d = self.desc
        d.lddx, d.lddw = _matrix("dX", dX, d.tokens, d.d, d.dtype), _matrix("dW", dW, d.vocab, d.d, d.grad_dtype)
        if weight is not None:
            _vector("weight", weight, d.tokens, torch.float32)
        _check(self.lib, None, self.lib.psgd_head_loss_grad(
            C.byref(self.desc), self._ws_ptr, _stream_for(stream, self.workspace, X, W, labels, loss, dX, dW, weight), X.data_ptr(),
            W.data_ptr(), labels.data_ptr(), weight.data_ptr() if weight is not None else None, loss.data_ptr(), dX.data_ptr(), dW.data_ptr(), 1 if accumulate else 0))


def _entries(name: str, t, tokens: int, top: int, types) -> int:
    """Checks tokens x top entries on the GPU, those of a token adjacent; how far apart tokens are."""
    strides = t.stride()
    if t.shape != (tokens, top) or t.dtype not in types or not t.is_cuda or (top > 1 and strides[1] != 1):
        raise ValueError("%s: %d x %d adjacent entries of %s on the GPU expected, got %s with strides %s of %s on %s"
                         % (name, tokens, top, types, tuple(t.shape), strides, t.dtype, t.device))
    ld = strides[0] if tokens > 1 else top
    if ld < top:
        raise ValueError("%s: rows that lie over each other (%d elements apart, %d entries)" % (name, ld, top))
    return ld


class HeadDistill:
    """Divergence of the head's probabilities softmax(X W^T / temperature) from a teacher's, of which the `top` largest logits are known,
    without logits in memory, and its gradients: psgd_head_distill and psgd_head_distill_grad with a torch-allocated workspace, for one
    set of sizes and types.

    index (tokens x top int64) and teacher (its logits, float32 or bfloat16) have the same strides.  Entries whose index lies outside
    [0, vocab) do not count, nor does a token without entries.  grad=False and streams: as for HeadLoss.
    """

    def __init__(self, tokens: int, d: int, vocab: int, top: int, dtype: int = PSGD_BF16, grad_dtype: Optional[int] = None, *,
                 grad: bool = True, piece_tokens: int = 0, device: str = "cuda"):
        self.lib = load_library()
        self.desc = HeadDesc(int(tokens), int(d), int(vocab), 0, 0, 0, 0, int(dtype),
                             int(dtype if grad_dtype is None else grad_dtype), int(piece_tokens))
        self.top, self.grad = int(top), bool(grad)
        sizes = [int(self.lib.psgd_head_distill_workspace_bytes(C.byref(self.desc), self.top, g)) for g in ([0, 1] if grad else [0])]
        if min(sizes) == 0:
            raise PsgdError(PSGD_E_INVALID_ARG, "sizes or types of the head")
        self.workspace_bytes = max(sizes)
        self.workspace, self._ws_ptr = _work_area(self.workspace_bytes, device)

    def _inputs(self, X, W, index, teacher, loss):
        import torch
        d = self.desc
        d.ldx, d.ldw = _matrix("X", X, d.tokens, d.d, d.dtype), _matrix("W", W, d.vocab, d.d, d.dtype)
        ld = _entries("index", index, d.tokens, self.top, (torch.int64,))
        _same("strides of index and teacher", ld, _entries("teacher", teacher, d.tokens, self.top, (torch.float32, torch.bfloat16)))
        _vector("loss", loss, d.tokens, torch.float32)
        return ld

    def loss(self, X, W, index, teacher, loss, temperature: float = 1.0, stream=None) -> None:
        """loss[t] <- sum_v q_tv log(q_tv / p_tv), 0 for tokens that do not count."""
        ld = self._inputs(X, W, index, teacher, loss)
        _check(self.lib, None, self.lib.psgd_head_distill(
            C.byref(self.desc), self._ws_ptr, _stream_for(stream, self.workspace, X, W, index, teacher, loss), X.data_ptr(), W.data_ptr(), self.top,
            index.data_ptr(), teacher.data_ptr(), _dtype_code(teacher), ld, float(temperature), loss.data_ptr()))

    def loss_grad(self, X, W, index, teacher, loss, dX, dW, temperature: float = 1.0, weight=None, accumulate: bool = False, stream=None) -> None:
        """loss as above; dX <- gradient of sum_t weight[t] loss[t] (weight None: the mean over the tokens that count), and
        dW <- (accumulate: +=) its gradient.  dX may be X itself; otherwise results overlap nothing."""
        import torch
        if not self.grad:
            raise ValueError("this HeadDistill has no workspace for gradients (grad=False)")
        ld = self._inputs(X, W, index, teacher, loss)
        d = self.desc
        d.lddx, d.lddw = _matrix("dX", dX, d.tokens, d.d, d.dtype), _matrix("dW", dW, d.vocab, d.d, d.grad_dtype)
        if weight is not None:
            _vector("weight", weight, d.tokens, torch.float32)
        _check(self.lib, None, self.lib.psgd_head_distill_grad(
            C.byref(self.desc), self._ws_ptr, _stream_for(stream, self.workspace, X, W, index, teacher, loss, dX, dW, weight), X.data_ptr(), W.data_ptr(),
            self.top, index.data_ptr(), teacher.data_ptr(), _dtype_code(teacher), ld, float(temperature), _ptr(weight), loss.data_ptr(), dX.data_ptr(),
            dW.data_ptr(), 1 if accumulate else 0))


class Act8:
    """An 8-bit checkpoint of an activation: codes (rows x ldc int8, ldc a multiple of 16, the first `cols` count) and
    scales (rows x ceil(cols / 32) uint8, contiguous)."""

    def __init__(self, codes, scales, cols: int):
        import torch
        rows, cols = int(codes.shape[0]), int(cols)
        if codes.dtype != torch.int8 or codes.dim() != 2 or codes.shape[1] < (cols + 15) // 16 * 16 or codes.stride(1) != 1 or not codes.is_cuda:
            raise ValueError("codes: an int8 matrix on the GPU with whole 16-byte pieces of adjacent columns expected")
        if scales.dtype != torch.uint8 or tuple(scales.shape) != (rows, -(-cols // ACT_GROUP)) or not scales.is_contiguous() or not scales.is_cuda:
            raise ValueError("scales: a contiguous %d x %d uint8 matrix on the GPU expected" % (rows, -(-cols // ACT_GROUP)))
        self.codes, self.scales, self.rows, self.cols = codes, scales, rows, cols
        self.ldc = int(codes.stride(0)) if rows > 1 else (cols + 15) // 16 * 16


def act_empty(rows: int, cols: int, device: str = "cuda") -> Act8:
    """Buffers for the checkpoint of a rows x cols activation."""
    import torch
    return Act8(torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=device),
                torch.empty((rows, -(-cols // ACT_GROUP)), dtype=torch.uint8, device=device), cols)


def act_store(X, kept: Act8, stream=None) -> None:
    """psgd_act_store: kept <- X in 8 bits."""
    lib = load_library()
    ld = _matrix("X", X, kept.rows, kept.cols)
    _check(lib, None, lib.psgd_act_store(_stream_for(stream, X, kept.codes, kept.scales), kept.rows, kept.cols, X.data_ptr(), _dtype_code(X), ld,
                                         kept.codes.data_ptr(), kept.ldc, kept.scales.data_ptr()))


def act_restore(kept: Act8, X, stream=None) -> None:
    """psgd_act_restore: X <- the values that kept stands for."""
    lib = load_library()
    ld = _matrix("X", X, kept.rows, kept.cols)
    _check(lib, None, lib.psgd_act_restore(_stream_for(stream, X, kept.codes, kept.scales), kept.rows, kept.cols, kept.codes.data_ptr(), kept.ldc,
                                           kept.scales.data_ptr(), X.data_ptr(), _dtype_code(X), ld))


def _kept_tensors(*kept):
    return [t for k in kept if k is not None for t in (k.codes, k.scales)]


def _same(name: str, a, b) -> None:
    if a != b:
        raise ValueError("%s: %s and %s differ" % (name, a, b))


def act_glu(gate, up, h, kept_gate: Act8, kept_up: Optional[Act8], act: int = PSGD_SILU, stream=None) -> None:
    """psgd_act_glu: h <- act(gate) * up (up None: act(gate)), and the checkpoints of gate and up."""
    lib = load_library()
    rows, cols, dt = kept_gate.rows, kept_gate.cols, _dtype_code(gate)
    ld_in, ld_h = _matrix("gate", gate, rows, cols), _matrix("h", h, rows, cols, dt)
    _same("presence of up and of its checkpoint", up is None, kept_up is None)
    if up is not None:
        _same("leading dimensions of gate and up", ld_in, _matrix("up", up, rows, cols, dt))
        _same("checkpoints of gate and up", (rows, cols, kept_gate.ldc), (kept_up.rows, kept_up.cols, kept_up.ldc))
    _check(lib, None, lib.psgd_act_glu(
        _stream_for(stream, gate, up, h, *_kept_tensors(kept_gate, kept_up)), rows, cols, int(act), dt, gate.data_ptr(), up.data_ptr() if up is not None else None, ld_in,
        h.data_ptr(), ld_h, kept_gate.codes.data_ptr(), kept_gate.scales.data_ptr(),
        kept_up.codes.data_ptr() if up is not None else None, kept_up.scales.data_ptr() if up is not None else None, kept_gate.ldc))


def act_glu_backward(kept_gate: Act8, kept_up: Optional[Act8], dh, dgate, dup, act: int = PSGD_SILU, stream=None) -> None:
    """psgd_act_glu_backward: dgate <- dh * up * act'(gate), dup <- dh * act(gate) (kept_up, dup None: dgate <- dh * act'(gate))."""
    lib = load_library()
    rows, cols, dt = kept_gate.rows, kept_gate.cols, _dtype_code(dh)
    ld_h, ld_out = _matrix("dh", dh, rows, cols), _matrix("dgate", dgate, rows, cols, dt)
    _same("presence of the checkpoint of up and of dup", kept_up is None, dup is None)
    if dup is not None:
        _same("leading dimensions of dgate and dup", ld_out, _matrix("dup", dup, rows, cols, dt))
        _same("checkpoints of gate and up", (rows, cols, kept_gate.ldc), (kept_up.rows, kept_up.cols, kept_up.ldc))
    _check(lib, None, lib.psgd_act_glu_backward(
        _stream_for(stream, dh, dgate, dup, *_kept_tensors(kept_gate, kept_up)), rows, cols, int(act), dt, kept_gate.codes.data_ptr(), kept_gate.scales.data_ptr(),
        kept_up.codes.data_ptr() if dup is not None else None, kept_up.scales.data_ptr() if dup is not None else None,
        kept_gate.ldc, dh.data_ptr(), ld_h, dgate.data_ptr(), dup.data_ptr() if dup is not None else None, ld_out))


class WeightGrad:
    """psgd_act_wgrad with a torch-allocated workspace, for one set of sizes and types: G = dY^T X from dY and the 8-bit
    checkpoint of X.  Calls on streams that do not wait for each other need an object each: they would share the workspace."""

    def __init__(self, tokens: int, out_features: int, in_features: int, dtype: int = PSGD_BF16,
                 grad_dtype: Optional[int] = None, *, device: str = "cuda"):
        self.lib = load_library()
        self.shape = (int(tokens), int(out_features), int(in_features))
        self.dtype, self.grad_dtype = int(dtype), int(dtype if grad_dtype is None else grad_dtype)
        self.workspace_bytes = int(self.lib.psgd_act_wgrad_workspace_bytes(*self.shape, self.dtype))
        if self.workspace_bytes == 0 or self.grad_dtype not in (PSGD_F32, PSGD_BF16):
            raise PsgdError(PSGD_E_INVALID_ARG, "sizes or types of the weight gradient")
        self.workspace, self._ws_ptr = _work_area(self.workspace_bytes, device)

    def run(self, dY, kept: Act8, G, accumulate: bool = False, stream=None) -> None:
        tokens, out_features, in_features = self.shape
        ldy = _matrix("dY", dY, tokens, out_features, self.dtype)
        ldg = _matrix("G", G, out_features, in_features, self.grad_dtype)
        _same("sizes of the checkpoint", (kept.rows, kept.cols), (tokens, in_features))
        _check(self.lib, None, self.lib.psgd_act_wgrad(
            self._ws_ptr, _stream_for(stream, self.workspace, dY, G, kept.codes, kept.scales), tokens, out_features, in_features, dY.data_ptr(), self.dtype, ldy,
            kept.codes.data_ptr(), kept.ldc, kept.scales.data_ptr(), G.data_ptr(), self.grad_dtype, ldg, 1 if accumulate else 0))


def norm(X, weight, bias, Y, stats=None, eps: float = 1e-5, add=None, total=None, stream=None) -> None:
    """psgd_norm: Y <- layer norm of the rows of X, or with add of total <- X + add (rounded to the type), times weight plus bias
    (one type; None: 1 and 0).  stats (rows x 2, float32): what NormGrad needs.  total or Y may be X or add itself."""
    lib = load_library()
    _same("presence of add and of total", add is None, total is None)
    (rows, cols), dt = X.shape, _dtype_code(X)
    ld_x, ld_y, ld_add, ld_total = _matrix("X", X, rows, cols), _matrix("Y", Y, rows, cols, dt), 0, 0
    if add is not None:
        ld_add, ld_total = _matrix("add", add, rows, cols, dt), _matrix("total", total, rows, cols, dt)
    if stats is not None:
        _pairs(stats, rows)
    w_dt = _params(cols, weight, bias)
    _check(lib, None, lib.psgd_norm(_stream_for(stream, X, weight, bias, Y, stats, add, total), rows, cols, dt, X.data_ptr(), ld_x, _ptr(add), ld_add,
                                    _ptr(weight), _ptr(bias), w_dt, float(eps), _ptr(total), ld_total, Y.data_ptr(), ld_y, _ptr(stats)))


def _pairs(stats, rows: int) -> None:
    if _dtype_code(stats) != PSGD_F32 or stats.shape != (rows, 2) or not stats.is_contiguous() or not stats.is_cuda:
        raise ValueError("stats: a contiguous %d x 2 float32 matrix on the GPU expected" % rows)


def _params(cols: int, a, b) -> int:
    """Checks two vectors of one type, each of which may be None; their type."""
    code = None
    for t in (a, b):
        if t is not None:
            if t.shape != (cols,) or not t.is_cuda or not t.is_contiguous():
                raise ValueError("%d contiguous elements on the GPU expected, got %s on %s" % (cols, tuple(t.shape), t.device))
            if code is not None and _dtype_code(t) != code:
                raise ValueError("element types of a weight and a bias: one expected")
            code = _dtype_code(t)
    return PSGD_F32 if code is None else code


class NormGrad:
    """psgd_norm_backward with a torch-allocated workspace, for one set of sizes and types.  Calls on streams that do not wait for
    each other need an object each: they would share the workspace."""

    def __init__(self, rows: int, cols: int, dtype: int = PSGD_BF16, w_dtype: Optional[int] = None, grad_dtype: Optional[int] = None, *,
                 device: str = "cuda"):
        self.lib = load_library()
        self.shape, self.dtype = (int(rows), int(cols)), int(dtype)
        self.w_dtype = int(dtype if w_dtype is None else w_dtype)
        self.grad_dtype = int(self.w_dtype if grad_dtype is None else grad_dtype)
        self.workspace_bytes = int(self.lib.psgd_norm_backward_workspace_bytes(*self.shape, self.dtype))
        if self.workspace_bytes == 0 or self.w_dtype not in (PSGD_F32, PSGD_BF16) or self.grad_dtype not in (PSGD_F32, PSGD_BF16):
            raise PsgdError(PSGD_E_INVALID_ARG, "sizes or types of the norm")
        self.workspace, self._ws_ptr = _work_area(self.workspace_bytes, device)

    def run(self, dY, X, weight, stats, dX, dweight=None, dbias=None, dtotal=None, accumulate: bool = False, stream=None) -> None:
        """X: what was normalised (norm's total, where there was one); dtotal: the gradient that reaches it past the norm.
        dX <- its gradient; dweight, dbias <- (accumulate: +=) theirs, each of which may be None.  dX may be dY, X or dtotal itself."""
        rows, cols = self.shape
        ld_dy, ld_x, ld_dx = (_matrix("dY", dY, rows, cols, self.dtype), _matrix("X", X, rows, cols, self.dtype),
                              _matrix("dX", dX, rows, cols, self.dtype))
        ld_dtotal = _matrix("dtotal", dtotal, rows, cols, self.dtype) if dtotal is not None else 0
        _pairs(stats, rows)
        if weight is not None and _params(cols, weight, None) != self.w_dtype:
            raise ValueError("weight: wrong element type %s" % weight.dtype)
        if (dweight is not None or dbias is not None) and _params(cols, dweight, dbias) != self.grad_dtype:
            raise ValueError("dweight, dbias: wrong element type")
        _check(self.lib, None, self.lib.psgd_norm_backward(
            self._ws_ptr, _stream_for(stream, self.workspace, dY, X, weight, stats, dX, dweight, dbias, dtotal), rows, cols, self.dtype, dY.data_ptr(),
            ld_dy, X.data_ptr(), ld_x, _ptr(weight), self.w_dtype, stats.data_ptr(), _ptr(dtotal), ld_dtotal, dX.data_ptr(), ld_dx, _ptr(dweight), _ptr(dbias),
            self.grad_dtype, 1 if accumulate else 0))


class ExpertOrder:
    """Tokens sorted by expert: place (tokens x slots int32: the row of each choice, -1 where it does not count), order (tokens * slots
    int32: the choice of each row, -1 behind the last) and offsets (experts + 1 int32: each expert's first row, and their number)."""

    def __init__(self, place, order, offsets):
        import torch
        if place.dim() != 2 or offsets.dim() != 1 or offsets.shape[0] < 2:
            raise ValueError("place: tokens x slots, offsets: experts + 1 elements expected, got %s and %s" % (tuple(place.shape), tuple(offsets.shape)))
        self.tokens, self.slots, self.experts = int(place.shape[0]), int(place.shape[1]), int(offsets.shape[0]) - 1
        if place.dtype != torch.int32 or not place.is_contiguous() or not place.is_cuda:
            raise ValueError("place: a contiguous int32 matrix on the GPU expected")
        _vector("order", order, self.tokens * self.slots, torch.int32)
        _vector("offsets", offsets, self.experts + 1, torch.int32)
        self.place, self.order, self.offsets = place, order, offsets


def expert_order_empty(tokens: int, slots: int, experts: int, device: str = "cuda") -> ExpertOrder:
    """Buffers for the order of tokens that choose `slots` of `experts` each."""
    import torch
    return ExpertOrder(torch.empty((tokens, slots), dtype=torch.int32, device=device), torch.empty(tokens * slots, dtype=torch.int32, device=device),
                       torch.empty(experts + 1, dtype=torch.int32, device=device))


class ExpertSort:
    """psgd_expert_sort with a torch-allocated workspace, for one set of sizes.  Calls on streams that do not wait for each other need an
    object each: they would share the workspace."""

    def __init__(self, tokens: int, slots: int, experts: int, *, device: str = "cuda"):
        self.lib = load_library()
        self.shape = (int(tokens), int(slots), int(experts))
        self.workspace_bytes = int(self.lib.psgd_expert_sort_workspace_bytes(*self.shape))
        if self.workspace_bytes == 0:
            raise PsgdError(PSGD_E_INVALID_ARG, "sizes of the sort")
        self.workspace, self._ws_ptr = _work_area(self.workspace_bytes, device)

    def run(self, choice, order: ExpertOrder, stream=None) -> None:
        """order <- the tokens sorted by choice (tokens x slots int64; outside [0, experts): the choice does not count)."""
        import torch
        _same("sizes of the order", (order.tokens, order.slots, order.experts), self.shape)
        if choice.dtype != torch.int64 or choice.shape != self.shape[:2] or not choice.is_contiguous() or not choice.is_cuda:
            raise ValueError("choice: a contiguous %d x %d int64 matrix on the GPU expected" % self.shape[:2])
        _check(self.lib, None, self.lib.psgd_expert_sort(
            self._ws_ptr, _stream_for(stream, self.workspace, choice, order.place, order.order, order.offsets), *self.shape, choice.data_ptr(), order.place.data_ptr(),
            order.order.data_ptr(), order.offsets.data_ptr()))


def _choice_weights(name: str, t, order: ExpertOrder):
    if t is not None and (_dtype_code(t) != PSGD_F32 or t.shape != (order.tokens, order.slots) or not t.is_contiguous() or not t.is_cuda):
        raise ValueError("%s: a contiguous %d x %d float32 matrix on the GPU expected" % (name, order.tokens, order.slots))


def expert_rows(X, order: ExpertOrder, Xs, stream=None) -> None:
    """psgd_expert_rows: row place[t, s] of Xs (tokens * slots rows) <- row t of X; rows behind the last stay as they are.
    The gradient of X is expert_combine of the gradient of Xs."""
    lib = load_library()
    cols, dt = X.shape[1], _dtype_code(X)
    ld, ld_s = _matrix("X", X, order.tokens, cols), _matrix("Xs", Xs, order.tokens * order.slots, cols, dt)
    _check(lib, None, lib.psgd_expert_rows(_stream_for(stream, X, Xs, order.place), order.tokens, order.slots, cols, dt, X.data_ptr(), ld,
                                           order.place.data_ptr(), Xs.data_ptr(), ld_s))


def expert_combine(Ys, order: ExpertOrder, Y, weight=None, stream=None) -> None:
    """psgd_expert_combine: row t of Y <- the sum of its choices' rows of Ys times weight[t, s] (None: 1)."""
    lib = load_library()
    cols, dt = Y.shape[1], _dtype_code(Y)
    ld_s, ld = _matrix("Ys", Ys, order.tokens * order.slots, cols, dt), _matrix("Y", Y, order.tokens, cols)
    _choice_weights("weight", weight, order)
    _check(lib, None, lib.psgd_expert_combine(_stream_for(stream, Ys, Y, weight, order.place), order.tokens, order.slots, cols, dt, Ys.data_ptr(),
                                              ld_s, order.place.data_ptr(), _ptr(weight), Y.data_ptr(), ld))


def expert_combine_backward(dY, Ys, order: ExpertOrder, dYs, weight=None, dweight=None, stream=None) -> None:
    """psgd_expert_combine_backward: row place[t, s] of dYs <- weight[t, s] times row t of dY, rows behind the last stay as they are;
    dweight[t, s] <- dY[t] . Ys[place[t, s]], 0 where there is no row (dweight None: Ys may be None).  dYs may be Ys itself."""
    lib = load_library()
    cols, dt, rows = dY.shape[1], _dtype_code(dY), order.tokens * order.slots
    ld, ld_ds = _matrix("dY", dY, order.tokens, cols), _matrix("dYs", dYs, rows, cols, dt)
    ld_s = _matrix("Ys", Ys, rows, cols, dt) if Ys is not None else 0
    if dweight is not None and Ys is None:
        raise ValueError("dweight needs Ys")
    _choice_weights("weight", weight, order)
    _choice_weights("dweight", dweight, order)
    _check(lib, None, lib.psgd_expert_combine_backward(
        _stream_for(stream, dY, Ys, dYs, weight, dweight, order.place), order.tokens, order.slots, cols, dt, dY.data_ptr(), ld, _ptr(Ys), ld_s,
        order.place.data_ptr(), _ptr(weight), dYs.data_ptr(), ld_ds, _ptr(dweight)))
