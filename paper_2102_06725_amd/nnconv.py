"""ctypes binding of libnnconv (include/nnconv.h).

The functions below carry the C names and only marshal arguments: device
pointers are Python ints (``tensor.data_ptr()``), streams are ints
(``torch.cuda.current_stream().cuda_stream``).  Every computation runs in
the HIP library; if it is missing, loading fails loudly.

``Conv2d`` is a small convenience on top: it takes torch tensors, sizes and
allocates the caller-owned workspace with torch, and raises on a non-OK
status.
"""
from __future__ import annotations

import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libnnconv.so")

# enums (same values as nnconv.h)
NNCONV_OK = 0
NNCONV_ERR_INVALID_ARG = 1
NNCONV_ERR_UNSUPPORTED = 2
NNCONV_ERR_WORKSPACE = 3
NNCONV_ERR_MISALIGNED = 4
NNCONV_ERR_HIP = 5
NNCONV_NCHW = 0
NNCONV_NHWC = 1
NNCONV_F16 = 0
NNCONV_BF16 = 1
NNCONV_F32 = 2
NNCONV_F8 = 3
NNCONV_FWD = 0
NNCONV_DGRAD = 1
NNCONV_WGRAD = 2
NNCONV_NOALLOC_WS_BYTES = 64 * 1024 * 1024
NNCONV_RECURRENCE_SAVE = 64
NNCONV_ADAMW_BLOCK = 64
# nnconv_tile: tiles of the implicit-GEMM forward / backward-data kernel
NNCONV_TILE_256x256_8W = 0
NNCONV_TILE_128x128_2S = 1
NNCONV_TILE_128x128 = 2
NNCONV_TILE_128x64 = 3
NNCONV_TILE_256x256_16W = 4
NNCONV_TILE_256x256_RING = 6
NNCONV_TILE_256x128_RING = 7
NNCONV_TILE_256x64_RING = 8
NNCONV_TILE_HALO_256x64 = 9
NNCONV_TILE_HALO_256x128 = 10
NNCONV_TILE_HALO_256x64_2T = 11
NNCONV_TILE_HALO_R256x128 = 12
NNCONV_TILE_HALO_R128x256 = 13
NNCONV_TILE_HALO_R224x256 = 14
NNCONV_TILE_HALO_R256x64S = 15
HALO_TILES = (NNCONV_TILE_HALO_256x64, NNCONV_TILE_HALO_256x128, NNCONV_TILE_HALO_256x64_2T,
              NNCONV_TILE_HALO_R256x128, NNCONV_TILE_HALO_R128x256, NNCONV_TILE_HALO_R224x256,
              NNCONV_TILE_HALO_R256x64S)
# largest raster span of the filter taps each halo tile's buffer holds
HALO_TILE_SPAN = {NNCONV_TILE_HALO_256x64: 128, NNCONV_TILE_HALO_256x128: 128,
                  NNCONV_TILE_HALO_256x64_2T: 128, NNCONV_TILE_HALO_R256x128: 64,
                  NNCONV_TILE_HALO_R128x256: 128, NNCONV_TILE_HALO_R224x256: 32,
                  NNCONV_TILE_HALO_R256x64S: 128}
# filter taps the halo tiles with register-held weights take (3x3 only)
HALO_TILE_TAPS = {NNCONV_TILE_HALO_R256x128: 9, NNCONV_TILE_HALO_R128x256: 9,
                  NNCONV_TILE_HALO_R224x256: 9, NNCONV_TILE_HALO_R256x64S: 9}
# the pass's reduction channel count the single-slice halo tile requires
HALO_TILE_RED = {NNCONV_TILE_HALO_R256x64S: 64}
TILES = (NNCONV_TILE_256x256_8W, NNCONV_TILE_128x128_2S, NNCONV_TILE_128x128, NNCONV_TILE_128x64,
         NNCONV_TILE_256x256_16W, NNCONV_TILE_256x256_RING, NNCONV_TILE_256x128_RING,
         NNCONV_TILE_256x64_RING)

EXPORTS = ("nnconv_version", "nnconv_last_hip_error", "nnconv_status_string", "nnconv_output_dims",
           "nnconv_workspace_size", "nnconv_fwd", "nnconv_dgrad", "nnconv_fwd_tile",
           "nnconv_dgrad_tile", "nnconv_wgrad", "nnconv_wgrad_noalloc",
           "nnconv_nchw_to_nhwc", "nnconv_nhwc_to_nchw", "nnconv_pad_channels",
           "nnconv_weight_kcrs_to_krsc", "nnconv_weight_krsc_to_kcrs",
           "nnconv_loss_scaler_init", "nnconv_loss_scaler_update", "nnconv_sgd_update",
           "nnconv_rmsnorm_fwd", "nnconv_rmsnorm_fwd_q8", "nnconv_rmsnorm_workspace_size",
           "nnconv_rmsnorm_bwd", "nnconv_recurrence_saved_size",
           "nnconv_recurrence_workspace_size", "nnconv_recurrence_fwd", "nnconv_recurrence_bwd",
           "nnconv_adamw_plan_size", "nnconv_adamw_plan_init", "nnconv_adamw_update")


class nnconv_desc(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in
                ("n", "c", "h", "w", "k", "r", "s", "stride_h", "stride_w", "pad_h", "pad_w",
                 "dil_h", "dil_w", "groups", "layout", "dtype")]


class nnconv_loss_scaler(ctypes.Structure):
    """Layout of the device-resident scaler state (24 bytes)."""
    _fields_ = [("scale", ctypes.c_float), ("factor", ctypes.c_float),
                ("interval", ctypes.c_int32), ("counter", ctypes.c_int32),
                ("skipped", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class nnconv_rmsnorm_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("c", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("group", ctypes.c_int32), ("eps", ctypes.c_float)]


class nnconv_recurrence_desc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("t", ctypes.c_int32), ("c", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("ld", ctypes.c_int64), ("ldy", ctypes.c_int64)]


class nnconv_adamw_tensor(ctypes.Structure):
    _fields_ = [("master", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("w16", ctypes.c_void_p),
                ("m", ctypes.c_void_p), ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("count", ctypes.c_int64),
                ("weight_decay", ctypes.c_float), ("grad_dtype", ctypes.c_int32),
                ("w16_dtype", ctypes.c_int32), ("state_dtype", ctypes.c_int32)]


class nnconv_adamw_plan(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("chunks", ctypes.c_int64),
                ("tensors", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class NNConvError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        extra = ""
        if status == NNCONV_ERR_HIP:
            extra = ", hipError %d" % nnconv_last_hip_error()
        super().__init__("%s: %s (status %d%s)" % (what or "libnnconv", status_string(status),
                                                   status, extra))


_lib = None

_VP = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_DESCP = ctypes.POINTER(nnconv_desc)


def load(path: str | None = None):
    """Load libnnconv.so (built in-tree by paper_2102_06725_amd.build)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise ImportError("libnnconv.so not found at %s; build it with "
                          "`python -m paper_2102_06725_amd.build`" % p)
    # torch ships its own HIP runtime whose SONAME matches the one libnnconv
    # links against.  Loading torch first makes the library bind to that same
    # runtime instance, so torch's device pointers and streams are valid in
    # it; loading libnnconv first would put a second runtime in the process.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = ctypes.CDLL(p)
    lib.nnconv_version.restype = _I32
    lib.nnconv_last_hip_error.restype = _I32
    lib.nnconv_status_string.argtypes = [ctypes.c_int]
    lib.nnconv_status_string.restype = ctypes.c_char_p
    lib.nnconv_output_dims.argtypes = [_DESCP, ctypes.POINTER(_I32), ctypes.POINTER(_I32)]
    lib.nnconv_workspace_size.argtypes = [_DESCP, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
    lib.nnconv_fwd.argtypes = [_DESCP, _VP, _VP, _VP, ctypes.c_float, _VP, ctypes.c_size_t, _VP]
    lib.nnconv_dgrad.argtypes = [_DESCP, _VP, _VP, _VP, ctypes.c_float, _VP, ctypes.c_size_t, _VP]
    lib.nnconv_wgrad_noalloc.argtypes = [_DESCP, _VP, _VP, _VP, _I32, ctypes.c_float, _I32,
                                         _VP, _VP]
    lib.nnconv_fwd_tile.argtypes = [_DESCP, _VP, _VP, _VP, ctypes.c_float, _VP, ctypes.c_size_t,
                                    _VP, _I32]
    lib.nnconv_dgrad_tile.argtypes = [_DESCP, _VP, _VP, _VP, ctypes.c_float, _VP,
                                      ctypes.c_size_t, _VP, _I32]
    lib.nnconv_wgrad.argtypes = [_DESCP, _VP, _VP, _VP, _I32, ctypes.c_float, _I32, _VP, _VP,
                                 ctypes.c_size_t, _VP]
    lib.nnconv_nchw_to_nhwc.argtypes = [_VP, _VP, _I32, _I32, _I32, _I32, _I32, _VP]
    lib.nnconv_nhwc_to_nchw.argtypes = [_VP, _VP, _I32, _I32, _I32, _I32, _VP]
    lib.nnconv_pad_channels.argtypes = [_VP, _VP, _I64, _I32, _I32, _VP]
    lib.nnconv_weight_kcrs_to_krsc.argtypes = [_VP, _VP, _I32, _I32, _I32, _I32, _I32, _VP]
    lib.nnconv_weight_krsc_to_kcrs.argtypes = [_VP, _VP, _I32, _I32, _I32, _I32, _VP]
    lib.nnconv_loss_scaler_init.argtypes = [_VP, ctypes.c_float, ctypes.c_float, _I32, _VP]
    lib.nnconv_loss_scaler_update.argtypes = [_VP, _VP, _VP]
    lib.nnconv_sgd_update.argtypes = [_I64, _VP, _VP, _VP, _I32, _VP, _VP, _VP, ctypes.c_float,
                                      ctypes.c_float, ctypes.c_float, _VP]
    _F32, _SZ, _SZP = ctypes.c_float, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)
    norm, rec = ctypes.POINTER(nnconv_rmsnorm_desc), ctypes.POINTER(nnconv_recurrence_desc)
    tens, plan = ctypes.POINTER(nnconv_adamw_tensor), ctypes.POINTER(nnconv_adamw_plan)
    lib.nnconv_rmsnorm_fwd.argtypes = [norm] + [_VP] * 7
    lib.nnconv_rmsnorm_fwd_q8.argtypes = [norm] + [_VP] * 8
    lib.nnconv_rmsnorm_workspace_size.argtypes = [norm, _SZP]
    lib.nnconv_rmsnorm_bwd.argtypes = [norm] + [_VP] * 7 + [_F32, _I32, _VP, _VP, _SZ, _VP]
    lib.nnconv_recurrence_saved_size.argtypes = [rec, _SZP]
    lib.nnconv_recurrence_workspace_size.argtypes = [rec, ctypes.c_int, _SZP]
    lib.nnconv_recurrence_fwd.argtypes = [rec] + [_VP] * 10 + [_SZ, _VP]
    lib.nnconv_recurrence_bwd.argtypes = [rec] + [_VP] * 13 + [_F32, _I32, _VP, _VP, _SZ, _VP]
    lib.nnconv_adamw_plan_size.argtypes = [tens, _I32, _SZP]
    lib.nnconv_adamw_plan_init.argtypes = [tens, _I32, _VP, _SZ, plan, _VP]
    lib.nnconv_adamw_update.argtypes = [plan, _VP, _F32, _F32, _F32, _F32, ctypes.c_uint32, _VP,
                                        _VP, _VP]
    for f in EXPORTS[3:]:
        getattr(lib, f).restype = ctypes.c_int
    if path is None:
        _lib = lib
    return lib


def make_desc(n, c, h, w, k, r, s, stride=(1, 1), pad=(0, 0), dil=(1, 1), groups=1,
              layout=NNCONV_NHWC, dtype=NNCONV_F16) -> nnconv_desc:
    def pair(v):
        return (v, v) if isinstance(v, int) else tuple(v)
    st, pd, dl = pair(stride), pair(pad), pair(dil)
    return nnconv_desc(n, c, h, w, k, r, s, st[0], st[1], pd[0], pd[1], dl[0], dl[1], groups,
                       layout, dtype)


# --- C entry points, same names -------------------------------------------

def nnconv_version() -> int:
    return load().nnconv_version()


def nnconv_last_hip_error() -> int:
    return load().nnconv_last_hip_error()


def status_string(status: int) -> str:
    return load().nnconv_status_string(int(status)).decode()


nnconv_status_string = status_string


def nnconv_output_dims(desc: nnconv_desc):
    p, q = _I32(), _I32()
    st = load().nnconv_output_dims(ctypes.byref(desc), ctypes.byref(p), ctypes.byref(q))
    return st, p.value, q.value


def nnconv_workspace_size(desc: nnconv_desc, pass_: int):
    b = ctypes.c_size_t()
    st = load().nnconv_workspace_size(ctypes.byref(desc), int(pass_), ctypes.byref(b))
    return st, b.value


def nnconv_fwd(desc, x, w, y, alpha, ws, ws_bytes, stream) -> int:
    return load().nnconv_fwd(ctypes.byref(desc), x, w, y, float(alpha), ws, ws_bytes, stream)


def nnconv_dgrad(desc, dy, w, dx, alpha, ws, ws_bytes, stream) -> int:
    return load().nnconv_dgrad(ctypes.byref(desc), dy, w, dx, float(alpha), ws, ws_bytes, stream)


def nnconv_fwd_tile(desc, x, w, y, alpha, ws, ws_bytes, stream, tile) -> int:
    return load().nnconv_fwd_tile(ctypes.byref(desc), x, w, y, float(alpha), ws, ws_bytes, stream,
                                  int(tile))


def nnconv_dgrad_tile(desc, dy, w, dx, alpha, ws, ws_bytes, stream, tile) -> int:
    return load().nnconv_dgrad_tile(ctypes.byref(desc), dy, w, dx, float(alpha), ws, ws_bytes,
                                    stream, int(tile))


def nnconv_wgrad(desc, x, dy, dw, dw_dtype, inv_loss_scale, accumulate, overflow_flag, ws,
                 ws_bytes, stream) -> int:
    return load().nnconv_wgrad(ctypes.byref(desc), x, dy, dw, int(dw_dtype),
                               float(inv_loss_scale), int(accumulate), overflow_flag, ws,
                               ws_bytes, stream)


def nnconv_wgrad_noalloc(desc, x, dy, dw, dw_dtype, inv_loss_scale, accumulate, overflow_flag,
                         stream) -> int:
    return load().nnconv_wgrad_noalloc(ctypes.byref(desc), x, dy, dw, int(dw_dtype),
                                       float(inv_loss_scale), int(accumulate), overflow_flag,
                                       stream)


def nnconv_nchw_to_nhwc(src, dst, n, c, h, w, c_pad, stream) -> int:
    return load().nnconv_nchw_to_nhwc(src, dst, n, c, h, w, c_pad, stream)


def nnconv_nhwc_to_nchw(src, dst, n, c, h, w, stream) -> int:
    return load().nnconv_nhwc_to_nchw(src, dst, n, c, h, w, stream)


def nnconv_pad_channels(src, dst, rows, c, c_pad, stream) -> int:
    return load().nnconv_pad_channels(src, dst, rows, c, c_pad, stream)


def nnconv_weight_kcrs_to_krsc(src, dst, k, cg, r, s, cg_pad, stream) -> int:
    return load().nnconv_weight_kcrs_to_krsc(src, dst, k, cg, r, s, cg_pad, stream)


def nnconv_weight_krsc_to_kcrs(src, dst, k, cg, r, s, stream) -> int:
    return load().nnconv_weight_krsc_to_kcrs(src, dst, k, cg, r, s, stream)


def nnconv_loss_scaler_init(state, initial_scale, factor, interval, stream) -> int:
    return load().nnconv_loss_scaler_init(state, float(initial_scale), float(factor),
                                          int(interval), stream)


def nnconv_loss_scaler_update(state, overflow_flag, stream) -> int:
    return load().nnconv_loss_scaler_update(state, overflow_flag, stream)


def nnconv_sgd_update(count, master, momentum, w16, w16_dtype, grad, state, overflow_flag, lr,
                      momentum_coef, weight_decay, stream) -> int:
    return load().nnconv_sgd_update(int(count), master, momentum, w16, int(w16_dtype), grad,
                                    state, overflow_flag, float(lr), float(momentum_coef),
                                    float(weight_decay), stream)


def nnconv_rmsnorm_fwd(desc, x, residual, gain, sum, y, rstd, stream) -> int:
    return load().nnconv_rmsnorm_fwd(ctypes.byref(desc), x, residual, gain, sum, y, rstd, stream)


def nnconv_rmsnorm_fwd_q8(desc, x, residual, gain, sum, q, scales, rstd, stream) -> int:
    return load().nnconv_rmsnorm_fwd_q8(ctypes.byref(desc), x, residual, gain, sum, q, scales,
                                        rstd, stream)


def nnconv_rmsnorm_workspace_size(desc):
    b = ctypes.c_size_t()
    st = load().nnconv_rmsnorm_workspace_size(ctypes.byref(desc), ctypes.byref(b))
    return st, b.value


def nnconv_rmsnorm_bwd(desc, sum, dy, dsum, gain, rstd, dx, dgain, inv_loss_scale, accumulate,
                       overflow_flag, ws, ws_bytes, stream) -> int:
    return load().nnconv_rmsnorm_bwd(ctypes.byref(desc), sum, dy, dsum, gain, rstd, dx, dgain,
                                     float(inv_loss_scale), int(accumulate), overflow_flag, ws,
                                     ws_bytes, stream)


def nnconv_recurrence_saved_size(desc):
    b = ctypes.c_size_t()
    st = load().nnconv_recurrence_saved_size(ctypes.byref(desc), ctypes.byref(b))
    return st, b.value


def nnconv_recurrence_workspace_size(desc, pass_: int):
    b = ctypes.c_size_t()
    st = load().nnconv_recurrence_workspace_size(ctypes.byref(desc), int(pass_), ctypes.byref(b))
    return st, b.value


def nnconv_recurrence_fwd(desc, x, f, bias, g, lengths, h0, y, ht, saved, ws, ws_bytes,
                          stream) -> int:
    return load().nnconv_recurrence_fwd(ctypes.byref(desc), x, f, bias, g, lengths, h0, y, ht,
                                        saved, ws, ws_bytes, stream)


def nnconv_recurrence_bwd(desc, x, f, bias, g, lengths, saved, dy, dht, dx, df, dg, dh0, dbias,
                          inv_loss_scale, accumulate, overflow_flag, ws, ws_bytes, stream) -> int:
    return load().nnconv_recurrence_bwd(ctypes.byref(desc), x, f, bias, g, lengths, saved, dy, dht,
                                        dx, df, dg, dh0, dbias, float(inv_loss_scale),
                                        int(accumulate), overflow_flag, ws, ws_bytes, stream)


def nnconv_adamw_plan_size(tensors, n):
    """tensors: a ctypes array of nnconv_adamw_tensor (None for n = 0)."""
    b = ctypes.c_size_t()
    st = load().nnconv_adamw_plan_size(tensors, int(n), ctypes.byref(b))
    return st, b.value


def nnconv_adamw_plan_init(tensors, n, table, table_bytes, plan, stream) -> int:
    return load().nnconv_adamw_plan_init(tensors, int(n), table, table_bytes, ctypes.byref(plan),
                                         stream)


def nnconv_adamw_update(plan, step, lr, beta1, beta2, eps, seed, state, overflow_flag,
                        stream) -> int:
    return load().nnconv_adamw_update(ctypes.byref(plan), step, float(lr), float(beta1),
                                      float(beta2), float(eps), int(seed), state, overflow_flag,
                                      stream)


def check(status: int, what: str = "") -> None:
    if status != NNCONV_OK:
        raise NNConvError(status, what)


# --- torch-tensor convenience ------------------------------------------------

def current_stream() -> int:
    """The current device's current stream as an int, without the Stream
    object that torch.cuda.current_stream() builds on each call (2.7 us of the
    9.1 us that a small Conv2d call took; 5.9 us now, 3.4 of them one launch)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


class Conv2d:
    """One convolution geometry bound to torch tensors on the current device.

    The workspace for each pass is a torch uint8 tensor owned by this object
    (allocated once, on first use)."""

    def __init__(self, n, c, h, w, k, r, s, stride=(1, 1), pad=(0, 0), dil=(1, 1), groups=1,
                 layout=NNCONV_NHWC, dtype=NNCONV_F16):
        self.desc = make_desc(n, c, h, w, k, r, s, stride, pad, dil, groups, layout, dtype)
        st, self.p, self.q = nnconv_output_dims(self.desc)
        check(st, "nnconv_output_dims")
        self._ws = {}
        self._sizes = {}  # pass -> (descriptor bytes, workspace bytes)

    def workspace(self, pass_: int, device=None):
        key = bytes(self.desc)
        size = self._sizes.get(pass_)
        if size is None or size[0] != key:
            st, nbytes = nnconv_workspace_size(self.desc, pass_)
            check(st, "nnconv_workspace_size")
            self._sizes[pass_] = size = (key, nbytes)
        nbytes = size[1]
        t = self._ws.get(pass_)
        if t is None or t.numel() < nbytes:
            import torch
            t = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device or "cuda")
            self._ws[pass_] = t
        return t, nbytes

    @staticmethod
    def _stream(stream):
        return stream if stream is not None else current_stream()

    def fwd(self, x, w, y, alpha=1.0, stream=None):
        ws, nb = self.workspace(NNCONV_FWD, x.device)
        check(nnconv_fwd(self.desc, x.data_ptr(), w.data_ptr(), y.data_ptr(), alpha,
                         ws.data_ptr(), nb, self._stream(stream)), "nnconv_fwd")

    def dgrad(self, dy, w, dx, alpha=1.0, stream=None):
        ws, nb = self.workspace(NNCONV_DGRAD, dy.device)
        check(nnconv_dgrad(self.desc, dy.data_ptr(), w.data_ptr(), dx.data_ptr(), alpha,
                           ws.data_ptr(), nb, self._stream(stream)), "nnconv_dgrad")

    def wgrad(self, x, dy, dw, dw_dtype=NNCONV_F32, inv_loss_scale=1.0, accumulate=0,
              overflow_flag=None, stream=None):
        ws, nb = self.workspace(NNCONV_WGRAD, x.device)
        flag = overflow_flag.data_ptr() if overflow_flag is not None else None
        check(nnconv_wgrad(self.desc, x.data_ptr(), dy.data_ptr(), dw.data_ptr(), dw_dtype,
                           inv_loss_scale, accumulate, flag, ws.data_ptr(), nb,
                           self._stream(stream)), "nnconv_wgrad")


def _ptr(t):
    return None if t is None else t.data_ptr()


class _Workspaces:
    """Workspaces of a handle, torch tensors that are allocated on first use.

    Each device, stream and kind has its own, so that calls on several streams do not share one,
    and each call that torch captures into a graph has one of the graph's memory, so that graphs
    of a handle may be replayed beside each other and beside its calls.  A workspace that became
    too small is kept until the handle goes: a graph that the caller captured by other means may
    hold its address."""

    def __init__(self):
        import torch
        self._held = {}
        self._kept = []
        self._capturing = torch.cuda.is_current_stream_capturing

    def get(self, kind, stream, nbytes, device):
        if device.type == "cuda" and self._capturing():
            return self._new(nbytes, stream, device)
        t = self._held.get((kind, stream, device))
        if t is None or t.numel() < nbytes:
            if t is not None:  # doubled, so that all that is kept is no more than what is in use
                self._kept.append(t)
                nbytes = max(nbytes, 2 * t.numel())
            t = self._held[kind, stream, device] = self._new(nbytes, stream, device)
        return t

    @staticmethod
    def _new(nbytes, stream, device):
        """Memory that is free on `stream`: another stream's may still be in use there, and
        torch hands it on in the order of the stream that it was allocated on."""
        import torch
        nbytes = max(nbytes, 1)
        if device.type != "cuda" or stream == current_stream():
            return torch.empty(nbytes, dtype=torch.uint8, device=device)
        s = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
        with torch.cuda.stream(s):
            return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _all_dense(tensors, dtype, count, gpu):
    """Whether the tensors, Nones aside, are dense ones of `count` elements on the device."""
    for t in tensors:
        if t is not None and not (t.dtype is dtype and t.numel() == count and t.is_contiguous() and t.get_device() == gpu):
            return False
    return True


class _Handle:
    """The checks that the handles below share: torch tensors of another type, size, layout or
    device than the call's are refused, since it would read or write past their end.  Other
    objects with data_ptr() are taken as they are.

    A call looks its tensors over in one go (a quarter of a microsecond each); only where
    that fails are they looked at one by one, for the name of the one to refuse."""

    def __init__(self, desc, dtype=None):
        import torch
        self.desc, self._lib, self._ref = desc, load(), ctypes.byref(desc)
        self._tensor, self._f32, self._i32 = torch.Tensor, torch.float32, torch.int32
        self._dtype = {NNCONV_F16: torch.float16, NNCONV_BF16: torch.bfloat16, NNCONV_F32: torch.float32}.get(dtype)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)

    def _gpu(self, name, t):
        """The device that a call's tensors have to be on."""
        if isinstance(t, self._tensor):
            return t.get_device()
        if t is None:
            raise ValueError("%s: %s is needed" % (type(self).__name__, name))
        return self._get_device()

    def _stream(self, stream, gpu):
        if gpu < 0 or gpu != self._get_device():
            raise ValueError("%s: the tensors are not on the current device" % type(self).__name__)
        if stream is not None:
            return stream
        return current_stream() if self._raw_stream is None else self._raw_stream(gpu)

    def _refuse(self, name, t, want):
        raise ValueError("%s: %s: %s with strides %s of %s on %s, where %s are expected" % (
            type(self).__name__, name, tuple(t.shape), t.stride(), t.dtype, t.device, want))

    def _dense(self, dtype, count, gpu, more=False, **tensors):
        """One by one: dense, of `count` elements (or more)."""
        for name, t in tensors.items():
            if isinstance(t, self._tensor) and not (
                    t.dtype is dtype and t.is_contiguous() and t.get_device() == gpu
                    and (t.numel() == count or more and t.numel() > count)):
                self._refuse(name, t, "%d%s dense elements of %s on device %d" % (count, " or more" if more else "", dtype, gpu))


class RMSNorm(_Handle):
    """Root-mean-square norm of [rows][c] torch tensors (dense, on the current device), with
    the residual's addition: nnconv_rmsnorm_*.  `rows` may be changed between calls (a serving
    program's batch).  Tensors that do not fit are refused with a ValueError."""

    def __init__(self, rows, c, dtype=NNCONV_F16, eps=1e-6, group=0):
        super().__init__(nnconv_rmsnorm_desc(rows, c, dtype, group, eps), dtype)
        self._ws = _Workspaces()
        self._nbytes = None

    @property
    def rows(self):
        return self.desc.rows

    @rows.setter
    def rows(self, rows):
        self.desc.rows = rows
        self._nbytes = None

    def _fits(self, rows, c, gpu, wide, channels, each):
        """Whether tensors of [rows][c], of c and of rows elements are these."""
        try:
            return (_all_dense(wide, self._dtype, rows * c, gpu) and _all_dense(channels, self._f32, c, gpu)
                    and _all_dense(each, self._f32, rows, gpu))
        except AttributeError:  # an object that is no tensor
            return False

    def fwd(self, x, gain, y, residual=None, sum=None, rstd=None, stream=None):
        rows, c, gpu = self.desc.rows, self.desc.c, self._gpu("x", x)
        if not self._fits(rows, c, gpu, (x, residual, sum, y), (gain,), (rstd,)):
            self._dense(self._dtype, rows * c, gpu, x=x, residual=residual, sum=sum, y=y)
            self._dense(self._f32, c, gpu, gain=gain)
            self._dense(self._f32, rows, gpu, rstd=rstd)
        check(self._lib.nnconv_rmsnorm_fwd(
            self._ref, x.data_ptr(), None if residual is None else residual.data_ptr(), _ptr(gain),
            None if sum is None else sum.data_ptr(), _ptr(y), None if rstd is None else rstd.data_ptr(),
            self._stream(stream, gpu)), "nnconv_rmsnorm_fwd")

    def fwd_q8(self, x, gain, q, scales, residual=None, sum=None, rstd=None, stream=None):
        """q: torch.float8_e4m3fn or uint8."""
        import torch
        rows, c, gpu = self.desc.rows, self.desc.c, self._gpu("x", x)
        if not self._fits(rows, c, gpu, (x, residual, sum), (gain,), (rstd,)):
            self._dense(self._dtype, rows * c, gpu, x=x, residual=residual, sum=sum)
            self._dense(self._f32, c, gpu, gain=gain)
            self._dense(self._f32, rows, gpu, rstd=rstd)
        q8 = torch.uint8 if getattr(q, "dtype", None) is torch.uint8 else torch.float8_e4m3fn
        self._dense(q8, rows * c, gpu, q=q)
        groups = -(-c // self.desc.group) if self.desc.group > 0 else 1
        self._dense(self._f32, rows * groups, gpu, scales=scales)
        check(self._lib.nnconv_rmsnorm_fwd_q8(
            self._ref, x.data_ptr(), _ptr(residual), _ptr(gain), _ptr(sum), _ptr(q), _ptr(scales), _ptr(rstd),
            self._stream(stream, gpu)), "nnconv_rmsnorm_fwd_q8")

    def bwd(self, sum, dy, gain, rstd, dx, dgain=None, dsum=None, inv_loss_scale=1.0,
            accumulate=0, overflow_flag=None, stream=None):
        rows, c, gpu = self.desc.rows, self.desc.c, self._gpu("sum", sum)
        if not self._fits(rows, c, gpu, (sum, dy, dsum, dx), (gain, dgain), (rstd,)):
            self._dense(self._dtype, rows * c, gpu, sum=sum, dy=dy, dsum=dsum, dx=dx)
            self._dense(self._f32, c, gpu, gain=gain, dgain=dgain)
            self._dense(self._f32, rows, gpu, rstd=rstd)
        if overflow_flag is not None:
            self._dense(self._i32, 1, gpu, more=True, overflow_flag=overflow_flag)
        stream = self._stream(stream, gpu)
        ws, nb = None, 0
        if dgain is not None:
            if self._nbytes is None:
                st, self._nbytes = nnconv_rmsnorm_workspace_size(self.desc)
                check(st, "nnconv_rmsnorm_workspace_size")
            nb = self._nbytes
            ws = self._ws.get("bwd", stream, nb, sum.device)
        check(self._lib.nnconv_rmsnorm_bwd(
            self._ref, sum.data_ptr(), _ptr(dy), _ptr(dsum), _ptr(gain), _ptr(rstd), _ptr(dx), _ptr(dgain),
            inv_loss_scale, accumulate, _ptr(overflow_flag), _ptr(ws), nb, stream), "nnconv_rmsnorm_bwd")


class GatedRecurrence(_Handle):
    """Gated linear recurrence over n sequences of t tokens with c channels:
    nnconv_recurrence_*.  ld and ldy: elements between the tokens of x, f, g (3 * c for the
    thirds of one projection's output, passed as views) and of y.  `n` and `t` may be changed
    between calls.  Tensors that do not fit are refused with a ValueError: x, f, g, y and their
    gradients may have any shape that ends in c and whose strides are those of n * t tokens."""

    def __init__(self, n, t, c, ld=None, ldy=None, dtype=NNCONV_F16):
        super().__init__(nnconv_recurrence_desc(n, t, c, dtype, c if ld is None else ld,
                                                c if ldy is None else ldy), dtype)
        self._ws = _Workspaces()
        self._sizes = {}  # pass -> workspace bytes of the present n and t

    @property
    def n(self):
        return self.desc.n

    @n.setter
    def n(self, n):
        self.desc.n = n
        self._sizes.clear()

    @property
    def t(self):
        return self.desc.t

    @t.setter
    def t(self, t):
        self.desc.t = t
        self._sizes.clear()

    def saved(self, device="cuda"):
        """A tensor for the states that fwd saves for bwd."""
        import torch
        st, nb = nnconv_recurrence_saved_size(self.desc)
        check(st, "nnconv_recurrence_saved_size")
        return torch.empty(max(nb // 4, 1), dtype=torch.float32, device=device)

    def _workspace(self, pass_, stream, x):
        nb = self._sizes.get(pass_)
        if nb is None:
            st, nb = nnconv_recurrence_workspace_size(self.desc, pass_)
            check(st, "nnconv_recurrence_workspace_size")
            self._sizes[pass_] = nb
        return (None if nb == 0 else self._ws.get(pass_, stream, nb, x.device)), nb

    def _fits(self, gpu, inputs, outputs, dense, saved):
        """Whether tensors of tokens ld and ldy elements apart, dense ones of (type, elements), and saved states are these."""
        d, dtype = self.desc, self._dtype
        n, t, c = d.n, d.t, d.c
        try:
            for tensors, ld in ((inputs, d.ld), (outputs, d.ldy)):
                # as most calls have them: [n][t][c] and [n * t][c]
                shape, strides = ((n, t, c), (t * ld, ld, 1)) if tensors[0].dim() == 3 else ((n * t, c), (ld, 1))
                for v in tensors:
                    if v is not None and not (v.dtype is dtype and v.shape == shape and v.stride() == strides
                                              and v.get_device() == gpu):
                        return False
            for kind, count, tensors in dense:
                if not _all_dense(tensors, kind, count, gpu):
                    return False
            return saved is None or (saved.dtype is self._f32 and saved.numel() >= self._saved_count()
                                     and saved.is_contiguous() and saved.get_device() == gpu)
        except AttributeError:  # an object that is no tensor
            return False

    def _tokens(self, ld, gpu, **tensors):
        """One by one: any shape that ends in c, with the strides of tokens ld elements apart."""
        d = self.desc
        for name, t in tensors.items():
            if isinstance(t, self._tensor) and not (
                    t.dtype is self._dtype and t.get_device() == gpu and self._laid_out(t, ld)):
                self._refuse(name, t, "%d * %d tokens of %d channels, %d elements apart, of %s on device %d" % (
                    d.n, d.t, d.c, ld, self._dtype, gpu))

    def _laid_out(self, t, ld):
        d, shape, strides = self.desc, t.shape, t.stride()
        if len(shape) == 0 or shape[-1] != d.c or t.numel() != d.n * d.t * d.c:
            return False
        if t.numel() == 0:
            return True
        if d.c > 1 and strides[-1] != 1:
            return False
        for size, stride in zip(shape[-2::-1], strides[-2::-1]):
            if size > 1 and stride != ld:
                return False
            ld *= size
        return True

    def _saved_count(self):
        d = self.desc
        return d.n * -(-d.t // NNCONV_RECURRENCE_SAVE) * d.c

    def fwd(self, x, f, bias, y, g=None, lengths=None, h0=None, ht=None, saved=None, stream=None):
        d, f32, gpu = self.desc, self._f32, self._gpu("x", x)
        n, c = d.n, d.c
        if not self._fits(gpu, (x, f, g), (y,), ((f32, c, (bias,)), (f32, n * c, (h0, ht)), (self._i32, n, (lengths,))), saved):
            self._tokens(d.ld, gpu, x=x, f=f, g=g)
            self._tokens(d.ldy, gpu, y=y)
            self._dense(f32, c, gpu, bias=bias)
            self._dense(f32, n * c, gpu, h0=h0, ht=ht)
            self._dense(self._i32, n, gpu, lengths=lengths)
            self._dense(f32, self._saved_count(), gpu, more=True, saved=saved)
        stream = self._stream(stream, gpu)
        ws, nb = self._workspace(NNCONV_FWD, stream, x)
        check(self._lib.nnconv_recurrence_fwd(
            self._ref, x.data_ptr(), _ptr(f), None if bias is None else bias.data_ptr(),
            None if g is None else g.data_ptr(), None if lengths is None else lengths.data_ptr(),
            None if h0 is None else h0.data_ptr(), _ptr(y), None if ht is None else ht.data_ptr(),
            None if saved is None else saved.data_ptr(), None if ws is None else ws.data_ptr(), nb, stream),
            "nnconv_recurrence_fwd")

    def bwd(self, x, f, bias, saved, dy, dx, df, g=None, dg=None, lengths=None, dht=None, dh0=None,
            dbias=None, inv_loss_scale=1.0, accumulate=0, overflow_flag=None, stream=None):
        d, f32, gpu = self.desc, self._f32, self._gpu("x", x)
        n, c = d.n, d.c
        if not self._fits(gpu, (x, f, g, dx, df, dg), (dy,),
                          ((f32, c, (bias, dbias)), (f32, n * c, (dht, dh0)), (self._i32, n, (lengths,))), saved):
            self._tokens(d.ld, gpu, x=x, f=f, g=g, dx=dx, df=df, dg=dg)
            self._tokens(d.ldy, gpu, dy=dy)
            self._dense(f32, c, gpu, bias=bias, dbias=dbias)
            self._dense(f32, n * c, gpu, dht=dht, dh0=dh0)
            self._dense(self._i32, n, gpu, lengths=lengths)
            self._dense(f32, self._saved_count(), gpu, more=True, saved=saved)
        if overflow_flag is not None:
            self._dense(self._i32, 1, gpu, more=True, overflow_flag=overflow_flag)
        stream = self._stream(stream, gpu)
        ws, nb = self._workspace(NNCONV_DGRAD, stream, x)
        check(self._lib.nnconv_recurrence_bwd(
            self._ref, x.data_ptr(), _ptr(f), _ptr(bias), _ptr(g), _ptr(lengths), _ptr(saved), _ptr(dy),
            _ptr(dht), _ptr(dx), _ptr(df), _ptr(dg), _ptr(dh0), _ptr(dbias), inv_loss_scale, accumulate,
            _ptr(overflow_flag), _ptr(ws), nb, stream), "nnconv_recurrence_bwd")


class AdamW(_Handle):
    """AdamW over a list of tensors: nnconv_adamw_*.

    Each entry of `tensors` is a dict with master, grad, m, v (and w16; m_scale and v_scale with
    8-bit moments) as dense torch tensors on the current device, and weight_decay.  Moments in 8
    bits are torch.float8_e4m3fn (m) and torch.float8_e5m2 (v), or uint8, with a byte of scale for
    every NNCONV_ADAMW_BLOCK elements.

    The plan holds the tensors' addresses, and the handle keeps the tensors: every step reads the
    gradients from the tensors that are in the list, so a backward pass has to write them there
    (a gradient tensor that is replaced, or set to None and made anew, is not seen).  Making the
    plan queues kernels and waits for them."""

    def __init__(self, tensors, seed=0):
        import torch
        super().__init__(nnconv_adamw_plan())
        codes = {torch.float32: NNCONV_F32, torch.float16: NNCONV_F16, torch.bfloat16: NNCONV_BF16}
        self.tensors, self.seed = list(tensors), seed
        n = len(self.tensors)
        arr = (nnconv_adamw_tensor * max(n, 1))()
        fp32, scale = {torch.float32}, {torch.uint8, torch.float8_e8m0fnu}
        m8, v8 = {torch.float8_e4m3fn, torch.uint8}, {torch.float8_e5m2, torch.uint8}
        gpu = self.tensors[0]["master"].get_device() if n else self._get_device()

        def address(key, v, size, types):
            if v.numel() != size or not v.is_contiguous():
                raise ValueError("AdamW: %s has another size than the master, or is not dense" % key)
            if v.dtype not in types:
                raise ValueError("AdamW: %s has type %s" % (key, v.dtype))
            if v.get_device() != gpu:
                raise ValueError("AdamW: %s is on %s, the first master on device %d" % (key, v.device, gpu))
            return v.data_ptr()

        for a, t in zip(arr, self.tensors):
            master, grad, w16 = t["master"], t["grad"], t.get("w16")
            count = master.numel()
            f8 = t.get("m_scale") is not None
            a.master = address("master", master, count, fp32)
            a.grad = address("grad", grad, count, (grad.dtype,))
            a.m, a.v = address("m", t["m"], count, m8 if f8 else fp32), address("v", t["v"], count, v8 if f8 else fp32)
            if w16 is not None:
                a.w16, a.w16_dtype = address("w16", w16, count, {torch.float16, torch.bfloat16}), codes[w16.dtype]
            if f8:
                blocks = -(-count // NNCONV_ADAMW_BLOCK)
                a.m_scale, a.v_scale = (address(k, t[k], blocks, scale) for k in ("m_scale", "v_scale"))
            a.count, a.weight_decay = count, t.get("weight_decay", 0.0)
            a.grad_dtype, a.state_dtype = codes.get(grad.dtype, -1), NNCONV_F8 if f8 else NNCONV_F32
        stream = self._stream(None, gpu)
        st, nb = nnconv_adamw_plan_size(arr, n)
        check(st, "nnconv_adamw_plan_size")
        self._table = torch.empty(max(nb, 1), dtype=torch.uint8, device=torch.device("cuda", gpu))
        self.plan, self._device = self.desc, gpu
        check(nnconv_adamw_plan_init(arr, n, self._table.data_ptr(), nb, self.plan, stream), "nnconv_adamw_plan_init")
        torch.cuda.current_stream().synchronize()  # the plan is there for steps on any stream

    def step(self, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, state=None, overflow_flag=None,
             stream=None):
        """step, overflow_flag: int32 tensors of one element; state: the loss scaler's."""
        gpu = self._device
        self._dense(self._i32, 1, gpu, more=True, step=step, overflow_flag=overflow_flag)
        if isinstance(state, self._tensor) and not (
                state.nbytes >= ctypes.sizeof(nnconv_loss_scaler) and state.is_contiguous() and state.get_device() == gpu):
            self._refuse("state", state, "the loss scaler's %d bytes on device %d" % (ctypes.sizeof(nnconv_loss_scaler), gpu))
        check(nnconv_adamw_update(self.plan, _ptr(step), lr, beta1, beta2, eps, self.seed, _ptr(state),
                                  _ptr(overflow_flag), self._stream(stream, gpu)), "nnconv_adamw_update")
