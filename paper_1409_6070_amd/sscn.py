"""ctypes binding of libsscn (include/sscn.h): argument marshalling only.

The functions ``sscn_*`` below carry the C names and signatures one to one.
``SparseDeepCNet`` is a convenience wrapper that allocates the caller-owned
device buffers with torch (workspace, gradients, logits) and passes raw
pointers plus torch's current HIP stream; every step of the computation runs
in the HIP kernels of the library.  If the library is not built, loading
fails with an error -- there is no fallback path.
"""

import ctypes
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsscn.so")

SSCN_F32, SSCN_BF16 = 0, 1
ARCHS = ("deepcnet", "deepcnin")  # sscn_arch values 0, 1
STATUS = {
    0: "SSCN_OK",
    1: "SSCN_ERR_INVALID_ARGUMENT",
    2: "SSCN_ERR_OUT_OF_RANGE",
    3: "SSCN_ERR_DUPLICATE_SITE",
    4: "SSCN_ERR_CAPACITY",
    5: "SSCN_ERR_BAD_STATE",
    6: "SSCN_ERR_HIP",
    7: "SSCN_ERR_WORKSPACE",
}
EXPORTED = [
    "sscn_net_create", "sscn_net_destroy", "sscn_status_string", "sscn_net_num_params", "sscn_net_param_shape",
    "sscn_net_workspace_bytes", "sscn_rulebook_build", "sscn_rulebook_build_grouped", "sscn_layer_sizes", "sscn_forward", "sscn_backward",
    "sscn_forward_stage", "sscn_backward_stage", "sscn_layer_view_get", "sscn_timing_enable", "sscn_timing_collect",
    "sscn_timing_launches",
    "sscn_set_dropout", "sscn_philox4x32_10", "sscn_sgd_step", "sscn_encode_workspace_bytes", "sscn_encode_strokes",
    "sscn_encode_strokes_static",
    "sscn_layer_norm_forward", "sscn_layer_norm_workspace_bytes", "sscn_layer_norm_backward",
    "sscn_orthogonalize_workspace_bytes", "sscn_orthogonalize", "sscn_muon_workspace_bytes", "sscn_muon_update",
    "sscn_net_muon_workspace_bytes", "sscn_muon_step", "sscn_head_norm_workspace_bytes", "sscn_set_head_norm",
]
KERNEL_CLASSES = ["rulebook", "gather_gemm", "wgrad", "wgrad_reduce", "pool_fwd", "pool_bwd", "head", "ground",
                  "dropout", "sgd", "conv_narrow"]


class SSCNError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        self.name = STATUS.get(status, str(status))
        super().__init__(f"{where}: {self.name}")


class NetDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32)
                for n in ("ell", "k", "c_in", "n_classes", "batch_max", "max_active", "dtype", "arch", "dropout")]


class LayerView(ctypes.Structure):
    _fields_ = [
        ("kind", ctypes.c_int32), ("side", ctypes.c_int32), ("channels", ctypes.c_int32),
        ("row_stride", ctypes.c_int32), ("window", ctypes.c_int32), ("capacity", ctypes.c_int32),
        ("count", ctypes.c_void_p), ("sites", ctypes.c_void_p), ("rules", ctypes.c_void_p),
        ("rules_t", ctypes.c_void_p), ("features", ctypes.c_void_p), ("grad", ctypes.c_void_p),
        ("argmax", ctypes.c_void_p), ("gmask", ctypes.c_void_p),
    ]


class OrthoMatrix(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("d_in", ctypes.c_void_p),
                ("in_stride", ctypes.c_int64), ("d_out", ctypes.c_void_p), ("out_stride", ctypes.c_int64)]


class MuonParam(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("d_w", ctypes.c_void_p),
                ("d_w_store", ctypes.c_void_p), ("d_g", ctypes.c_void_p), ("d_v", ctypes.c_void_p),
                ("lr", ctypes.c_float), ("weight_decay", ctypes.c_float), ("scale", ctypes.c_float),
                ("orthogonal", ctypes.c_int32)]


class MuonOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("lr_rest", ctypes.c_float), ("momentum", ctypes.c_float),
                ("weight_decay", ctypes.c_float), ("nesterov", ctypes.c_int32), ("softmax", ctypes.c_int32),
                ("steps", ctypes.c_int32), ("h_coef", ctypes.c_void_p)]


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Loads libsscn.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_1409_6070_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32, VP, SZ = ctypes.POINTER, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
    I64, F32 = ctypes.c_int64, ctypes.c_float
    sig = {
        "sscn_net_create": (I32, [P(NetDesc), P(VP)]),
        "sscn_net_destroy": (None, [VP]),
        "sscn_status_string": (ctypes.c_char_p, [I32]),
        "sscn_net_num_params": (I32, [VP]),
        "sscn_net_param_shape": (I32, [VP, I32, P(ctypes.c_int64), P(ctypes.c_int64)]),
        "sscn_net_workspace_bytes": (I32, [VP, P(SZ)]),
        "sscn_rulebook_build": (I32, [VP, VP, I32, I32, VP, SZ, VP]),
        "sscn_rulebook_build_grouped": (I32, [VP, VP, VP, I32, I32, VP, SZ, VP]),
        "sscn_layer_sizes": (I32, [VP, P(I32), VP]),
        "sscn_forward": (I32, [VP, VP, P(VP), P(VP), VP, VP, VP, VP]),
        "sscn_backward": (I32, [VP, P(VP), P(VP), VP, VP]),
        "sscn_forward_stage": (I32, [VP, I32, VP]),
        "sscn_backward_stage": (I32, [VP, I32, VP]),
        "sscn_layer_view_get": (I32, [VP, I32, P(LayerView)]),
        "sscn_timing_enable": (I32, [VP, ctypes.c_uint32]),
        "sscn_timing_collect": (I32, [VP, I32, P(I32), P(ctypes.c_float), VP]),
        "sscn_timing_launches": (I32, [VP, I32, P(I32), P(ctypes.c_float), I32, P(I32), VP]),
        "sscn_set_dropout": (I32, [VP, P(ctypes.c_double), I32, ctypes.c_uint64]),
        "sscn_philox4x32_10": (None, [P(ctypes.c_uint32), P(ctypes.c_uint32), P(ctypes.c_uint32)]),
        "sscn_sgd_step": (I32, [VP, P(VP), P(VP), P(VP), P(VP), P(VP), ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                VP]),
        "sscn_encode_workspace_bytes": (I32, [I32, I32, I32, P(SZ)]),
        "sscn_encode_strokes": (I32, [I32, I32, VP, I32, VP, VP, I32, I32, VP, VP, I32, P(I32), VP, SZ, VP]),
        "sscn_encode_strokes_static": (I32, [I32, I32, VP, I32, VP, VP, I32, I32, VP, VP, I32, P(I32), VP]),
        "sscn_layer_norm_forward": (I32, [I32, VP, I64, I64, I32, VP, VP, F32, VP, I64, VP]),
        "sscn_layer_norm_workspace_bytes": (I32, [I32, I64, I32, P(SZ)]),
        "sscn_layer_norm_backward": (I32, [I32, VP, I64, VP, I64, I64, I32, VP, F32, VP, I64, VP, VP, VP, SZ, VP]),
        "sscn_orthogonalize_workspace_bytes": (I32, [I32, P(OrthoMatrix), P(SZ)]),
        "sscn_orthogonalize": (I32, [I32, I32, P(OrthoMatrix), I32, P(F32), VP, SZ, VP]),
        "sscn_muon_workspace_bytes": (I32, [I32, P(MuonParam), P(SZ)]),
        "sscn_muon_update": (I32, [I32, I32, P(MuonParam), F32, I32, I32, P(F32), VP, SZ, VP]),
        "sscn_net_muon_workspace_bytes": (I32, [VP, P(MuonOptions), P(SZ)]),
        "sscn_muon_step": (I32, [VP, P(VP), P(VP), P(VP), P(VP), P(VP), P(MuonOptions), VP, SZ, VP]),
        "sscn_head_norm_workspace_bytes": (I32, [VP, P(SZ)]),
        "sscn_set_head_norm": (I32, [VP, VP, VP, VP, VP, F32, VP, SZ]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int, where: str):
    if status != 0:
        raise SSCNError(status, where)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# ---------------------------------------------------------------------------
# the C calls, same names


def sscn_net_create(desc: NetDesc) -> int:
    h = ctypes.c_void_p()
    _check(load_library().sscn_net_create(ctypes.byref(desc), ctypes.byref(h)), "sscn_net_create")
    return h.value


def sscn_net_destroy(net: int) -> None:
    load_library().sscn_net_destroy(net)


def sscn_status_string(status: int) -> str:
    return load_library().sscn_status_string(status).decode()


def sscn_net_num_params(net: int) -> int:
    return load_library().sscn_net_num_params(net)


def sscn_net_param_shape(net: int, layer: int):
    r, c = ctypes.c_int64(), ctypes.c_int64()
    _check(load_library().sscn_net_param_shape(net, layer, ctypes.byref(r), ctypes.byref(c)), "sscn_net_param_shape")
    return r.value, c.value


def sscn_net_workspace_bytes(net: int) -> int:
    b = ctypes.c_size_t()
    _check(load_library().sscn_net_workspace_bytes(net, ctypes.byref(b)), "sscn_net_workspace_bytes")
    return b.value


def sscn_rulebook_build(net: int, d_coords: int, n: int, batch: int, d_ws: int, ws_bytes: int, stream: int) -> None:
    _check(load_library().sscn_rulebook_build(net, d_coords, n, batch, d_ws, ws_bytes, stream), "sscn_rulebook_build")


def sscn_rulebook_build_grouped(net: int, d_coords: int, d_sample_begin: int, n: int, batch: int, d_ws: int,
                                ws_bytes: int, stream: int) -> None:
    _check(load_library().sscn_rulebook_build_grouped(net, d_coords, d_sample_begin, n, batch, d_ws, ws_bytes, stream),
           "sscn_rulebook_build_grouped")


def sscn_layer_sizes(net: int, nlayers: int, stream: int) -> List[int]:
    arr = (ctypes.c_int32 * nlayers)()
    _check(load_library().sscn_layer_sizes(net, arr, stream), "sscn_layer_sizes")
    return list(arr)


def _ptr_array(ptrs: Sequence[int]):
    return (ctypes.c_void_p * len(ptrs))(*ptrs)


def sscn_forward(net, d_feats, W_ptrs, b_ptrs, d_labels, d_logits, d_loss, stream) -> None:
    _check(load_library().sscn_forward(net, d_feats, _ptr_array(W_ptrs), _ptr_array(b_ptrs), d_labels, d_logits,
                                       d_loss, stream), "sscn_forward")


def sscn_backward(net, dW_ptrs, db_ptrs, d_dfeats, stream) -> None:
    _check(load_library().sscn_backward(net, _ptr_array(dW_ptrs), _ptr_array(db_ptrs), d_dfeats, stream),
           "sscn_backward")


def sscn_forward_stage(net, stage, stream) -> None:
    _check(load_library().sscn_forward_stage(net, stage, stream), "sscn_forward_stage")


def sscn_backward_stage(net, stage, stream) -> None:
    _check(load_library().sscn_backward_stage(net, stage, stream), "sscn_backward_stage")


def sscn_layer_view_get(net, layer) -> LayerView:
    v = LayerView()
    _check(load_library().sscn_layer_view_get(net, layer, ctypes.byref(v)), "sscn_layer_view_get")
    return v


def sscn_set_dropout(net, rates: Optional[Sequence[float]], seed: int) -> None:
    rates = list(rates or [])
    arr = (ctypes.c_double * max(len(rates), 1))(*rates)
    _check(load_library().sscn_set_dropout(net, arr if rates else None, len(rates), seed & (2 ** 64 - 1)),
           "sscn_set_dropout")


def sscn_philox4x32_10(counter: Sequence[int], key: Sequence[int]) -> List[int]:
    c = (ctypes.c_uint32 * 4)(*counter)
    k = (ctypes.c_uint32 * 2)(*key)
    out = (ctypes.c_uint32 * 4)()
    load_library().sscn_philox4x32_10(c, k, out)
    return list(out)


def sscn_sgd_step(net, W32_ptrs, W_ptrs, b_ptrs, vW_ptrs, vb_ptrs, lr, momentum, weight_decay, stream) -> None:
    _check(load_library().sscn_sgd_step(net, _ptr_array(W32_ptrs), _ptr_array(W_ptrs) if W_ptrs is not None else None,
                                        _ptr_array(b_ptrs), _ptr_array(vW_ptrs), _ptr_array(vb_ptrs), lr, momentum,
                                        weight_decay, stream), "sscn_sgd_step")


def sscn_encode_workspace_bytes(N: int, batch_max: int, max_sites: int) -> int:
    out = ctypes.c_size_t()
    _check(load_library().sscn_encode_workspace_bytes(N, batch_max, max_sites, ctypes.byref(out)),
           "sscn_encode_workspace_bytes")
    return out.value


def sscn_encode_strokes(N, dtype, d_points, n_points, d_begin, d_sample, n_strokes, batch, d_coords, d_feats,
                        max_sites, d_ws, ws_bytes, stream) -> int:
    """Returns the site count; raises SSCNError (the count is in .count) on failure."""
    cnt = ctypes.c_int32(0)
    st = load_library().sscn_encode_strokes(N, dtype, d_points, n_points, d_begin, d_sample, n_strokes, batch,
                                            d_coords, d_feats, max_sites, ctypes.byref(cnt), d_ws, ws_bytes, stream)
    if st != 0:
        err = SSCNError(st, "sscn_encode_strokes")
        err.count = cnt.value
        raise err
    return cnt.value


ENCODE_STATIC_SCRATCH_BYTES = 16 << 20  # SSCN_ENCODE_STATIC_SCRATCH_BYTES


def sscn_encode_strokes_static(N, dtype, d_points, n_points, d_begin, d_sample, n_strokes, batch, d_coords,
                               d_feats, max_sites, stream) -> int:
    """sscn_encode_strokes without a workspace (the library's fixed per-GPU scratch); returns the site count."""
    cnt = ctypes.c_int32(0)
    st = load_library().sscn_encode_strokes_static(N, dtype, d_points, n_points, d_begin, d_sample, n_strokes,
                                                   batch, d_coords, d_feats, max_sites, ctypes.byref(cnt), stream)
    if st != 0:
        err = SSCNError(st, "sscn_encode_strokes_static")
        err.count = cnt.value
        raise err
    return cnt.value


def sscn_timing_enable(net, class_mask: int) -> None:
    _check(load_library().sscn_timing_enable(net, class_mask), "sscn_timing_enable")


def sscn_timing_collect(net, kernel_class: int, stream):
    n, ms = ctypes.c_int32(), ctypes.c_float()
    _check(load_library().sscn_timing_collect(net, kernel_class, ctypes.byref(n), ctypes.byref(ms), stream),
           "sscn_timing_collect")
    return n.value, ms.value


def sscn_timing_launches(net, kernel_class: int, capacity: int, stream):
    tags = (ctypes.c_int32 * max(capacity, 1))()
    ms = (ctypes.c_float * max(capacity, 1))()
    n = ctypes.c_int32()
    _check(load_library().sscn_timing_launches(net, kernel_class, tags, ms, capacity, ctypes.byref(n), stream),
           "sscn_timing_launches")
    k = min(n.value, capacity)
    return list(tags[:k]), list(ms[:k]), n.value


def sscn_layer_norm_forward(dtype, d_x, x_stride, rows, cols, d_gain, d_shift, eps, d_y, y_stride, stream) -> None:
    _check(load_library().sscn_layer_norm_forward(dtype, d_x, x_stride, rows, cols, d_gain, d_shift, eps, d_y, y_stride,
                                                  stream), "sscn_layer_norm_forward")


def sscn_layer_norm_workspace_bytes(dtype, rows, cols) -> int:
    b = ctypes.c_size_t()
    _check(load_library().sscn_layer_norm_workspace_bytes(dtype, rows, cols, ctypes.byref(b)),
           "sscn_layer_norm_workspace_bytes")
    return b.value


def sscn_layer_norm_backward(dtype, d_dy, dy_stride, d_x, x_stride, rows, cols, d_gain, eps, d_dx, dx_stride, d_dgain,
                             d_dshift, d_ws, ws_bytes, stream) -> None:
    _check(load_library().sscn_layer_norm_backward(dtype, d_dy, dy_stride, d_x, x_stride, rows, cols, d_gain, eps, d_dx,
                                                   dx_stride, d_dgain, d_dshift, d_ws, ws_bytes, stream),
           "sscn_layer_norm_backward")


def sscn_orthogonalize_workspace_bytes(matrices) -> int:
    """matrices: a ctypes array of OrthoMatrix (rows and cols are read)."""
    b = ctypes.c_size_t()
    _check(load_library().sscn_orthogonalize_workspace_bytes(len(matrices), matrices, ctypes.byref(b)),
           "sscn_orthogonalize_workspace_bytes")
    return b.value


def sscn_orthogonalize(dtype, matrices, steps, coef, d_ws, ws_bytes, stream) -> None:
    _check(load_library().sscn_orthogonalize(dtype, len(matrices), matrices, steps, coef, d_ws, ws_bytes, stream),
           "sscn_orthogonalize")


def sscn_muon_workspace_bytes(params) -> int:
    """params: a ctypes array of MuonParam (rows, cols and orthogonal are read)."""
    b = ctypes.c_size_t()
    _check(load_library().sscn_muon_workspace_bytes(len(params), params, ctypes.byref(b)), "sscn_muon_workspace_bytes")
    return b.value


def sscn_muon_update(dtype, params, momentum, nesterov, steps, coef, d_ws, ws_bytes, stream) -> None:
    _check(load_library().sscn_muon_update(dtype, len(params), params, momentum, nesterov, steps, coef, d_ws, ws_bytes,
                                           stream), "sscn_muon_update")


def sscn_net_muon_workspace_bytes(net, options: MuonOptions) -> int:
    b = ctypes.c_size_t()
    _check(load_library().sscn_net_muon_workspace_bytes(net, ctypes.byref(options), ctypes.byref(b)),
           "sscn_net_muon_workspace_bytes")
    return b.value


def sscn_muon_step(net, W32_ptrs, W_ptrs, b_ptrs, vW_ptrs, vb_ptrs, options: MuonOptions, d_ws, ws_bytes, stream) -> None:
    _check(load_library().sscn_muon_step(net, _ptr_array(W32_ptrs), _ptr_array(W_ptrs) if W_ptrs is not None else None,
                                         _ptr_array(b_ptrs), _ptr_array(vW_ptrs), _ptr_array(vb_ptrs),
                                         ctypes.byref(options), d_ws, ws_bytes, stream), "sscn_muon_step")


def sscn_head_norm_workspace_bytes(net) -> int:
    b = ctypes.c_size_t()
    _check(load_library().sscn_head_norm_workspace_bytes(net, ctypes.byref(b)), "sscn_head_norm_workspace_bytes")
    return b.value


def sscn_set_head_norm(net, d_gain, d_shift, d_dgain, d_dshift, eps, d_ws, ws_bytes) -> None:
    _check(load_library().sscn_set_head_norm(net, d_gain, d_shift, d_dgain, d_dshift, eps, d_ws, ws_bytes),
           "sscn_set_head_norm")


# ---------------------------------------------------------------------------
# convenience wrapper

NORM_MAX_COLS = 1 << 20  # SSCN_NORM_MAX_COLS
# coefficients (a, b, c) of the quintic commonly used with Muon
MUON_COEF = (3.4445, -4.7750, 2.0315)
_TYPES = {"f32": (SSCN_F32, torch.float32), "bf16": (SSCN_BF16, torch.bfloat16)}


def _gpu_device(device) -> torch.device:
    d = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


# the current stream's handle; the public way to it costs 2 us a call, as much as a launch
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(device: torch.device, call, *args):
    """call(stream, ...) on the device's current stream, with the device current."""
    if device.index == torch.cuda.current_device():
        return call(_raw_stream(device.index), *args)
    with torch.cuda.device(device):
        return call(_raw_stream(device.index), *args)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _row_stride(t: torch.Tensor, what: str) -> int:
    """Elements between the rows of a matrix whose rows are contiguous and do not overlap."""
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: rows must be contiguous")
    if rows <= 1:
        return cols
    if t.stride(0) < cols:
        raise ValueError(f"{what}: rows overlap")
    return t.stride(0)


def _coef_array(coef, steps):
    """[steps][3] float32 from one triple for every step, or a triple per step."""
    rows = [coef] * steps if not hasattr(coef[0], "__len__") else list(coef)
    _need(len(rows) == steps and all(len(r) == 3 for r in rows), "coef: one (a, b, c), or one per step")
    return (ctypes.c_float * max(3 * steps, 1))(*[x for r in rows for x in r])


class SparseDeepCNet:
    """DeepCNet(ell, k) or DeepCNiN(ell, k) on the GPU through libsscn; torch supplies memory and the stream."""

    def __init__(self, ell: int, k: int, c_in: int, n_classes: int, batch_max: int, max_active: int,
                 dtype: str = "bf16", device: str = "cuda", arch: str = "deepcnet", dropout: bool = False):
        if dtype not in ("f32", "bf16"):
            raise ValueError(dtype)
        if arch not in ARCHS:
            raise ValueError(arch)
        self.ell, self.k, self.c_in, self.n_classes = ell, k, c_in, n_classes
        self.dtype = dtype
        self.arch = arch
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.device = torch.device(device)
        self.nlayers = (3 * ell + 3) if arch == "deepcnin" else (2 * ell + 2)
        desc = NetDesc(ell, k, c_in, n_classes, batch_max, max_active, SSCN_BF16 if dtype == "bf16" else SSCN_F32,
                       ARCHS.index(arch), int(bool(dropout)))
        self.handle = sscn_net_create(desc)
        self.ws_bytes = sscn_net_workspace_bytes(self.handle)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.param_shapes = [sscn_net_param_shape(self.handle, i) for i in range(sscn_net_num_params(self.handle))]
        self.dW = [torch.empty(r, c, dtype=torch.float32, device=self.device) for r, c in self.param_shapes]
        self.db = [torch.empty(c, dtype=torch.float32, device=self.device) for _, c in self.param_shapes]
        self.loss = torch.empty(1, dtype=torch.float32, device=self.device)
        self.logits = None
        self._keep = []
        self._muon_ws = None
        self._norm_bufs = self._norm_keep = None

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            try:
                sscn_net_destroy(h)
            except Exception:
                pass
            self.handle = None

    # -- calls ---------------------------------------------------------------
    def rulebook_build(self, coords: torch.Tensor, batch: int, sample_begin: Optional[torch.Tensor] = None) -> None:
        """coords [n][3] int32 (b, y, x); with sample_begin (int32 [batch + 1] on the device) the sites are
        grouped by sample and the grouped build is used."""
        assert coords.dtype == torch.int32 and coords.is_contiguous() and coords.device.type == "cuda"
        self.batch = batch
        self.n = int(coords.shape[0])
        self._coords = coords
        if sample_begin is None:
            sscn_rulebook_build(self.handle, coords.data_ptr() if self.n else None, self.n, batch, self.ws.data_ptr(),
                                self.ws_bytes, _stream())
        else:
            assert sample_begin.dtype == torch.int32 and sample_begin.is_contiguous()
            assert sample_begin.device.type == "cuda" and int(sample_begin.numel()) == batch + 1
            self._sample_begin = sample_begin
            sscn_rulebook_build_grouped(self.handle, coords.data_ptr() if self.n else None, sample_begin.data_ptr(),
                                        self.n, batch, self.ws.data_ptr(), self.ws_bytes, _stream())

    def set_dropout(self, rates: Optional[Sequence[float]], seed: int = 0) -> None:
        """Dropout rates per level (ell + 2: each convolution that is not 1x1, then the softmax
        input) for the following training passes; None switches it off."""
        sscn_set_dropout(self.handle, rates, seed)

    def layer_sizes(self) -> List[int]:
        return sscn_layer_sizes(self.handle, self.nlayers, _stream())

    def forward(self, feats: torch.Tensor, Ws: Sequence[torch.Tensor], bs: Sequence[torch.Tensor],
                labels: Optional[torch.Tensor]):
        """Forward pass; ``labels=None`` is inference (logits only, no loss, no backward)."""
        assert feats.dtype == self.tdtype and feats.is_contiguous()
        assert labels is None or labels.dtype == torch.int32
        for W in Ws:
            assert W.dtype == self.tdtype and W.is_contiguous()
        for b in bs:
            assert b.dtype == torch.float32 and b.is_contiguous()
        if self.logits is None or self.logits.shape[0] != self.batch:
            self.logits = torch.empty(self.batch, self.n_classes, dtype=torch.float32, device=self.device)
        self._keep = [feats, list(Ws), list(bs), labels]
        sscn_forward(self.handle, feats.data_ptr() if feats.numel() else None, [W.data_ptr() for W in Ws],
                     [b.data_ptr() for b in bs], labels.data_ptr() if labels is not None else None,
                     self.logits.data_ptr(), self.loss.data_ptr() if labels is not None else None, _stream())
        return self.logits, (self.loss if labels is not None else None)

    def backward(self, want_dfeats: bool = False):
        dfeats = None
        if want_dfeats:
            dfeats = torch.empty(self.n, self.c_in, dtype=self.tdtype, device=self.device)
        sscn_backward(self.handle, [t.data_ptr() for t in self.dW], [t.data_ptr() for t in self.db],
                      dfeats.data_ptr() if (dfeats is not None and self.n) else None, _stream())
        return self.dW, self.db, dfeats

    def sgd_step(self, W32: Sequence[torch.Tensor], W: Optional[Sequence[torch.Tensor]], bs: Sequence[torch.Tensor],
                 vW: Sequence[torch.Tensor], vb: Sequence[torch.Tensor], lr: float, momentum: float = 0.0,
                 weight_decay: float = 0.0) -> None:
        """SGD update from the last backward's gradients: fp32 masters W32 (and biases, velocities)
        in place, then the storage copies W the next forward reads."""
        for t in list(W32) + list(bs) + list(vW) + list(vb):
            assert t.dtype == torch.float32 and t.is_contiguous()
        if W is not None:
            for t in W:
                assert t.dtype == self.tdtype and t.is_contiguous()
        sscn_sgd_step(self.handle, [t.data_ptr() for t in W32], [t.data_ptr() for t in W] if W is not None else None,
                      [t.data_ptr() for t in bs], [t.data_ptr() for t in vW], [t.data_ptr() for t in vb], lr,
                      momentum, weight_decay, _stream())

    def muon_step(self, W32: Sequence[torch.Tensor], W: Optional[Sequence[torch.Tensor]], bs: Sequence[torch.Tensor],
                  vW: Sequence[torch.Tensor], vb: Sequence[torch.Tensor], lr: float, lr_rest: float,
                  momentum: float = 0.95, weight_decay: float = 0.0, nesterov: bool = True, softmax: bool = False,
                  coef=MUON_COEF, steps: int = 5) -> None:
        """Muon's update from the last backward's gradients, in the place of sgd_step: orthogonalised updates of
        the convolutions (and with softmax=True of the softmax layer's matrix), momentum SGD with lr_rest elsewhere."""
        for what, ts in (("W32", W32), ("W", W), ("bs", bs), ("vW", vW), ("vb", vb)):
            sizes = [r * c if "W" in what else c for r, c in self.param_shapes]
            _need(what == "W" and ts is None or [t.numel() for t in ts if t.device.type == self.device.type] == sizes,
                  f"{what}: one array of each parameter's size on {self.device.type}")
        for t in list(W32) + list(bs) + list(vW) + list(vb):
            assert t.dtype == torch.float32 and t.is_contiguous()
        if W is not None:
            for t in W:
                assert t.dtype == self.tdtype and t.is_contiguous()
        arr = _coef_array(coef, steps)
        opt = MuonOptions(lr, lr_rest, momentum, weight_decay, int(nesterov), int(softmax), steps, ctypes.addressof(arr))
        if self._muon_ws is None:  # for either choice of softmax: a captured step keeps pointing at it
            need = max(sscn_net_muon_workspace_bytes(self.handle, MuonOptions(softmax=s)) for s in (0, 1))
            self._muon_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        sscn_muon_step(self.handle, [t.data_ptr() for t in W32], [t.data_ptr() for t in W] if W is not None else None,
                       [t.data_ptr() for t in bs], [t.data_ptr() for t in vW], [t.data_ptr() for t in vb], opt,
                       self._muon_ws.data_ptr(), self._muon_ws.numel(), _stream())

    def set_head_norm(self, gain: Optional[torch.Tensor], shift: Optional[torch.Tensor] = None, eps: float = 1e-5):
        """Layer norm of the softmax layer's input with the given gain and shift ([C_last] float32, read by every
        following pass); returns (dgain, dshift), which each backward overwrites: the same two tensors at every
        call, so that a pass captured before keeps its buffers. None switches it off."""
        if gain is None:
            sscn_set_head_norm(self.handle, None, None, None, None, 0.0, None, 0)
            return None
        c = self.param_shapes[-1][0]
        for t in (gain, shift):
            assert t is not None and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == c and t.device.type == "cuda"
        if self._norm_bufs is None:
            ws = torch.empty(sscn_head_norm_workspace_bytes(self.handle), dtype=torch.uint8, device=self.device)
            self._norm_bufs = [ws] + [torch.empty(c, dtype=torch.float32, device=self.device) for _ in range(2)]
        ws, dgain, dshift = self._norm_bufs
        sscn_set_head_norm(self.handle, gain.data_ptr(), shift.data_ptr(), dgain.data_ptr(), dshift.data_ptr(), eps,
                           ws.data_ptr(), ws.numel())
        self._norm_keep = (gain, shift)
        return dgain, dshift

    def timing(self, classes: Sequence[str]) -> None:
        """Bracket launches of the named kernel classes with HIP events (empty: off)."""
        mask = 0
        for c in classes:
            mask |= 1 << KERNEL_CLASSES.index(c)
        sscn_timing_enable(self.handle, mask)

    def timing_collect(self, kernel_class: str):
        """(launches, total milliseconds) of a class since the last collect."""
        return sscn_timing_collect(self.handle, KERNEL_CLASSES.index(kernel_class), _stream())

    def timing_launches(self, kernel_class: str, capacity: int = 65536):
        """Per-launch records of a class since the last collect: [(tag, milliseconds)], launch order."""
        tags, ms, _ = sscn_timing_launches(self.handle, KERNEL_CLASSES.index(kernel_class), capacity, _stream())
        return list(zip(tags, ms))

    def forward_stage(self, stage: int) -> None:
        sscn_forward_stage(self.handle, stage, _stream())

    def backward_stage(self, stage: int) -> None:
        sscn_backward_stage(self.handle, stage, _stream())

    # -- inspection ----------------------------------------------------------
    def _slice(self, ptr: int, nbytes: int, dtype) -> torch.Tensor:
        off = ptr - self.ws.data_ptr()
        assert 0 <= off and off + nbytes <= self.ws_bytes
        return self.ws[off: off + nbytes].view(dtype)

    def layer_view(self, layer: int, n: Optional[int] = None) -> dict:
        """Tensors viewing layer `layer` in the workspace, trimmed to n active rows (+ the ground row)."""
        v = sscn_layer_view_get(self.handle, layer)
        if n is None:
            n = self.layer_sizes()[layer]
        es = 2 if self.dtype == "bf16" else 4
        out = dict(kind=v.kind, side=v.side, channels=v.channels, row_stride=v.row_stride, window=v.window,
                   capacity=v.capacity, n=n)
        rs = v.row_stride
        out["features"] = self._slice(v.features, (n + 1) * rs * es, self.tdtype).view(n + 1, rs)
        out["grad"] = self._slice(v.grad, (n + 1) * rs * es, self.tdtype).view(n + 1, rs)
        out["sites"] = self._slice(v.sites, max(n, 0) * 4, torch.int32) if n else torch.zeros(0, dtype=torch.int32)
        if layer > 0:
            A = v.window
            out["rules"] = self._slice(v.rules, (n + 1) * A * 4, torch.int32).view(n + 1, A)
            if v.argmax:
                out["argmax"] = self._slice(v.argmax, (n + 1) * rs, torch.uint8).view(n + 1, rs)
            if v.gmask:
                out["gmask"] = self._slice(v.gmask, (n + 1) * 2, torch.int16)
        return out

    def rules_t(self, layer: int, n_below: int) -> torch.Tensor:
        v = sscn_layer_view_get(self.handle, layer)
        if v.kind == 1:
            return self._slice(v.rules_t, (n_below + 1) * v.window * 4, torch.int32).view(n_below + 1, v.window)
        return self._slice(v.rules_t, (n_below + 1) * 4, torch.int32)


class StrokeEncoder:
    """Pen paths -> sparse input with 9 features per site (Section 2.4) on the GPU, through
    sscn_encode_strokes; holds the scratch and output buffers for batches within its limits."""

    def __init__(self, N: int, batch_max: int, max_sites: int, dtype: str = "bf16", device: str = "cuda"):
        if dtype not in ("f32", "bf16"):
            raise ValueError(dtype)
        self.N, self.batch_max, self.max_sites, self.dtype = N, batch_max, max_sites, dtype
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.device = torch.device(device)
        self.ws_bytes = sscn_encode_workspace_bytes(N, batch_max, max_sites)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.coords = torch.empty(max(max_sites, 1), 3, dtype=torch.int32, device=self.device)
        self.feats = torch.empty(max(max_sites, 1), 9, dtype=self.tdtype, device=self.device)

    def encode(self, points: torch.Tensor, stroke_begin: torch.Tensor, stroke_sample: torch.Tensor, batch: int):
        """(coords [n, 3], feats [n, 9]) views of the encoder's buffers (valid until the next call)."""
        for t in (points, stroke_begin, stroke_sample):
            assert t.dtype == torch.int32 and t.is_contiguous() and t.device.type == "cuda"
        if batch > self.batch_max:
            raise SSCNError(4, "StrokeEncoder.encode")
        n_strokes = int(stroke_sample.shape[0])
        n = sscn_encode_strokes(self.N, SSCN_BF16 if self.dtype == "bf16" else SSCN_F32,
                                points.data_ptr() if points.numel() else None, int(points.shape[0]),
                                stroke_begin.data_ptr(), stroke_sample.data_ptr() if n_strokes else None, n_strokes,
                                batch, self.coords.data_ptr(), self.feats.data_ptr(), self.max_sites,
                                self.ws.data_ptr(), self.ws_bytes, _stream())
        return self.coords[:n], self.feats[:n]


class LayerNorm:
    """Layer norm of feature rows [rows, cols] over their columns, through sscn_layer_norm_*; holds the backward
    pass's workspace for up to rows_max rows, from the first backward pass on. One stream at a time, and kept until
    its calls have run."""

    def __init__(self, cols: int, rows_max: int, dtype: str = "bf16", eps: float = 1e-5, device: str = "cuda"):
        if dtype not in _TYPES:
            raise ValueError(dtype)
        self.cols, self.rows_max, self.dtype, self.eps = cols, rows_max, dtype, eps
        self.code, self.tdtype = _TYPES[dtype]
        self.ws_bytes = sscn_layer_norm_workspace_bytes(self.code, rows_max, cols)
        self.device = _gpu_device(device)
        self.ws = self.ws_ptr = None

    # (messages are made only where they are raised: the calls below are a few microseconds long)
    def _rows(self, t: torch.Tensor, what: str):
        """(rows, elements between rows) of a matrix for this norm."""
        if t.dtype != self.tdtype or t.device != self.device or t.dim() != 2 or t.shape[1] != self.cols:
            raise ValueError(f"{what}: [rows, {self.cols}] {self.dtype} on {self.device}")
        if t.is_contiguous():
            return t.shape[0], self.cols
        return t.shape[0], _row_stride(t, what)

    def _param(self, t: Optional[torch.Tensor], what: str):
        if t is None:
            return None
        if t.dtype != torch.float32 or t.device != self.device or t.numel() != self.cols or not t.is_contiguous():
            raise ValueError(f"{what}: [{self.cols}] float32 on {self.device}")
        return t.data_ptr()

    def forward(self, x: torch.Tensor, gain: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """out (may be x) or a new contiguous tensor; gain and shift [cols] float32, None for 1 and 0."""
        rows, xs = self._rows(x, "x")
        if out is None:
            out, ys = torch.empty((rows, self.cols), dtype=self.tdtype, device=self.device), self.cols
        else:
            n, ys = self._rows(out, "out")
            _need(n == rows, "out: as many rows as x")
        g, s = self._param(gain, "gain"), self._param(shift, "shift")
        _launch(self.device, self._forward, x.data_ptr(), xs, rows, g, s, out.data_ptr(), ys)
        return out

    def _forward(self, stream, x, xs, rows, g, s, y, ys):
        sscn_layer_norm_forward(self.code, x, xs, rows, self.cols, g, s, self.eps, y, ys, stream)

    def backward(self, dy: torch.Tensor, x: torch.Tensor, gain: Optional[torch.Tensor] = None,
                 dx: Optional[torch.Tensor] = None):
        """(dx, dgain, dshift) from the output's gradient and the forward's input; dx may be given (dy and x too)."""
        rows, xs = self._rows(x, "x")
        n, ds = self._rows(dy, "dy")
        _need(n == rows, "dy: as many rows as x")
        if rows > self.rows_max:
            raise ValueError(f"rows: at most {self.rows_max}")
        if dx is None:
            dx, os = torch.empty((rows, self.cols), dtype=self.tdtype, device=self.device), self.cols
        else:
            n, os = self._rows(dx, "dx")
            _need(n == rows, "dx: as many rows as x")
        g = self._param(gain, "gain")
        if self.ws is None:
            self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
            self.ws_ptr = self.ws.data_ptr()
        dgain, dshift = torch.empty((2, self.cols), dtype=torch.float32, device=self.device).unbind(0)
        _launch(self.device, self._backward, dy.data_ptr(), ds, x.data_ptr(), xs, rows, g, dx.data_ptr(), os,
                dgain.data_ptr(), dshift.data_ptr())
        return dx, dgain, dshift

    def _backward(self, stream, dy, ds, x, xs, rows, g, dx, os, dgain, dshift):
        sscn_layer_norm_backward(self.code, dy, ds, x, xs, rows, self.cols, g, self.eps, dx, os, dgain, dshift,
                                 self.ws_ptr, self.ws_bytes, stream)


class Orthogonalizer:
    """Newton-Schulz orthogonalisation of matrices of fixed shapes, through sscn_orthogonalize; holds the workspace.
    coef: (a, b, c) for every step, or one triple per step. One stream at a time, and kept until its calls have
    run."""

    def __init__(self, shapes: Sequence, dtype: str = "bf16", coef=MUON_COEF, steps: int = 5, device: str = "cuda"):
        if dtype not in _TYPES:
            raise ValueError(dtype)
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        self.code, self.tdtype = _TYPES[dtype]
        self.steps, self.coef = steps, _coef_array(coef, steps)
        self._mats = (OrthoMatrix * len(self.shapes))(*[OrthoMatrix(rows=r, cols=c) for r, c in self.shapes])
        self.ws_bytes = sscn_orthogonalize_workspace_bytes(self._mats)
        self.device = _gpu_device(device)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)

    def orthogonalize(self, mats: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None):
        """out (may be mats) or new contiguous matrices, in the order of the shapes."""
        if out is None:
            out = [torch.empty(r, c, dtype=self.tdtype, device=self.device) for r, c in self.shapes]
        _need(len(mats) == len(out) == len(self.shapes), f"{len(self.shapes)} matrices")
        ins, outs = [t.data_ptr() for t in mats], [t.data_ptr() for t in out]
        apart = {i for i, o in zip(ins, outs) if i != o}
        _need(len(set(outs)) == len(outs) and apart.isdisjoint(outs), "out: each its own array, or its own matrix")
        for m, i, o, shape, a, b in zip(self._mats, mats, out, self.shapes, ins, outs):
            for t, what in ((i, "matrix"), (o, "out")):
                if t.shape != shape or t.dtype != self.tdtype or t.device != self.device:
                    raise ValueError(f"{what}: {shape} {self.tdtype} on {self.device}")
            m.d_in, m.in_stride = a, _row_stride(i, "matrix")
            m.d_out, m.out_stride = b, _row_stride(o, "out")
        _launch(self.device, lambda st: sscn_orthogonalize(self.code, self._mats, self.steps, self.coef,
                                                           self.ws.data_ptr(), self.ws_bytes, st))
        return out


class Muon:
    """Muon's update of parameter arrays of fixed shapes, through sscn_muon_update; holds the workspace. Matrices
    take the orthogonalised update (orthogonal[i] says otherwise), vectors momentum SGD without weight decay.
    dtype is that of the storage copies. One stream at a time, and kept until its calls have run."""

    def __init__(self, shapes: Sequence, dtype: str = "bf16", coef=MUON_COEF, steps: int = 5,
                 orthogonal: Optional[Sequence[bool]] = None, device: str = "cuda"):
        if dtype not in _TYPES:
            raise ValueError(dtype)
        self.shapes = [tuple(int(n) for n in s) for s in shapes]
        _need(all(len(s) in (1, 2) for s in self.shapes), "shapes: vectors and matrices")
        orthogonal = [len(s) == 2 for s in self.shapes] if orthogonal is None else [bool(o) for o in orthogonal]
        _need(len(orthogonal) == len(self.shapes), f"orthogonal: {len(self.shapes)} truth values")
        self.code, self.tdtype = _TYPES[dtype]
        self.steps, self.coef = steps, _coef_array(coef, steps)
        self._params = (MuonParam * len(self.shapes))(*[
            MuonParam(rows=s[0] if len(s) == 2 else 1, cols=s[-1], orthogonal=int(o),
                      scale=max(1.0, s[-1] / s[0]) ** 0.5 if len(s) == 2 else 1.0)
            for s, o in zip(self.shapes, orthogonal)])
        self.ws_bytes = sscn_muon_workspace_bytes(self._params)
        self.device = _gpu_device(device)
        self.ws = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=self.device)

    def step(self, W32: Sequence[torch.Tensor], W: Optional[Sequence[Optional[torch.Tensor]]],
             grads: Sequence[torch.Tensor], vs: Sequence[torch.Tensor], lr: float, momentum: float = 0.95,
             weight_decay: float = 0.0, nesterov: bool = True, lr_rest: Optional[float] = None) -> None:
        """Updates the masters W32 and velocities vs in place and rewrites the copies W (None: no copies); lr_rest
        (default lr) is the rate of the arrays that are not orthogonalised."""
        n = len(self.shapes)
        W = [None] * n if W is None else W
        _need(len(W32) == len(W) == len(grads) == len(vs) == n, f"{n} arrays")
        for p, s, w, c, g, v in zip(self._params, self.shapes, W32, W, grads, vs):
            for t in (w, g, v):
                if t.shape != s or t.dtype != torch.float32 or t.device != self.device or not t.is_contiguous():
                    raise ValueError(f"parameter: {s} float32 on {self.device}, contiguous")
            if c is not None and (c.shape != s or c.dtype != self.tdtype or c.device != self.device
                                  or not c.is_contiguous()):
                raise ValueError(f"copy: {s} {self.tdtype} on {self.device}, contiguous")
            p.d_w, p.d_g, p.d_v = w.data_ptr(), g.data_ptr(), v.data_ptr()
            p.d_w_store = None if c is None else c.data_ptr()
            p.lr = lr if p.orthogonal or lr_rest is None else lr_rest
            p.weight_decay = weight_decay if len(s) == 2 else 0.0
        _need(len({p.d_w for p in self._params}) == n, "an array is named twice")
        _launch(self.device, lambda st: sscn_muon_update(self.code, self._params, momentum, int(nesterov), self.steps,
                                                         self.coef, self.ws.data_ptr(), self.ws_bytes, st))
