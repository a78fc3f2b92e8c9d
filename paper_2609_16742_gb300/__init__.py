"""Python binding of libct, the carry-through checksum inference library.

Argument marshalling only: every step of inference, verification, fault
injection and re-execution runs in the library's CUDA kernels (see
``include/ct.h``).  The functions keep the C names.  Device buffers are
passed as PyTorch CUDA tensors (or raw integer addresses); PyTorch supplies
device memory and streams, nothing else.

Importing this package does not need a GPU; calling into the library does,
and there is no fallback: if ``_lib/libct.so`` is missing, every call raises.
"""
from __future__ import annotations

import array
import ctypes
import functools
import operator
import os
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libct.so")

CT_FP32, CT_FP16 = 0, 1
CT_OP_CONV, CT_OP_MAXPOOL, CT_OP_GAP, CT_OP_FC = 0, 1, 2, 3
CT_ROLE_CT, CT_ROLE_NONE, CT_ROLE_PASS, CT_ROLE_AUTO = 0, 1, 2, 3
CT_BUF_WEIGHT, CT_BUF_ACT = 0, 1
CT_DS_PASS, CT_DS_ZERO = 0, 1
CT_PROTECT_NONE, CT_PROTECT_WIDEN, CT_PROTECT_REPLACE = 0, 1, 2
CT_FLAG_SIMT_ONLY = 1
CT_FLAG_LAYERWISE = 2
FAM_TC, FAM_SIMT, FAM_FC, FAM_POOL, FAM_OTHER = 0, 1, 2, 3, 4

_STATUS = {0: "CT_OK", 1: "CT_EINVAL", 2: "CT_ENOMEM", 3: "CT_ECUDA", 4: "CT_ESTATE",
           5: "CT_ERANGE", 6: "CT_EUNSUPPORTED", 7: "CT_EDEVICE"}

# every exported symbol of include/ct.h
EXPORTS = ["ct_build", "ct_set_threshold", "ct_get_threshold", "ct_infer", "ct_inject",
           "ct_clear_faults", "ct_reexecute", "ct_infer_reexec", "ct_run_host", "ct_calibrate", "ct_buffer_count",
           "ct_buffer_info", "ct_profile_enable", "ct_profile_read", "ct_launches_per_infer", "ct_kernel_count",
           "ct_fi_threshold",
           "ct_copy_activation", "ct_device_error", "ct_destroy", "ct_strerror",
           "ct_reexecute_noalloc", "ct_campaign_batched", "ct_resolve_roles",
           "ct_reexecute_prepare", "ct_infer_batches", "ct_run_host_batches",
           "ct_fp8_quantize", "ct_fp8_matmul", "ct_fp8_linear", "ct_fp8_linear_workspace",
           "ct_logprobs", "ct_logprobs_grad", "ct_ops_device_error",
           "ct_adapters", "ct_adapters_workspace", "ct_adapters_grad", "ct_adapters_grad_workspace",
           "ct_clip_grads", "ct_clip_grads_workspace", "ct_verify_drafts", "ct_verify_drafts_workspace"]

CT_NOALLOC_SCRATCH_BYTES = 16 * 1024 * 1024
CT_DT_F32, CT_DT_F16, CT_DT_BF16 = 0, 1, 2
CT_MAX_TOP_K = 32
CT_MAX_RANK = 128
CT_MAX_ADAPTERS = 65534
CT_MAX_DRAFTS = 64
CT_NORM_2, CT_NORM_INF = 0, 1


class CtError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        super().__init__("%s: %s (%s)" % (what, _STATUS.get(status, status), _strerror(status)))


class LayerDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("op", "src", "dst", "res", "cin", "cout", "k", "stride", "pad", "role", "bn",
                 "relu", "final", "ct_shift", "groups")]


class ModelDesc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("layers", ctypes.POINTER(LayerDesc)),
                ("in_c", ctypes.c_int32), ("in_h", ctypes.c_int32), ("in_w", ctypes.c_int32),
                ("n_classes", ctypes.c_int32), ("bn_eps", ctypes.c_double)]


class FaultDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("layer", ctypes.c_int32), ("element", ctypes.c_int64),
                ("bit", ctypes.c_int32)]


class BuildOpts(ctypes.Structure):
    _fields_ = [("precision", ctypes.c_int32), ("protect", ctypes.c_int32),
                ("ds_mode", ctypes.c_int32), ("device", ctypes.c_int32),
                ("max_batch", ctypes.c_int32), ("flags", ctypes.c_uint32)]


_lib = None


def lib():
    """The loaded libct.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libct.so is not built (%s); run paper_2609_16742_gb300.build.build()"
                               % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
        P = ctypes.POINTER
        sig = {
            "ct_build": [P(ModelDesc), P(ctypes.c_void_p), P(BuildOpts), P(vp)],
            "ct_set_threshold": [vp, dbl, dbl],
            "ct_get_threshold": [vp, P(dbl), P(dbl)],
            "ct_infer": [vp, vp, i32, vp, vp, vp, vp],
            "ct_inject": [vp, i32, i32, i64, i32],
            "ct_clear_faults": [vp],
            "ct_reexecute": [vp, vp, i32, vp, vp, vp, P(i32), vp],
            "ct_infer_reexec": [vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, vp, P(i32), vp],
            "ct_reexecute_noalloc": [vp, vp, i32, vp, vp, vp, P(i32), vp],
            "ct_run_host": [vp, vp, i32, vp, vp, vp, P(i32), vp],
            "ct_calibrate": [vp, i64, dbl, P(dbl), P(dbl)],
            "ct_fi_threshold": [vp, vp, i64, dbl, dbl, P(dbl)],
            "ct_buffer_count": [vp, i32, P(i32)],
            "ct_buffer_info": [vp, i32, i32, P(i32), P(i32), P(i64), P(i32)],
            "ct_profile_enable": [vp, i32],
            "ct_profile_read": [vp, i32, P(i64), P(dbl), P(dbl)],
            "ct_launches_per_infer": [vp, P(i32)],
            "ct_kernel_count": [vp, P(i64)],
            "ct_copy_activation": [vp, i32, i32, vp, vp, P(i32), P(i32), P(i32), P(i32), P(i32), vp],
            "ct_device_error": [vp, P(ctypes.c_uint32)],
            "ct_campaign_batched": [vp, vp, i32, P(FaultDesc), i32, vp, vp, vp, vp],
            "ct_resolve_roles": [P(ModelDesc), P(i32)],
            "ct_reexecute_prepare": [vp, i32],
            "ct_infer_batches": [vp, i32, i32, P(vp), P(vp), P(vp), P(vp), P(i32), vp],
            "ct_run_host_batches": [vp, i32, i32, P(vp), P(vp), P(vp), P(vp), P(i32), vp],
            "ct_fp8_quantize": [vp, i32, i64, i64, i64, i32, vp, i64, vp, i64, i64, vp],
            "ct_fp8_matmul": [vp, i64, vp, i64, i64, vp, i64, vp, i64, i64, vp, i32, vp, i32, i64, i64, i64, i64, vp],
            "ct_fp8_linear": [vp, i32, i64, vp, i64, vp, i64, i64, vp, i32, vp, i32, i64, i64, i64, i64, vp,
                              ctypes.c_size_t, vp],
            "ct_fp8_linear_workspace": [i64, i64, P(ctypes.c_size_t)],
            "ct_logprobs": [vp, i32, i64, vp, i64, i64, i32, vp, vp, vp, vp, vp, vp],
            "ct_logprobs_grad": [vp, i32, i64, vp, i64, i64, vp, vp, vp, vp, vp, i64, vp],
            "ct_ops_device_error": [P(ctypes.c_uint32)],
            "ct_adapters_workspace": [i64, i64, i64, i64, i64, P(ctypes.c_size_t)],
            "ct_adapters": [vp, i32, i64, vp, i32, i64, vp, i64, i64, vp, i64, i64, i32, vp, vp, i64, i64, i64, i64, i64, i32, vp,
                            ctypes.c_size_t, vp],
            "ct_adapters_grad_workspace": [i64, i64, i64, i64, i64, P(ctypes.c_size_t)],
            "ct_adapters_grad": [vp, i32, i64, vp, i32, i64, vp, i64, i64, vp, i64, i64, i32, vp, vp, i64, i64, i64, i64, i64,
                                 vp, i32, i64, vp, vp, i32, vp, ctypes.c_size_t, vp],
            "ct_clip_grads_workspace": [i64, i64, P(ctypes.c_size_t)],
            "ct_clip_grads": [vp, i64, i32, dbl, vp, vp, vp, ctypes.c_size_t, vp],
            "ct_verify_drafts_workspace": [i64, i64, i64, i64, P(ctypes.c_size_t)],
            "ct_verify_drafts": [vp, i32, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, i64, i64, i64, vp, vp, vp, vp,
                                 ctypes.c_size_t, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        L.ct_destroy.argtypes = [vp]
        L.ct_destroy.restype = None
        L.ct_strerror.argtypes = [ctypes.c_int]
        L.ct_strerror.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _strerror(s: int) -> str:
    try:
        return lib().ct_strerror(int(s)).decode()
    except Exception:
        return "?"


def _check(s: int, what: str):
    if s != 0:
        raise CtError(s, what)


def _ptr(t) -> Optional[int]:
    """Device or host address of a torch tensor / numpy array / int / None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_OPS = {"conv": CT_OP_CONV, "maxpool": CT_OP_MAXPOOL, "gap": CT_OP_GAP, "fc": CT_OP_FC}
_ROLES = {"ct": CT_ROLE_CT, "none": CT_ROLE_NONE, "pass": CT_ROLE_PASS, "auto": CT_ROLE_AUTO}
_ROLE_NAMES = {v: k for k, v in _ROLES.items()}


class Model:
    """Handle of a built model (owns the C ct_model)."""

    def __init__(self, handle: int, n_classes: int, in_shape, precision: str, protect: bool,
                 max_batch: int):
        self.handle = ctypes.c_void_p(handle)
        self.n_classes = n_classes
        self.in_shape = tuple(in_shape)
        self.precision = precision
        self.protect = protect
        self.max_batch = max_batch

    def close(self):
        if self.handle:
            lib().ct_destroy(self.handle)
            self.handle = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _layer_descs(layers: Sequence):
    n = len(layers)
    arr = (LayerDesc * n)()
    for i, L in enumerate(layers):
        arr[i] = LayerDesc(_OPS[L.op], L.src, L.dst, L.res, L.cin, L.cout, L.k, L.stride, L.pad,
                           _ROLES.get(L.ct, CT_ROLE_NONE), int(L.bn), int(L.relu), int(L.final),
                           int(L.ct_shift), int(getattr(L, "groups", 1)))
    return arr


def ct_resolve_roles(layers: Sequence, in_shape, n_classes: int) -> List[Optional[str]]:
    """Sec. II-A residual rule as the library applies it: the effective role
    of every convolution ("ct", "none", "pass"; "auto" resolved), None for
    other layers.  Raises CtError (CT_EINVAL) when a "ct" role breaks the rule."""
    arr = _layer_descs(layers)
    desc = ModelDesc(len(layers), arr, in_shape[0], in_shape[1], in_shape[2], n_classes, 1e-5)
    out = (ctypes.c_int32 * len(layers))()
    _check(lib().ct_resolve_roles(ctypes.byref(desc), out), "ct_resolve_roles")
    return [None if r < 0 else _ROLE_NAMES[r] for r in out]


def ct_build(layers: Sequence, params: Sequence[dict], in_shape, n_classes: int,
             precision: str = "fp32", protect: bool = True, ds_mode: str = "pass",
             device: int = 0, max_batch: int = 64, simt_only: bool = False,
             bn_eps: float = 1e-5, replace: bool = False, layerwise: bool = False) -> Model:
    """Build a model from synth-style layers and float32 parameter dicts.

    protect=True adds the carry-through filters as extra channels (widened);
    replace=True builds the paper's prune-and-replace construction instead;
    layerwise=True keeps one kernel per layer: for the LeNet-5 shape, and for
    1x1 shortcuts that would otherwise run in their block's first launch."""
    n = len(layers)
    arr = _layer_descs(layers)
    keep = []
    wp = (ctypes.c_void_p * (6 * n))()
    for i, (L, p) in enumerate(zip(layers, params)):
        for j, key in enumerate(("w", "b", "gamma", "beta", "mean", "var")):
            if key in p:
                a = np.ascontiguousarray(p[key], dtype=np.float32)
                keep.append(a)
                wp[6 * i + j] = a.ctypes.data
    desc = ModelDesc(n, arr, in_shape[0], in_shape[1], in_shape[2], n_classes, bn_eps)
    mode = CT_PROTECT_REPLACE if replace else (CT_PROTECT_WIDEN if protect else CT_PROTECT_NONE)
    opts = BuildOpts(CT_FP16 if precision == "fp16" else CT_FP32, mode,
                     CT_DS_ZERO if ds_mode == "zero" else CT_DS_PASS, device, max_batch,
                     (CT_FLAG_SIMT_ONLY if simt_only else 0) | (CT_FLAG_LAYERWISE if layerwise else 0))
    h = ctypes.c_void_p()
    _check(lib().ct_build(ctypes.byref(desc), wp, ctypes.byref(opts), ctypes.byref(h)), "ct_build")
    return Model(h.value, n_classes, in_shape, precision, protect or replace, max_batch)


def ct_build_workload(wl, params=None, **kw) -> Model:
    import synth
    if params is None:
        params = synth.make_params(wl.layers, wl.seed)
    kw.setdefault("precision", wl.precision)
    kw.setdefault("max_batch", wl.batch)
    kw.setdefault("bn_eps", wl.bn_eps)
    return ct_build(wl.layers, params, wl.in_shape, wl.n_classes, **kw)


def ct_set_threshold(m: Model, reference: float, tau: float):
    _check(lib().ct_set_threshold(m.handle, reference, tau), "ct_set_threshold")


def ct_get_threshold(m: Model):
    r, t = ctypes.c_double(), ctypes.c_double()
    _check(lib().ct_get_threshold(m.handle, ctypes.byref(r), ctypes.byref(t)), "ct_get_threshold")
    return r.value, t.value


def ct_infer(m: Model, input_dev, batch: int, logits_dev, S_dev=None, flag_dev=None, stream=None):
    _check(lib().ct_infer(m.handle, _ptr(input_dev), batch, _ptr(logits_dev), _ptr(S_dev),
                          _ptr(flag_dev), _stream(stream)), "ct_infer")


def ct_inject(m: Model, kind: int, layer: int, element: int, bit: int):
    _check(lib().ct_inject(m.handle, kind, layer, element, bit), "ct_inject")


def ct_clear_faults(m: Model):
    _check(lib().ct_clear_faults(m.handle), "ct_clear_faults")


def ct_reexecute(m: Model, input_dev, batch: int, flag_dev, logits_dev, S_dev=None,
                 stream=None) -> int:
    n = ctypes.c_int32()
    _check(lib().ct_reexecute(m.handle, _ptr(input_dev), batch, _ptr(flag_dev), _ptr(logits_dev),
                              _ptr(S_dev), ctypes.byref(n), _stream(stream)), "ct_reexecute")
    return n.value


def ct_reexecute_prepare(m: Model, max_images: int):
    """Capture the re-execution graphs of every padded size up to max_images."""
    _check(lib().ct_reexecute_prepare(m.handle, max_images), "ct_reexecute_prepare")


def _ptr_array(items):
    """ctypes array of addresses (None entries stay NULL), or None for None."""
    if items is None:
        return None
    return (ctypes.c_void_p * max(len(items), 1))(*[_ptr(t) for t in items])


def ct_infer_batches(m: Model, inputs_dev, batch: int, logits_dev, S_dev, flag_dev, stream=None) -> int:
    """Inference of a list of device-resident batches with each batch's
    flagged images re-run two batches later (Sec. II-B); returns the images
    re-run.  Each argument is a list with one device tensor per batch."""
    n = ctypes.c_int32()
    _check(lib().ct_infer_batches(m.handle, len(inputs_dev), batch, _ptr_array(inputs_dev), _ptr_array(logits_dev),
                                  _ptr_array(S_dev), _ptr_array(flag_dev), ctypes.byref(n), _stream(stream)),
           "ct_infer_batches")
    return n.value


def ct_run_host_batches(m: Model, inputs_host, batch: int, logits_host, S_host=None, flag_host=None,
                        stream=None) -> int:
    """ct_infer_batches for host buffers (numpy arrays or pinned CPU tensors):
    input copies and result copies overlap the device's work."""
    n = ctypes.c_int32()
    _check(lib().ct_run_host_batches(m.handle, len(inputs_host), batch, _ptr_array(inputs_host),
                                     _ptr_array(logits_host), _ptr_array(S_host), _ptr_array(flag_host),
                                     ctypes.byref(n), _stream(stream)), "ct_run_host_batches")
    return n.value


def ct_infer_reexec(m: Model, input_dev, batch: int, logits_dev, S_dev=None, flag_dev=None,
                    prev_input_dev=None, prev_batch: int = 0, prev_flag_dev=None, prev_logits_dev=None,
                    prev_S_dev=None, stream=None) -> int:
    """ct_infer of a new batch that re-executes the previous batch's flagged
    images as extra rows of the same inference; returns how many were re-run."""
    n = ctypes.c_int32()
    _check(lib().ct_infer_reexec(m.handle, _ptr(input_dev), batch, _ptr(logits_dev), _ptr(S_dev), _ptr(flag_dev),
                                 _ptr(prev_input_dev), prev_batch, _ptr(prev_flag_dev), _ptr(prev_logits_dev),
                                 _ptr(prev_S_dev), ctypes.byref(n), _stream(stream)), "ct_infer_reexec")
    return n.value


def ct_campaign_batched(m: Model, input_dev, batch: int, faults, S_dev, top1_dev, flag_dev, stream=None):
    """Many faults in one launch.  faults: rows (kind, layer, element, bit);
    outputs [n_faults, batch] device tensors (float32, int32, uint8)."""
    f = np.asarray(faults, dtype=np.int64).reshape(-1, 4)
    arr = (FaultDesc * max(len(f), 1))()
    for i, (kind, layer, el, bit) in enumerate(f.tolist()):
        arr[i] = FaultDesc(kind, layer, el, bit)
    _check(lib().ct_campaign_batched(m.handle, _ptr(input_dev), batch, arr, len(f), _ptr(S_dev), _ptr(top1_dev),
                                     _ptr(flag_dev), _stream(stream)), "ct_campaign_batched")


def ct_reexecute_noalloc(m: Model, input_dev, batch: int, flag_dev, logits_dev, S_dev=None,
                         stream=None) -> int:
    """ct_reexecute without allocation: its scratch is a static device array."""
    n = ctypes.c_int32()
    _check(lib().ct_reexecute_noalloc(m.handle, _ptr(input_dev), batch, _ptr(flag_dev),
                                      _ptr(logits_dev), _ptr(S_dev), ctypes.byref(n),
                                      _stream(stream)), "ct_reexecute_noalloc")
    return n.value


def ct_run_host(m: Model, input_host: np.ndarray, logits_host: np.ndarray, S_host=None,
                flag_host=None, stream=None) -> int:
    assert input_host.dtype == np.float32 and input_host.flags.c_contiguous
    n = ctypes.c_int32()
    _check(lib().ct_run_host(m.handle, _ptr(input_host), input_host.shape[0], _ptr(logits_host),
                             _ptr(S_host), _ptr(flag_host), ctypes.byref(n), _stream(stream)),
           "ct_run_host")
    return n.value


def ct_calibrate(S_host: np.ndarray, alpha: float):
    S = np.ascontiguousarray(S_host, dtype=np.float32)
    r, t = ctypes.c_double(), ctypes.c_double()
    _check(lib().ct_calibrate(S.ctypes.data, S.size, alpha, ctypes.byref(r), ctypes.byref(t)),
           "ct_calibrate")
    return r.value, t.value


def ct_fi_threshold(S_host: np.ndarray, critical: np.ndarray, reference: float, alpha: float) -> float:
    """Sec. II-C FI-based threshold from campaign trials (S, critical)."""
    S = np.ascontiguousarray(S_host, dtype=np.float32)
    c = np.ascontiguousarray(critical, dtype=np.uint8)
    if S.shape != c.shape:
        raise ValueError("S and critical must have the same shape")
    t = ctypes.c_double()
    _check(lib().ct_fi_threshold(S.ctypes.data, c.ctypes.data, S.size, reference, alpha, ctypes.byref(t)),
           "ct_fi_threshold")
    return t.value


def ct_buffers(m: Model, batch: int) -> List[tuple]:
    """[(kind, layer, n_elements, bits)] from ct_buffer_count / ct_buffer_info."""
    n = ctypes.c_int32()
    _check(lib().ct_buffer_count(m.handle, batch, ctypes.byref(n)), "ct_buffer_count")
    out = []
    for i in range(n.value):
        k, l, b = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        e = ctypes.c_int64()
        _check(lib().ct_buffer_info(m.handle, batch, i, ctypes.byref(k), ctypes.byref(l),
                                    ctypes.byref(e), ctypes.byref(b)), "ct_buffer_info")
        out.append((k.value, l.value, e.value, b.value))
    return out


def ct_profile_enable(m: Model, on: bool = True):
    _check(lib().ct_profile_enable(m.handle, int(on)), "ct_profile_enable")


def ct_profile_read(m: Model, family: int):
    n, ms, fl = ctypes.c_int64(), ctypes.c_double(), ctypes.c_double()
    _check(lib().ct_profile_read(m.handle, family, ctypes.byref(n), ctypes.byref(ms),
                                 ctypes.byref(fl)), "ct_profile_read")
    return n.value, ms.value, fl.value


def ct_kernel_count(m: Model) -> int:
    """Library kernels launched for m since the previous call (then reset)."""
    n = ctypes.c_int64()
    _check(lib().ct_kernel_count(m.handle, ctypes.byref(n)), "ct_kernel_count")
    return n.value


def ct_launches_per_infer(m: Model) -> int:
    n = ctypes.c_int32()
    _check(lib().ct_launches_per_infer(m.handle, ctypes.byref(n)), "ct_launches_per_infer")
    return n.value


def ct_copy_activation(m: Model, slot: int, batch: int, stream=None):
    """(data, cs) of a stored slot as float64 arrays: data [batch, C, H, W],
    cs [batch, H, W] or None."""
    C, H, W, hc, eb = (ctypes.c_int32() for _ in range(5))
    _check(lib().ct_copy_activation(m.handle, slot, batch, None, None, ctypes.byref(C),
                                    ctypes.byref(H), ctypes.byref(W), ctypes.byref(hc),
                                    ctypes.byref(eb), _stream(stream)), "ct_copy_activation")
    dt = np.float32 if eb.value == 4 else np.float16
    data = np.empty((batch, H.value, W.value, C.value), dt)
    cs = np.empty((batch, H.value, W.value), dt) if hc.value else None
    _check(lib().ct_copy_activation(m.handle, slot, batch, data.ctypes.data,
                                    None if cs is None else cs.ctypes.data, None, None, None,
                                    None, None, _stream(stream)), "ct_copy_activation")
    data = data.astype(np.float64).transpose(0, 3, 1, 2)
    return data, (None if cs is None else cs.astype(np.float64))


def ct_device_error(m: Model) -> int:
    c = ctypes.c_uint32()
    _check(lib().ct_device_error(m.handle, ctypes.byref(c)), "ct_device_error")
    return c.value


def ct_destroy(m: Model):
    m.close()


# ---------------------------------------------------------------------------
# The 8-bit answer head: operators on PyTorch CUDA tensors, without a model.
#
# Tensors are checked here (device, type, shape, unit column stride) and
# passed on with their row pitches; ValueError names the offending argument.
# Outputs that are not given are allocated on the call's stream.  `stream`:
# None (the current one), a torch stream, or a raw cudaStream_t; inputs made
# on another stream must be ordered before it by the caller, as for any
# PyTorch kernel.  Autograd does not track these calls: while it records, a
# tensor that requires a gradient is refused, as its gradient would be lost in
# silence (pass t.detach(), or call under torch.no_grad()); gradients are calls
# of their own, ct_logprobs_grad and the product with the transposed weights.
# The calls are short next to Python's own cost, so the checks read each
# attribute once and build no message unless they fail.
# ---------------------------------------------------------------------------
class _TorchNames:
    """What the operators use of torch, looked up once."""

    def __init__(self):
        import torch
        self.torch = torch
        self.empty, self.empty_strided = torch.empty, torch.empty_strided
        self.f32, self.u8, self.i64, self.e4m3 = torch.float32, torch.uint8, torch.int64, torch.float8_e4m3fn
        self.dtypes = {torch.float32: CT_DT_F32, torch.float16: CT_DT_F16, torch.bfloat16: CT_DT_BF16}
        self.bytes = {self.e4m3: 0, self.u8: 0}
        tensor, get = torch.Tensor, operator.attrgetter
        self.is_contiguous, self.get_device, self.numel, self.data_ptr = tensor.is_contiguous, tensor.get_device, tensor.numel, tensor.data_ptr
        self.requires_grad, self.dtype, self.shape = get("requires_grad"), get("dtype"), get("shape")
        self.current_device = torch.cuda.current_device
        self.recording = torch.is_grad_enabled
        # of tensors written in place, so that autograd notices where a graph still wants what was there
        self.raise_versions = torch.autograd.graph.increment_version
        # the raw handle of the current stream; torch.cuda.current_stream builds a Stream object first
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)


_names = None


def _T():
    global _names
    if _names is None:
        _names = _TorchNames()
    return _names


class _Call:
    """One call's stream: its raw handle, and the contexts that make it (for
    allocations) and the tensors' device current while the call runs.  Only
    used where the call's stream or device is not the current one."""

    def __init__(self, device, stream):
        import contextlib
        import torch
        self.stack = contextlib.ExitStack()
        self.stack.enter_context(torch.cuda.device(device))
        if stream is not None:
            if isinstance(stream, int):
                stream = torch.cuda.ExternalStream(stream, device=device)
            self.stack.enter_context(torch.cuda.stream(stream))
        self.handle = torch.cuda.current_stream(device).cuda_stream

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        return self.stack.__exit__(*exc)


def _elsewhere(f, device, stream, *args):
    """f(*args, stream=None) with the call's device and stream current."""
    with _Call(device, stream):
        return f(*args)


def _tracked(name):
    return ValueError("%s requires a gradient, which this call does not pass on: detach it, or call under torch.no_grad()" % name)


def _bad_matrix(t, name, dtypes, shape, device):
    if t.dim() != 2 or t.dtype not in dtypes or not t.is_cuda:
        return ValueError("%s: a 2-D CUDA tensor of %s is wanted, got %s %s on %s"
                          % (name, "/".join(str(d) for d in dtypes), t.dtype, tuple(t.shape), t.device))
    if shape is not None and tuple(t.shape) != shape:
        return ValueError("%s: shape %s is wanted, got %s" % (name, shape, tuple(t.shape)))
    if device is not None and t.device != device:
        return ValueError("%s is on %s, the other tensors on %s" % (name, t.device, device))
    if t.requires_grad and _names.recording():
        return _tracked(name)
    return ValueError("%s: its columns must be contiguous (strides %s)" % (name, t.stride()))


def _matrix(t, name, dtypes, shape=None, device=None):
    """(rows, columns, row pitch) of a 2-D CUDA tensor with unit column stride."""
    size = t.shape
    if len(size) != 2 or t.dtype not in dtypes or not t.is_cuda or (shape is not None and size != shape) or \
            (device is not None and t.device != device) or (t.requires_grad and _names.recording()):
        raise _bad_matrix(t, name, dtypes, shape, device)
    m, n = size
    s0, s1 = t.stride()
    if s1 != 1 and n > 1:
        raise _bad_matrix(t, name, dtypes, shape, device)
    return m, n, s0 if m > 1 or s0 > n else n


def _vector(t, name, dtype, n, device):
    if t.dtype != dtype or t.shape != (n,) or t.device != device or (n > 1 and t.stride(0) != 1):
        raise ValueError("%s: a contiguous %s tensor of %d values on %s is wanted, got %s %s on %s"
                         % (name, dtype, n, device, t.dtype, tuple(t.shape), t.device))
    if t.requires_grad and _names.recording():
        raise _tracked(name)
    return t.data_ptr()


def _scales(t, name, shape, device):
    if t.shape != shape or t.dtype != _names.f32 or t.device != device:
        raise ValueError("%s: a float32 tensor of shape %s on %s is wanted, got %s %s on %s"
                         % (name, shape, device, t.dtype, tuple(t.shape), t.device))
    if t.requires_grad and _names.recording():
        raise _tracked(name)
    s0, s1 = t.stride()
    return t.data_ptr(), s0, s1


def _fp8_weights(wq, ws, k, device):
    """(n, pointer arguments) of 8-bit weights [n, k] and their scales."""
    n, kw, ldw = _matrix(wq, "wq", _names.bytes, None, device)
    if kw != k:
        raise ValueError("wq has %d columns, the activations %d" % (kw, k))
    return n, (wq.data_ptr(), ldw) + _scales(ws, "ws", ((n + 127) // 128, (k + 127) // 128), device)


def _fp8_out(out, out_dtype, m, n, device):
    """(y, its ct_dtype, its row pitch)"""
    if out is None:
        code = _names.dtypes.get(out_dtype)
        if code is None:
            raise ValueError("out_dtype: float32, float16 or bfloat16 is wanted, got %s" % out_dtype)
        return _names.empty((m, n), dtype=out_dtype, device=device), code, n
    if out_dtype is not None and out.dtype != out_dtype:
        raise ValueError("out is %s, out_dtype %s" % (out.dtype, out_dtype))
    ldy = _matrix(out, "out", _names.dtypes, (m, n), device)[2]
    return out, _names.dtypes[out.dtype], ldy


def ct_fp8_quantize(x, block_rows: int = 1, q=None, scale=None, stream=None):
    """(q, scale): x [m, k] in e4m3 with one power-of-two scale for each
    block of block_rows x 128 values (1: activations, 128: weights).  q
    [m, k] float8_e4m3fn has a row pitch that is a multiple of 16 bytes, as the
    products want it; scale is float32 [ceil(m / block_rows), ceil(k / 128)]."""
    T = _names or _T()
    m, k, ldx = _matrix(x, "x", T.dtypes)
    if block_rows not in (1, 128):
        raise ValueError("block_rows is 1 or 128, got %r" % (block_rows,))
    dev = x.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_fp8_quantize, dev, stream, x, block_rows, q, scale)
    rows, kb = (m + block_rows - 1) // block_rows, (k + 127) // 128
    if q is None:
        ldq = (k + 15) // 16 * 16
        q = T.empty_strided((m, k), (ldq, 1), dtype=T.e4m3, device=dev)
    else:
        ldq = _matrix(q, "q", T.bytes, (m, k), dev)[2]
    if scale is not None:
        sp, s0, s1 = _scales(scale, "scale", (rows, kb), dev)
    elif block_rows == 1:
        # activations: [block][row], the order in which the products read them
        scale = T.empty_strided((rows, kb), (1, rows), dtype=T.f32, device=dev)
        sp, s0, s1 = scale.data_ptr(), 1, rows
    else:
        scale = T.empty((rows, kb), dtype=T.f32, device=dev)
        sp, s0, s1 = scale.data_ptr(), kb, 1
    st = (_lib or lib()).ct_fp8_quantize(x.data_ptr(), T.dtypes[x.dtype], m, k, ldx, block_rows, q.data_ptr(), ldq, sp, s0, s1,
                                         T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_fp8_quantize")
    return q, scale


def ct_fp8_matmul(xq, xs, wq, ws, bias=None, relu: bool = False, out_dtype=None, out=None, stream=None):
    """y [m, n] = act(x w^T + bias) of 8-bit operands: xq [m, k] with scales xs
    [m, ceil(k / 128)], wq [n, k] with scales ws [ceil(n / 128), ceil(k / 128)]
    (any strides).  out_dtype: float32 unless `out` or another type is given."""
    T = _names or _T()
    m, k, ldx = _matrix(xq, "xq", T.bytes)
    dev = xq.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_fp8_matmul, dev, stream, xq, xs, wq, ws, bias, relu, out_dtype, out)
    n, w = _fp8_weights(wq, ws, k, dev)
    x = _scales(xs, "xs", (m, (k + 127) // 128), dev)
    b = None if bias is None else _vector(bias, "bias", T.f32, n, dev)
    y, code, ldy = _fp8_out(out, T.f32 if out is None and out_dtype is None else out_dtype, m, n, dev)
    st = (_lib or lib()).ct_fp8_matmul(xq.data_ptr(), ldx, *x, *w, b, 1 if relu else 0, y.data_ptr(), code, ldy, m, n, k,
                                       T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_fp8_matmul")
    return y


@functools.lru_cache(maxsize=256)
def _linear_workspace(m, k):
    need = ctypes.c_size_t()
    _check(lib().ct_fp8_linear_workspace(m, k, ctypes.byref(need)), "ct_fp8_linear_workspace")
    return need.value


def ct_fp8_linear(x, wq, ws, bias=None, relu: bool = False, out_dtype=None, out=None, stream=None):
    """act(x W^T + bias) with 8-bit weights on float32 / float16 / bfloat16
    activations x [m, k], quantised on the way (1 x 128 blocks).  out_dtype: x's
    type unless `out` or another type is given."""
    T = _names or _T()
    m, k, ldx = _matrix(x, "x", T.dtypes)
    dev = x.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_fp8_linear, dev, stream, x, wq, ws, bias, relu, out_dtype, out)
    n, w = _fp8_weights(wq, ws, k, dev)
    b = None if bias is None else _vector(bias, "bias", T.f32, n, dev)
    y, code, ldy = _fp8_out(out, x.dtype if out is None and out_dtype is None else out_dtype, m, n, dev)
    need = _linear_workspace(m, k)
    work = T.empty(need, dtype=T.u8, device=dev)
    st = (_lib or lib()).ct_fp8_linear(x.data_ptr(), T.dtypes[x.dtype], ldx, *w, b, 1 if relu else 0, y.data_ptr(), code, ldy,
                                       m, n, k, work.data_ptr(), need, T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_fp8_linear")
    return y


def ct_logprobs(logits, ids=None, top_k: int = 0, stream=None):
    """(logprob, entropy, lse, top_logprob, top_id) of logits [rows, vocab]:
    the log probability of token ids[r] (int64; -1: none, 0; logprob is None
    without ids), the entropy and log normaliser of each row (float32), and
    its top_k most probable tokens (float32 / int64 [rows, top_k])."""
    T = _names or _T()
    rows, vocab, ld = _matrix(logits, "logits", T.dtypes)
    dev = logits.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_logprobs, dev, stream, logits, ids, top_k)
    idp = None if ids is None else _vector(ids, "ids", T.i64, rows, dev)
    if not 0 <= top_k <= CT_MAX_TOP_K:
        raise ValueError("top_k is 0 to %d, got %r" % (CT_MAX_TOP_K, top_k))
    lp = None if ids is None else T.empty(rows, dtype=T.f32, device=dev)
    entropy = T.empty(rows, dtype=T.f32, device=dev)
    lse = T.empty(rows, dtype=T.f32, device=dev)
    top_lp = T.empty((rows, top_k), dtype=T.f32, device=dev)
    top_id = T.empty((rows, top_k), dtype=T.i64, device=dev)
    st = (_lib or lib()).ct_logprobs(logits.data_ptr(), T.dtypes[logits.dtype], ld, idp, rows, vocab, top_k,
                                     None if lp is None else lp.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
                                     top_lp.data_ptr(), top_id.data_ptr(), T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_logprobs")
    return lp, entropy, lse, top_lp, top_id


def ct_logprobs_grad(logits, ids, lse, entropy, g_logprob=None, g_entropy=None, out=None, stream=None):
    """Gradient of sum(g_logprob * logprob + g_entropy * entropy) with respect
    to the logits, in their type; lse and entropy are ct_logprobs' outputs.  A
    given token keeps its own term g_logprob also where its logit is -inf.
    `out` may be `logits`."""
    T = _names or _T()
    rows, vocab, ld = _matrix(logits, "logits", T.dtypes)
    dev = logits.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_logprobs_grad, dev, stream, logits, ids, lse, entropy, g_logprob, g_entropy, out)
    if lse is None or (g_logprob is not None and ids is None) or (g_entropy is not None and entropy is None):
        raise ValueError("lse is needed, ids for g_logprob, entropy for g_entropy")
    f32 = T.f32
    idp = None if ids is None else _vector(ids, "ids", T.i64, rows, dev)
    lsep = _vector(lse, "lse", f32, rows, dev)
    hp = None if entropy is None else _vector(entropy, "entropy", f32, rows, dev)
    gp = None if g_logprob is None else _vector(g_logprob, "g_logprob", f32, rows, dev)
    ghp = None if g_entropy is None else _vector(g_entropy, "g_entropy", f32, rows, dev)
    if out is None:
        out, ldd = T.empty((rows, vocab), dtype=logits.dtype, device=dev), vocab
    else:
        ldd = _matrix(out, "out", (logits.dtype,), (rows, vocab), dev)[2]
    st = (_lib or lib()).ct_logprobs_grad(logits.data_ptr(), T.dtypes[logits.dtype], ld, idp, rows, vocab, lsep, hp, gp, ghp,
                                          out.data_ptr(), ldd, T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_logprobs_grad")
    return out


# ---------------------------------------------------------------------------
# Adapting and answering: what trains beside the head's frozen 8-bit weights, and
# how its rows of logits become tokens.  The rules of the operators above hold.
# ---------------------------------------------------------------------------
def _bad_stack(t, name, dtype, shape, device):
    if t.dim() != 3 or t.dtype != dtype or t.device != device or (shape is not None and tuple(t.shape) != shape):
        return ValueError("%s: a 3-D tensor of %s%s on %s is wanted, got %s %s on %s"
                          % (name, dtype, "" if shape is None else " of shape %s" % (shape,), device, t.dtype, tuple(t.shape), t.device))
    if t.requires_grad and _names.recording():
        return _tracked(name)
    return ValueError("%s: its columns must be contiguous (strides %s)" % (name, t.stride()))


def _stack(t, name, dtype, shape, device):
    """(its address, matrix stride, row stride) of a stack of matrices with unit column stride."""
    size = t.shape
    if len(size) != 3 or t.dtype != dtype or t.device != device or (shape is not None and size != shape) or \
            (t.requires_grad and _names.recording()):
        raise _bad_stack(t, name, dtype, shape, device)
    s0, s1, s2 = t.stride()
    if s2 != 1 and size[2] > 1:
        raise _bad_stack(t, name, dtype, shape, device)
    return t.data_ptr(), s0, s1


def _adapters(x, a, b, ids, scale):
    """(rows, adapters, rank, k, n, x's pitch, pointer arguments) of checked adapters for activations x."""
    T = _names
    t, k, ldx = _matrix(x, "x", T.dtypes)
    dev, dt = x.device, a.dtype
    if dt not in T.dtypes or (x.dtype != dt and x.dtype != T.f32):
        raise ValueError("a: float32, float16 or bfloat16 is wanted, and x of its type or float32; got a %s, x %s" % (dt, x.dtype))
    ap = _stack(a, "a", dt, None, dev)
    count, rank = a.shape[0], a.shape[1]
    if a.shape[2] != k:
        raise ValueError("a has %d columns, x %d" % (a.shape[2], k))
    if b.dim() != 3:
        raise _bad_stack(b, "b", dt, None, dev)
    n = b.shape[1]
    bp = _stack(b, "b", dt, (count, n, rank), dev)
    if rank > CT_MAX_RANK:
        raise ValueError("a: a rank of at most %d is wanted, got %d" % (CT_MAX_RANK, rank))
    if ids is None:
        if count != 1:
            raise ValueError("ids are needed where there are %d adapters" % count)
        idp = None
    else:
        idp = _vector(ids, "ids", T.i64, t, dev)
    sp = None if scale is None else _vector(scale, "scale", T.f32, count, dev)
    return t, count, rank, k, n, ldx, ap + bp + (T.dtypes[dt], idp, sp)


@functools.lru_cache(maxsize=256)
def _adapters_workspace(grad, t, count, rank, k, n):
    need = ctypes.c_size_t()
    name = "ct_adapters_grad_workspace" if grad else "ct_adapters_workspace"
    _check(getattr(lib(), name)(t, count, rank, k, n, ctypes.byref(need)), name)
    return need.value


def ct_adapters(y, x, a, b, ids=None, scale=None, relu: bool = False, stream=None):
    """y [t, n] += scale[i] * (x A[i]^T) B[i]^T in place, with i = ids[row], then
    a ReLU if asked: low-rank adapters a [adapters, rank, k], b [adapters, n,
    rank] beside the shared projection that gave y.  ids int64 [t] in any order
    (-1: no adapter; None: one adapter for all rows); scale float32
    [adapters].  a and b are of one type, x of that or float32, y of any; y may
    be x, and shares no value with b or ids.  Returns y."""
    T = _names or _T()
    t, count, rank, k, n, ldx, w = _adapters(x, a, b, ids, scale)
    dev = x.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_adapters, dev, stream, y, x, a, b, ids, scale, relu)
    ldy = _matrix(y, "y", T.dtypes, (t, n), dev)[2]
    need = _adapters_workspace(False, t, count, rank, k, n)
    work = T.empty(need, dtype=T.u8, device=dev)
    st = (_lib or lib()).ct_adapters(y.data_ptr(), T.dtypes[y.dtype], ldy, x.data_ptr(), T.dtypes[x.dtype], ldx, *w, t, count, rank,
                                     k, n, 1 if relu else 0, work.data_ptr(), need, T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_adapters")
    T.raise_versions(y)
    return y


def ct_adapters_grad(dy, x, a, b, ids=None, scale=None, dx=None, grad_dtype=None, stream=None):
    """(dx, da, db): gradients of ct_adapters (without its ReLU) for the gradient
    dy [t, n] of its output.  dx [t, k], if given, is added to in place (the shared
    projection's part; None: not wanted) and shares no value with dy, x or a.  da
    and db are new, of a's type or grad_dtype = float32; dy is of a's type or
    float32."""
    T = _names or _T()
    t, count, rank, k, n, ldx, w = _adapters(x, a, b, ids, scale)
    dev = x.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_adapters_grad, dev, stream, dy, x, a, b, ids, scale, dx, grad_dtype)
    dt = a.dtype
    lddy = _matrix(dy, "dy", (dt, T.f32), (t, n), dev)[2]
    if grad_dtype is None:
        grad_dtype = dt
    elif grad_dtype != dt and grad_dtype != T.f32:
        raise ValueError("grad_dtype: %s or float32 is wanted, got %s" % (dt, grad_dtype))
    dxp, dx_code, lddx = None, CT_DT_F32, 0
    if dx is not None:
        lddx = _matrix(dx, "dx", T.dtypes, (t, k), dev)[2]
        dxp, dx_code = dx.data_ptr(), T.dtypes[dx.dtype]
    da = T.empty((count, rank, k), dtype=grad_dtype, device=dev)
    db = T.empty((count, n, rank), dtype=grad_dtype, device=dev)
    need = _adapters_workspace(True, t, count, rank, k, n)
    work = T.empty(need, dtype=T.u8, device=dev)
    st = (_lib or lib()).ct_adapters_grad(dy.data_ptr(), T.dtypes[dy.dtype], lddy, x.data_ptr(), T.dtypes[x.dtype], ldx, *w, t, count,
                                          rank, k, n, dxp, dx_code, lddx, da.data_ptr(), db.data_ptr(), T.dtypes[grad_dtype],
                                          work.data_ptr(), need, T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_adapters_grad")
    if dx is not None:
        T.raise_versions(dx)
    return dx, da, db


def _layout(t, name):
    """(rows, columns, row pitch) of a tensor whose values are dense in memory in some order of its dimensions, or a matrix with a pitch."""
    if t.is_contiguous():
        n = t.numel()
        return 1, n, n
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1) and t.stride(0) >= t.shape[1]:
        return t.shape[0], t.shape[1], t.stride(0)
    size = 1
    for stride, n in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride != size:
            raise ValueError("%s: dense values or a matrix with contiguous columns are wanted, got shape %s strides %s"
                             % (name, tuple(t.shape), t.stride()))
        size *= n
    return 1, size, size


def _bad_values(t, name, device):
    if t.dtype in _names.dtypes and t.device == device:
        return _tracked(name)
    return ValueError("%s: a tensor of %s on %s is wanted, got %s on %s"
                      % (name, "/".join(str(d) for d in _names.dtypes), device, t.dtype, t.device))


def _dense_table(grads, outs, index):
    """(values, table) of ct_tensor rows where every tensor is contiguous and nothing is to be refused, else None.  Attributes are
    taken of all tensors at a time: a loop over them would cost more than the kernels."""
    T = _names
    every = grads if outs is grads else grads + outs
    if not all(map(T.is_contiguous, every)) or set(map(T.get_device, every)) != {index} or \
            (T.recording() and any(map(T.requires_grad, every))):
        return None
    types = list(map(T.dtype, grads))
    codes = list(map(T.dtypes.get, types))
    if None in codes:
        return None
    n, numel, ptr = len(grads), list(map(T.numel, grads)), list(map(T.data_ptr, grads))
    to = ptr
    if outs is not grads:
        if list(map(T.dtype, outs)) != types or list(map(T.shape, outs)) != list(map(T.shape, grads)):
            return None
        to = list(map(T.data_ptr, outs))
    table = array.array("q", bytes(56 * n))
    sizes = array.array("q", numel)
    table[0::7], table[1::7], table[2::7] = array.array("q", ptr), array.array("q", to), array.array("q", [1]) * n
    table[3::7] = table[4::7] = table[5::7] = sizes
    table[6::7] = array.array("q", codes)
    return sum(numel), table


def _clip_table(grads, out, dev):
    """(values, table) of ct_tensor rows, tensor by tensor."""
    index, codes, recording, values, table = dev.index, _names.dtypes, _names.recording(), 0, []
    for i, t in enumerate(grads):
        code = codes.get(t.dtype)
        if code is None or t.get_device() != index or (recording and t.requires_grad):
            raise _bad_values(t, "grads[%d]" % i, dev)
        rows, cols, ld = _layout(t, "grads[%d]" % i)
        p, ldo = t.data_ptr(), ld
        o = p
        if out is not None:
            q = out[i]
            if q.dtype != t.dtype or q.shape != t.shape:
                raise ValueError("out[%d]: %s %s is wanted, got %s %s" % (i, t.dtype, tuple(t.shape), q.dtype, tuple(q.shape)))
            if q.get_device() != index or (recording and q.requires_grad):
                raise _bad_values(q, "out[%d]" % i, dev)
            o = q.data_ptr()
            ldo = _layout(q, "out[%d]" % i)[2]
            if q.stride() != t.stride() and not (t.is_contiguous() and q.is_contiguous()):
                # matrices of different pitches
                if t.dim() != 2 or (t.shape[1] > 1 and (t.stride(1) != 1 or q.stride(1) != 1)):
                    raise ValueError("out[%d]: strides %s are wanted, got %s" % (i, t.stride(), q.stride()))
                rows, cols = t.shape
                ld, ldo = t.stride(0), q.stride(0)
        values += rows * cols
        table += (p, o, rows, cols, ld, ldo, code)
    return values, array.array("q", table)


@functools.lru_cache(maxsize=256)
def _clip_workspace(n, values):
    need = ctypes.c_size_t()
    _check(lib().ct_clip_grads_workspace(n, values, ctypes.byref(need)), "ct_clip_grads_workspace")
    return need.value


def ct_clip_grads(grads, max_norm, kind: float = 2.0, out=None, stream=None):
    """(norm, norms): the norm of the values of all tensors `grads` together
    (float32, no dimension) and of each (float32 [len(grads)]), and the values
    times min(1, max_norm / norm), in place or into `out` (tensors of the same
    types, shapes and strides).  kind: 2 or infinity.  A norm that is NaN or infinite scales
    nothing.  Types may differ from tensor to tensor; none may overlap another."""
    T = _names or _T()
    grads = list(grads)
    if not grads:
        raise ValueError("grads: at least one tensor is wanted")
    n = len(grads)
    if out is not None:
        out = list(out)
        if len(out) != n:
            raise ValueError("out: %d tensors are wanted, got %d" % (n, len(out)))
    if kind != 2 and kind != float("inf"):
        raise ValueError("kind is 2 or infinity, got %r" % (kind,))
    max_norm = float(max_norm)
    if not max_norm >= 0:
        raise ValueError("max_norm: a number of at least 0 is wanted, got %r" % (max_norm,))
    dev = grads[0].device
    if dev.type != "cuda":
        raise ValueError("grads[0]: a CUDA tensor is wanted, got one on %s" % dev)
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_clip_grads, dev, stream, grads, max_norm, kind, out)
    index = dev.index
    fast = _dense_table(grads, grads if out is None else out, index)
    values, table = fast if fast is not None else _clip_table(grads, out, dev)
    norm = T.empty((), dtype=T.f32, device=dev)
    norms = T.empty(n, dtype=T.f32, device=dev)
    need = _clip_workspace(n, values)
    work = T.empty(need, dtype=T.u8, device=dev)
    st = (_lib or lib()).ct_clip_grads(table.buffer_info()[0], n, CT_NORM_2 if kind == 2 else CT_NORM_INF, max_norm, norms.data_ptr(),
                                       norm.data_ptr(), work.data_ptr(), need, T.raw_stream(index))
    if st:
        raise CtError(st, "ct_clip_grads")
    T.raise_versions(grads if out is None else out)
    return norm, norms


@functools.lru_cache(maxsize=256)
def _verify_workspace(sequences, drafts, vocab, most):
    need = ctypes.c_size_t()
    _check(lib().ct_verify_drafts_workspace(sequences, drafts, vocab, most, ctypes.byref(need)), "ct_verify_drafts_workspace")
    return need.value


def ct_verify_drafts(logits, drafts, offsets, max_drafts: int, uniform, noise, draft_logits=None, temperature=None, stream=None):
    """(accepted, token, logprob): drafted tokens held against the target's
    probabilities.  Sequence b has the drafts offsets[b] to offsets[b + 1] - 1 of
    drafts (int64) and as many rows of logits and one more, from row offsets[b] + b
    on; draft_logits [drafts, vocab] are what the drafts were drawn from (None: they
    are certain).  uniform float32 [drafts] in [0, 1) and noise float32 [sequences,
    vocab], exponentially distributed, are the random numbers; temperature
    float32 [sequences] (None: 1; 0: the most probable token).
    accepted int64 [sequences]; token int64 and logprob float32 [sequences,
    max_drafts + 1]: the drafts that stand and the token after them, then -1 and 0."""
    T = _names or _T()
    rows, vocab, ld = _matrix(logits, "logits", T.dtypes)
    dev = logits.device
    if stream is not None or dev.index != T.current_device():
        return _elsewhere(ct_verify_drafts, dev, stream, logits, drafts, offsets, max_drafts, uniform, noise, draft_logits, temperature)
    if drafts.dim() != 1 or offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("drafts and offsets: 1-D tensors are wanted, got shapes %s and %s" % (tuple(drafts.shape), tuple(offsets.shape)))
    count, batch = drafts.shape[0], offsets.shape[0] - 1
    if rows != count + batch:
        raise ValueError("logits: %d rows are wanted (%d drafts, %d sequences), got %d" % (count + batch, count, batch, rows))
    if not 0 <= max_drafts <= CT_MAX_DRAFTS:
        raise ValueError("max_drafts is 0 to %d, got %r" % (CT_MAX_DRAFTS, max_drafts))
    dp, op = _vector(drafts, "drafts", T.i64, count, dev), _vector(offsets, "offsets", T.i64, batch + 1, dev)
    up = _vector(uniform, "uniform", T.f32, count, dev)
    ldn = _matrix(noise, "noise", (T.f32,), (batch, vocab), dev)[2]
    tp = None if temperature is None else _vector(temperature, "temperature", T.f32, batch, dev)
    qp, ldq = None, 0
    if draft_logits is not None:
        ldq = _matrix(draft_logits, "draft_logits", (logits.dtype,), (count, vocab), dev)[2]
        qp = draft_logits.data_ptr()
    accepted = T.empty(batch, dtype=T.i64, device=dev)
    token = T.empty((batch, max_drafts + 1), dtype=T.i64, device=dev)
    logprob = T.empty((batch, max_drafts + 1), dtype=T.f32, device=dev)
    need = _verify_workspace(batch, count, vocab, max_drafts)
    work = T.empty(need, dtype=T.u8, device=dev)
    st = (_lib or lib()).ct_verify_drafts(logits.data_ptr(), T.dtypes[logits.dtype], ld, qp, ldq, dp, op, up, noise.data_ptr(), ldn, tp,
                                          batch, count, vocab, max_drafts, accepted.data_ptr(), token.data_ptr(), logprob.data_ptr(),
                                          work.data_ptr(), need, T.raw_stream(dev.index))
    if st:
        raise CtError(st, "ct_verify_drafts")
    return accepted, token, logprob


def ct_ops_device_error() -> int:
    """Reads and clears the current device's error word of these operators."""
    c = ctypes.c_uint32()
    _check(lib().ct_ops_device_error(ctypes.byref(c)), "ct_ops_device_error")
    return c.value
