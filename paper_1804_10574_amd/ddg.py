"""ctypes binding of libddg.so: same names as include/ddg.h, argument marshalling only."""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import List, Optional, Sequence

import numpy as np

DDG_F32, DDG_BF16 = 0, 1
DDG_OPT_SGD, DDG_OPT_ADAM = 0, 1
_STATUS = {0: "DDG_OK", 1: "DDG_ERR_INVALID_ARG", 2: "DDG_ERR_SHAPE", 3: "DDG_ERR_STATE",
           4: "DDG_ERR_OOM", 5: "DDG_ERR_DEVICE"}

_HERE = os.path.dirname(os.path.abspath(__file__))


def library_path() -> str:
    return os.path.join(_HERE, "libddg.so")


class DDGError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


class BlockDesc(C.Structure):
    _fields_ = [("kind", C.c_int), ("cin", C.c_int), ("cmid", C.c_int), ("cout", C.c_int),
                ("stride", C.c_int), ("projection", C.c_int)]


class ModuleDesc(C.Structure):
    _fields_ = [("K", C.c_int), ("k", C.c_int), ("batch", C.c_int), ("in_c", C.c_int),
                ("in_h", C.c_int), ("in_w", C.c_int), ("num_blocks", C.c_int),
                ("blocks", C.POINTER(BlockDesc)), ("num_classes", C.c_int), ("compute", C.c_int),
                ("momentum", C.c_float), ("weight_decay", C.c_float), ("bn_eps", C.c_float),
                ("stream", C.c_void_p), ("forward_stream", C.c_void_p), ("dry_run", C.c_int),
                ("stale_jacobian", C.c_int)]


class DropoutDesc(C.Structure):
    _fields_ = [("rows", C.c_int), ("cols", C.c_int), ("dtype", C.c_int), ("p", C.c_float), ("seed", C.c_uint64),
                ("ld_x", C.c_long), ("ld_y", C.c_long), ("stream", C.c_void_p), ("dry_run", C.c_int)]


class JoinDesc(C.Structure):
    _fields_ = [("rows", C.c_int), ("cols", C.c_int), ("dtype", C.c_int), ("eps", C.c_float), ("p", C.c_float),
                ("seed", C.c_uint64), ("ld_y", C.c_long), ("ld_residual", C.c_long), ("ld_x", C.c_long),
                ("ld_out", C.c_long), ("group", C.c_int), ("stream", C.c_void_p), ("dry_run", C.c_int)]


class VocabDesc(C.Structure):
    _fields_ = [("tokens", C.c_int), ("dim", C.c_int), ("vocab", C.c_int), ("dtype", C.c_int), ("ld_h", C.c_long),
                ("ld_w", C.c_long), ("ld_dh", C.c_long), ("ld_dw", C.c_long), ("dw_f32", C.c_int),
                ("stream", C.c_void_p), ("dry_run", C.c_int), ("unaligned", C.c_int)]


class RotaryDesc(C.Structure):
    _fields_ = [("rows", C.c_int), ("heads", C.c_int), ("dim", C.c_int), ("dtype", C.c_int), ("rot", C.c_int), ("interleaved", C.c_int),
                ("base", C.c_double), ("factor", C.c_double), ("context", C.c_double), ("low", C.c_double), ("high", C.c_double), ("magnitude", C.c_float),
                ("ld_x", C.c_long), ("ld_y", C.c_long), ("stream", C.c_void_p), ("dry_run", C.c_int)]


class LinearDesc(C.Structure):
    _fields_ = [("rows", C.c_int), ("sequences", C.c_int), ("heads", C.c_int), ("kv_heads", C.c_int), ("dim_k", C.c_int), ("dim_v", C.c_int),
                ("dtype", C.c_int), ("slots", C.c_int), ("scale", C.c_float), ("ld_q", C.c_long), ("ld_k", C.c_long), ("ld_v", C.c_long), ("ld_o", C.c_long),
                ("stream", C.c_void_p), ("dry_run", C.c_int)]


class GatedJoinDesc(C.Structure):
    _fields_ = [("rows", C.c_int), ("cols", C.c_int), ("dtype", C.c_int), ("eps", C.c_float), ("scale", C.c_float), ("residual_scale", C.c_float),
                ("group", C.c_int), ("gate", C.c_int), ("ld_y", C.c_long), ("ld_gate", C.c_long), ("ld_residual", C.c_long), ("ld_x", C.c_long),
                ("ld_out", C.c_long), ("stream", C.c_void_p), ("dry_run", C.c_int)]


_lib = None


def load_library():
    """Load libddg.so built in-tree (python -m paper_1804_10574_amd.build). Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: build it first (python paper_1804_10574_amd/build.py). "
            "There is no CPU fallback.")
    lib = C.CDLL(path)
    vp, st = C.c_void_p, C.c_int
    sig = {
        "ddg_module_create": (st, [C.POINTER(ModuleDesc), C.POINTER(vp)]),
        "ddg_module_destroy": (st, [vp]),
        "ddg_param_count": (C.c_size_t, [vp]),
        "ddg_out_shape": (st, [vp, C.POINTER(C.c_int), C.POINTER(C.c_int), C.POINTER(C.c_int)]),
        "ddg_device_bytes": (C.c_size_t, [vp]),
        "ddg_set_params": (st, [vp, vp, C.c_int]),
        "ddg_set_velocity": (st, [vp, vp, C.c_int]),
        "ddg_get_params": (st, [vp, vp]),
        "ddg_get_velocity": (st, [vp, vp]),
        "ddg_get_grad": (st, [vp, vp, C.POINTER(C.c_int)]),
        "ddg_forward": (st, [vp, C.c_long, vp, vp]),
        "ddg_backward_delayed": (st, [vp, C.c_long, vp, vp, vp, vp, C.POINTER(C.c_int)]),
        "ddg_update": (st, [vp, C.c_long, C.c_float]),
        "ddg_set_optimizer": (st, [vp, C.c_int, C.c_float, C.c_float, C.c_float]),
        "ddg_set_moment2": (st, [vp, vp, C.c_int]),
        "ddg_get_moment2": (st, [vp, vp]),
        "ddg_set_update_count": (st, [vp, C.c_long]),
        "ddg_get_update_count": (C.c_long, [vp]),
        "ddg_pipeline_set_optimizer": (st, [vp, C.c_int, C.c_float, C.c_float, C.c_float]),
        "ddg_set_bn_momentum": (st, [vp, C.c_float]),
        "ddg_running_count": (C.c_size_t, [vp]),
        "ddg_get_running": (st, [vp, vp]),
        "ddg_set_running": (st, [vp, vp]),
        "ddg_forward_eval": (st, [vp, vp, vp, vp, vp, vp]),
        "ddg_forward_eval_static": (st, [vp, vp, vp, vp, vp, vp]),
        "ddg_pipeline_forward_eval": (st, [vp, vp, vp, vp, vp]),
        "ddg_pipeline_set_bn_momentum": (st, [vp, C.c_float]),
        "ddg_module_sync": (st, [vp]),
        "ddg_ring_slots": (C.c_int, [vp]),
        "ddg_ring_slot_bytes": (C.c_size_t, [vp]),
        "ddg_get_ring_slot": (st, [vp, C.c_int, vp]),
        "ddg_set_ring_slot": (st, [vp, C.c_int, vp]),
        "ddg_set_time": (st, [vp, C.c_long]),
        "ddg_get_time": (C.c_long, [vp]),
        "ddg_pipeline_time": (C.c_long, [vp]),
        "ddg_pipeline_set_time": (st, [vp, C.c_long]),
        "ddg_pipeline_mail_bytes": (C.c_size_t, [vp, C.c_int]),
        "ddg_pipeline_get_mail": (st, [vp, C.c_int, vp, C.POINTER(C.c_long)]),
        "ddg_pipeline_set_mail": (st, [vp, C.c_int, vp, C.c_long]),
        "ddg_pipeline_create": (st, [C.POINTER(ModuleDesc), C.c_int, C.POINTER(vp), C.POINTER(vp)]),
        "ddg_pipeline_destroy": (st, [vp]),
        "ddg_pipeline_module": (vp, [vp, C.c_int]),
        "ddg_pipeline_step": (st, [vp, vp, vp, C.c_float, vp]),
        "ddg_pipeline_set_graphs": (st, [vp, C.c_int]),
        "ddg_pipeline_get_h": (st, [vp, C.c_int, vp]),
        "ddg_pipeline_get_delta": (st, [vp, C.c_int, vp, C.POINTER(C.c_long)]),
        "ddg_pipeline_sync": (st, [vp]),
        "ddg_profile_kinds": (C.c_int, []),
        "ddg_profile_kind_name": (C.c_char_p, [C.c_int]),
        "ddg_profile_enable": (st, [vp, C.c_int]),
        "ddg_profile_read": (st, [vp, C.c_int, C.POINTER(C.c_long), C.POINTER(C.c_double),
                                  C.POINTER(C.c_double), C.POINTER(C.c_double)]),
        "ddg_profile_reset": (st, [vp]),
        "ddg_dropout": (st, [C.POINTER(DropoutDesc), C.c_uint64, vp, vp]),
        "ddg_join_norm": (st, [C.POINTER(JoinDesc), C.c_uint64] + [vp] * 6),
        "ddg_join_norm_q8": (st, [C.POINTER(JoinDesc), C.c_uint64] + [vp] * 7),
        "ddg_join_norm_workspace": (C.c_size_t, [C.POINTER(JoinDesc)]),
        "ddg_join_norm_backward": (st, [C.POINTER(JoinDesc), C.c_uint64] + [vp] * 9 + [C.c_size_t]),
        "ddg_vocab_loss_workspace": (C.c_size_t, [C.POINTER(VocabDesc), C.c_int]),
        "ddg_vocab_loss": (st, [C.POINTER(VocabDesc)] + [vp] * 10 + [C.c_size_t]),
        "ddg_rotary_table": (st, [C.POINTER(RotaryDesc), vp]),
        "ddg_rotary": (st, [C.POINTER(RotaryDesc), vp, vp, C.c_long, vp, C.c_int, vp]),
        "ddg_linear_attention_workspace": (C.c_size_t, [C.POINTER(LinearDesc), C.c_int]),
        "ddg_linear_attention": (st, [C.POINTER(LinearDesc)] + [vp] * 10 + [C.c_size_t]),
        "ddg_linear_attention_backward": (st, [C.POINTER(LinearDesc)] + [vp] * 14 + [C.c_size_t]),
        "ddg_linear_attention_step": (st, [C.POINTER(LinearDesc)] + [vp] * 8),
        "ddg_gated_join": (st, [C.POINTER(GatedJoinDesc)] + [vp] * 9),
        "ddg_gated_join_workspace": (C.c_size_t, [C.POINTER(GatedJoinDesc)]),
        "ddg_gated_join_backward": (st, [C.POINTER(GatedJoinDesc)] + [vp] * 15 + [C.c_size_t]),
        "ddg_last_error": (C.c_char_p, []),
        "ddg_version": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


EXPORTS = ["ddg_module_create", "ddg_module_destroy", "ddg_param_count", "ddg_out_shape",
           "ddg_device_bytes", "ddg_set_params", "ddg_set_velocity", "ddg_get_params", "ddg_get_velocity", "ddg_get_grad",
           "ddg_forward", "ddg_backward_delayed", "ddg_update", "ddg_module_sync",
           "ddg_set_optimizer", "ddg_set_moment2", "ddg_get_moment2", "ddg_set_update_count", "ddg_get_update_count",
           "ddg_pipeline_set_optimizer",
           "ddg_set_bn_momentum", "ddg_running_count", "ddg_get_running", "ddg_set_running", "ddg_forward_eval", "ddg_forward_eval_static",
           "ddg_pipeline_forward_eval", "ddg_pipeline_set_bn_momentum",
           "ddg_pipeline_create", "ddg_pipeline_destroy", "ddg_pipeline_module", "ddg_pipeline_step",
           "ddg_pipeline_set_graphs", "ddg_pipeline_get_h", "ddg_pipeline_get_delta", "ddg_pipeline_sync", "ddg_profile_kinds",
           "ddg_profile_kind_name", "ddg_profile_enable", "ddg_profile_read", "ddg_profile_reset",
           "ddg_ring_slots", "ddg_ring_slot_bytes", "ddg_get_ring_slot", "ddg_set_ring_slot", "ddg_set_time", "ddg_get_time",
           "ddg_pipeline_time", "ddg_pipeline_set_time", "ddg_pipeline_mail_bytes", "ddg_pipeline_get_mail",
           "ddg_pipeline_set_mail",
           "ddg_dropout", "ddg_join_norm", "ddg_join_norm_q8", "ddg_join_norm_workspace", "ddg_join_norm_backward",
           "ddg_vocab_loss_workspace", "ddg_vocab_loss",
           "ddg_rotary_table", "ddg_rotary", "ddg_linear_attention_workspace", "ddg_linear_attention", "ddg_linear_attention_backward",
           "ddg_linear_attention_step", "ddg_gated_join", "ddg_gated_join_workspace", "ddg_gated_join_backward",
           "ddg_last_error", "ddg_version"]


def _check(status: int):
    if status != 0:
        raise DDGError(status, load_library().ddg_last_error().decode())


def version() -> str:
    return load_library().ddg_version().decode()


def profile_kinds() -> List[str]:
    lib = load_library()
    return [lib.ddg_profile_kind_name(i).decode() for i in range(lib.ddg_profile_kinds())]


def _ptr(t) -> Optional[int]:
    """Device (or host) address of a torch tensor / numpy array / int / None."""
    if t is None:
        return None
    try:
        return t.data_ptr()
    except AttributeError:
        return t if isinstance(t, int) else t.ctypes.data


def make_desc(K, k, batch, in_chw, blocks: Sequence[Sequence[int]], num_classes, compute, momentum,
              weight_decay, bn_eps, stream=None, dry_run=False, forward_stream=None, stale_jacobian=False):
    arr = (BlockDesc * len(blocks))(*[BlockDesc(*b) for b in blocks])
    d = ModuleDesc(K, k, batch, in_chw[0], in_chw[1], in_chw[2], len(blocks), arr, num_classes,
                   compute, momentum, weight_decay, bn_eps, stream, forward_stream, 1 if dry_run else 0,
                   1 if stale_jacobian else 0)
    d._keep = arr
    return d


class Module:
    """One module G(k): ddg_forward / ddg_backward_delayed / ddg_update."""

    def __init__(self, desc: ModuleDesc = None, handle=None, owner=None):
        self._lib = load_library()
        self._owner = owner
        if handle is not None:
            self._h = C.c_void_p(handle)
            return
        h = C.c_void_p()
        _check(self._lib.ddg_module_create(C.byref(desc), C.byref(h)))
        self._h = h

    def close(self):
        if self._owner is None and self._h:
            self._lib.ddg_module_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def param_count(self) -> int:
        return int(self._lib.ddg_param_count(self._h))

    def device_bytes(self) -> int:
        return int(self._lib.ddg_device_bytes(self._h))

    def out_shape(self):
        c, h, w = C.c_int(), C.c_int(), C.c_int()
        _check(self._lib.ddg_out_shape(self._h, C.byref(c), C.byref(h), C.byref(w)))
        return c.value, h.value, w.value

    def set_params(self, src, is_device=False):
        if not is_device:
            src = np.ascontiguousarray(src, np.float32)
            assert src.size == self.param_count()
        _check(self._lib.ddg_set_params(self._h, _ptr(src), 1 if is_device else 0))

    def set_velocity(self, src, is_device=False):
        if not is_device:
            src = np.ascontiguousarray(src, np.float32)
            assert src.size == self.param_count()
        _check(self._lib.ddg_set_velocity(self._h, _ptr(src), 1 if is_device else 0))

    def set_optimizer(self, kind, beta1=0.9, beta2=0.999, eps=1e-8):
        _check(self._lib.ddg_set_optimizer(self._h, kind, beta1, beta2, eps))

    def set_moment2(self, src, is_device=False):
        if not is_device:
            src = np.ascontiguousarray(src, np.float32)
            assert src.size == self.param_count()
        _check(self._lib.ddg_set_moment2(self._h, _ptr(src), 1 if is_device else 0))

    def get_moment2(self):
        out, st = self._get(self._lib.ddg_get_moment2)
        _check(st)
        return out

    def set_update_count(self, n):
        _check(self._lib.ddg_set_update_count(self._h, n))

    def get_update_count(self) -> int:
        return int(self._lib.ddg_get_update_count(self._h))

    def _get(self, fn):
        out = np.empty(self.param_count(), np.float32)
        return out, fn(self._h, _ptr(out))

    # evaluation: running BN estimates (per conv unit in parameter order: mean[C], variance[C])
    def set_bn_momentum(self, rho):
        _check(self._lib.ddg_set_bn_momentum(self._h, rho))

    def running_count(self) -> int:
        return int(self._lib.ddg_running_count(self._h))

    def get_running(self):
        out = np.empty(self.running_count(), np.float32)
        _check(self._lib.ddg_get_running(self._h, _ptr(out)))
        return out

    def set_running(self, src):
        src = np.ascontiguousarray(src, np.float32)
        assert src.size == self.running_count()
        _check(self._lib.ddg_set_running(self._h, _ptr(src)))

    def forward_eval(self, h_in, h_out=None, labels=None, loss_out=None, logits_out=None):
        _check(self._lib.ddg_forward_eval(self._h, _ptr(h_in), _ptr(h_out), _ptr(labels), _ptr(loss_out),
                                          _ptr(logits_out)))

    def forward_eval_static(self, h_in, h_out=None, labels=None, loss_out=None, logits_out=None):
        _check(self._lib.ddg_forward_eval_static(self._h, _ptr(h_in), _ptr(h_out), _ptr(labels), _ptr(loss_out),
                                                 _ptr(logits_out)))

    def get_params(self):
        out = np.empty(self.param_count(), np.float32)
        _check(self._lib.ddg_get_params(self._h, _ptr(out)))
        return out

    def get_velocity(self):
        out = np.empty(self.param_count(), np.float32)
        _check(self._lib.ddg_get_velocity(self._h, _ptr(out)))
        return out

    def get_grad(self):
        out = np.empty(self.param_count(), np.float32)
        valid = C.c_int()
        _check(self._lib.ddg_get_grad(self._h, _ptr(out), C.byref(valid)))
        return out if valid.value else None

    def forward(self, t, h_in, h_out):
        _check(self._lib.ddg_forward(self._h, t, _ptr(h_in), _ptr(h_out)))

    def backward_delayed(self, t, delta_in=None, labels=None, delta_out=None, loss_out=None) -> bool:
        did = C.c_int()
        _check(self._lib.ddg_backward_delayed(self._h, t, _ptr(delta_in), _ptr(labels), _ptr(delta_out),
                                              _ptr(loss_out), C.byref(did)))
        return bool(did.value)

    def update(self, t, lr):
        _check(self._lib.ddg_update(self._h, t, lr))

    def sync(self):
        _check(self._lib.ddg_module_sync(self._h))

    # checkpoint of the delay ring: raw slots (bytes of the compute type) and the iteration counter
    def ring_slots(self) -> int:
        return int(self._lib.ddg_ring_slots(self._h))

    def get_ring_slot(self, slot):
        out = np.empty(int(self._lib.ddg_ring_slot_bytes(self._h)), np.uint8)
        _check(self._lib.ddg_get_ring_slot(self._h, slot, _ptr(out)))
        return out

    def set_ring_slot(self, slot, src):
        src = np.ascontiguousarray(src, np.uint8)
        assert src.size == int(self._lib.ddg_ring_slot_bytes(self._h))
        _check(self._lib.ddg_set_ring_slot(self._h, slot, _ptr(src)))

    def set_time(self, t):
        _check(self._lib.ddg_set_time(self._h, t))

    def get_time(self) -> int:
        return int(self._lib.ddg_get_time(self._h))

    def profile_enable(self, on=True):
        _check(self._lib.ddg_profile_enable(self._h, 1 if on else 0))

    def profile_reset(self):
        _check(self._lib.ddg_profile_reset(self._h))

    def profile_read(self):
        """-> {kind name: (launches, total_ms, algorithmic bytes, algorithmic flops)}"""
        out = {}
        for i, name in enumerate(profile_kinds()):
            n, ms, nb, fl = C.c_long(), C.c_double(), C.c_double(), C.c_double()
            _check(self._lib.ddg_profile_read(self._h, i, C.byref(n), C.byref(ms), C.byref(nb), C.byref(fl)))
            out[name] = (n.value, ms.value, nb.value, fl.value)
        return out


class Pipeline:
    """K modules as concurrent streams: ddg_pipeline_*."""

    def __init__(self, descs: Sequence[ModuleDesc], streams: Optional[Sequence[int]] = None):
        self._lib = load_library()
        K = len(descs)
        arr = (ModuleDesc * K)(*descs)
        self._keep = (arr, list(descs))
        sp = None
        if streams is not None:
            sp = (C.c_void_p * K)(*[C.c_void_p(s) for s in streams])
        h = C.c_void_p()
        _check(self._lib.ddg_pipeline_create(arr, K, sp, C.byref(h)))
        self._h = h
        self.K = K
        self.batch = descs[0].batch

    def close(self):
        if self._h:
            self._lib.ddg_pipeline_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def module(self, k) -> Module:
        return Module(handle=self._lib.ddg_pipeline_module(self._h, k), owner=self)

    def step(self, x, labels, lr, loss_out=None):
        _check(self._lib.ddg_pipeline_step(self._h, _ptr(x), _ptr(labels), lr, _ptr(loss_out)))

    def set_graphs(self, on: bool):
        _check(self._lib.ddg_pipeline_set_graphs(self._h, 1 if on else 0))

    def set_optimizer(self, kind, beta1=0.9, beta2=0.999, eps=1e-8):
        _check(self._lib.ddg_pipeline_set_optimizer(self._h, kind, beta1, beta2, eps))

    def set_bn_momentum(self, rho):
        _check(self._lib.ddg_pipeline_set_bn_momentum(self._h, rho))

    def forward_eval(self, x, labels=None, loss_out=None, logits_out=None):
        _check(self._lib.ddg_pipeline_forward_eval(self._h, _ptr(x), _ptr(labels), _ptr(loss_out), _ptr(logits_out)))

    def sync(self):
        _check(self._lib.ddg_pipeline_sync(self._h))

    # checkpoint of the pipeline's own state: the iteration counter and the error gradients in flight
    def time(self) -> int:
        return int(self._lib.ddg_pipeline_time(self._h))

    def set_time(self, t):
        _check(self._lib.ddg_pipeline_set_time(self._h, t))

    def get_mail(self, k):
        """-> (raw bytes of the gradient in flight to module k, its iteration), or (None, -1)."""
        out = np.empty(int(self._lib.ddg_pipeline_mail_bytes(self._h, k)), np.uint8)
        it = C.c_long()
        _check(self._lib.ddg_pipeline_get_mail(self._h, k, _ptr(out), C.byref(it)))
        return (out, it.value) if it.value >= 0 else (None, -1)

    def set_mail(self, k, src, iteration):
        src = np.ascontiguousarray(src, np.uint8)
        assert src.size == int(self._lib.ddg_pipeline_mail_bytes(self._h, k))
        _check(self._lib.ddg_pipeline_set_mail(self._h, k, _ptr(src), iteration))

    def get_h(self, k):
        c, h, w = self.module(k).out_shape()
        out = np.empty((self.batch, h, w, c), np.float32)
        _check(self._lib.ddg_pipeline_get_h(self._h, k, _ptr(out)))
        return out

    def get_delta(self, k):
        c, h, w = self.module(k).out_shape()
        out = np.empty((self.batch, h, w, c), np.float32)
        it = C.c_long()
        _check(self._lib.ddg_pipeline_get_delta(self._h, k, _ptr(out), C.byref(it)))
        return (out, it.value) if it.value >= 0 else (None, -1)


# ---- operators of token models: a descriptor each, tensors and workspace are the caller's --------
# (Small calls take as long as the host needs for them: functions and descriptors are looked up once.)

def _bytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size() if hasattr(t, "data_ptr") else t.nbytes


class Dropout:
    """ddg_dropout on [rows][cols]: the same call on the error gradient is its backward pass."""

    def __init__(self, rows, cols, dtype, p, seed=0, ld_x=0, ld_y=0, stream=None, dry_run=False):
        self.desc = DropoutDesc(rows, cols, dtype, p, seed, ld_x, ld_y, stream, 1 if dry_run else 0)
        self._d, self._call = C.byref(self.desc), load_library().ddg_dropout

    def __call__(self, x, y, step=0):
        status = self._call(self._d, step, _ptr(x), _ptr(y))
        if status:
            _check(status)


class JoinNorm:
    """Join of a residual branch with its norm: ddg_join_norm, ddg_join_norm_q8, ddg_join_norm_backward."""

    def __init__(self, rows, cols, dtype, eps=1e-6, p=0.0, seed=0, ld_y=0, ld_residual=0, ld_x=0, ld_out=0, group=0,
                 stream=None, dry_run=False):
        self.desc = JoinDesc(rows, cols, dtype, eps, p, seed, ld_y, ld_residual, ld_x, ld_out, group, stream,
                             1 if dry_run else 0)
        lib = load_library()
        self._d, self._space = C.byref(self.desc), lib.ddg_join_norm_workspace
        self._forward, self._q8, self._backward = lib.ddg_join_norm, lib.ddg_join_norm_q8, lib.ddg_join_norm_backward

    def workspace_bytes(self) -> int:
        """Bytes that `backward` needs for d_gain."""
        return int(self._space(self._d))

    def forward(self, y, residual, gain, out, x_out=None, rstd=None, step=0):
        status = self._forward(self._d, step, _ptr(y), _ptr(residual), _ptr(gain), _ptr(x_out), _ptr(out), _ptr(rstd))
        if status:
            _check(status)

    def forward_q8(self, y, residual, gain, q, scale, x_out=None, rstd=None, step=0):
        status = self._q8(self._d, step, _ptr(y), _ptr(residual), _ptr(gain), _ptr(x_out), _ptr(q), _ptr(scale), _ptr(rstd))
        if status:
            _check(status)

    def backward(self, x, rstd, gain, d_out, d_x=None, d_residual=None, d_y=None, d_gain=None, workspace=None, step=0):
        status = self._backward(self._d, step, _ptr(x), _ptr(rstd), _ptr(gain), _ptr(d_out), _ptr(d_x), _ptr(d_residual), _ptr(d_y),
                                _ptr(d_gain), _ptr(workspace), _bytes(workspace))
        if status:
            _check(status)


@functools.lru_cache(maxsize=None)
def _is_int32(dtype) -> bool:
    return str(dtype).rpartition(".")[2] == "int32"


def _int32(t, name):
    """Whole numbers are 64 bits in torch and numpy unless asked otherwise; addresses are the caller's word."""
    dtype = getattr(t, "dtype", None)
    if dtype is None:
        return
    whole = t.is_contiguous() if hasattr(t, "is_contiguous") else t.flags.c_contiguous
    if not whole or not _is_int32(dtype):
        raise DDGError(1, f"{name} must be int32, next to each other ({dtype}, strides {t.stride() if hasattr(t, 'stride') else t.strides})")


def _on_device(t, name):
    """Kernels fault on memory of the host that is not pinned."""
    if isinstance(t, np.ndarray) or not (getattr(t, "is_cuda", True) or t.is_pinned()):
        raise DDGError(1, f"{name} must be on the device: copy it there")


def _index(t, name, count):
    """`count` int32 numbers or more on the device, next to each other."""
    try:
        if t is None or t.is_cuda and t.numel() >= count and t.is_contiguous() and _is_int32(t.dtype):
            return
    except AttributeError:                                     # addresses, arrays
        pass
    _int32(t, name)
    _on_device(t, name)
    if hasattr(t, "numel") and t.numel() < count:
        raise DDGError(1, f"{name} must be {count} or more numbers ({t.numel()})")


class VocabLoss:
    """ddg_vocab_loss: softmax cross entropy over a vocabulary and its gradients, without the logits. unaligned: workspace_bytes
    leaves room for an h or w off 16 bytes."""

    def __init__(self, tokens, dim, vocab, dtype, ld_h=0, ld_w=0, ld_dh=0, ld_dw=0, dw_f32=False, stream=None, dry_run=False,
                 unaligned=False):
        self.desc = VocabDesc(tokens, dim, vocab, dtype, ld_h, ld_w, ld_dh, ld_dw, 1 if dw_f32 else 0, stream,
                              1 if dry_run else 0, 1 if unaligned else 0)
        lib = load_library()
        self._d, self._call, self._space = C.byref(self.desc), lib.ddg_vocab_loss, lib.ddg_vocab_loss_workspace

    def workspace_bytes(self, gradients=True) -> int:
        return int(self._space(self._d, 1 if gradients else 0))

    def __call__(self, h, w, targets, weights=None, loss=None, row_loss=None, lse=None, dh=None, dw=None, workspace=None):
        _int32(targets, "targets")
        status = self._call(self._d, _ptr(h), _ptr(w), _ptr(targets), _ptr(weights), _ptr(loss), _ptr(row_loss), _ptr(lse), _ptr(dh),
                            _ptr(dw), _ptr(workspace), _bytes(workspace))
        if status:
            _check(status)


class Rotary:
    """ddg_rotary on [rows][heads * dim]; inverse=True on the error gradient is its backward pass. `table` is what table() returns, copied to
    the device once; its 64-bit words may be of any 8-byte type there, next to each other."""

    def __init__(self, rows, heads, dim, dtype, rot=0, interleaved=False, base=10000.0, factor=1.0, context=0, low=1.0, high=32.0, magnitude=1.0, ld_x=0,
                 ld_y=0, stream=None, dry_run=False):
        self.desc = RotaryDesc(rows, heads, dim, dtype, rot, 1 if interleaved else 0, base, factor, context, low, high, magnitude, ld_x, ld_y, stream,
                               1 if dry_run else 0)
        lib = load_library()
        self._d, self._call, self._table = C.byref(self.desc), lib.ddg_rotary, lib.ddg_rotary_table
        self._need = (rot or dim) // 2 * 8

    def table(self) -> np.ndarray:
        """The frequencies as 64-bit fractions of a turn, on the host."""
        out = np.empty(max(1, (self.desc.rot or self.desc.dim) // 2), np.uint64)
        _check(self._table(self._d, _ptr(out)))
        return out

    def _look_at(self, table):
        _on_device(table, "table")
        if hasattr(table, "element_size") and (table.element_size() != 8 or table.numel() * 8 < self._need or not table.is_contiguous()):
            raise DDGError(1, f"table must be {self._need // 8} words of 64 bits, next to each other ({table.numel()} of {table.element_size()} bytes)")

    def __call__(self, x, y, table, positions=None, first=0, inverse=False):
        try:
            source, words, target = x.data_ptr(), table.data_ptr(), y.data_ptr()
            ready = table.is_cuda and table.itemsize == 8 and table.nbytes >= self._need and table.is_contiguous()
        except AttributeError:                                 # addresses, arrays
            source, words, target, ready = _ptr(x), _ptr(table), _ptr(y), False
        if not ready:
            self._look_at(table)
        _index(positions, "positions", self.desc.rows)
        status = self._call(self._d, source, _ptr(positions), first, words, 1 if inverse else 0, target)
        if status:
            _check(status)


class LinearAttention:
    """Linear attention with a decay for each head: ddg_linear_attention, ddg_linear_attention_backward, ddg_linear_attention_step."""

    def __init__(self, rows, heads, dim_k, dim_v, dtype, sequences=1, kv_heads=0, scale=None, slots=0, ld_q=0, ld_k=0, ld_v=0, ld_o=0, stream=None,
                 dry_run=False):
        if scale is None:
            scale = dim_k ** -0.5 if dim_k > 0 else 1.0
        self.desc = LinearDesc(rows, sequences, heads, kv_heads, dim_k, dim_v, dtype, slots, scale, ld_q, ld_k, ld_v, ld_o, stream, 1 if dry_run else 0)
        lib = load_library()
        self._d, self._space = C.byref(self.desc), lib.ddg_linear_attention_workspace
        self._forward, self._backward, self._step = lib.ddg_linear_attention, lib.ddg_linear_attention_backward, lib.ddg_linear_attention_step

    def workspace_bytes(self, backward=False) -> int:
        return int(self._space(self._d, 1 if backward else 0))

    def forward(self, q, k, v, log_decay, o, starts=None, slots=None, state_in=None, state_out=None, workspace=None):
        _index(starts, "starts", self.desc.sequences + 1)
        _index(slots, "slots", self.desc.sequences)
        status = self._forward(self._d, _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(starts), _ptr(slots), _ptr(state_in), _ptr(o), _ptr(state_out),
                               _ptr(workspace), _bytes(workspace))
        if status:
            _check(status)

    def backward(self, q, k, v, log_decay, d_o, dq=None, dk=None, dv=None, starts=None, slots=None, state_in=None, d_state_out=None, d_state_in=None,
                 workspace=None):
        _index(starts, "starts", self.desc.sequences + 1)
        _index(slots, "slots", self.desc.sequences)
        status = self._backward(self._d, _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(starts), _ptr(slots), _ptr(state_in), _ptr(d_o), _ptr(d_state_out),
                                _ptr(dq), _ptr(dk), _ptr(dv), _ptr(d_state_in), _ptr(workspace), _bytes(workspace))
        if status:
            _check(status)

    def step(self, q, k, v, log_decay, o, slots=None, state_in=None, state_out=None):
        """One row of every sequence."""
        _index(slots, "slots", self.desc.rows)
        status = self._step(self._d, _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(slots), _ptr(state_in), _ptr(o), _ptr(state_out))
        if status:
            _check(status)


GATES = {"none": 0, "column": 1, "plain": 2, "sigmoid": 3, "silu": 4}


class GatedJoin:
    """Norm after a block, its gate, the residual and the norm before the next block: ddg_gated_join, ddg_gated_join_backward. gate: a key of GATES."""

    def __init__(self, rows, cols, dtype, eps=1e-6, gate="none", group=0, scale=1.0, residual_scale=1.0, ld_y=0, ld_gate=0, ld_residual=0, ld_x=0, ld_out=0,
                 stream=None, dry_run=False):
        if gate not in GATES:
            raise DDGError(1, f"gate must be one of {', '.join(GATES)} ({gate!r})")
        self.desc = GatedJoinDesc(rows, cols, dtype, eps, scale, residual_scale, group, GATES[gate], ld_y, ld_gate, ld_residual, ld_x, ld_out, stream,
                                  1 if dry_run else 0)
        lib = load_library()
        self._d, self._space = C.byref(self.desc), lib.ddg_gated_join_workspace
        self._forward, self._backward = lib.ddg_gated_join, lib.ddg_gated_join_backward

    def workspace_bytes(self) -> int:
        """Bytes that `backward` needs for sums over rows."""
        return int(self._space(self._d))

    def forward(self, y, gate, residual, gain_y, gain_x, x_out=None, out=None, rstd_y=None, rstd_x=None):
        status = self._forward(self._d, _ptr(y), _ptr(gate), _ptr(residual), _ptr(gain_y), _ptr(gain_x), _ptr(x_out), _ptr(out), _ptr(rstd_y), _ptr(rstd_x))
        if status:
            _check(status)

    def backward(self, y, rstd_y, gate, x, rstd_x, gain_y, gain_x, d_out=None, d_x=None, d_residual=None, d_y=None, d_gate=None, d_gain_y=None, d_gain_x=None,
                 workspace=None):
        status = self._backward(self._d, _ptr(y), _ptr(rstd_y), _ptr(gate), _ptr(x), _ptr(rstd_x), _ptr(gain_y), _ptr(gain_x), _ptr(d_out), _ptr(d_x),
                                _ptr(d_residual), _ptr(d_y), _ptr(d_gate), _ptr(d_gain_y), _ptr(d_gain_x), _ptr(workspace), _bytes(workspace))
        if status:
            _check(status)
