"""ctypes declarations of the C ABI in include/hieravg.h (argument marshalling
only: every step of the hot path runs in the HIP library).  Loading fails
loudly when the library has not been built; there is no other code path."""

import ctypes
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhieravg.so")

OK, EINVAL, EHIP, ENONFINITE, ESIZE = 0, -1, -2, -3, -4
KIND_SOFTMAX, KIND_MLP, KIND_AVERAGING = 0, 1, 2
MODEL_SOFTMAX_3072_10, MODEL_MLP_3072_512_10, MODEL_MLP_150528_1024_1000, MODEL_AVERAGING_11_7M = 0, 1, 2, 3


class Config(ctypes.Structure):
    _fields_ = [
        ("P", ctypes.c_int32), ("S", ctypes.c_int32), ("K1", ctypes.c_int32), ("K2", ctypes.c_int32),
        ("B", ctypes.c_int32), ("kind", ctypes.c_int32),
        ("in_dim", ctypes.c_int64), ("hidden", ctypes.c_int64), ("classes", ctypes.c_int64),
        ("n_samples", ctypes.c_int64),
        ("noise_std", ctypes.c_float), ("lr", ctypes.c_float), ("momentum", ctypes.c_float),
        ("init_std", ctypes.c_float), ("grad_std", ctypes.c_float),
        ("seed", ctypes.c_uint64),
        ("update_mode", ctypes.c_int32),
        ("k_global", ctypes.c_int32),
        ("weight_decay", ctypes.c_float),
        ("avg_momentum", ctypes.c_int32),
    ]


class AdamWConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [
        ("seed", ctypes.c_uint64), ("state_bits", ctypes.c_int32)]


class AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("param_type", ctypes.c_int32), ("grad_type", ctypes.c_int32), ("copy_type", ctypes.c_int32)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("type", ctypes.c_int32)]


class Adapters(ctypes.Structure):
    _fields_ = [("down", ctypes.c_void_p), ("up", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("in_", ctypes.c_int64), ("out", ctypes.c_int64),
                ("n", ctypes.c_int32), ("rank", ctypes.c_int32), ("type", ctypes.c_int32)]


_H = ctypes.c_void_p
_I, _L, _Z = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
# name -> (restype, argtypes); the exported symbols of include/hieravg.h
SIGNATURES = {
    "hieravg_create": (_H, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                            ctypes.c_float, ctypes.c_int32, ctypes.c_uint64]),
    "hieravg_create_config": (_H, [ctypes.POINTER(Config)]),
    "hieravg_round": (ctypes.c_int, [_H]),
    "hieravg_params": (ctypes.c_int, [_H, ctypes.c_void_p, ctypes.c_size_t]),
    "hieravg_set_params": (ctypes.c_int, [_H, ctypes.c_void_p, ctypes.c_size_t]),
    "hieravg_destroy": (None, [_H]),
    "hieravg_set_lr": (ctypes.c_int, [_H, ctypes.c_float]),
    "hieravg_set_batch": (ctypes.c_int, [_H, ctypes.c_int32]),
    "hieravg_set_step_count": (ctypes.c_int, [_H, ctypes.c_int64]),
    "hieravg_check_finite": (ctypes.c_int, [_H]),
    "hieravg_momentum": (ctypes.c_int, [_H, ctypes.c_void_p, ctypes.c_size_t]),
    "hieravg_set_momentum": (ctypes.c_int, [_H, ctypes.c_void_p, ctypes.c_size_t]),
    "hieravg_evaluate": (ctypes.c_int, [_H, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64,
                                        ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]),
    "hieravg_evaluate_noalloc": (ctypes.c_int, [_H, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64,
                                                ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]),
    "hieravg_scores": (ctypes.c_int, [_H, _I, _I, _L, _I, _H, _H, _H, _H]),
    "hieravg_last_error": (ctypes.c_char_p, []),
    "hieravg_dim": (ctypes.c_int64, [_H]),
    "hieravg_step_count": (ctypes.c_int64, [_H]),
    "hieravg_last_indices": (ctypes.c_int, [_H, ctypes.c_void_p, ctypes.c_size_t]),
    "hieravg_set_stream": (ctypes.c_int, [_H, ctypes.c_void_p]),
    "hieravg_sync": (ctypes.c_int, [_H]),
    "hieravg_profile": (ctypes.c_int, [_H, ctypes.c_int]),
    "hieravg_profile_read": (ctypes.c_int, [_H, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double),
                                            ctypes.c_int]),
    "hieravg_kernel_classes": (ctypes.c_int, []),
    "hieravg_time_kernel": (ctypes.c_int, [_H, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_double)]),
    "hieravg_kernel_class_name": (ctypes.c_char_p, [ctypes.c_int]),
    "hieravg_log_probs_scratch": (_Z, [_L, _L, _I]),
    "hieravg_log_probs": (ctypes.c_int, [_H, _I, _L, _L, _L, _H, _I, _I, _H, _H, _H, _H, _H, _H, _Z, _H]),
    "hieravg_log_probs_grad": (ctypes.c_int, [_H, _I, _L, _L, _L, _H, _I, _H, _H, _H, _H, _H, _L, _H]),
    "hieravg_adamw_state_size": (_L, [ctypes.POINTER(_L), _I]),
    "hieravg_adamw_create": (_H, [ctypes.POINTER(AdamWConfig), ctypes.POINTER(AdamWTensor), _I, _H, _H, _H, _H]),
    "hieravg_adamw_step": (ctypes.c_int, [_H, _H, _H]),
    "hieravg_adamw_step_scaled": (ctypes.c_int, [_H, _H, _H, _H]),
    "hieravg_adamw_set_lr": (ctypes.c_int, [_H, ctypes.c_double, _H]),
    "hieravg_adamw_set_steps": (ctypes.c_int, [_H, _L, _H]),
    "hieravg_adamw_steps": (_L, [_H]),
    "hieravg_adamw_lr": (ctypes.c_int, [_H, ctypes.POINTER(ctypes.c_double)]),
    "hieravg_adamw_destroy": (None, [_H]),
    "hieravg_quantize_blocks": (ctypes.c_int, [_H, _I, _L, _L, _L, _I, _H, _H, _H, _H, _H]),
    "hieravg_block_product_scratch": (_Z, [_L, _L, _L]),
    "hieravg_block_product": (ctypes.c_int, [_H, _H, _I, _H, _H, _I, _L, _L, _L, _H, _I, _L, _H, _Z, _H]),
    "hieravg_grad_norm_scratch": (_Z, [_H, _I]),
    "hieravg_grad_norm": (ctypes.c_int, [_H, _I, ctypes.c_double, _H, _H, _H, _H, _Z, _H]),
    "hieravg_scale_tensors": (ctypes.c_int, [_H, _H, _I, _H, _H]),
    "hieravg_verify_drafts_scratch": (_Z, [_L, _I, _L, _I]),
    "hieravg_verify_drafts": (ctypes.c_int, [_H, _I, _L, _I, _L, _L, _H, _I, _L, _H, _I, _H, _H, _H, _H, _H, _H, _H,
                                             _Z, _H]),
    "hieravg_adapter_product_scratch": (_Z, [_L, ctypes.POINTER(Adapters)]),
    "hieravg_adapter_product": (ctypes.c_int, [ctypes.POINTER(Adapters), _H, _L, _L, _H, _I, _H, _L, _H, _I, _L, _H,
                                               _H, _Z, _H]),
    "hieravg_adapter_grad_scratch": (_Z, [_L, ctypes.POINTER(Adapters), _I]),
    "hieravg_adapter_dx_scratch": (_Z, [_L, ctypes.POINTER(Adapters)]),
    "hieravg_adapter_grad": (ctypes.c_int, [ctypes.POINTER(Adapters), _H, _L, _L, _H, _L, _H, _I, _H, _H, _L, _H, _I,
                                            _L, _H, _H, _I, _H, _Z, _H]),
}

_lib = None


def lib():
    """The loaded library with its signatures declared."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built (run __graft_entry__.build())")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


class HierAvgError(RuntimeError):
    pass


def check(rc):
    if rc != OK:
        msg = lib().hieravg_last_error().decode()
        raise HierAvgError(f"hieravg error {rc}: {msg}")
    return rc
