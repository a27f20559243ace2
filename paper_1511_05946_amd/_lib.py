"""ctypes loader for libacdc.so (the HIP library built in-tree).

Fails loudly when the library is missing: there is no CPU fallback.
"""

from __future__ import annotations

import ctypes
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libacdc.so")

_lib = None

# Exported symbols and their signatures (mirrors include/acdc.h and
# include/acdc_train.h).
_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I32 = ctypes.c_int32
_U32 = ctypes.c_uint32
_SZ = ctypes.c_size_t
_F = ctypes.c_float
_D = ctypes.c_double
# logits, dtype, stride, targets, target_bits: the head of every loss's arguments
_LOGITS = [_P, _I32, _I64, _P, _I32]
SIGNATURES = {
    "acdc_supported": (ctypes.c_int, [_I32, _U32]),
    "acdc_prepare": (ctypes.c_int, [_I32, _U32]),
    "acdc_saved_bytes": (_SZ, [_I64, _I32, _I32, _U32]),
    "acdc_forward_workspace_size": (_SZ, [_I64, _I32, _I32, _U32]),
    "acdc_backward_workspace_size": (_SZ, [_I64, _I32, _I32, _U32, ctypes.c_int]),
    "acdc_forward": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _I64, _I32, _I32, _U32, _P, _SZ, _P, _SZ, _P]),
    "acdc_forward_noalloc": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, _I64, _I32, _I32, _U32, _P, _SZ, _P]),
    "acdc_backward": (ctypes.c_int,
                      [_P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P, _P, _P, _I64, _I32, _I32, _U32, _P, _SZ, _P]),
    "acdc_profile_enable": (ctypes.c_int, [ctypes.c_int]),
    "acdc_profile_read": (ctypes.c_int, [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]),
    "acdc_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "acdc_last_hip_error": (ctypes.c_int, []),
    "acdc_sync_timeouts": (ctypes.c_int, [ctypes.POINTER(ctypes.c_int64), ctypes.c_int]),
    "acdc_logprob_forward": (ctypes.c_int, [*_LOGITS, _I64, _I32, _P, _P, _P, _P, _SZ, _P]),
    "acdc_logprob_workspace_size": (_SZ, [_I64, _I32, _I32]),
    "acdc_logprob_backward": (ctypes.c_int, [*_LOGITS, _P, _P, _P, _P, _P, _I64, _I64, _I32, _P]),
    "acdc_policy_loss": (ctypes.c_int,
                         [*_LOGITS, _P, _P, _P, _P, _I64, _I32, _P, _P, _P, _P, _I64, _P, _P, _P, _SZ, _P]),
    "acdc_policy_workspace_size": (_SZ, [_I64, _I32, _I32]),
    "acdc_preference_loss": (ctypes.c_int,
                             [*_LOGITS, _P, _I32, _P, _I64, _I32, _I64, _P, _P, _P, _P, _I64, _P, _P, _P, _SZ, _P]),
    "acdc_preference_workspace_size": (_SZ, [_I64, _I32, _I32, _I64]),
    "acdc_adamw_step": (ctypes.c_int, [_P, _I32, _D, _D, _D, _I64, _P, _P]),
    "acdc_grad_norm": (ctypes.c_int, [_P, _P, _P, _I32, _F, _P, _P, _SZ, _P]),
    "acdc_grad_norm_workspace_size": (_SZ, [_P, _I32]),
}


class LibraryMissing(RuntimeError):
    pass


def lib():
    """The loaded library (loaded once)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise LibraryMissing(
                f"{LIB_PATH} is not built; run `python -m paper_1511_05946_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


_binding = None


def binding():
    """The native part of the training operators' binding (loaded once)."""
    global _binding
    if _binding is None:
        lib()
        path = os.path.join(os.path.dirname(LIB_PATH), "_train_binding.so")
        if not os.path.exists(path):
            raise LibraryMissing(f"{path} is not built; run `python -m paper_1511_05946_amd.build`")
        import importlib.util

        import torch  # noqa: F401  (the module's own libraries)
        spec = importlib.util.spec_from_file_location("paper_1511_05946_amd._train_binding", path)
        _binding = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(_binding)
    return _binding


def status_string(rc: int) -> str:
    return lib().acdc_status_string(int(rc)).decode()
