"""ctypes loader for libscoot.so (built in-tree by ``build.py``).

Loading never falls back to anything: a missing or stale library raises.
"""
import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libscoot.so")

_lib = None

c_int, c_i64, c_dbl, c_vp = C.c_int, C.c_int64, C.c_double, C.c_void_p
P_dbl, P_int, P_i64 = C.POINTER(C.c_double), C.POINTER(C.c_int), C.POINTER(C.c_int64)
P_i32, P_f32, P_u32 = C.POINTER(C.c_int32), C.POINTER(C.c_float), C.POINTER(C.c_uint32)

# name -> argtypes (every function returns int)
SIGNATURES = {
    "scoot_abi_version": [],
    "scoot_status_string": [c_int],
    "scoot_last_error": [],
    "scoot_gp_factor_host": [P_dbl, P_dbl, c_int, c_int, P_dbl, c_dbl, c_dbl, c_dbl, P_dbl, P_dbl],
    "scoot_gp_fit": [P_dbl, P_dbl, c_int, c_int, P_dbl, c_dbl, c_dbl, c_dbl, c_int, c_vp, C.POINTER(c_vp)],
    "scoot_gp_factor_host_ex": [P_dbl, P_dbl, c_int, c_int, c_int, P_dbl, P_dbl, P_dbl, c_dbl, c_dbl, c_dbl,
                                P_dbl, P_dbl],
    "scoot_gp_fit_ex": [P_dbl, P_dbl, c_int, c_int, c_int, P_dbl, P_dbl, P_dbl, c_dbl, c_dbl, c_dbl, c_int, c_vp,
                        C.POINTER(c_vp)],
    "scoot_gp_fit_device": [P_dbl, P_dbl, c_int, c_int, c_int, P_dbl, P_dbl, P_dbl, c_dbl, c_dbl, c_dbl, c_int,
                            c_vp, C.POINTER(c_vp)],
    "scoot_gp_destroy": [c_vp],
    "scoot_gp_nll": [P_dbl, P_dbl, c_int, c_int, c_int, P_dbl, P_dbl, c_dbl, P_dbl, P_dbl, P_dbl],
    "scoot_gp_mle": [P_dbl, P_dbl, c_int, c_int, c_int, P_dbl, P_dbl, c_dbl, P_dbl, P_dbl, c_int, P_dbl, P_dbl,
                     P_int],
    "scoot_gp_nll_warp": [P_dbl, P_dbl, c_int, c_int, c_int, c_dbl, P_dbl, P_dbl, P_dbl],
    "scoot_gp_mle_warp": [P_dbl, P_dbl, c_int, c_int, c_int, c_dbl, P_dbl, P_dbl, c_int, P_dbl, P_dbl, P_int],
    "scoot_gp_nll_device": [P_dbl, P_dbl, c_int, c_int, c_int, P_dbl, P_dbl, c_dbl, c_int, P_dbl, P_dbl, P_dbl,
                            c_vp],
    "scoot_gp_mle_device": [P_dbl, P_dbl, c_int, c_int, c_int, P_dbl, P_dbl, c_dbl, c_int, P_dbl, P_dbl, c_int,
                            P_dbl, P_dbl, P_int, c_vp],
    "scoot_posterior": [c_vp, c_vp, c_i64, c_vp, c_vp, c_vp],
    "scoot_acq_ei": [c_vp, c_vp, c_i64, c_int, c_dbl, c_dbl, c_vp, c_vp],
    "scoot_ehvi_front": [P_dbl, c_int, c_int, P_dbl, P_dbl, P_int, P_int],
    "scoot_acq_ehvi": [C.POINTER(c_vp), C.POINTER(c_vp), c_int, c_i64, c_int, P_dbl, c_int, P_dbl, c_vp, c_vp],
    "scoot_forest_create": [P_i32, P_f32, P_i32, P_i32, P_i32, P_i64, c_int, c_int, C.POINTER(c_vp)],
    "scoot_forest_destroy": [c_vp],
    "scoot_forest_train": [P_dbl, P_dbl, c_int, c_int, c_int, c_int, C.c_uint64, c_int, c_i64, P_i32, P_dbl, P_i32,
                           P_i32, P_dbl, P_i64, P_i64],
    "scoot_forest_train_create": [P_dbl, P_dbl, c_int, c_int, c_int, c_int, C.c_uint64, c_int, C.POINTER(c_vp)],
    "scoot_vote_threshold": [c_dbl, c_int, P_i64],
    "scoot_rf_feasibility": [c_vp, c_vp, c_i64, c_dbl, c_vp, c_vp, c_vp, c_vp],
    "scoot_suggest_topq": [c_vp, c_vp, c_i64, c_int, c_int, c_vp, c_vp, c_vp, c_vp],
    "scoot_suggest_topq_noalloc": [c_vp, c_vp, c_i64, c_int, c_int, c_vp, c_vp, c_vp, c_vp],
    "scoot_delta_update": [P_dbl, P_int, c_int, c_int],
    "scoot_score_pool": [C.POINTER(c_vp), c_int, c_vp, c_vp, c_i64, c_dbl, c_dbl, P_dbl, c_int, P_dbl,
                         c_dbl, c_int, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp],
    "scoot_suggest_kb_workspace": [C.POINTER(c_vp), c_int, c_i64, c_int, C.POINTER(C.c_uint64)],
    "scoot_suggest_kb": [C.POINTER(c_vp), c_int, c_vp, c_vp, c_i64, P_dbl, c_int, P_dbl, c_dbl, c_int, c_vp,
                         C.c_uint64, P_i64, P_dbl, P_int, c_vp],
    "scoot_ucb_beta": [c_int, P_dbl],
    "scoot_acq_mace": [c_vp, c_vp, c_i64, c_int, c_dbl, c_dbl, c_dbl, c_vp, c_vp, c_vp, c_vp],
    "scoot_pareto_front3": [c_vp, c_vp, c_vp, c_vp, c_i64, c_int, c_vp, c_vp, c_vp],
    "scoot_random_pick": [c_vp, c_i64, C.c_uint64, c_int, c_vp, c_vp, c_vp],
    "scoot_suggest_mace": [c_vp, c_vp, c_vp, c_i64, c_dbl, c_dbl, c_dbl, c_dbl, C.c_uint64, c_int, c_vp, c_vp,
                           c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp],
    "scoot_score_pool_ex": [C.POINTER(c_vp), c_int, c_vp, c_vp, c_vp, c_i64, c_dbl, c_dbl, P_dbl, c_int, P_dbl,
                            c_dbl, c_int, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp],
    "scoot_suggest_kb_ex": [C.POINTER(c_vp), c_int, c_vp, c_vp, c_vp, c_i64, P_dbl, c_int, P_dbl, c_dbl, c_int, c_vp,
                            C.c_uint64, P_i64, P_dbl, P_int, c_vp, c_vp, c_vp],
    "scoot_suggest_mace_ex": [c_vp, c_vp, c_vp, c_vp, c_i64, c_dbl, c_dbl, c_dbl, c_dbl, C.c_uint64, c_int, c_vp,
                              c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp],
    "scoot_sobol_pool": [P_u32, P_u32, c_int, P_i32, c_i64, c_i64, P_dbl, P_dbl, c_int, c_vp, c_vp, c_vp],
    "scoot_known_constraints": [c_vp, c_i64, c_int, P_dbl, P_dbl, c_int, c_vp, c_vp],
    "scoot_suggest": [P_dbl, P_dbl, C.POINTER(C.c_uint8), c_int, c_int, c_vp, c_vp, P_dbl, P_i32, P_dbl, P_int,
                      c_vp],
    "scoot_kv_assign": [c_vp, c_vp, c_int, c_int, c_vp, c_int, c_i64, c_vp, c_int, c_i64, c_vp, c_vp, c_vp, c_vp,
                        c_vp, c_vp],
    "scoot_kv_write": [c_vp, c_vp, c_int, c_i64, c_int, c_int, c_i64, c_i64, c_i64, c_i64, c_vp, c_vp, c_vp, c_int,
                       c_i64, c_int, C.c_float, C.c_float, c_vp],
    "scoot_kv_attention_workspace": [c_i64, c_int, c_int, c_int, c_int, c_i64, c_i64, c_int, C.POINTER(C.c_uint64)],
    "scoot_kv_attention": [c_vp, c_int, c_i64, c_int, c_int, c_int, c_i64, c_i64, c_vp, c_vp, c_int, c_i64, c_int, c_vp,
                           c_int, c_i64, c_vp, c_vp, c_int, c_i64, c_i64, C.c_float, c_int, C.c_float, C.c_float,
                           c_vp, c_i64, c_i64, c_vp, C.c_uint64, c_vp],
}
RESTYPES = {"scoot_status_string": C.c_char_p, "scoot_last_error": C.c_char_p}


class ScootError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{message} (status {status})")
        self.status = status


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2408_04323_amd.build.build() "
                               "(the scoring path has no CPU fallback)")
        # torch ships its own HIP runtime; loaded first, it is the one the
        # library binds to, so device memory and streams are shared.  Loaded
        # after the library, a second runtime ends up in the process and the
        # library's first allocation fails.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        L = C.CDLL(LIB_PATH)
        for name, args in SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = RESTYPES.get(name, c_int)
        _lib = L
    return _lib


def check(status, what):
    if status != 0:
        L = lib()
        raise ScootError(status, f"{what}: {L.scoot_status_string(status).decode()}: "
                                 f"{L.scoot_last_error().decode()}")


def kv_module(raw_stream):
    """The module that makes the key/value cache calls from torch tensors, bound to the loaded library; ``raw_stream``
    gives a device's current stream."""
    path = os.path.join(HERE, "_kv_torch.so")
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2408_04323_amd.build.build()")
    from . import _kv_torch
    at = [C.cast(getattr(lib(), name), c_vp).value
          for name in ("scoot_kv_assign", "scoot_kv_write", "scoot_kv_attention_workspace", "scoot_kv_attention")]
    _kv_torch.bind(*at, raw_stream)
    return _kv_torch
