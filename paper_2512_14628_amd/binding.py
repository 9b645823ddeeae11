"""ctypes binding of the C ABI declared in include/hsadmm.h (argument marshalling only).

Device buffers are torch tensors (or raw integer device addresses); torch is used for device memory
and streams and for nothing else.  torch is imported before the library is loaded so that the HIP
runtime the library links against is the one already in the process.
"""
from __future__ import annotations

import array
import ctypes
import os
import struct
import subprocess
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
SRC_PATH = os.path.join(_HERE, "csrc", "hsadmm.hip")
INCLUDE_DIR = os.path.join(_ROOT, "include")
# HSADMM_LIB: load this build of the library instead of the in-tree one (e.g. one whose host code carries sanitizers)
LIB_PATH = os.environ.get("HSADMM_LIB") or os.path.join(_HERE, "libhsadmm.so")

MODE_NONE, MODE_FILTER, MODE_CHANNEL, MODE_BOTH = 0, 1, 2, 3
TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
MX_FP8, MX_FP4 = 0, 1
MAX_REPLICAS = 16

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fPIC", "-shared",
]

EXPORTS = ("hsadmm_plan_create", "hsadmm_plan_destroy", "hsadmm_plan_sizes", "hsadmm_project",
           "hsadmm_compact", "hsadmm_expand", "hsadmm_strerror", "hsadmm_version",
           "hsadmm_kernel_timing_enable", "hsadmm_kernel_timing_read", "hsadmm_kernel_timing_read_n", "hsadmm_kernel_name",
           "hsadmm_project_frozen", "hsadmm_mask_or", "hsadmm_compact_sum", "hsadmm_node_coefficients",
           "hsadmm_plan_set_node_weights", "hsadmm_project_weighted", "hsadmm_dual_inter", "hsadmm_residuals",
           "hsadmm_average", "hsadmm_mask_drift", "hsadmm_expand_dual", "hsadmm_project_compact",
           "hsadmm_project_weighted_compact", "hsadmm_project_frozen_compact",
           "hsadmm_project_weighted_frozen", "hsadmm_project_weighted_frozen_compact",
           "hsadmm_retrain_project", "hsadmm_retrain_expand",
           "hsadmm_adapt_penalties", "hsadmm_scale_layers", "hsadmm_project_compact_static",
           "hsadmm_step", "hsadmm_selection_from_mask", "hsadmm_kernel_grid", "hsadmm_plan_estimates",
           "hsadmm_layer_sqnorms", "hsadmm_stopping_test", "hsadmm_plan_create_nested",
           "hsadmm_gradient_norms", "hsadmm_adamw_coefficients", "hsadmm_plan_state_blocks", "hsadmm_adamw",
           "hsadmm_compact_mx", "hsadmm_expand_mx",
           "hsadmm_embedding", "hsadmm_embedding_workspace", "hsadmm_embedding_gradient", "hsadmm_dropout",
           "hsadmm_softmax_loss_workspace", "hsadmm_softmax_loss")
KERNEL_COUNT = 52


class HsadmmError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__("%s failed: %s (code %d)" % (what, hsadmm_strerror(code), code))
        self.code = code


class _Layer(ctypes.Structure):
    _fields_ = [("elem_off", ctypes.c_int64), ("c_out", ctypes.c_int32), ("c_in", ctypes.c_int32),
                ("khw", ctypes.c_int32), ("mode", ctypes.c_int32), ("k", ctypes.c_int32),
                ("k_in", ctypes.c_int32)]


class _Nest(ctypes.Structure):
    _fields_ = [("span", ctypes.c_int32), ("k_coarse", ctypes.c_int32)]


# hsadmm_step_args_t, field by field, in declaration order: (name, C type, how the binding fills it).
#   "dev": device buffer (torch tensor, integer address or None)
_vp = ctypes.c_void_p
_STEP_FIELDS = (
    ("struct_bytes", ctypes.c_size_t, "sizeof"),
    ("W_replicas", ctypes.POINTER(_vp), "replicas"),
    ("R", ctypes.c_int32, "replica_count"),
    ("mappings_cached", ctypes.c_int32, "flag"),
    ("U", _vp, "dev"), ("U_out", _vp, "dev"), ("Zg", _vp, "dev"), ("Vd", _vp, "dev"), ("coef", _vp, "dev"),
    ("Zi_prev", _vp, "dev"), ("mask_frozen", _vp, "dev"), ("sel_prev", _vp, "dev"),
    ("Z", _vp, "dev"), ("Wbar", _vp, "dev"), ("mask", _vp, "dev"), ("sqnorm", _vp, "dev"), ("sel", _vp, "dev"),
    ("packed", _vp, "dev"), ("layer_off", _vp, "dev"), ("kept_idx", _vp, "dev"), ("residuals", _vp, "dev"),
    ("workspace", _vp, "dev"),
    ("workspace_bytes", ctypes.c_size_t, "workspace_size"),
    ("hip_stream", _vp, "stream"),
)


class _StepArgs(ctypes.Structure):
    _fields_ = [(name, ctype) for name, ctype, _ in _STEP_FIELDS]


class _AdamwCoef(ctypes.Structure):
    _fields_ = [("decay", ctypes.c_float), ("step_size", ctypes.c_float), ("root", ctypes.c_float),
                ("noise", ctypes.c_uint32)]


# hsadmm_adamw_args_t, field by field, in declaration order.  W .. W_low are HOST arrays of device addresses.
_ADAMW_FIELDS = (
    ("struct_bytes", ctypes.c_size_t), ("R", ctypes.c_int32), ("grad_type", ctypes.c_int32),
    ("state_bits", ctypes.c_int32), ("noise", ctypes.c_uint32),
    ("W", _vp), ("G", _vp), ("M", _vp), ("V", _vp), ("M_scale", _vp), ("V_scale", _vp), ("W_low", _vp),
    ("Z", _vp), ("U", _vp), ("rho", _vp), ("grad_scale", _vp), ("coef", _vp),
    ("lr", ctypes.c_double), ("beta_one", ctypes.c_double), ("beta_two", ctypes.c_double),
    ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("step", ctypes.c_int64), ("hip_stream", _vp),
)


class _AdamwArgs(ctypes.Structure):
    _fields_ = list(_ADAMW_FIELDS)


# hsadmm_softmax_loss_args_t, field by field, in declaration order
_LOSS_FIELDS = (
    ("struct_bytes", ctypes.c_size_t), ("layer", ctypes.c_int32), ("type", ctypes.c_int32), ("index_bits", ctypes.c_int32),
    ("mean", ctypes.c_int32), ("accumulate", ctypes.c_int32), ("reserved", ctypes.c_int32), ("n", ctypes.c_int64),
    ("x_stride", ctypes.c_int64), ("dx_stride", ctypes.c_int64), ("scale", ctypes.c_double),
    ("W", _vp), ("X", _vp), ("labels", _vp), ("loss", _vp), ("lse", _vp), ("total", _vp), ("dX", _vp), ("G", _vp),
    ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t), ("hip_stream", _vp),
)


class _LossArgs(ctypes.Structure):
    _fields_ = list(_LOSS_FIELDS)


# the same structure written at once (native sizes and alignment)
_LOSS_PACK = struct.Struct("N6i3qd9PNP")
_ADAMW_PACK = struct.Struct("N3iI12P5dqP")
_COEF_BYTES = ctypes.sizeof(_AdamwCoef)


_lib = None


def build_library(verbose: bool = False) -> str:
    """Compile csrc/hsadmm.hip for gfx950 with hipcc into libhsadmm.so (in-tree)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB_PATH + ".tmp.%d" % os.getpid()
    cmd = [hipcc, *HIPCC_FLAGS, "-I", INCLUDE_DIR, "-I", os.path.dirname(SRC_PATH), "-o", tmp, SRC_PATH]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or res.returncode != 0:
        print(res.stdout)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed (%d): %s" % (res.returncode, " ".join(cmd)))
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


def load_library():
    """Load libhsadmm.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libhsadmm.so is missing at %s: build it first "
                           "(python -c 'import __graft_entry__ as g; g.build()')" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp = ctypes.c_void_p
    lib.hsadmm_plan_create.argtypes = [ctypes.POINTER(_Layer), ctypes.c_int32, ctypes.c_int32,
                                       ctypes.POINTER(vp)]
    lib.hsadmm_plan_create.restype = ctypes.c_int
    lib.hsadmm_plan_create_nested.argtypes = [ctypes.POINTER(_Layer), ctypes.POINTER(_Nest), ctypes.c_int32,
                                              ctypes.c_int32, ctypes.POINTER(vp)]
    lib.hsadmm_plan_create_nested.restype = ctypes.c_int
    lib.hsadmm_plan_destroy.argtypes = [vp]
    lib.hsadmm_plan_destroy.restype = None
    lib.hsadmm_plan_sizes.argtypes = [vp, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64),
                                      ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_size_t)]
    lib.hsadmm_plan_sizes.restype = ctypes.c_int
    lib.hsadmm_project.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp,
                                   ctypes.c_size_t, vp]
    lib.hsadmm_project.restype = ctypes.c_int
    lib.hsadmm_project_compact.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                           ctypes.c_size_t, vp]
    lib.hsadmm_project_compact.restype = ctypes.c_int
    lib.hsadmm_project_compact_static.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp, vp,
                                                  vp, vp]
    lib.hsadmm_project_compact_static.restype = ctypes.c_int
    lib.hsadmm_step.argtypes = [vp, ctypes.POINTER(_StepArgs)]
    lib.hsadmm_step.restype = ctypes.c_int
    lib.hsadmm_selection_from_mask.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_selection_from_mask.restype = ctypes.c_int
    lib.hsadmm_project_frozen.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp]
    lib.hsadmm_project_frozen.restype = ctypes.c_int
    lib.hsadmm_project_frozen_compact.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp,
                                                  ctypes.c_int32, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_project_frozen_compact.restype = ctypes.c_int
    lib.hsadmm_mask_or.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp]
    lib.hsadmm_mask_or.restype = ctypes.c_int
    lib.hsadmm_expand_dual.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_expand_dual.restype = ctypes.c_int
    lib.hsadmm_mask_drift.argtypes = [vp, vp, vp, vp, vp]
    lib.hsadmm_mask_drift.restype = ctypes.c_int
    lib.hsadmm_average.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, ctypes.c_int64, vp, vp]
    lib.hsadmm_average.restype = ctypes.c_int
    lib.hsadmm_compact_sum.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_compact_sum.restype = ctypes.c_int
    f64p = ctypes.POINTER(ctypes.c_double)
    f32p = ctypes.POINTER(ctypes.c_float)
    lib.hsadmm_node_coefficients.argtypes = [f64p, f64p, ctypes.c_int32, ctypes.c_double, ctypes.c_int32,
                                             ctypes.c_int32, f32p, f32p]
    lib.hsadmm_node_coefficients.restype = ctypes.c_int
    lib.hsadmm_plan_set_node_weights.argtypes = [vp, f32p, f32p]
    lib.hsadmm_plan_set_node_weights.restype = ctypes.c_int
    lib.hsadmm_project_weighted.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp, vp, vp,
                                            ctypes.c_size_t, vp]
    lib.hsadmm_project_weighted.restype = ctypes.c_int
    lib.hsadmm_project_weighted_compact.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp, vp,
                                                    vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_project_weighted_compact.restype = ctypes.c_int
    lib.hsadmm_project_weighted_frozen.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp, vp]
    lib.hsadmm_project_weighted_frozen.restype = ctypes.c_int
    lib.hsadmm_project_weighted_frozen_compact.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp,
                                                           vp, ctypes.c_int32, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_project_weighted_frozen_compact.restype = ctypes.c_int
    lib.hsadmm_retrain_project.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp,
                                           ctypes.c_int32, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_retrain_project.restype = ctypes.c_int
    lib.hsadmm_retrain_expand.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_retrain_expand.restype = ctypes.c_int
    dp, fp = ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_float)
    lib.hsadmm_adapt_penalties.argtypes = [dp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_double,
                                           ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                           dp, dp, fp, fp]
    lib.hsadmm_adapt_penalties.restype = ctypes.c_int
    lib.hsadmm_scale_layers.argtypes = [vp, vp, vp, vp]
    lib.hsadmm_scale_layers.restype = ctypes.c_int
    lib.hsadmm_residuals.argtypes = [vp, ctypes.POINTER(vp), ctypes.c_int32, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_residuals.restype = ctypes.c_int
    lib.hsadmm_dual_inter.argtypes = [vp, vp, vp, vp, vp]
    lib.hsadmm_dual_inter.restype = ctypes.c_int
    lib.hsadmm_compact.argtypes = [vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_compact.restype = ctypes.c_int
    lib.hsadmm_expand.argtypes = [vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_expand.restype = ctypes.c_int
    lib.hsadmm_strerror.argtypes = [ctypes.c_int]
    lib.hsadmm_strerror.restype = ctypes.c_char_p
    lib.hsadmm_version.argtypes = []
    lib.hsadmm_version.restype = ctypes.c_int
    lib.hsadmm_kernel_timing_enable.argtypes = [vp, ctypes.c_int]
    lib.hsadmm_kernel_timing_enable.restype = ctypes.c_int
    lib.hsadmm_kernel_timing_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.hsadmm_kernel_timing_read.restype = ctypes.c_int
    lib.hsadmm_kernel_timing_read_n.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64),
                                                ctypes.c_int32]
    lib.hsadmm_kernel_timing_read_n.restype = ctypes.c_int
    lib.hsadmm_layer_sqnorms.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_layer_sqnorms.restype = ctypes.c_int
    lib.hsadmm_stopping_test.argtypes = [ctypes.POINTER(ctypes.c_int64), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                         dp, dp, dp, dp, ctypes.c_double,
                                         ctypes.c_double, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
    lib.hsadmm_stopping_test.restype = ctypes.c_int
    lib.hsadmm_gradient_norms.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_double, vp, vp,
                                          vp, ctypes.c_size_t, vp]
    lib.hsadmm_gradient_norms.restype = ctypes.c_int
    lib.hsadmm_adamw_coefficients.argtypes = [ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                              ctypes.c_int64, ctypes.c_uint32, ctypes.POINTER(_AdamwCoef)]
    lib.hsadmm_adamw_coefficients.restype = ctypes.c_int
    lib.hsadmm_plan_state_blocks.argtypes = [vp, ctypes.POINTER(ctypes.c_int64)]
    lib.hsadmm_plan_state_blocks.restype = ctypes.c_int
    lib.hsadmm_adamw.argtypes = [vp, vp]
    lib.hsadmm_adamw.restype = ctypes.c_int
    lib.hsadmm_compact_mx.argtypes = [vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_compact_mx.restype = ctypes.c_int
    lib.hsadmm_expand_mx.argtypes = [vp, vp, vp, ctypes.c_int32, ctypes.c_int32, vp, vp,
                                     vp, vp, vp, ctypes.c_size_t, vp]
    lib.hsadmm_expand_mx.restype = ctypes.c_int
    i32, i64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.hsadmm_embedding.argtypes = [vp, i32, vp, i32, vp, i32, i64, ctypes.c_float, vp, i64, vp]
    lib.hsadmm_embedding.restype = ctypes.c_int
    lib.hsadmm_embedding_workspace.argtypes = [vp, i32, i64, ctypes.POINTER(size)]
    lib.hsadmm_embedding_workspace.restype = ctypes.c_int
    lib.hsadmm_embedding_gradient.argtypes = [vp, i32, vp, i32, i64, vp, i64, i32, ctypes.c_float, i32, vp, vp, size, vp]
    lib.hsadmm_embedding_gradient.restype = ctypes.c_int
    lib.hsadmm_dropout.argtypes = [vp, vp, i64, vp, i64, vp, i64, i64, i64, i32, ctypes.c_double, ctypes.c_uint64,
                                   ctypes.c_uint64, vp, vp]
    lib.hsadmm_dropout.restype = ctypes.c_int
    lib.hsadmm_softmax_loss_workspace.argtypes = [vp, i32, i64, i32, i32, ctypes.POINTER(size)]
    lib.hsadmm_softmax_loss_workspace.restype = ctypes.c_int
    lib.hsadmm_softmax_loss.argtypes = [vp, vp]
    lib.hsadmm_softmax_loss.restype = ctypes.c_int
    lib.hsadmm_kernel_grid.argtypes = [vp, ctypes.c_int]
    lib.hsadmm_kernel_grid.restype = ctypes.c_int
    lib.hsadmm_plan_estimates.argtypes = [vp]
    lib.hsadmm_plan_estimates.restype = ctypes.c_int
    lib.hsadmm_kernel_name.argtypes = [ctypes.c_int]
    lib.hsadmm_kernel_name.restype = ctypes.c_char_p
    _lib = lib
    return lib


def exported_symbols():
    """Names include/hsadmm.h declares, each resolved in the loaded library."""
    lib = load_library()
    return {name: getattr(lib, name) for name in EXPORTS}


def hsadmm_strerror(code: int) -> str:
    return load_library().hsadmm_strerror(int(code)).decode()


def hsadmm_version() -> int:
    return int(load_library().hsadmm_version())


def _ptr(x) -> Optional[int]:
    """Device address of a torch tensor, or an integer address passed through; None -> NULL."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return int(x.data_ptr())


def _nbytes(x) -> int:
    return x.nbytes


def _stream(stream) -> Optional[int]:
    if stream is None:
        return int(torch.cuda.current_stream().cuda_stream) or None
    if isinstance(stream, int):
        return stream or None
    return int(stream.cuda_stream) or None


class Plan:
    """Owner of an hsadmm_plan_t*.  `table` has the columns elem_off, c_out, c_in, khw, mode, k and, when it
    holds layers under both constraints (mode 3), k_in.  With the columns span and k_coarse (runs of channels,
    hsadmm_nest_t) the plan is made by hsadmm_plan_create_nested."""

    def __init__(self, table, pack_align_elems: int = 1):
        lib = load_library()
        L = len(table["c_out"])
        arr = (_Layer * max(L, 1))()
        for i in range(L):
            arr[i].elem_off = int(table["elem_off"][i])
            arr[i].c_out = int(table["c_out"][i])
            arr[i].c_in = int(table["c_in"][i])
            arr[i].khw = int(table["khw"][i])
            arr[i].mode = int(table["mode"][i])
            arr[i].k = int(table["k"][i])
            arr[i].k_in = int(table["k_in"][i]) if "k_in" in table else 0
        handle = ctypes.c_void_p()
        self.handle = None
        if "span" in table:
            nest = (_Nest * max(L, 1))()
            for i in range(L):
                nest[i].span = int(table["span"][i])
                nest[i].k_coarse = int(table["k_coarse"][i])
            rc = lib.hsadmm_plan_create_nested(arr, nest, L, int(pack_align_elems), ctypes.byref(handle))
            if rc != 0:
                raise HsadmmError(rc, "hsadmm_plan_create_nested")
        else:
            rc = lib.hsadmm_plan_create(arr, L, int(pack_align_elems), ctypes.byref(handle))
            if rc != 0:
                raise HsadmmError(rc, "hsadmm_plan_create")
        self.handle = handle
        self.n_layers = L
        self.pack_align_elems = int(pack_align_elems)
        a, g, c, w = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_size_t()
        rc = lib.hsadmm_plan_sizes(self.handle, ctypes.byref(a), ctypes.byref(g), ctypes.byref(c),
                                   ctypes.byref(w))
        if rc != 0:
            raise HsadmmError(rc, "hsadmm_plan_sizes")
        self.arena_elems, self.groups_total = a.value, g.value
        self.packed_capacity_elems, self.workspace_bytes = c.value, w.value
        self.state_blocks = hsadmm_plan_state_blocks(self)
        self.device = torch.cuda.current_device()
        self.widths = [int(c) for c in table["c_in"]]          # (columns of the layers that have one row a token)

    def close(self):
        if getattr(self, "handle", None):
            load_library().hsadmm_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def hsadmm_kernel_timing_enable(plan: Plan, enable: bool) -> None:
    rc = load_library().hsadmm_kernel_timing_enable(plan.handle, 1 if enable else 0)
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_kernel_timing_enable")


def hsadmm_kernel_timing_read(plan: Plan):
    """{kernel name: (total milliseconds, launches)} since the last read."""
    lib = load_library()
    ms = (ctypes.c_double * KERNEL_COUNT)()
    cnt = (ctypes.c_int64 * KERNEL_COUNT)()
    rc = lib.hsadmm_kernel_timing_read_n(plan.handle, ms, cnt, KERNEL_COUNT)
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_kernel_timing_read")
    return {lib.hsadmm_kernel_name(i).decode(): (float(ms[i]), int(cnt[i])) for i in range(KERNEL_COUNT)}


def hsadmm_plan_estimates(plan: Plan) -> bool:
    """Whether this plan's un-predicted projection forms a prediction inside pass 1 (see include/hsadmm.h)."""
    return bool(load_library().hsadmm_plan_estimates(plan.handle))


def hsadmm_kernel_grids(plan: Plan):
    """{kernel name: workgroups of its latest timed launch on this plan} (0: not launched with timing on)."""
    lib = load_library()
    return {lib.hsadmm_kernel_name(i).decode(): int(lib.hsadmm_kernel_grid(plan.handle, i)) for i in range(KERNEL_COUNT)}


def hsadmm_project(plan: Plan, W_replicas: Sequence, U, Z, Wbar, mask, sqnorm, workspace,
                   stream=None, workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_project(plan.handle, ptrs, R, _ptr(U), _ptr(Z), _ptr(Wbar), _ptr(mask), _ptr(sqnorm),
                            _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project")
    return rc


def hsadmm_project_compact(plan: Plan, W_replicas: Sequence, U, Z, Wbar, mask, sqnorm, packed, layer_off, kept_idx,
                           workspace, stream=None, workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_project_compact(plan.handle, ptrs, R, _ptr(U), _ptr(Z), _ptr(Wbar), _ptr(mask), _ptr(sqnorm),
                                    _ptr(packed), _ptr(layer_off), _ptr(kept_idx), _ptr(workspace), wb,
                                    _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_compact")
    return rc


def hsadmm_project_compact_static(plan: Plan, W_replicas: Sequence, U, Z, Wbar, mask, sqnorm, packed, layer_off,
                                  kept_idx, stream=None, check: bool = True) -> int:
    """hsadmm_project_compact on the library's static scratch array (no workspace argument, no allocation)."""
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    rc = lib.hsadmm_project_compact_static(plan.handle, ptrs, R, _ptr(U), _ptr(Z), _ptr(Wbar), _ptr(mask),
                                           _ptr(sqnorm), _ptr(packed), _ptr(layer_off), _ptr(kept_idx),
                                           _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_compact_static")
    return rc


def hsadmm_step(plan: Plan, W_replicas: Sequence, stream=None, workspace_bytes: Optional[int] = None,
                check: bool = True, **fields) -> int:
    """hsadmm_step: every form of the projection step through one argument structure.  Keyword arguments are the
    device-buffer fields of hsadmm_step_args_t (U, Z, mask, packed, sel_prev, ...) and the flag mappings_cached;
    fields that are not given stay NULL."""
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    args = _StepArgs()
    known = {name for name, _, how in _STEP_FIELDS if how in ("dev", "flag")}
    unknown = set(fields) - known
    if unknown:
        raise TypeError("hsadmm_step has no field(s) %s" % ", ".join(sorted(unknown)))
    for name, _, how in _STEP_FIELDS:
        if how == "sizeof":
            value = ctypes.sizeof(_StepArgs)
        elif how == "replicas":
            value = ptrs
        elif how == "replica_count":
            value = R
        elif how == "flag":
            value = 1 if fields.get(name) else 0
        elif how == "dev":
            value = _ptr(fields.get(name))
        elif how == "workspace_size":
            ws = fields.get("workspace")
            value = int(workspace_bytes) if workspace_bytes is not None else (0 if ws is None or isinstance(ws, int)
                                                                             else _nbytes(ws))
        else:
            value = _stream(stream)
        setattr(args, name, value)
    rc = lib.hsadmm_step(plan.handle, ctypes.byref(args))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_step")
    return rc


def hsadmm_selection_from_mask(plan: Plan, mask, sel, workspace, stream=None, workspace_bytes: Optional[int] = None,
                               check: bool = True) -> int:
    """sel[g] = rank of group g among its layer's groups kept by `mask`, -1 if not kept."""
    lib = load_library()
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_selection_from_mask(plan.handle, _ptr(mask), _ptr(sel), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_selection_from_mask")
    return rc


def hsadmm_project_frozen(plan: Plan, W_replicas: Sequence, U, Z, Wbar, mask, stream=None, check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    rc = lib.hsadmm_project_frozen(plan.handle, ptrs, R, _ptr(U), _ptr(Z), _ptr(Wbar), _ptr(mask), _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_frozen")
    return rc


def hsadmm_project_frozen_compact(plan: Plan, W_replicas: Sequence, U, Z, Wbar, mask, mappings_cached: bool, packed,
                                  layer_off, kept_idx, workspace, stream=None, workspace_bytes: Optional[int] = None,
                                  check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_project_frozen_compact(plan.handle, ptrs, R, _ptr(U), _ptr(Z), _ptr(Wbar), _ptr(mask),
                                           1 if mappings_cached else 0, _ptr(packed), _ptr(layer_off),
                                           _ptr(kept_idx), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_frozen_compact")
    return rc


def hsadmm_mask_or(plan: Plan, masks: Sequence, out, stream=None, check: bool = True) -> int:
    lib = load_library()
    M = len(masks)
    ptrs = (ctypes.c_void_p * max(M, 1))(*[_ptr(m) for m in masks])
    rc = lib.hsadmm_mask_or(plan.handle, ptrs, M, _ptr(out), _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_mask_or")
    return rc


def hsadmm_mask_drift(plan: Plan, mask_a, mask_b, drift, stream=None, check: bool = True) -> int:
    """Section 4.5: drift[l] = groups of layer l whose kept flag differs between the two masks."""
    rc = load_library().hsadmm_mask_drift(plan.handle, _ptr(mask_a), _ptr(mask_b), _ptr(drift), _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_mask_drift")
    return rc


def hsadmm_average(plan: Plan, bufs: Sequence, n_elems: int, out, stream=None, check: bool = True) -> int:
    """Eq. (11): out = mean of the M buffers (each n_elems floats)."""
    lib = load_library()
    M = len(bufs)
    ptrs = (ctypes.c_void_p * max(M, 1))(*[_ptr(b) for b in bufs])
    rc = lib.hsadmm_average(plan.handle, ptrs, M, int(n_elems), _ptr(out), _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_average")
    return rc


def hsadmm_node_coefficients(rho1, rho2, lam: float, M: int, P: int):
    """Eq. (9) weights as two lists of L floats (host computation inside the library)."""
    lib = load_library()
    L = len(rho1)
    r1 = (ctypes.c_double * L)(*[float(x) for x in rho1])
    r2 = (ctypes.c_double * L)(*[float(x) for x in rho2])
    a = (ctypes.c_float * L)()
    b = (ctypes.c_float * L)()
    rc = lib.hsadmm_node_coefficients(r1, r2, L, float(lam), int(M), int(P), a, b)
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_node_coefficients")
    return list(a), list(b)


def hsadmm_adapt_penalties(residuals, rho1, rho2, P: int, n_out: int, mu: float, tau_incr: float, tau_decr: float,
                           rho1_max: float, rho2_max: float):
    """Residual balancing per layer and level (host computation inside the library).  residuals: 4*L floats on the
    host, rows as hsadmm_residuals writes them.  Returns (rho1, rho2, scale_u, scale_v) as lists of L numbers."""
    lib = load_library()
    L = len(rho1)
    flat = [float(x) for row in residuals for x in (row if hasattr(row, "__len__") else [row])]
    if len(flat) != 4 * L or len(rho2) != L:
        raise ValueError("residuals need 4 entries per layer, rho1 and rho2 one")
    sq = (ctypes.c_double * (4 * L))(*flat)
    r1 = (ctypes.c_double * L)(*[float(x) for x in rho1])
    r2 = (ctypes.c_double * L)(*[float(x) for x in rho2])
    su = (ctypes.c_float * L)()
    sv = (ctypes.c_float * L)()
    rc = lib.hsadmm_adapt_penalties(sq, L, int(P), int(n_out), float(mu), float(tau_incr), float(tau_decr),
                                    float(rho1_max), float(rho2_max), r1, r2, su, sv)
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_adapt_penalties")
    return list(r1), list(r2), list(su), list(sv)


def hsadmm_layer_sqnorms(plan: Plan, X, out, workspace, stream=None, workspace_bytes: Optional[int] = None,
                         check: bool = True) -> int:
    """out[l] = squared Frobenius norm of layer l of the arena X (fp64, on the device)."""
    lib = load_library()
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_layer_sqnorms(plan.handle, _ptr(X), _ptr(out), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_layer_sqnorms")
    return rc


def hsadmm_stopping_test(n_elems, P: int, n_out: int, rho1, rho2, residuals, magnitudes, eps_abs: float,
                         eps_rel: float):
    """Section 3.4's stopping test on the host.  n_elems: elements per layer; residuals: 4*L numbers, magnitudes:
    5*L numbers (rows as in the header).  Returns (list of L flags, all_done)."""
    lib = load_library()
    L = len(n_elems)
    ne = (ctypes.c_int64 * L)(*[int(x) for x in n_elems])

    def flat(x, rows):
        v = [float(y) for r in x for y in (r if hasattr(r, "__len__") else [r])]
        if len(v) != rows * L:
            raise ValueError("%d numbers per layer expected" % rows)
        return (ctypes.c_double * len(v))(*v)
    if len(rho1) != L or len(rho2) != L:
        raise ValueError("one penalty per layer and level")
    r1 = (ctypes.c_double * L)(*[float(x) for x in rho1])
    r2 = (ctypes.c_double * L)(*[float(x) for x in rho2])
    done = (ctypes.c_int32 * L)()
    every = ctypes.c_int32(-1)
    rc = lib.hsadmm_stopping_test(ne, L, int(P), int(n_out), r1, r2, flat(residuals, 4), flat(magnitudes, 5),
                                  float(eps_abs), float(eps_rel), done, ctypes.byref(every))
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_stopping_test")
    return list(done), bool(every.value)


def hsadmm_scale_layers(plan: Plan, X, factor, stream=None, check: bool = True) -> int:
    """X *= factor[layer] on the device (factor: L floats on the device)."""
    lib = load_library()
    rc = lib.hsadmm_scale_layers(plan.handle, _ptr(X), _ptr(factor), _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_scale_layers")
    return rc


def hsadmm_plan_set_node_weights(plan: Plan, a, b) -> None:
    lib = load_library()
    L = plan.n_layers
    if len(a) != L or len(b) != L:
        raise ValueError("a and b need one entry per layer")
    fa = (ctypes.c_float * L)(*[float(x) for x in a])
    fb = (ctypes.c_float * L)(*[float(x) for x in b])
    rc = lib.hsadmm_plan_set_node_weights(plan.handle, fa, fb)
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_plan_set_node_weights")


def hsadmm_project_weighted(plan: Plan, W_replicas: Sequence, U, Zg, Vd, Z, Wbar, mask, sqnorm, workspace,
                            stream=None, workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_project_weighted(plan.handle, ptrs, R, _ptr(U), _ptr(Zg), _ptr(Vd), _ptr(Z), _ptr(Wbar),
                                     _ptr(mask), _ptr(sqnorm), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_weighted")
    return rc


def hsadmm_project_weighted_compact(plan: Plan, W_replicas: Sequence, U, Zg, Vd, Z, Wbar, mask, sqnorm, packed,
                                    layer_off, kept_idx, workspace, stream=None,
                                    workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_project_weighted_compact(plan.handle, ptrs, R, _ptr(U), _ptr(Zg), _ptr(Vd), _ptr(Z), _ptr(Wbar),
                                             _ptr(mask), _ptr(sqnorm), _ptr(packed), _ptr(layer_off),
                                             _ptr(kept_idx), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_weighted_compact")
    return rc


def hsadmm_project_weighted_frozen(plan: Plan, W_replicas: Sequence, U, Zg, Vd, Z, Wbar, mask, stream=None,
                                   check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    rc = lib.hsadmm_project_weighted_frozen(plan.handle, ptrs, R, _ptr(U), _ptr(Zg), _ptr(Vd), _ptr(Z), _ptr(Wbar),
                                            _ptr(mask), _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_weighted_frozen")
    return rc


def hsadmm_project_weighted_frozen_compact(plan: Plan, W_replicas: Sequence, U, Zg, Vd, Z, Wbar, mask,
                                           mappings_cached: bool, packed, layer_off, kept_idx, workspace, stream=None,
                                           workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_project_weighted_frozen_compact(plan.handle, ptrs, R, _ptr(U), _ptr(Zg), _ptr(Vd), _ptr(Z),
                                                    _ptr(Wbar), _ptr(mask), 1 if mappings_cached else 0,
                                                    _ptr(packed), _ptr(layer_off), _ptr(kept_idx), _ptr(workspace),
                                                    wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_project_weighted_frozen_compact")
    return rc


def hsadmm_retrain_project(plan: Plan, W_replicas: Sequence, U, Zg, Vd, Z, Wbar, mask, mappings_cached: bool,
                           packed, layer_off, kept_idx, residuals, workspace, stream=None,
                           workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """hsadmm_project_weighted_frozen_compact that also writes rows 0 and 1 of `residuals` (Z in: previous z_i)."""
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_retrain_project(plan.handle, ptrs, R, _ptr(U), _ptr(Zg), _ptr(Vd), _ptr(Z), _ptr(Wbar),
                                    _ptr(mask), 1 if mappings_cached else 0, _ptr(packed), _ptr(layer_off),
                                    _ptr(kept_idx), _ptr(residuals), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_retrain_project")
    return rc


def hsadmm_retrain_expand(plan: Plan, packed, mask, dst, Zi, Vd, z_prev, residuals, workspace, stream=None,
                          workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """hsadmm_expand_dual that also writes rows 2 and 3 of `residuals` (z_prev: the previous global consensus)."""
    lib = load_library()
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_retrain_expand(plan.handle, _ptr(packed), _ptr(mask), _ptr(dst), _ptr(Zi), _ptr(Vd), _ptr(z_prev),
                                   _ptr(residuals), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_retrain_expand")
    return rc


def hsadmm_residuals(plan: Plan, W_replicas: Sequence, Zi, Zi_prev, Zg, Zg_prev, out, workspace, stream=None,
                     workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    R = len(W_replicas)
    ptrs = (ctypes.c_void_p * max(R, 1))(*[_ptr(w) for w in W_replicas])
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_residuals(plan.handle, ptrs, R, _ptr(Zi), _ptr(Zi_prev), _ptr(Zg), _ptr(Zg_prev), _ptr(out),
                              _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_residuals")
    return rc


def hsadmm_dual_inter(plan: Plan, Zi, Zg, Vd, stream=None, check: bool = True) -> int:
    rc = load_library().hsadmm_dual_inter(plan.handle, _ptr(Zi), _ptr(Zg), _ptr(Vd), _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_dual_inter")
    return rc


def hsadmm_compact_sum(plan: Plan, src0, src1, mask, packed, layer_off, kept_idx, workspace, stream=None,
                       workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_compact_sum(plan.handle, _ptr(src0), _ptr(src1), _ptr(mask), _ptr(packed), _ptr(layer_off),
                                _ptr(kept_idx), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_compact_sum")
    return rc


def hsadmm_compact(plan: Plan, src, mask, packed, layer_off, kept_idx, workspace, stream=None,
                   workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_compact(plan.handle, _ptr(src), _ptr(mask), _ptr(packed), _ptr(layer_off), _ptr(kept_idx),
                            _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_compact")
    return rc


def hsadmm_expand(plan: Plan, packed, mask, dst, workspace, stream=None,
                  workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    lib = load_library()
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_expand(plan.handle, _ptr(packed), _ptr(mask), _ptr(dst), _ptr(workspace), wb,
                           _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_expand")
    return rc


def hsadmm_expand_dual(plan: Plan, packed, mask, dst, Zi, Vd, workspace, stream=None,
                       workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """hsadmm_expand with Vd <- Vd + (Zi - dst) (Eq. (13)) applied in the same pass."""
    lib = load_library()
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = lib.hsadmm_expand_dual(plan.handle, _ptr(packed), _ptr(mask), _ptr(dst), _ptr(Zi), _ptr(Vd), _ptr(workspace),
                                wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_expand_dual")
    return rc


class _Unfit(Exception):
    """Arguments that do not go together, above all a tensor that cannot be the buffer it was given as."""


def _fit(buffers, name: str, dtype, elems: int) -> list:
    """Device addresses of buffers (see _ptr; None -> 0).  Arenas come in several element types, and the library sees addresses
    only: a tensor has to hold `elems` elements of `dtype` (None: of one byte each) in a row, or kernels would run past its
    end.  An integer address is the caller's word."""
    at = []
    for x in buffers:
        if x is None:
            x = 0
        elif not isinstance(x, int):
            if ((x.element_size() != 1 if dtype is None else x.dtype is not dtype) or (elems and x.numel() < elems) or
                    not x.is_contiguous()):
                raise _Unfit("%s: %s of %s, where %d elements of %s have to lie in a row" % (
                    name, tuple(x.shape), x.dtype, elems, dtype or "one byte"))
            x = x.data_ptr()
        at.append(x)
    return at


def _fit_bytes(x, name: str, nbytes: int) -> int:
    """Address of a buffer of that many bytes, whatever a tensor's type."""
    if isinstance(x, int):
        return x
    if _nbytes(x) < nbytes or not x.is_contiguous():
        raise _Unfit("%s: %s of %s, where %d bytes have to lie in a row" % (name, tuple(x.shape), x.dtype, nbytes))
    return x.data_ptr()


def _refused(what: str, why: _Unfit, check: bool) -> int:
    """INVALID_ARGUMENT, as the library itself would have it."""
    if check:
        raise HsadmmError(-1, "%s (%s)" % (what, why))
    return -1


_F32 = torch.float32
_GRAD_DTYPES = {TYPE_F32: _F32, TYPE_BF16: torch.bfloat16, TYPE_F16: torch.float16}


def hsadmm_gradient_norms(plan: Plan, G: Sequence, max_norm: float, norm, scale, workspace, grad_type: int = TYPE_F32,
                          stream=None, workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """Norms of the replicas' gradients and the factors that clip them (NaN: not finite); either output may be None.  Tensors
    of another type than grad_type, or too short, are refused (INVALID_ARGUMENT)."""
    R, grad = len(G), _GRAD_DTYPES.get(grad_type)
    if R > MAX_REPLICAS or grad is None:                      # (the library refuses these as such)
        at, norm_at, scale_at = [_ptr(g) or 0 for g in G], _ptr(norm), _ptr(scale)
    else:
        try:
            at = _fit(G, "G", grad, plan.arena_elems)
            norm_at = 0 if norm is None else _fit((norm,), "norm", torch.float64, R)[0]
            scale_at = 0 if scale is None else _fit((scale,), "scale", _F32, R)[0]
        except _Unfit as why:
            return _refused("hsadmm_gradient_norms", why, check)
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    at = array.array("Q", at)
    rc = load_library().hsadmm_gradient_norms(plan.handle, at.buffer_info()[0], R, int(grad_type), float(max_norm), norm_at,
                                              scale_at, _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_gradient_norms")
    return rc


def hsadmm_adamw_coefficients(lr: float, beta_one: float, beta_two: float, weight_decay: float, step: int,
                              noise: int = 0):
    """(decay, step_size, root, noise) of an AdamW step; as bytes on the device (three floats, one uint32) they are
    hsadmm_adamw's `coef`.  noise 0: a number taken from step."""
    out = _AdamwCoef()
    rc = load_library().hsadmm_adamw_coefficients(float(lr), float(beta_one), float(beta_two), float(weight_decay),
                                                  int(step), int(noise) & 0xFFFFFFFF, ctypes.byref(out))
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_adamw_coefficients")
    return out.decay, out.step_size, out.root, out.noise


def hsadmm_plan_state_blocks(plan: Plan) -> int:
    """Length of the scale arrays of 8-bit optimizer states."""
    n = ctypes.c_int64()
    rc = load_library().hsadmm_plan_state_blocks(plan.handle, ctypes.byref(n))
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_plan_state_blocks")
    return n.value


def hsadmm_adamw(plan: Plan, W: Sequence, G: Sequence, M: Sequence, V: Sequence, *, grad_type: int = TYPE_F32,
                 state_bits: int = 32, M_scale: Optional[Sequence] = None, V_scale: Optional[Sequence] = None,
                 W_low: Optional[Sequence] = None, Z=None, U=None, rho=None, grad_scale=None, coef=None,
                 lr: Optional[float] = None, beta_one: float = 0.9, beta_two: float = 0.999, eps: float = 1e-8,
                 weight_decay: float = 0.0, step: int = 1, noise: int = 0, stream=None, check: bool = True) -> int:
    """One AdamW step of every layer of every replica.  W, G, M, V (and M_scale, V_scale, W_low where they are given): one
    buffer per replica; the other arguments are the fields of hsadmm_adamw_args_t.  `step` is 1 for the first step and grows by
    one a step; with 8-bit states codes are rounded with numbers made of `noise`, or of `step` where noise is 0, so one of them
    has to differ from step to step.  `coef` stands for lr, weight_decay, step and noise.  A call without lr and without coef is
    refused (INVALID_ARGUMENT), as are tensors of other types than grad_type and state_bits say, or too short."""
    R, n, grad = len(W), plan.arena_elems, _GRAD_DTYPES.get(grad_type)
    fit = _fit
    if R > MAX_REPLICAS or grad is None or (state_bits != 32 and state_bits != 8):       # (the library refuses these as such)
        fit = lambda buffers, *_: [_ptr(x) or 0 for x in buffers]        # noqa: E731
    state = _F32 if state_bits != 8 else None
    lists = [("W", W, _F32, n), ("G", G, grad, n), ("M", M, state, n), ("V", V, state, n)]
    if M_scale is not None or V_scale is not None or W_low is not None:
        lists += [("M_scale", M_scale, _F32, plan.state_blocks), ("V_scale", V_scale, _F32, plan.state_blocks),
                  ("W_low", W_low, grad, n)]
    at, places = array.array("Q"), []       # one HOST array for all lists, and where each of them starts in it
    try:
        for name, buffers, dtype, elems in lists:
            if buffers is None:
                places.append(None)
                continue
            if len(buffers) != R:
                raise ValueError("hsadmm_adamw: %d buffers in %s, %d replicas" % (len(buffers), name, R))
            places.append(8 * len(at))
            at.extend(fit(buffers, name, dtype, elems))
        first = at.buffer_info()[0]
        fields = [0 if place is None else first + place for place in places] + [0] * (7 - len(places))
        if Z is not None or U is not None or rho is not None:
            fields += fit((Z, U), "Z, U", _F32, n) + fit((rho,), "rho", _F32, plan.n_layers)
        else:
            fields += (0, 0, 0)
        fields += fit((grad_scale,), "grad_scale", _F32, R)
        fields.append(0 if coef is None else _fit_bytes(coef, "coef", _COEF_BYTES))
        if lr is None:
            if coef is None:
                raise _Unfit("neither lr nor coef")
            lr = 0.0
    except _Unfit as why:
        return _refused("hsadmm_adamw", why, check)
    args = _ADAMW_PACK.pack(_ADAMW_PACK.size, R, grad_type, state_bits, noise & 0xFFFFFFFF, *fields, lr, beta_one, beta_two, eps,
                            weight_decay, step, _stream(stream) or 0)
    rc = load_library().hsadmm_adamw(plan.handle, args)
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_adamw")
    return rc


def hsadmm_compact_mx(plan: Plan, src0, src1, mask, format: int, codes, scales, layer_off, kept_idx, workspace, stream=None,
                      workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """hsadmm_compact (src1 None) or hsadmm_compact_sum into codes of MX_FP8 or MX_FP4 and a scale byte per 32 of them.  Tensors
    of other types, or arenas too short, are refused (INVALID_ARGUMENT); codes and scales have to have room for what the mask
    keeps, which only the caller knows."""
    try:
        src = _fit((src0, src1), "src0, src1", _F32, plan.arena_elems)
        out = _fit((codes, scales), "codes, scales", None, 0)
    except _Unfit as why:
        return _refused("hsadmm_compact_mx", why, check)
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = load_library().hsadmm_compact_mx(plan.handle, src[0], src[1], _ptr(mask), int(format), out[0], out[1], _ptr(layer_off),
                                          _ptr(kept_idx), _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_compact_mx")
    return rc


def hsadmm_expand_mx(plan: Plan, codes: Sequence, scales: Sequence, format: int, mask, dst, Zi, Vd, workspace, stream=None,
                     workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """The mean of the nodes' quantised buffers, scattered to full layout; with Zi and Vd also Vd <- Vd + (Zi - dst).  Tensors
    of other types, or arenas too short, are refused (INVALID_ARGUMENT)."""
    if len(codes) != len(scales):
        raise ValueError("hsadmm_expand_mx: %d buffers of codes, %d of scales" % (len(codes), len(scales)))
    try:
        at = array.array("Q", _fit([*codes, *scales], "codes, scales", None, 0))      # HOST array of both lists
        full = _fit((dst, Zi, Vd), "dst, Zi, Vd", _F32, plan.arena_elems)
    except _Unfit as why:
        return _refused("hsadmm_expand_mx", why, check)
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    M, first = len(codes), at.buffer_info()[0]
    rc = load_library().hsadmm_expand_mx(plan.handle, first, first + 8 * M, M, int(format), _ptr(mask), full[0], full[1], full[2],
                                         _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_expand_mx")
    return rc


_INDEX_DTYPES = {32: torch.int32, 64: torch.int64}


def _width(plan: Plan, layer: int) -> int:
    """Columns of a layer's rows (0: no such layer, which the library refuses)."""
    return plan.widths[layer] if 0 <= layer < plan.n_layers else 0


def _count(ids, n: Optional[int]) -> int:
    """How many tokens there are: n, or a tensor's length."""
    if n is not None:
        return int(n)
    if ids is None or isinstance(ids, int):
        raise _Unfit("n has to be given with an address")
    return ids.numel()


def _here(plan: Plan, *tensors) -> None:
    """Tensors have to lie on the plan's device (which the library compares with the current one)."""
    for x in tensors:
        if x is not None and not isinstance(x, int) and x.get_device() != plan.device:
            raise _Unfit("a tensor on %s, not on the plan's device" % x.device)


def _rows(x, name: str, dtype, n: int, width: int):
    """Device address and stride of n rows of `width` elements: a tensor of two dimensions whose rows lie in one piece, at least
    their width apart.  An integer address (the caller's word) stands for rows without gaps."""
    if x is None or isinstance(x, int):
        return x or 0, width
    if x.dtype is not dtype or x.dim() != 2 or x.shape[0] != n or x.shape[1] != width or (
            n > 0 and width > 1 and x.stride(1) != 1) or (n > 1 and x.stride(0) < width):
        raise _Unfit("%s: %s of %s with strides %s, where %d rows of %d elements of %s have to lie apart" % (
            name, tuple(x.shape), x.dtype, tuple(x.stride()), n, width, dtype))
    return x.data_ptr(), x.stride(0) if n > 1 else width


def hsadmm_embedding(plan: Plan, layer: int, W, ids, out, *, scale: float = 1.0, type: int = TYPE_F32, index_bits: int = 32,
                     n: Optional[int] = None, stream=None, check: bool = True) -> int:
    """out[i] = scale W[ids[i]], rows of the layer in the arena W; zeros where ids[i] is no token.  `n` only with addresses in the
    place of tensors.  Tensors of other types or shapes, or on another device, are refused (INVALID_ARGUMENT)."""
    dtype, width = _GRAD_DTYPES.get(type), _width(plan, layer)
    try:
        n = _count(ids, n)
        _here(plan, W, ids, out)
        if dtype is None or index_bits not in _INDEX_DTYPES:               # (the library refuses these as such)
            at, ids_at, out_at, stride = _ptr(W), _ptr(ids), _ptr(out), width
        else:
            at = _fit((W,), "W", dtype, plan.arena_elems)[0]
            ids_at = _fit((ids,), "ids", _INDEX_DTYPES[index_bits], n)[0]
            out_at, stride = _rows(out, "out", dtype, n, width)
    except _Unfit as why:
        return _refused("hsadmm_embedding", why, check)
    rc = load_library().hsadmm_embedding(plan.handle, int(layer), at, int(type), ids_at, int(index_bits), n, float(scale), out_at,
                                         stride, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_embedding")
    return rc


def hsadmm_embedding_workspace(plan: Plan, layer: int, n: int) -> int:
    """Bytes of the workspace of hsadmm_embedding_gradient for n tokens."""
    nbytes = ctypes.c_size_t()
    rc = load_library().hsadmm_embedding_workspace(plan.handle, int(layer), int(n), ctypes.byref(nbytes))
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_embedding_workspace")
    return nbytes.value


def hsadmm_embedding_gradient(plan: Plan, layer: int, ids, dY, G, workspace, *, scale: float = 1.0, accumulate: bool = False,
                              type: int = TYPE_F32, index_bits: int = 32, n: Optional[int] = None, stream=None,
                              workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """The layer's rows of the gradient arena G: the scaled sums of their tokens' rows of dY (added to what G holds with
    `accumulate`).  Tensors of other types or shapes, or on another device, are refused (INVALID_ARGUMENT)."""
    dtype, width = _GRAD_DTYPES.get(type), _width(plan, layer)
    try:
        n = _count(ids, n)
        _here(plan, ids, dY, G, workspace)
        if dtype is None or index_bits not in _INDEX_DTYPES:
            at, ids_at, dy_at, stride = _ptr(G), _ptr(ids), _ptr(dY), width
        else:
            at = _fit((G,), "G", dtype, plan.arena_elems)[0]
            ids_at = _fit((ids,), "ids", _INDEX_DTYPES[index_bits], n)[0]
            dy_at, stride = _rows(dY, "dY", dtype, n, width)
    except _Unfit as why:
        return _refused("hsadmm_embedding_gradient", why, check)
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    rc = load_library().hsadmm_embedding_gradient(plan.handle, int(layer), ids_at, int(index_bits), n, dy_at, stride, int(type),
                                                  float(scale), 1 if accumulate else 0, at, _ptr(workspace), wb, _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_embedding_gradient")
    return rc


def hsadmm_dropout(plan: Plan, X, Y, p: float, seed: int, call: int, *, residual=None, type: int = TYPE_F32, rows: Optional[int] = None,
                   width: Optional[int] = None, call_device=None, stream=None, check: bool = True) -> int:
    """Y = X without a share p of its elements, the others scaled up, plus the residual.  Which ones follows from seed and call (or
    the 64-bit number at call_device, read when the kernel runs): the same call on Y's gradient is X's.  Tensors of two dimensions;
    rows and width only with addresses in their place.  Tensors of other types or shapes, or on another device, are refused (INVALID_ARGUMENT)."""
    dtype = _GRAD_DTYPES.get(type)
    try:
        if X is not None and not isinstance(X, int) and X.dim() == 2:
            rows, width = X.shape[0] if rows is None else rows, X.shape[1] if width is None else width
        if rows is None or width is None:
            raise _Unfit("X: two dimensions, or rows and width")
        _here(plan, X, residual, Y, call_device)
        if dtype is None:
            at = [(_ptr(x) or 0, width) for x in (X, residual, Y)]
        else:
            at = [_rows(x, name, dtype, rows, width) for name, x in (("X", X), ("residual", residual), ("Y", Y))]
        call_at = 0 if call_device is None else _fit_bytes(call_device, "call_device", 8)
    except _Unfit as why:
        return _refused("hsadmm_dropout", why, check)
    rc = load_library().hsadmm_dropout(plan.handle, at[0][0], at[0][1], at[1][0], at[1][1], at[2][0], at[2][1], int(rows), int(width),
                                       int(type), float(p), int(seed) & (2 ** 64 - 1), int(call) & (2 ** 64 - 1), call_at,
                                       _stream(stream))
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_dropout")
    return rc


def hsadmm_softmax_loss_workspace(plan: Plan, layer: int, n: int, type: int = TYPE_F32, gradients: bool = True) -> int:
    """Bytes of the workspace of hsadmm_softmax_loss for n rows, with gradients or for the losses alone."""
    nbytes = ctypes.c_size_t()
    rc = load_library().hsadmm_softmax_loss_workspace(plan.handle, int(layer), int(n), int(type), 1 if gradients else 0,
                                                      ctypes.byref(nbytes))
    if rc != 0:
        raise HsadmmError(rc, "hsadmm_softmax_loss_workspace")
    return nbytes.value


def hsadmm_softmax_loss(plan: Plan, layer: int, W, X, labels, *, workspace, loss=None, lse=None, total=None, dX=None, G=None,
                        mean: bool = True, scale: float = 1.0, accumulate: bool = False, type: int = TYPE_F32, index_bits: int = 32,
                        n: Optional[int] = None, stream=None, workspace_bytes: Optional[int] = None, check: bool = True) -> int:
    """Softmax cross entropy of X times the layer's rows of the arena W against labels, and its gradients; outputs that are None are
    not wanted.  The other arguments are the fields of hsadmm_softmax_loss_args_t.  Tensors of other types or shapes, or on
    another device, are refused (INVALID_ARGUMENT)."""
    dtype, width = _GRAD_DTYPES.get(type), _width(plan, layer)
    try:
        n = _count(labels, n)
        _here(plan, W, X, labels, workspace, loss, lse, total, dX, G)
        if dtype is None or index_bits not in _INDEX_DTYPES:
            arenas, (x_at, x_stride), (dx_at, dx_stride), labels_at = [_ptr(W), _ptr(G) or 0], (_ptr(X), width), (_ptr(dX) or 0, width), _ptr(labels)
        else:
            arenas = _fit((W, G), "W, G", dtype, plan.arena_elems)
            labels_at = _fit((labels,), "labels", _INDEX_DTYPES[index_bits], n)[0]
            x_at, x_stride = _rows(X, "X", dtype, n, width)
            dx_at, dx_stride = _rows(dX, "dX", dtype, n, width)
        each = _fit((loss, lse), "loss, lse", _F32, n) + _fit((total,), "total", _F32, 2)
    except _Unfit as why:
        return _refused("hsadmm_softmax_loss", why, check)
    wb = _nbytes(workspace) if workspace_bytes is None else int(workspace_bytes)
    args = _LOSS_PACK.pack(_LOSS_PACK.size, int(layer), int(type), int(index_bits), 1 if mean else 0, 1 if accumulate else 0, 0, n,
                           x_stride, dx_stride, float(scale), arenas[0], x_at or 0, labels_at or 0, *each, dx_at, arenas[1],
                           _ptr(workspace) or 0, wb, _stream(stream) or 0)
    rc = load_library().hsadmm_softmax_loss(plan.handle, args)
    if check and rc != 0:
        raise HsadmmError(rc, "hsadmm_softmax_loss")
    return rc
