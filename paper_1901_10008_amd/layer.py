"""ctypes binding of libsk_layer.so (include/sk_layer.h) with the same names: norms around a block, mixture-of-experts layers, verification of
drafted tokens (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import os
from typing import Sequence

from .binding import DTYPE_CODE, SkError

HERE = os.path.dirname(os.path.abspath(__file__))

SK_ACT_NONE, SK_ACT_SIGMOID, SK_ACT_SILU, SK_ACT_TANH, SK_ACT_GELU, SK_ACT_RELU = range(6)
SK_NORM_RMS, SK_NORM_LAYER = range(2)
SK_MOE_SOFTMAX, SK_MOE_SIGMOID = range(2)

LAYER_SYMBOLS = [
    "sk_layer_params_default", "sk_norm_plan_create", "sk_norm_plan_destroy", "sk_norm_launch", "sk_moe_plan_create", "sk_moe_plan_destroy", "sk_moe_launch",
    "sk_moe_plan_info", "sk_verify_plan_create", "sk_verify_plan_destroy", "sk_verify_launch", "sk_verify_plan_info",
]


def _fields(kind, names):
    return [(n, kind) for n in names.split()]


class LayerParams(C.Structure):
    _fields_ = [("host_only", C.c_int32), ("workgroups", C.c_int32), ("reserved", C.c_int32 * 2)]


class sk_norm_problem(C.Structure):
    _fields_ = (_fields(C.c_int32, "dtype residual_dtype kind rows dim post gate_act gate_rows") + _fields(C.c_float, "eps residual_scale block_scale")
                + _fields(C.c_int32, "reserved") + _fields(C.c_int64, "block_stride gate_stride residual_stride residual_out_stride next_stride")
                + _fields(C.c_void_p, "n_rows block gate residual post_weight post_bias pre_weight pre_bias residual_out next"))


class sk_moe_problem(C.Structure):
    _fields_ = (_fields(C.c_int32, "dtype router_dtype rows dim experts top_k ffn shared_ffn act scoring normalize") + _fields(C.c_float, "scale")
                + _fields(C.c_int64, "x_stride out_stride router_stride up_expert_stride down_expert_stride up_row_stride down_row_stride")
                + _fields(C.c_void_p, "n_rows x router router_bias gate up down shared_gate shared_up shared_down out expert_ids expert_weights"))


class sk_verify_problem(C.Structure):
    _fields_ = (_fields(C.c_int32, "dtype sequences rows vocab") + _fields(C.c_float, "temperature") + _fields(C.c_int32, "reserved")
                + _fields(C.c_int64, "logits_stride draft_stride")
                + _fields(C.c_void_p, "first_row logits drafted draft_logits temperatures accept_random sample_random tokens accepted"))


def layer_lib_path() -> str:
    return os.path.join(HERE, "libsk_layer.so")


_lib = None


def layer_lib():
    """The loaded shared library.  Raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = layer_lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_1901_10008_amd.build` (hipcc, gfx950). There is no CPU fallback.")
    L = C.CDLL(path)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    L.sk_layer_params_default.restype = None
    L.sk_layer_params_default.argtypes = [C.POINTER(LayerParams)]
    for kind, problem in (("norm", sk_norm_problem), ("moe", sk_moe_problem), ("verify", sk_verify_problem)):
        for name, args in {"plan_create": [C.POINTER(problem), i32, C.POINTER(LayerParams), C.POINTER(vp)], "plan_destroy": [vp], "launch": [vp, vp],
                           "plan_info": [vp, C.POINTER(i32), C.POINTER(i64)]}.items():
            if kind == "norm" and name == "plan_info":
                continue
            f = getattr(L, f"sk_{kind}_{name}")
            f.restype, f.argtypes = C.c_int, args
    L.sk_last_error.restype = C.c_char_p  # of the libsuperkernel.so that this library is linked to
    L.sk_last_error.argtypes = []
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise SkError(status, (layer_lib().sk_last_error() or b"").decode())


def sk_layer_params_default(**overrides) -> LayerParams:
    p = LayerParams()
    layer_lib().sk_layer_params_default(C.byref(p))
    for k, v in overrides.items():
        if not hasattr(p, k):
            raise AttributeError(k)
        setattr(p, k, v)
    return p


def _make(kind, fields):
    p = kind()
    for k, v in fields.items():
        if not hasattr(p, k):
            raise AttributeError(k)
        setattr(p, k, DTYPE_CODE[v] if k.endswith("dtype") and isinstance(v, str) else v)
    return p


def make_norm_problem(**fields) -> sk_norm_problem:
    """sk_norm_problem from its fields by name (device addresses as numbers, element types as "bf16", "f16", "f32" or their codes); those not named
    are 0, residual_dtype is dtype."""
    return _make(sk_norm_problem, {"residual_dtype": fields.get("dtype", 0)} | fields)


def make_moe_problem(**fields) -> sk_moe_problem:
    """sk_moe_problem from its fields by name, as make_norm_problem; router_dtype is dtype if it is not named."""
    return _make(sk_moe_problem, {"router_dtype": fields.get("dtype", 0)} | fields)


def make_verify_problem(**fields) -> sk_verify_problem:
    """sk_verify_problem from its fields by name, as make_norm_problem."""
    return _make(sk_verify_problem, fields)


class _Plan:
    """Owner of a handle (destroyed on close() / garbage collection)."""

    kind, problem = "", None

    def __init__(self, handle: int, keepalive=None):
        self.handle = handle
        self.keepalive = keepalive

    def close(self):
        if self.handle:
            h, self.handle = self.handle, None
            _check(getattr(layer_lib(), f"sk_{self.kind}_plan_destroy")(h))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class NormPlan(_Plan):
    kind, problem = "norm", sk_norm_problem


class MoePlan(_Plan):
    kind, problem = "moe", sk_moe_problem


class VerifyPlan(_Plan):
    kind, problem = "verify", sk_verify_problem


def _create(plan, problems, params, keepalive):
    n = len(problems)
    arr = (plan.problem * max(n, 1))(*problems)
    out = C.c_void_p()
    _check(getattr(layer_lib(), f"sk_{plan.kind}_plan_create")(arr if n else None, n, C.byref(params) if params is not None else None, C.byref(out)))
    return plan(out.value, keepalive)


def _info(plan):
    launches, workspace = C.c_int32(), C.c_int64()
    _check(getattr(layer_lib(), f"sk_{plan.kind}_plan_info")(plan.handle, C.byref(launches), C.byref(workspace)))
    return launches.value, workspace.value


def sk_norm_plan_create(problems: Sequence[sk_norm_problem], params: LayerParams | None = None, keepalive=None) -> NormPlan:
    return _create(NormPlan, problems, params, keepalive)


def sk_norm_plan_destroy(plan: NormPlan) -> None:
    plan.close()


def sk_norm_launch(plan: NormPlan, stream: int = 0) -> None:
    _check(layer_lib().sk_norm_launch(plan.handle, stream))


def sk_moe_plan_create(problems: Sequence[sk_moe_problem], params: LayerParams | None = None, keepalive=None) -> MoePlan:
    return _create(MoePlan, problems, params, keepalive)


def sk_moe_plan_destroy(plan: MoePlan) -> None:
    plan.close()


def sk_moe_launch(plan: MoePlan, stream: int = 0) -> None:
    _check(layer_lib().sk_moe_launch(plan.handle, stream))


def sk_moe_plan_info(plan: MoePlan):
    """(kernel launches of sk_moe_launch, bytes of the workspace)."""
    return _info(plan)


def sk_verify_plan_create(problems: Sequence[sk_verify_problem], params: LayerParams | None = None, keepalive=None) -> VerifyPlan:
    return _create(VerifyPlan, problems, params, keepalive)


def sk_verify_plan_destroy(plan: VerifyPlan) -> None:
    plan.close()


def sk_verify_launch(plan: VerifyPlan, stream: int = 0) -> None:
    _check(layer_lib().sk_verify_launch(plan.handle, stream))


def sk_verify_plan_info(plan: VerifyPlan):
    """(kernel launches of sk_verify_launch, bytes of the workspace)."""
    return _info(plan)
