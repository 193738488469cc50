"""ctypes binding of libsk_cache.so (include/sk_cache.h) with the same names: attention's side of decoder layers over paged
key/value caches, and the account of pages (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import os
from typing import Iterable, Sequence

from .binding import DTYPE_CODE, SkError

HERE = os.path.dirname(os.path.abspath(__file__))

CACHE_SYMBOLS = [
    "sk_attn_params_default", "sk_attn_plan_create", "sk_attn_plan_destroy", "sk_attn_append", "sk_attn_launch", "sk_attn_plan_info",
    "sk_pages_create", "sk_pages_destroy", "sk_pages_resize", "sk_pages_fork", "sk_pages_compact", "sk_pages_apply", "sk_pages_state",
    "sk_pages_copy",
]


class sk_attn_problem(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "q_heads", "kv_heads", "head_dim", "page_tokens", "num_pages", "sequences", "pages_per_sequence",
                                         "rows", "max_new", "window", "sinks", "rotary_dim", "neighbours", "positions")] + [
        ("eps", C.c_float), ("scale", C.c_float), ("reserved", C.c_int32)] + [(n, C.c_int64) for n in (
            "page_stride", "kv_head_stride", "token_stride", "qkv_row_stride", "q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride")] + [
        (n, C.c_void_p) for n in ("k", "v", "page_table", "lengths", "first_row", "qkv", "q_weight", "k_weight", "cos", "sin", "q", "out")]


class AttnParams(C.Structure):
    _fields_ = [("host_only", C.c_int32), ("workgroups", C.c_int32), ("reserved", C.c_int32 * 2)]


class sk_page_array(C.Structure):
    _fields_ = [("base", C.c_void_p), ("page_bytes", C.c_int64)]


def cache_lib_path() -> str:
    return os.path.join(HERE, "libsk_cache.so")


_lib = None


def cache_lib():
    """The loaded shared library.  Raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    path = cache_lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_1901_10008_amd.build` (hipcc, gfx950). There is no CPU fallback.")
    L = C.CDLL(path)
    vp, i32 = C.c_void_p, C.c_int32
    L.sk_attn_params_default.restype = None
    L.sk_attn_params_default.argtypes = [C.POINTER(AttnParams)]
    for name, args in {
        "sk_attn_plan_create": [C.POINTER(sk_attn_problem), i32, C.POINTER(AttnParams), C.POINTER(vp)],
        "sk_attn_plan_destroy": [vp],
        "sk_attn_append": [vp, vp],
        "sk_attn_launch": [vp, vp],
        "sk_attn_plan_info": [vp, C.POINTER(i32), C.POINTER(C.c_int64)],
        "sk_pages_create": [i32, i32, i32, i32, C.POINTER(vp)],
        "sk_pages_destroy": [vp],
        "sk_pages_resize": [vp, vp, vp, i32],
        "sk_pages_fork": [vp, i32, vp, i32],
        "sk_pages_compact": [vp],
        "sk_pages_apply": [vp, C.POINTER(sk_page_array), i32, vp, vp],
        "sk_pages_state": [vp, C.POINTER(i32), C.POINTER(i32), i32, C.POINTER(i32), vp],
        "sk_pages_copy": [C.POINTER(sk_page_array), i32, i32, vp, vp, i32, vp],
    }.items():
        getattr(L, name).restype = C.c_int
        getattr(L, name).argtypes = args
    L.sk_last_error.restype = C.c_char_p  # of the libsuperkernel.so that this library is linked to
    L.sk_last_error.argtypes = []
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise SkError(status, (cache_lib().sk_last_error() or b"").decode())


# ---- attention plans -----------------------------------------------------------------------------------------------------------

def sk_attn_params_default(**overrides) -> AttnParams:
    p = AttnParams()
    cache_lib().sk_attn_params_default(C.byref(p))
    for k, v in overrides.items():
        if not hasattr(p, k):
            raise AttributeError(k)
        setattr(p, k, v)
    return p


def make_attn_problem(**fields) -> sk_attn_problem:
    """sk_attn_problem from its fields by name (device addresses as numbers, the element type as "bf16", "f16" or its code); those
    not named are 0."""
    p = sk_attn_problem()
    for k, v in fields.items():
        if not hasattr(p, k):
            raise AttributeError(k)
        setattr(p, k, DTYPE_CODE[v] if k == "dtype" and isinstance(v, str) else v)
    return p


class _Owner:
    """Owner of a handle (destroyed on close() / garbage collection)."""

    destroy = ""

    def __init__(self, handle: int, keepalive=None):
        self.handle = handle
        self.keepalive = keepalive

    def close(self):
        if self.handle:
            h, self.handle = self.handle, None
            _check(getattr(cache_lib(), self.destroy)(h))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


class AttnPlan(_Owner):
    destroy = "sk_attn_plan_destroy"


class Pages(_Owner):
    destroy = "sk_pages_destroy"


def sk_attn_plan_create(problems: Sequence[sk_attn_problem], params: AttnParams | None = None, keepalive=None) -> AttnPlan:
    n = len(problems)
    arr = (sk_attn_problem * max(n, 1))(*problems)
    out = C.c_void_p()
    _check(cache_lib().sk_attn_plan_create(arr if n else None, n, C.byref(params) if params is not None else None, C.byref(out)))
    return AttnPlan(out.value, keepalive)


def sk_attn_plan_destroy(plan: AttnPlan) -> None:
    plan.close()


def sk_attn_append(plan: AttnPlan, stream: int = 0) -> None:
    _check(cache_lib().sk_attn_append(plan.handle, stream))


def sk_attn_launch(plan: AttnPlan, stream: int = 0) -> None:
    _check(cache_lib().sk_attn_launch(plan.handle, stream))


def sk_attn_plan_info(plan: AttnPlan):
    """(kernel launches of sk_attn_launch, bytes of the workspace)."""
    launches, workspace = C.c_int32(), C.c_int64()
    _check(cache_lib().sk_attn_plan_info(plan.handle, C.byref(launches), C.byref(workspace)))
    return launches.value, workspace.value


# ---- pages ---------------------------------------------------------------------------------------------------------------------

def make_ids(numbers: Iterable[int]):
    """Numbers of sequences, tokens or pages as the calls take them (a ctypes array, which may be kept)."""
    numbers = list(numbers)
    return (C.c_int32 * len(numbers))(*numbers)


def _ids(numbers):
    return numbers if isinstance(numbers, C.Array) and numbers._type_ is C.c_int32 else make_ids(numbers)


def make_page_arrays(arrays):
    """Arrays of pages from (device address, bytes of a page) pairs, as the calls take them (a ctypes array, which may be kept)."""
    arrays = [sk_page_array(a, n) for a, n in arrays]
    return (sk_page_array * len(arrays))(*arrays)


def sk_pages_create(num_pages: int, page_tokens: int, sequences: int, pages_per_sequence: int) -> Pages:
    out = C.c_void_p()
    _check(cache_lib().sk_pages_create(num_pages, page_tokens, sequences, pages_per_sequence, C.byref(out)))
    p = Pages(out.value)
    p.columns = pages_per_sequence
    return p


def sk_pages_destroy(pages: Pages) -> None:
    pages.close()


def sk_pages_resize(pages: Pages, sequences, tokens) -> None:
    if len(sequences) != len(tokens):
        raise ValueError("as many numbers of tokens as sequences are wanted")
    s, t = _ids(sequences), _ids(tokens)
    _check(cache_lib().sk_pages_resize(pages.handle, C.addressof(s), C.addressof(t), len(s)))


def sk_pages_fork(pages: Pages, from_: int, to) -> None:
    t = _ids(to)
    _check(cache_lib().sk_pages_fork(pages.handle, from_, C.addressof(t), len(t)))


def sk_pages_compact(pages: Pages) -> None:
    _check(cache_lib().sk_pages_compact(pages.handle))


def sk_pages_apply(pages: Pages, arrays, page_table: int = 0, stream: int = 0) -> None:
    _check(cache_lib().sk_pages_apply(pages.handle, arrays, len(arrays), page_table, stream))


def sk_pages_state(pages: Pages, sequence: int | None = None):
    """(free pages, pending copies), or of a sequence (tokens, its row of the page table)."""
    if sequence is None:
        free, pending = C.c_int32(), C.c_int32()
        _check(cache_lib().sk_pages_state(pages.handle, C.byref(free), C.byref(pending), 0, None, None))
        return free.value, pending.value
    tokens, row = C.c_int32(), (C.c_int32 * pages.columns)()
    _check(cache_lib().sk_pages_state(pages.handle, None, None, sequence, C.byref(tokens), C.addressof(row)))
    return tokens.value, list(row)


def sk_pages_copy(arrays, num_pages: int, from_, to, stream: int = 0) -> None:
    if len(from_) != len(to):
        raise ValueError("as many pages to copy from as to copy to are wanted")
    f, t = _ids(from_), _ids(to)
    _check(cache_lib().sk_pages_copy(arrays, len(arrays), num_pages, C.addressof(f), C.addressof(t), len(f), stream))
