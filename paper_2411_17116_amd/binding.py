"""Binding of libstarattn.so (see include/star_attn.h for the contract): queries through ctypes, the
calls that enqueue work through the extension module built from csrc/marshal.cpp, or through ctypes too, at some
4 us of host time more, where it has not been built or does not load with this torch."""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import warnings
from typing import Optional

import torch

F32 = 0
BF16 = 1
ANCHOR_FIRST = 0
ANCHOR_PREVIOUS = 1
ANCHOR_EXTERNAL = 2
ANCHOR_PER_BLOCK = 3
ANCHOR_ALL_BLOCKS = 4

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None
_MARSHAL = None       # the calls that enqueue work: the extension module, bound to _LIB's entry points, or _CtypesCalls


class StarAttnError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"star_attn: {what} (status {code})")
        self.code = code


class StarShape(ctypes.Structure):
    """Mirror of `star_attn_shape`."""
    _fields_ = [
        ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("ctx_len", ctypes.c_int64), ("block", ctypes.c_int64), ("anchor", ctypes.c_int64),
        ("cache_capacity", ctypes.c_int64),
        ("softmax_scale", ctypes.c_float), ("reserved2", ctypes.c_float),
    ]

    @classmethod
    def make(cls, dtype, batch, n_q_heads, n_kv_heads, head_dim, ctx_len, block, anchor,
             cache_capacity, softmax_scale=0.0) -> "StarShape":
        if isinstance(dtype, torch.dtype):
            dtype = {torch.float32: F32, torch.bfloat16: BF16}.get(dtype, -1)
        elif isinstance(dtype, str):
            dtype = {"fp32": F32, "bf16": BF16}.get(dtype, -1)
        return cls(int(dtype), int(batch), int(n_q_heads), int(n_kv_heads), int(head_dim), 0,
                   int(ctx_len), int(block), int(anchor), int(cache_capacity),
                   float(softmax_scale), 0.0)


class StarRotary(ctypes.Structure):
    """Mirror of `star_attn_rotary`."""
    _fields_ = [
        ("rope_theta", ctypes.c_double), ("pos0", ctypes.c_int64), ("positions", ctypes.c_void_p),
        ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p), ("norm_eps", ctypes.c_float),
        ("n_axes", ctypes.c_int32), ("axis", ctypes.c_uint8 * 64),
    ]


def _pointer(t, what, dtype=None, shape=None):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("star_attn tensors must be contiguous")
    if (dtype is not None and t.dtype != dtype) or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{what}: {tuple(t.shape)} {t.dtype} given" + (f", {tuple(shape)} wanted" if shape else ""))
    return t.data_ptr()


class Rotary:
    """How a call's queries and keys are normed per head and rotated (`star_attn_rotary`); holds on to its tensors.

    q_norm, k_norm: weights [d] in the storage dtype, None: not normed.  positions: int64 [B, n_tokens, n_axes] (or [B,
    n_tokens]) of the call's tokens, None: they follow each other from pos0 on (in phase 2 behind the cache).  sections: how many of
    the d / 2 frequencies each axis turns, one after the other; or `axis`: every frequency's axis."""

    def __init__(self, rope_theta: float, q_norm=None, k_norm=None, eps: float = 1e-6, pos0: int = 0, positions=None,
                 sections=None, axis=None):
        if sections is not None and axis is not None:
            raise ValueError("sections or axis, not both")
        if sections is not None:
            axis = [a for a, n in enumerate(sections) for _ in range(n)]
        axes = [0] if axis is None else [int(a) for a in axis]
        n_axes = len(sections) if sections is not None else max(axes) + 1
        if positions is not None:
            n_axes = max(n_axes, positions.shape[2]) if positions.dim() == 3 else 1
            if positions.dim() not in (2, 3) or (positions.dim() == 3 and positions.shape[2] != n_axes) or max(axes) >= n_axes:
                raise ValueError("positions are [batch, tokens, axes]")
        if axis is not None and (len(axes) not in (32, 64) or min(axes) < 0):
            raise ValueError("an axis for each of the d / 2 frequencies is wanted")
        for w in (q_norm, k_norm):
            if w is not None and w.dim() != 1:
                raise ValueError("norm weights are [head_dim]")
        norms = {(w.shape[0], w.element_size()) for w in (q_norm, k_norm) if w is not None}
        if len(norms) > 1:
            raise ValueError("norm weights are [head_dim] in the storage dtype")
        self.tensors = (q_norm, k_norm, positions)
        self.c = StarRotary(float(rope_theta), int(pos0), _pointer(positions, "positions", torch.int64), _pointer(q_norm, "q_norm"),
                            _pointer(k_norm, "k_norm"), float(eps), n_axes, (ctypes.c_uint8 * 64)(*axes))
        size, item = next(iter(norms), (0, 0))
        tokens = (0, 0) if positions is None else tuple(positions.shape[:2])
        self.held = _HeldRotary(self.c, size, item, 0 if axis is None else len(axes), *tokens)


class _HeldRotary(ctypes.Structure):
    """A call's checks of it are made where its arguments are read: the extension module, or _CtypesCalls."""
    _fields_ = [("c", StarRotary), ("norm", ctypes.c_int32), ("item", ctypes.c_int32), ("frequencies", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("tokens", ctypes.c_int64)]

    def of(self, shape: StarShape, n_tokens: int) -> StarRotary:
        if self.norm and (self.norm != shape.head_dim or self.item != (4 if shape.dtype == F32 else 2)):
            raise ValueError("norm weights are [head_dim] in the storage dtype")
        if self.c.positions and (self.batch, self.tokens) != (shape.batch, n_tokens):
            raise ValueError("positions of other tokens than the call's")
        if self.frequencies and 2 * self.frequencies != shape.head_dim:
            raise ValueError("an axis for each of the d / 2 frequencies is wanted")
        return self.c


class StarQ4(ctypes.Structure):
    """Mirror of `star_attn_q4_cache`."""
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


class Q4Cache:
    """A cache held in four bits (`star_attn_q4_cache`): uint8 codes [B, Hkv, cache_capacity, d / 2] and exponents
    [B, Hkv, cache_capacity, d / 32] of K and of V, the caller's tensors (alloc_q4_cache makes them)."""

    def __init__(self, shape: StarShape, k_codes, k_scales, v_codes, v_scales):
        rows = (shape.batch, shape.n_kv_heads, shape.cache_capacity)
        sizes = {"codes": rows + (shape.head_dim // 2,), "scales": rows + (shape.head_dim // 32,)}
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.c = StarQ4(*(_pointer(getattr(self, n), n, torch.uint8, sizes[n[2:]]) for n, _ in StarQ4._fields_))
        self.held = _HeldQ4(self.c, shape.batch, shape.n_kv_heads, shape.head_dim, 0, shape.cache_capacity)


class _HeldQ4(ctypes.Structure):
    _fields_ = [("c", StarQ4), ("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("unused", ctypes.c_int32), ("rows", ctypes.c_int64)]

    def of(self, shape: StarShape) -> StarQ4:
        if (self.batch, self.heads, self.head_dim, self.rows) != (shape.batch, shape.n_kv_heads, shape.head_dim, shape.cache_capacity):
            raise ValueError("a four-bit cache of another shape than the call's")
        return self.c


class PlanInfo(ctypes.Structure):
    """Mirror of `star_attn_plan_info`."""
    _fields_ = [
        ("decode", ctypes.c_int32), ("flat", ctypes.c_int32), ("n_splits", ctypes.c_int32),
        ("non_temporal", ctypes.c_int32), ("steps_per_batch", ctypes.c_int32),
        ("tile_rows", ctypes.c_int32), ("split_len", ctypes.c_int64),
        ("workspace_bytes", ctypes.c_int64),
    ]


class Phase1PlanInfo(ctypes.Structure):
    """Mirror of `star_attn_phase1_plan_info`."""
    _fields_ = [
        ("queued", ctypes.c_int32), ("tile_rows", ctypes.c_int32), ("wavefronts", ctypes.c_int32),
        ("group", ctypes.c_int32), ("n_tiles", ctypes.c_int64),
    ]


def lib_path() -> str:
    return os.path.join(_HERE, "libstarattn.so")


def load_library():
    """Load the built library; raises if it has not been built (no fallback)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2411_17116_amd.build`")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER(StarShape)
    vp, sz, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
    lib.star_attn_workspace_bytes.restype = sz
    lib.star_attn_workspace_bytes.argtypes = [P, i64]
    lib.star_attn_phase1.restype = ctypes.c_int
    lib.star_attn_phase1.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.star_attn_phase1_anchor.restype = ctypes.c_int
    lib.star_attn_phase1_anchor.argtypes = [P, ctypes.c_int, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                            vp, sz, vp]
    lib.star_attn_phase1_workspace_bytes.restype = sz
    lib.star_attn_phase1_workspace_bytes.argtypes = [P, ctypes.c_int]
    dbl = ctypes.c_double
    lib.star_attn_phase1_rope.restype = ctypes.c_int
    lib.star_attn_phase1_rope.argtypes = [P, dbl, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.star_attn_phase2_rope.restype = ctypes.c_int
    lib.star_attn_phase2_rope.argtypes = [P, dbl, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                          sz, vp]
    lib.star_attn_rope.restype = ctypes.c_int
    lib.star_attn_rope.argtypes = [P, ctypes.c_int32, i64, i64, dbl, vp, vp, vp]
    lib.star_attn_phase2.restype = ctypes.c_int
    lib.star_attn_phase2.argtypes = [P, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.star_attn_phase2_static.restype = ctypes.c_int
    lib.star_attn_phase2_static.argtypes = [P, i64, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.star_attn_phase2_partial.restype = ctypes.c_int
    lib.star_attn_phase2_partial.argtypes = [P, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.star_attn_merge.restype = ctypes.c_int
    lib.star_attn_merge.argtypes = [P, i64, i64, vp, vp, vp, vp, vp, vp]
    lib.star_attn_status_string.restype = ctypes.c_char_p
    lib.star_attn_status_string.argtypes = [ctypes.c_int]
    lib.star_attn_phase2_plan.restype = ctypes.c_int
    lib.star_attn_phase2_plan.argtypes = [P, i64, i64, ctypes.c_int, ctypes.POINTER(PlanInfo)]
    lib.star_attn_phase1_plan.restype = ctypes.c_int
    lib.star_attn_phase1_plan.argtypes = [P, ctypes.c_int, ctypes.POINTER(Phase1PlanInfo)]
    R, C4 = ctypes.POINTER(StarRotary), ctypes.POINTER(StarQ4)
    for name, kinds in {
            "qk_norm_rope": [P, R, i64, vp, vp, vp, vp, vp],
            "phase1_norm_rope": [P, R, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
            "phase2_norm_rope": [P, R, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
            "q4_store": [P, i64, i64, vp, vp, i64, i64, C4, vp],
            "q4_load": [P, i64, i64, C4, vp, vp, i64, i64, vp],
            "phase2_q4": [P, R, i64, i64, vp, vp, vp, C4, vp, vp, vp, vp, sz, vp],
            "phase2_q4_partial": [P, i64, i64, vp, vp, vp, C4, vp, vp, vp, sz, vp],
            "phase2_q4_plan": [P, i64, i64, ctypes.c_int, ctypes.POINTER(PlanInfo)]}.items():
        getattr(lib, "star_attn_" + name).restype = ctypes.c_int
        getattr(lib, "star_attn_" + name).argtypes = kinds
    lib.star_attn_q4_workspace_bytes.restype = sz
    lib.star_attn_q4_workspace_bytes.argtypes = [P, i64]
    lib.star_attn_kernel_path.restype = ctypes.c_char_p
    lib.star_attn_kernel_path.argtypes = [P]
    _LIB = lib
    return lib


def _bind(lib) -> None:
    """Load the extension module and hand it the library's entry points."""
    global _MARSHAL
    path = os.path.join(_HERE, "_marshal.so")
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2411_17116_amd.build`")
    if not hasattr(_MARSHAL, "bind"):
        loader = importlib.machinery.ExtensionFileLoader("_marshal", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
        loader.exec_module(module)
    else:
        module = _MARSHAL
    names = ("phase1", "phase1_anchor", "phase1_rope", "phase2", "phase2_rope", "phase2_static",
             "phase2_partial", "merge", "rope")
    q4_names = ("qk_norm_rope", "phase1_norm_rope", "phase2_norm_rope", "q4_store", "q4_load", "phase2_q4", "phase2_q4_partial")
    addresses = lambda names: tuple(ctypes.cast(getattr(lib, "star_attn_" + n), ctypes.c_void_p).value for n in names)
    module.bind(StarShape, addresses(names))
    if hasattr(lib, "star_attn_phase2_q4"):
        module.bind_q4(addresses(q4_names))
    _MARSHAL = module


class _CtypesCalls:
    """The extension module's calls by ctypes alone: same arguments, same refusals."""
    # what follows the shape and precedes the stream: t a tensor's address, w and its bytes, q behind its shape[1],
    # m behind its shape[0] and shape[3]; i and d numbers; 4 a four-bit cache
    _KINDS = {"phase1": "tttttttw", "phase1_anchor": "itttttttttw", "phase1_rope": "ditttttttw", "phase2": "iqtttttttw",
              "phase2_rope": "diiqtttttttw", "phase2_static": "iqttttt", "phase2_partial": "iqttttttw", "merge": "mtttt"}
    _Q4_KINDS = {"phase2_q4_partial": "iqtt4ttw"}

    def __init__(self, lib):
        self._rope, kinds = lib.star_attn_rope, dict(self._KINDS)
        if hasattr(lib, "star_attn_phase2_q4"):
            self._lib = lib
            kinds.update(self._Q4_KINDS)
        for name, kinds in kinds.items():
            setattr(self, name, self._entry(getattr(lib, "star_attn_" + name), kinds))

    @staticmethod
    def _address(t):
        if t is None:
            return None
        if not t.is_contiguous():
            raise ValueError("star_attn tensors must be contiguous")
        return t.data_ptr()

    def _entry(self, fn, kinds):
        def call(shape, *args):
            *values, stream = args
            if len(values) != len(kinds):
                raise TypeError("wrong number of arguments")
            out = [ctypes.byref(shape)]
            for kind, x in zip(kinds, values):
                if kind == "q":
                    out.append(x.shape[1])
                elif kind == "m":
                    out += [x.shape[0], x.shape[3]]
                out.append(x if kind in "id" else ctypes.byref(x.of(shape)) if kind == "4" else self._address(x))
                if kind == "w":
                    out.append(0 if x is None else x.numel() * x.element_size())
            return fn(*out, stream)
        return call

    def rope(self, shape, X, Y, theta, pos0, stream):
        return self._rope(ctypes.byref(shape), X.shape[2], X.shape[1], pos0, theta, self._address(X), self._address(Y), stream)


    def qk_norm_rope(self, shape, tokens, rotary, Q, K, Yq, Yk, stream):
        return self._lib.star_attn_qk_norm_rope(ctypes.byref(shape), ctypes.byref(rotary.of(shape, tokens)), tokens,
                                                *map(self._address, (Q, K, Yq, Yk)), stream)

    def phase1_norm_rope(self, shape, rotary, Q, K, V, O, LSE, Kc, Vc, ws, stream):
        return self._lib.star_attn_phase1_norm_rope(ctypes.byref(shape), ctypes.byref(rotary.of(shape, shape.ctx_len)),
                                                    *map(self._address, (Q, K, V, O, LSE, Kc, Vc, ws)), _nbytes(ws), stream)

    def phase2_norm_rope(self, shape, cached, Q, rotary, K, V, Kc, Vc, O_part, LSE_part, O, ws, stream):
        q = Q.shape[1]
        return self._lib.star_attn_phase2_norm_rope(ctypes.byref(shape), ctypes.byref(rotary.of(shape, q)), cached, q,
                                                    *map(self._address, (Q, K, V, Kc, Vc, O_part, LSE_part, O, ws)), _nbytes(ws), stream)

    def q4_store(self, shape, row, rows, K, V, plain_row, cache, stream):
        return self._lib.star_attn_q4_store(ctypes.byref(shape), row, rows, self._address(K), self._address(V), K.shape[2], plain_row,
                                            ctypes.byref(cache.of(shape)), stream)

    def q4_load(self, shape, row, rows, K, V, plain_row, cache, stream):
        return self._lib.star_attn_q4_load(ctypes.byref(shape), row, rows, ctypes.byref(cache.of(shape)), self._address(K), self._address(V),
                                           K.shape[2], plain_row, stream)

    def phase2_q4(self, shape, cached, Q, rotary, K, V, cache, O_part, LSE_part, O, ws, stream):
        q = Q.shape[1]
        rotary = None if rotary is None else ctypes.byref(rotary.of(shape, q))
        return self._lib.star_attn_phase2_q4(ctypes.byref(shape), rotary, cached, q, *map(self._address, (Q, K, V)), ctypes.byref(cache.of(shape)),
                                             *map(self._address, (O_part, LSE_part, O, ws)), _nbytes(ws), stream)


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def _calls():
    global _MARSHAL
    if _MARSHAL is None:
        lib = load_library()
        try:
            _bind(lib)
        except (ImportError, OSError) as e:
            warnings.warn(f"star_attn calls go through ctypes, some 4 us of host time more each: {e}")
            _MARSHAL = _CtypesCalls(lib)
    return _MARSHAL


def status_string(code: int) -> str:
    return load_library().star_attn_status_string(int(code)).decode()


def kernel_path(shape: StarShape) -> Optional[str]:
    r = load_library().star_attn_kernel_path(ctypes.byref(shape))
    return r.decode() if r else None


def phase2_plan(shape: StarShape, cache_len: int, q_len: int, want_parts: bool = False) -> PlanInfo:
    """star_attn_phase2_plan: what a phase-2 call with these arguments would run."""
    info = PlanInfo()
    _check(load_library().star_attn_phase2_plan(ctypes.byref(shape), int(cache_len), int(q_len),
                                                int(bool(want_parts)), ctypes.byref(info)))
    return info


def phase1_plan(shape: StarShape, anchor_mode: int = ANCHOR_FIRST) -> Phase1PlanInfo:
    """star_attn_phase1_plan: which set-up a phase-1 call would take."""
    info = Phase1PlanInfo()
    _check(load_library().star_attn_phase1_plan(ctypes.byref(shape), int(anchor_mode), ctypes.byref(info)))
    return info


def workspace_bytes(shape: StarShape, max_q_len: int) -> int:
    return int(load_library().star_attn_workspace_bytes(ctypes.byref(shape), int(max_q_len)))


# The current stream's handle comes from torch's own raw look-up (0.3 us; a torch.cuda.Stream object made
# for its handle 3 us).
_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _RAW_STREAM is not None and torch.cuda.is_initialized():
        return _RAW_STREAM(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _check(rc: int):
    if rc != 0:
        raise StarAttnError(rc, status_string(rc))


def alloc_cache(shape: StarShape, device="cuda"):
    """Caller-owned K/V caches [B, Hkv, cache_capacity, d] in the shape's dtype."""
    dt = torch.float32 if shape.dtype == F32 else torch.bfloat16
    dims = (shape.batch, shape.n_kv_heads, shape.cache_capacity, shape.head_dim)
    return torch.zeros(dims, dtype=dt, device=device), torch.zeros(dims, dtype=dt, device=device)


def alloc_workspace(shape: StarShape, max_q_len: int, device="cuda") -> torch.Tensor:
    n = workspace_bytes(shape, max_q_len)
    if n == 0:
        raise StarAttnError(-1, "invalid shape for workspace query")
    return torch.empty(n, dtype=torch.uint8, device=device)


def phase1(shape: StarShape, Q, K, V, O_ctx, K_cache, V_cache, LSE_ctx=None,
           workspace=None, stream=None) -> None:
    """star_attn_phase1: context encoding; fills O_ctx, the caches and LSE_ctx."""
    _check(_calls().phase1(shape, Q, K, V, O_ctx, LSE_ctx, K_cache, V_cache, workspace, _stream(stream)))


def phase1_workspace_bytes(shape: StarShape, anchor_mode: int) -> int:
    return int(load_library().star_attn_phase1_workspace_bytes(ctypes.byref(shape), int(anchor_mode)))


def phase1_anchor(shape: StarShape, anchor_mode: int, Q, K, V, O_ctx, K_cache, V_cache,
                  K_anchor=None, V_anchor=None, LSE_ctx=None, workspace=None, stream=None) -> None:
    """star_attn_phase1_anchor: phase 1 under an anchor variant of the ablation study."""
    _check(_calls().phase1_anchor(shape, int(anchor_mode), Q, K, V, K_anchor, V_anchor, O_ctx, LSE_ctx,
                                  K_cache, V_cache, workspace, _stream(stream)))


def phase1_rope(shape: StarShape, rope_theta: float, Q, K, V, O_ctx, K_cache, V_cache, pos0=0,
                LSE_ctx=None, workspace=None, stream=None) -> None:
    """star_attn_phase1_rope: phase 1 on unrotated Q (rotated in place) and K."""
    _check(_calls().phase1_rope(shape, float(rope_theta), int(pos0), Q, K, V, O_ctx, LSE_ctx, K_cache, V_cache,
                                workspace, _stream(stream)))


def phase2_rope(shape: StarShape, rope_theta: float, cache_len: int, Qq, Kq, Vq, K_cache, V_cache,
                O, workspace, pos0=0, O_part=None, LSE_part=None, stream=None) -> None:
    """star_attn_phase2_rope: phase 2 on unrotated Qq (rotated in place) and Kq."""
    _check(_calls().phase2_rope(shape, float(rope_theta), int(pos0), int(cache_len), Qq, Kq, Vq, K_cache, V_cache,
                                O_part, LSE_part, O, workspace, _stream(stream)))


def rope(shape: StarShape, X, Y, rope_theta: float, pos0=0, stream=None) -> None:
    """star_attn_rope: rotate X [B, T, H, d] into Y (may be X), token t at pos0 + t."""
    _check(_calls().rope(shape, X, Y, float(rope_theta), int(pos0), _stream(stream)))


def phase2(shape: StarShape, cache_len: int, Qq, Kq, Vq, K_cache, V_cache, O, workspace,
           O_part=None, LSE_part=None, stream=None) -> None:
    """star_attn_phase2: appends Kq/Vq at cache_len, then global attention of the
    q_len = Qq.shape[1] new tokens; fills O (and the per-part outputs if given)."""
    _check(_calls().phase2(shape, int(cache_len), Qq, Kq, Vq, K_cache, V_cache, O_part, LSE_part, O, workspace,
                           _stream(stream)))


STATIC_SCRATCH_BYTES = 16 << 20


def phase2_static(shape: StarShape, cache_len: int, Qq, Kq, Vq, K_cache, V_cache, O,
                  stream=None) -> None:
    """star_attn_phase2_static: star_attn_phase2 with the library's static scratch
    in place of a workspace (allocates nothing; calls must not overlap on a GPU)."""
    _check(_calls().phase2_static(shape, int(cache_len), Qq, Kq, Vq, K_cache, V_cache, O, _stream(stream)))


def phase2_partial(shape: StarShape, cache_len: int, Qq, K_cache, V_cache, A, LSE, workspace,
                   Kq=None, Vq=None, stream=None) -> None:
    """star_attn_phase2_partial: one host's pair (A, LSE) for the q_len = Qq.shape[1]
    new tokens; with Kq/Vq the query host's share (append, then attend causally)."""
    _check(_calls().phase2_partial(shape, int(cache_len), Qq, Kq, Vq, K_cache, V_cache, A, LSE, workspace,
                                   _stream(stream)))


def merge(shape: StarShape, A_parts, LSE_parts, O=None, A=None, LSE=None, stream=None) -> None:
    """star_attn_merge: Eq. 3-4 over the n_parts = A_parts.shape[0] gathered pairs."""
    _check(_calls().merge(shape, A_parts, LSE_parts, O, A, LSE, _stream(stream)))


def qk_norm_rope(shape: StarShape, rotary: Rotary, Q, K, Yq, Yk, stream=None) -> None:
    """star_attn_qk_norm_rope: queries Q and keys K [B, T, H, d] (either may be None) normed per head and rotated into
    Yq and Yk (which may be Q and K)."""
    tokens = (Q if Q is not None else K).shape[1]
    _check(_calls().qk_norm_rope(shape, tokens, rotary.held, Q, K, Yq, Yk, _stream(stream)))


def phase1_norm_rope(shape: StarShape, rotary: Rotary, Q, K, V, O_ctx, K_cache, V_cache, LSE_ctx=None, workspace=None,
                     stream=None) -> None:
    """star_attn_phase1_norm_rope: phase 1 on queries (normed and rotated in place) and keys as they are projected."""
    _check(_calls().phase1_norm_rope(shape, rotary.held, Q, K, V, O_ctx, LSE_ctx, K_cache, V_cache, workspace, _stream(stream)))


def phase2_norm_rope(shape: StarShape, rotary: Rotary, cache_len: int, Qq, Kq, Vq, K_cache, V_cache, O, workspace,
                     O_part=None, LSE_part=None, stream=None) -> None:
    """star_attn_phase2_norm_rope: phase 2 on queries (normed and rotated in place) and keys as they are projected."""
    _check(_calls().phase2_norm_rope(shape, int(cache_len), Qq, rotary.held, Kq, Vq, K_cache, V_cache, O_part, LSE_part, O,
                                     workspace, _stream(stream)))


def alloc_q4_cache(shape: StarShape, device="cuda") -> Q4Cache:
    """A caller-owned cache in four bits, all zeros."""
    rows = (shape.batch, shape.n_kv_heads, shape.cache_capacity)
    return Q4Cache(shape, *(torch.zeros(rows + (shape.head_dim // n,), dtype=torch.uint8, device=device) for n in (2, 32) * 2))


def q4_workspace_bytes(shape: StarShape, max_q_len: int) -> int:
    return int(load_library().star_attn_q4_workspace_bytes(ctypes.byref(shape), int(max_q_len)))


def alloc_q4_workspace(shape: StarShape, max_q_len: int, device="cuda") -> torch.Tensor:
    n = q4_workspace_bytes(shape, max_q_len)
    if n == 0:
        raise StarAttnError(-1, "invalid shape for workspace query")
    return torch.empty(n, dtype=torch.uint8, device=device)


def q4_store(shape: StarShape, first_row: int, n_rows: int, K, V, cache: Q4Cache, plain_row=None, stream=None) -> None:
    """star_attn_q4_store: rows [plain_row, plain_row + n_rows) of K and V [B, Hkv, rows, d] (by default those of the same
    numbers) into rows [first_row, first_row + n_rows) of the cache."""
    _check(_calls().q4_store(shape, int(first_row), int(n_rows), K, V, int(first_row if plain_row is None else plain_row), cache.held,
                             _stream(stream)))


def q4_load(shape: StarShape, first_row: int, n_rows: int, cache: Q4Cache, K, V, plain_row=None, stream=None) -> None:
    """star_attn_q4_load: the same rows of the cache into K and V, as what their codes stand for."""
    _check(_calls().q4_load(shape, int(first_row), int(n_rows), K, V, int(first_row if plain_row is None else plain_row), cache.held,
                            _stream(stream)))


def phase2_q4(shape: StarShape, cache_len: int, Qq, Kq, Vq, cache: Q4Cache, O, workspace, rotary: Optional[Rotary] = None,
              O_part=None, LSE_part=None, stream=None) -> None:
    """star_attn_phase2_q4: files Kq/Vq in the four-bit cache at cache_len, then attends to all it holds; with `rotary`, Qq
    (in place) and Kq are normed and rotated first."""
    _check(_calls().phase2_q4(shape, int(cache_len), Qq, None if rotary is None else rotary.held, Kq, Vq, cache.held, O_part, LSE_part, O,
                              workspace, _stream(stream)))


def phase2_q4_partial(shape: StarShape, cache_len: int, Qq, cache: Q4Cache, A, LSE, workspace, Kq=None, Vq=None, stream=None) -> None:
    """star_attn_phase2_q4_partial: one host's pair (A, LSE) over a four-bit cache (see phase2_partial)."""
    _check(_calls().phase2_q4_partial(shape, int(cache_len), Qq, Kq, Vq, cache.held, A, LSE, workspace, _stream(stream)))


def phase2_q4_plan(shape: StarShape, cache_len: int, q_len: int, want_parts: bool = False) -> PlanInfo:
    """star_attn_phase2_q4_plan: what a phase2_q4 call with these arguments would run."""
    info = PlanInfo()
    _check(load_library().star_attn_phase2_q4_plan(ctypes.byref(shape), int(cache_len), int(q_len), int(bool(want_parts)),
                                                   ctypes.byref(info)))
    return info
