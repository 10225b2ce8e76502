"""ctypes binding of liblibra.so: the same entry points as include/libra.h, argument
marshalling only.  Tensors are torch CUDA tensors (device memory and streams come from
torch); every computation runs in the library's kernels.

Importing this module loads the library and raises if it has not been built — there is
no CPU fallback.
"""
from __future__ import annotations

import collections
import ctypes
import functools
import inspect
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "liblibra.so")
if not os.path.exists(_SO):
    raise ImportError(f"{_SO} is missing: run `python -m paper_2607_23250_b200.build` (needs nvcc)")
_lib = ctypes.CDLL(_SO)

LIBRA_DIR_Q, LIBRA_DIR_KV, LIBRA_DIR_PAIR = 1, 2, 4
LIBRA_WEIGHT_PAIRS, LIBRA_WEIGHT_BLOCKS = 0, 1
KERNEL_FWD, KERNEL_BWD_DKDV, KERNEL_BWD_DQ, KERNEL_BWD_PREP, KERNEL_BWD_FUSED, KERNEL_BWD_POST = 1, 2, 3, 4, 5, 6
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_PLAN_MISMATCH, ERR_CUDA = -1, -2, -3, -4
ERR_OVERFLOW, ERR_TIMEOUT, ERR_BAD_SEQLENS, ERR_NO_DEVICE = -5, -6, -7, -8
ERR_SCRATCH_TOO_SMALL = -9

EXPORTS = ["libra_plan_tiles", "libra_plan_tiles_window", "libra_plan_info", "libra_plan_status", "libra_plan_export",
           "libra_plan_export_pairs", "libra_plan_fused_ctas", "libra_plan_destroy", "libra_attn_pool_fwd", "libra_attn_pool_bwd_workspace_bytes",
           "libra_attn_pool_bwd", "libra_attn_pool_bwd_noalloc_max_bytes", "libra_attn_pool_bwd_noalloc",
           "libra_ckpt8_pack", "libra_ckpt8_unpack", "libra_attn_pool_bwd_ckpt8_workspace_bytes", "libra_attn_pool_bwd_ckpt8",
           "libra_tap_schedule", "libra_busy_times", "libra_tile_times", "libra_plan_set_wait_limit_ns", "libra_plan_inject_stall", "libra_plan_set_timing", "libra_kernel_time_ms", "libra_kernel_times_ms", "libra_selftest_wait_timeout", "libra_launch_count",
           "libra_strerror"]


class PlanOpts(ctypes.Structure):
    _fields_ = [("n_workers", ctypes.c_int), ("directions", ctypes.c_int), ("tile_kv", ctypes.c_int),
                ("n_heads_kv", ctypes.c_int), ("total_tokens", ctypes.c_int64), ("weight_model", ctypes.c_int),
                ("cost_block", ctypes.c_int), ("unit_cost_q", ctypes.c_int), ("unit_cost_kv", ctypes.c_int),
                ("pair_chunk", ctypes.c_int)]


class Dims(ctypes.Structure):
    _fields_ = [("total_tokens", ctypes.c_int64), ("n_samples", ctypes.c_int), ("hq", ctypes.c_int),
                ("hkv", ctypes.c_int), ("head_dim", ctypes.c_int), ("softmax_scale", ctypes.c_float)]


class _Ckpt8Pointers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v", "out", "q_exp", "k_exp", "v_exp", "out_exp")]


# An 8-bit checkpoint: int8 values [T, H, d] and exponent bytes (uint8) [T, H, d / 32] of each tensor, or None.
Ckpt8 = collections.namedtuple("Ckpt8", "q k v out q_exp k_exp v_exp out_exp", defaults=[None] * 8)

_lib.libra_strerror.restype = ctypes.c_char_p
_lib.libra_attn_pool_bwd_ckpt8_workspace_bytes.restype = ctypes.c_size_t
_lib.libra_launch_count.restype = ctypes.c_int64
_lib.libra_attn_pool_bwd_workspace_bytes.restype = ctypes.c_size_t
_lib.libra_attn_pool_bwd_noalloc_max_bytes.restype = ctypes.c_size_t
_vp = ctypes.c_void_p


class LibraError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        super().__init__(f"{what}: {_lib.libra_strerror(code).decode()} ({code})")


def _check(code, what):
    if code != 0:
        raise LibraError(code, what)


def _ptr(t):
    return _vp(t.data_ptr()) if t is not None else _vp(0)


def _np(a):
    return a.ctypes.data_as(_vp) if a is not None else _vp(0)


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return _vp(s.cuda_stream)


def _on_its_stream(f):
    """f(..., stream=s) as `with torch.cuda.stream(s): f(...)`: tensors and workspaces that the call allocates belong to s.  (Of the
    current stream's memory, one that is freed at the end of the call would be handed out again while the kernels on s still use it.)"""
    at = list(inspect.signature(f).parameters).index("stream")

    @functools.wraps(f)
    def call(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None:
            return f(*args, **kw)
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream.cuda_stream)
        with torch.cuda.stream(stream):
            return f(*args, **kw)
    return call


def libra_selftest_wait_timeout(limit_ns: int):
    """(status, nanoseconds waited) of a wait on a barrier nothing arrives on; status is ERR_TIMEOUT by design."""
    st, ns = ctypes.c_int(), ctypes.c_int()
    _check(_lib.libra_selftest_wait_timeout(ctypes.c_uint32(limit_ns), ctypes.byref(st), ctypes.byref(ns)),
           "libra_selftest_wait_timeout")
    return st.value, ns.value


def launch_count() -> int:
    return int(_lib.libra_launch_count())


class Plan:
    """Owner of a libra_plan_t."""

    def __init__(self, handle, cu_seqlens):
        self._h = handle
        self.cu_seqlens = cu_seqlens  # kept alive for the attention calls

    def info(self, direction=LIBRA_DIR_Q):
        nt, nb = ctypes.c_int64(), ctypes.c_int64()
        w, tile, h = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
        _check(_lib.libra_plan_info(self._h, direction, ctypes.byref(nt), ctypes.byref(w), ctypes.byref(nb),
                                    ctypes.byref(tile), ctypes.byref(h)), "libra_plan_info")
        return dict(n_tiles=nt.value, n_workers=w.value, n_blocks=nb.value, tile=tile.value, n_heads=h.value)

    def status(self) -> int:
        return int(_lib.libra_plan_status(self._h))

    def export(self, direction=LIBRA_DIR_Q):
        i = self.info(direction)
        nt, w = i["n_tiles"], i["n_workers"]
        res = dict(weight=np.empty(nt, np.int64), order=np.empty(nt, np.int32), cta_of_tile=np.empty(nt, np.int32),
                   cta_offsets=np.empty(w + 1, np.int32), cta_tiles=np.empty(nt, np.int32),
                   loads=np.empty(w, np.int64))
        _check(_lib.libra_plan_export(self._h, direction, _np(res["weight"]), _np(res["order"]),
                                      _np(res["cta_of_tile"]), _np(res["cta_offsets"]), _np(res["cta_tiles"]),
                                      _np(res["loads"])), "libra_plan_export")
        res["n_blocks"] = i["n_blocks"]
        return res

    def export_pairs(self):
        """(key_block, query_chunk) of every pair-block and the chunk size in tokens (LIBRA_DIR_PAIR plans)."""
        nb = self.info(LIBRA_DIR_PAIR)["n_blocks"]
        kb, qc, chunk = np.empty(nb, np.int32), np.empty(nb, np.int32), ctypes.c_int()
        _check(_lib.libra_plan_export_pairs(self._h, _np(kb), _np(qc), ctypes.byref(chunk)), "libra_plan_export_pairs")
        return kb, qc, chunk.value

    def fused_ctas(self) -> int:
        """CTAs that take a pair tile together in the fused backward: 1, or 2 where it runs on pairs of CTAs; 0: a windowed
        plan whose backward takes the two-kernel form."""
        n = int(_lib.libra_plan_fused_ctas(self._h))
        _check(min(n, 0), "libra_plan_fused_ctas")
        return n

    def busy_times(self, which=KERNEL_FWD):
        direction = LIBRA_DIR_PAIR if which == KERNEL_BWD_FUSED else (LIBRA_DIR_KV if which == KERNEL_BWD_DKDV else LIBRA_DIR_Q)
        try:
            w = self.info(direction)["n_workers"]
        except LibraError:
            if which != KERNEL_BWD_DKDV:
                raise
            w = self.info(LIBRA_DIR_Q)["n_workers"]   # key-major lists may be the library's own; all directions have as many
        out = np.zeros(w, np.uint64)
        _check(_lib.libra_busy_times(self._h, which, _np(out)), "libra_busy_times")
        return out

    def set_wait_limit_ns(self, ns: int):
        _check(_lib.libra_plan_set_wait_limit_ns(self._h, ctypes.c_uint64(ns)), "libra_plan_set_wait_limit_ns")

    def inject_stall(self, enabled=True):
        _check(_lib.libra_plan_inject_stall(self._h, 1 if enabled else 0), "libra_plan_inject_stall")

    def set_timing(self, enabled=True):
        _check(_lib.libra_plan_set_timing(self._h, 1 if enabled else 0), "libra_plan_set_timing")

    def kernel_time_ms(self, which=KERNEL_FWD) -> float:
        ms = ctypes.c_float()
        _check(_lib.libra_kernel_time_ms(self._h, which, ctypes.byref(ms)), "libra_kernel_time_ms")
        return float(ms.value)

    def tile_times(self, which=KERNEL_FWD):
        """Nanoseconds each tile took in the last launch of the forward (query-major tiles) or the fused backward
        (pair tiles), indexed by tile id (uint32 numpy array)."""
        nt = self.info(LIBRA_DIR_PAIR if which == KERNEL_BWD_FUSED else LIBRA_DIR_Q)["n_tiles"]
        out = np.zeros(nt, dtype=np.uint32)
        _check(_lib.libra_tile_times(self._h, which, _np(out)), "libra_tile_times")
        return out

    def kernel_times_ms(self, which=KERNEL_FWD, capacity=64):
        """Durations (ms) of the most recent recorded launches of kernel `which`, oldest first."""
        buf = (ctypes.c_float * capacity)()
        n = ctypes.c_int()
        _check(_lib.libra_kernel_times_ms(self._h, which, buf, ctypes.c_int(capacity), ctypes.byref(n)),
               "libra_kernel_times_ms")
        return [float(buf[i]) for i in range(n.value)]

    def destroy(self):
        if self._h:
            _lib.libra_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def libra_plan_tiles(cu_seqlens: torch.Tensor, n_heads: int, tile_q: int, n_workers: int = 0,
                     directions: int = 0, tile_kv: int = 0, n_heads_kv: int = 0, total_tokens: int = 0,
                     stream=None, weight_model: int = 0, cost_block: int = 0, unit_cost_q: int = 0,
                     unit_cost_kv: int = 0, pair_chunk: int = 0, window: int = 0, sinks: int = 0) -> Plan:
    """window > 0: a query sees the last `window` positions of its sample, its own among them, and the sample's first
    `sinks` (libra_plan_tiles_window); 0: all of its sample's past."""
    assert cu_seqlens.is_cuda and cu_seqlens.dtype == torch.int32 and cu_seqlens.is_contiguous()
    opts = PlanOpts(n_workers, directions, tile_kv, n_heads_kv, total_tokens, weight_model, cost_block,
                    unit_cost_q, unit_cost_kv, pair_chunk)
    h = _vp()
    if window != 0 or sinks != 0:
        window, sinks = (max(-1, min(x, 2 ** 31 - 1)) for x in (window, sinks))   # (no sample is longer)
        _check(_lib.libra_plan_tiles_window(_ptr(cu_seqlens), ctypes.c_int(cu_seqlens.numel() - 1), ctypes.c_int(n_heads),
                                            ctypes.c_int(tile_q), ctypes.byref(opts), ctypes.c_int(window),
                                            ctypes.c_int(sinks), _stream(stream), ctypes.byref(h)),
               "libra_plan_tiles_window")
        return Plan(h, cu_seqlens)
    _check(_lib.libra_plan_tiles(_ptr(cu_seqlens), ctypes.c_int(cu_seqlens.numel() - 1), ctypes.c_int(n_heads),
                                 ctypes.c_int(tile_q), ctypes.byref(opts), _stream(stream), ctypes.byref(h)),
           "libra_plan_tiles")
    return Plan(h, cu_seqlens)


def _dims(q, k, plan, scale):
    T, hq, d = q.shape
    return Dims(T, plan.cu_seqlens.numel() - 1, hq, k.shape[1], d, 0.0 if scale is None else float(scale))


def _chk(*ts):
    for t in ts:
        assert t.is_cuda and t.is_contiguous(), "expected contiguous CUDA tensors"


def _chk_qkv(q, k, v):
    _chk(q, k, v)
    assert q.dtype == k.dtype == v.dtype == torch.bfloat16
    T, hq, d = q.shape
    assert k.shape == v.shape and k.shape[0] == T and k.shape[2] == d, "shapes of q, k and v do not match"
    assert k.get_device() == v.get_device() == q.get_device(), "tensors on different devices"
    return T, hq, d


def _given(what, t, n, dtype, like):
    """A tensor of n values that the kernels read or write as a whole."""
    assert (t.dtype is dtype and t.numel() == n and t.is_cuda and t.is_contiguous() and t.get_device() == like.get_device()), \
        f"{what}: expected {n} contiguous values of {dtype} on {like.device}"


def _workspace(workspace, need, like):
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=like.device)
    assert workspace.is_cuda and workspace.is_contiguous() and workspace.get_device() == like.get_device()
    size = workspace.numel() * workspace.element_size()
    assert size >= need, f"workspace of {size} bytes, the call needs {need}"
    return workspace


def _chk_bwd(q, k, v, out, lse, dout, dq, dk, dv):
    T, hq, _ = _chk_qkv(q, k, v)
    n, n_kv = q.numel(), k.numel()
    _given("lse", lse, hq * T, torch.float32, q)
    for what, t, size in (("out", out, n), ("dout", dout, n), ("dq", dq, n), ("dk", dk, n_kv), ("dv", dv, n_kv)):
        _given(what, t, size, torch.bfloat16, q)


@_on_its_stream
def libra_attn_pool_fwd(q, k, v, plan: Plan, out=None, lse=None, scale=None, stream=None):
    """out [T,Hq,d] bf16, lse [Hq,T] fp32 (allocated with torch when not given)."""
    T, hq, _ = _chk_qkv(q, k, v)
    out = torch.empty_like(q) if out is None else out
    lse = torch.empty((hq, T), dtype=torch.float32, device=q.device) if lse is None else lse
    _given("out", out, q.numel(), torch.bfloat16, q)
    _given("lse", lse, hq * T, torch.float32, q)
    dims = _dims(q, k, plan, scale)
    _check(_lib.libra_attn_pool_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(plan.cu_seqlens), plan._h, _ptr(out), _ptr(lse),
                                    ctypes.byref(dims), _stream(stream)), "libra_attn_pool_fwd")
    return out, lse


def libra_attn_pool_bwd_workspace_bytes(plan: Plan, q, k) -> int:
    dims = _dims(q, k, plan, None)
    return int(_lib.libra_attn_pool_bwd_workspace_bytes(plan._h, ctypes.byref(dims)))


@_on_its_stream
def libra_attn_pool_bwd(q, k, v, out, lse, dout, plan: Plan, dq=None, dk=None, dv=None, workspace=None,
                        scale=None, stream=None):
    """dq, dk, dv bf16 and `workspace` (libra_attn_pool_bwd_workspace_bytes of this plan: plans of the same size may differ) are
    allocated with torch when not given."""
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    _chk_bwd(q, k, v, out, lse, dout, dq, dk, dv)
    dims = _dims(q, k, plan, scale)
    workspace = _workspace(workspace, int(_lib.libra_attn_pool_bwd_workspace_bytes(plan._h, ctypes.byref(dims))), q)
    _check(_lib.libra_attn_pool_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _ptr(dout),
                                    _ptr(plan.cu_seqlens), plan._h, _ptr(dq), _ptr(dk), _ptr(dv), _ptr(workspace),
                                    ctypes.byref(dims), _stream(stream)), "libra_attn_pool_bwd")
    return dq, dk, dv


def libra_attn_pool_bwd_noalloc_max_bytes() -> int:
    return int(_lib.libra_attn_pool_bwd_noalloc_max_bytes())


def libra_attn_pool_bwd_noalloc(q, k, v, out, lse, dout, plan: Plan, dq, dk, dv, scale=None, stream=None):
    """Backward that takes no workspace and allocates nothing: dq, dk, dv must be passed in.
    Raises LibraError(ERR_SCRATCH_TOO_SMALL) when the pool exceeds the library's built-in scratch."""
    _chk_bwd(q, k, v, out, lse, dout, dq, dk, dv)
    dims = _dims(q, k, plan, scale)
    _check(_lib.libra_attn_pool_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _ptr(dout),
                                            _ptr(plan.cu_seqlens), plan._h, _ptr(dq), _ptr(dk), _ptr(dv),
                                            ctypes.byref(dims), _stream(stream)), "libra_attn_pool_bwd_noalloc")
    return dq, dk, dv


def _ckpt8_dims_of(tensors):
    """dims of (q, k, v, out), each [T, H, *] or None; heads of 1 where there is no tensor with them."""
    T = d = hq = hkv = None
    here = torch.cuda.current_device()
    for i, t in enumerate(tensors):
        if t is None:
            continue
        assert t.is_cuda and t.is_contiguous() and t.dim() == 3, "expected contiguous 3-D CUDA tensors"
        assert t.device.index == here, "tensor on another device than the current one"
        n, h, w = t.shape
        heads = hkv if i in (1, 2) else hq
        assert (T is None or (n, w) == (T, d)) and (heads is None or heads == h), "shapes do not match"
        T, d = n, w
        if i in (1, 2):
            hkv = h
        else:
            hq = h
    assert T is not None, "no tensor"
    return Dims(T, 0, hq or 1, hkv or 1, d, 0.0)


def _ckpt8_args(ckpt):
    """Checks a checkpoint's tensors -> pointers, dims."""
    dims = _ckpt8_dims_of(ckpt[:4])
    T, w = dims.total_tokens, dims.head_dim // 32
    for i in range(4):
        val, exp = ckpt[i], ckpt[4 + i]
        if val is None:
            assert exp is None, "exponents without values"
            continue
        assert val.dtype is torch.int8 and exp is not None and exp.dtype is torch.uint8
        assert exp.is_contiguous() and exp.device == val.device
        assert exp.shape == (T, dims.hkv if i in (1, 2) else dims.hq, w), "exponents of another shape"
    return _Ckpt8Pointers(*[None if t is None else t.data_ptr() for t in ckpt]), dims


def _packed(shapes, dtype, device):
    """Contiguous tensors of these shapes (None: none) in one allocation; every size is a multiple of 16 bytes but the last ones'.
    (An allocation each costs more than the kernels of a small layer.)"""
    sizes = [0 if x is None else x[0] * x[1] * x[2] for x in shapes]
    room = torch.empty(sum(sizes), dtype=dtype, device=device)
    at, out = 0, []
    for x, n in zip(shapes, sizes):
        out.append(None if x is None else room.as_strided(x, (x[1] * x[2], x[2], 1), at))
        at += n
    return out


@_on_its_stream
def libra_ckpt8_pack(q=None, k=None, v=None, out=None, ckpt: Ckpt8 = None, stream=None) -> Ckpt8:
    """8-bit checkpoint of the bf16 tensors given (q, out [T, Hq, d], k, v [T, Hkv, d]); into `ckpt` when that is given, else
    into memory of its own, all of it one allocation: any of the tensors keeps all of it alive."""
    xs = (q, k, v, out)
    assert all(x is None or x.dtype is torch.bfloat16 for x in xs)
    dims = _ckpt8_dims_of(xs)
    if ckpt is None:
        d, device = dims.head_dim, next(x for x in xs if x is not None).device
        shapes = [None if x is None else tuple(x.shape) for x in xs]
        both = _packed(shapes + [x and (x[0], x[1], d // 32) for x in shapes], torch.int8, device)
        ckpt = Ckpt8(*both[:4], *[x if x is None else x.view(torch.uint8) for x in both[4:]])
        c = _Ckpt8Pointers(*[None if t is None else t.data_ptr() for t in ckpt])
    else:
        c, _ = _ckpt8_args(ckpt)
        for x, val in zip(xs, ckpt):
            assert x is None or (val is not None and val.shape == x.shape), "the checkpoint has another shape"
    _check(_lib.libra_ckpt8_pack(*[_ptr(x) for x in xs], ctypes.byref(c), ctypes.byref(dims), _stream(stream)),
           "libra_ckpt8_pack")
    return ckpt


@_on_its_stream
def libra_ckpt8_unpack(ckpt: Ckpt8, q=None, k=None, v=None, out=None, stream=None):
    """(q, k, v, out) as bf16, into the tensors given, None for those that the checkpoint does not hold.  Those not given are views of
    one allocation: any of them keeps all alive, and they share a version counter, so that for autograd a change of one in place is
    a change of all."""
    c, dims = _ckpt8_args(ckpt)
    xs = [q, k, v, out]
    for x, val in zip(xs, ckpt):
        assert x is None or (val is not None and x.dtype is torch.bfloat16 and x.is_contiguous() and x.shape == val.shape
                             and x.device == val.device)
    shapes = [tuple(val.shape) if x is None and val is not None else None for x, val in zip(xs, ckpt)]
    if any(shapes):
        new = _packed(shapes, torch.bfloat16, next(val for val in ckpt if val is not None).device)
        xs = [y if x is None else x for x, y in zip(xs, new)]
    _check(_lib.libra_ckpt8_unpack(ctypes.byref(c), *[_ptr(x) for x in xs], ctypes.byref(dims), _stream(stream)),
           "libra_ckpt8_unpack")
    return tuple(xs)


def _ckpt8_dims(ckpt, plan, scale):
    c, dims = _ckpt8_args(ckpt)
    assert all(t is not None for t in ckpt), "the backward pass needs q, k, v and out"
    dims.n_samples = plan.cu_seqlens.numel() - 1
    dims.softmax_scale = 0.0 if scale is None else float(scale)
    return c, dims


def libra_attn_pool_bwd_ckpt8_workspace_bytes(plan: Plan, ckpt: Ckpt8) -> int:
    return int(_lib.libra_attn_pool_bwd_ckpt8_workspace_bytes(plan._h, ctypes.byref(_ckpt8_dims(ckpt, plan, None)[1])))


@_on_its_stream
def libra_attn_pool_bwd_ckpt8(ckpt: Ckpt8, lse, dout, plan: Plan, dq=None, dk=None, dv=None, workspace=None, scale=None,
                              stream=None):
    """Backward of the tensors that `ckpt` stands for -> dq, dk, dv.  `workspace`: libra_attn_pool_bwd_ckpt8_workspace_bytes of this
    plan, which is more than libra_attn_pool_bwd takes (the restored q, k and v)."""
    c, dims = _ckpt8_dims(ckpt, plan, scale)
    assert dout.shape == ckpt.q.shape and lse.shape == (dims.hq, dims.total_tokens)
    new = lambda like: torch.empty(like.shape, dtype=torch.bfloat16, device=like.device)  # noqa: E731
    dq, dk, dv = new(ckpt.q) if dq is None else dq, new(ckpt.k) if dk is None else dk, new(ckpt.v) if dv is None else dv
    _given("lse", lse, lse.numel(), torch.float32, ckpt.q)
    for what, t, like in (("dout", dout, ckpt.q), ("dq", dq, ckpt.q), ("dk", dk, ckpt.k), ("dv", dv, ckpt.v)):
        _given(what, t, like.numel(), torch.bfloat16, ckpt.q)
    workspace = _workspace(workspace, int(_lib.libra_attn_pool_bwd_ckpt8_workspace_bytes(plan._h, ctypes.byref(dims))), dout)
    _check(_lib.libra_attn_pool_bwd_ckpt8(ctypes.byref(c), _ptr(lse), _ptr(dout), _ptr(plan.cu_seqlens), plan._h, _ptr(dq),
                                          _ptr(dk), _ptr(dv), _ptr(workspace), ctypes.byref(dims), _stream(stream)),
           "libra_attn_pool_bwd_ckpt8")
    return dq, dk, dv


@_on_its_stream
def libra_vrsp_work(sample_offsets: torch.Tensor, seq_first_sample: torch.Tensor, stream=None) -> torch.Tensor:
    """F_i = sum of squared raw-sample lengths of packed sequence i (int64, on the device)."""
    for t in (sample_offsets, seq_first_sample):
        assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()
    D = seq_first_sample.numel() - 1
    work = torch.empty(D, dtype=torch.int64, device=sample_offsets.device)
    _check(_lib.libra_vrsp_work(_ptr(sample_offsets), _ptr(seq_first_sample), ctypes.c_int(D), _ptr(work),
                                _stream(stream)), "libra_vrsp_work")
    return work


@_on_its_stream
def libra_vrsp_place(work: torch.Tensor, pool_size: int, stream=None):
    """Algorithm 1 on the device -> dict(order, pool_of_seq, pool_load) of device tensors."""
    assert work.is_cuda and work.dtype == torch.int64 and work.is_contiguous()
    D = work.numel()
    dev = work.device
    order = torch.empty(D, dtype=torch.int32, device=dev)
    pool_of_seq = torch.empty(D, dtype=torch.int32, device=dev)
    pool_load = torch.empty(max(D // max(pool_size, 1), 1), dtype=torch.int64, device=dev)
    scratch = torch.empty(D, dtype=torch.int32, device=dev)
    _check(_lib.libra_vrsp_place(_ptr(work), ctypes.c_int(D), ctypes.c_int(pool_size), _ptr(order), _ptr(pool_of_seq),
                                 _ptr(pool_load), _ptr(scratch), _stream(stream)), "libra_vrsp_place")
    return dict(order=order, pool_of_seq=pool_of_seq, pool_load=pool_load)


class TapOpts(ctypes.Structure):
    _fields_ = [("cp", ctypes.c_int), ("block", ctypes.c_int), ("n_shards", ctypes.c_int), ("hq", ctypes.c_int),
                ("hkv", ctypes.c_int), ("head_dim", ctypes.c_int), ("tau_num", ctypes.c_int), ("tau_den", ctypes.c_int)]


_lib.libra_tap_num_tiles.restype = ctypes.c_int64


@_on_its_stream
def libra_tap_plan(cu_seqlens: torch.Tensor, seq_offsets, cp: int, block: int, n_shards: int, hq: int, hkv: int,
                   head_dim: int, tau_num: int = 3, tau_den: int = 100, stream=None):
    """Tiles, Algorithm 2 and the exchange volumes of one pool -> dict of device tensors
    (sigma, loads, fwd_bytes [W, W], bwd_bytes [W, W], comm_total, status)."""
    assert cu_seqlens.is_cuda and cu_seqlens.dtype == torch.int32 and cu_seqlens.is_contiguous()
    so = (ctypes.c_int32 * len(seq_offsets))(*[int(x) for x in seq_offsets])
    P = len(seq_offsets) - 1
    W = P * cp
    NT = int(_lib.libra_tap_num_tiles(so, ctypes.c_int(P), ctypes.c_int(block), ctypes.c_int(n_shards)))
    if NT <= 0:
        raise RuntimeError("libra_tap_num_tiles: bad arguments")
    dev = cu_seqlens.device
    out = dict(sigma=torch.empty(NT, dtype=torch.int32, device=dev), loads=torch.empty(W, dtype=torch.int64, device=dev),
               fwd_bytes=torch.empty((W, W), dtype=torch.int64, device=dev),
               bwd_bytes=torch.empty((W, W), dtype=torch.int64, device=dev),
               comm_total=torch.empty(1, dtype=torch.int64, device=dev), status=torch.empty(1, dtype=torch.int32, device=dev))
    opts = TapOpts(cp, block, n_shards, hq, hkv, head_dim, tau_num, tau_den)
    _check(_lib.libra_tap_plan(_ptr(cu_seqlens), ctypes.c_int(cu_seqlens.numel() - 1), so, ctypes.c_int(P),
                               ctypes.byref(opts), _ptr(out["sigma"]), _ptr(out["loads"]), _ptr(out["fwd_bytes"]),
                               _ptr(out["bwd_bytes"]), _ptr(out["comm_total"]), _ptr(out["status"]), _stream(stream)),
           "libra_tap_plan")
    return out


@_on_its_stream
def libra_tap_schedule(cu_seqlens: torch.Tensor, seq_offsets, sigma: torch.Tensor, cp: int, block: int, n_shards: int,
                       hq: int, hkv: int, head_dim: int, capacity: int = 0, stream=None) -> torch.Tensor:
    """Transfer records [n, 6] (kind, src, dst, tok0, ntok, shard) implied by assignment `sigma` (device int32).
    When `capacity` is 0 the records are taken in one call with room for as many as most assignments imply, and in a
    second one when that was not enough."""
    assert cu_seqlens.is_cuda and cu_seqlens.dtype == torch.int32 and sigma.is_cuda and sigma.dtype == torch.int32
    so = (ctypes.c_int32 * len(seq_offsets))(*[int(x) for x in seq_offsets])
    P = len(seq_offsets) - 1
    opts = TapOpts(cp, block, n_shards, hq, hkv, head_dim, 3, 100)
    dev = cu_seqlens.device
    n = torch.zeros(1, dtype=torch.int64, device=dev)

    def call(cap):
        rec = torch.empty((max(cap, 1), 6), dtype=torch.int32, device=dev)
        _check(_lib.libra_tap_schedule(_ptr(cu_seqlens), ctypes.c_int(cu_seqlens.numel() - 1), so, ctypes.c_int(P),
                                       ctypes.byref(opts), _ptr(sigma), _ptr(rec), ctypes.c_int64(cap), _ptr(n),
                                       _stream(stream)), "libra_tap_schedule")
        return rec

    if capacity > 0:
        rec = call(capacity)
        return rec[:min(capacity, int(n.item()))]
    room = sigma.numel() + 65536
    rec = call(room)
    count = int(n.item())
    if count > room:
        rec = call(count)
    return rec[:count]
