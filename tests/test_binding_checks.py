"""What the binding refuses before the library is called: tensors that the kernels would read or write out of range.

No device: tensors of host memory say that they are on one, and the library's calls are recorded instead of made."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

lb = None      # the binding, once the library is built

NEED, NEED_CKPT = 1000, 5000       # workspace sizes that the library answers


@pytest.fixture(autouse=True, scope="module")
def binding():
    global lb
    from paper_2607_23250_b200 import build
    build.build()
    from paper_2607_23250_b200 import binding
    lb = binding


class Dev(torch.Tensor):
    """Host memory that says it is on a device."""
    is_cuda = property(lambda self: True)


class Calls:
    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append(name)
            return {"libra_attn_pool_bwd_workspace_bytes": NEED, "libra_attn_pool_bwd_ckpt8_workspace_bytes": NEED_CKPT}.get(name, 0)
        return call


@pytest.fixture
def calls(monkeypatch):
    made = Calls()
    monkeypatch.setattr(lb, "_lib", made)
    monkeypatch.setattr(lb, "_stream", lambda stream=None: ctypes.c_void_p(0))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    return made


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(Dev)


def _args(T=10, hq=4, hkv=2, d=64):
    q, kv = (T, hq, d), (T, hkv, d)
    ckpt = lb.Ckpt8(*(_t(*s, dtype=torch.int8) for s in (q, kv, kv, q)), *(_t(*s[:2], d // 32, dtype=torch.uint8) for s in (q, kv, kv, q)))
    return dict(q=_t(*q), k=_t(*kv), v=_t(*kv), out=_t(*q), lse=_t(hq, T, dtype=torch.float32), dout=_t(*q), dq=_t(*q), dk=_t(*kv),
                dv=_t(*kv), ckpt=ckpt)


PLAN = SimpleNamespace(_h=ctypes.c_void_p(0), cu_seqlens=torch.zeros(3, dtype=torch.int32))


def _call(name, a, **kw):
    if name == "ckpt8":
        return lb.libra_attn_pool_bwd_ckpt8(a["ckpt"], a["lse"], a["dout"], PLAN, a["dq"], a["dk"], a["dv"], **kw)
    if name == "fwd":
        return lb.libra_attn_pool_fwd(a["q"], a["k"], a["v"], PLAN, a["out"], a["lse"])
    f = lb.libra_attn_pool_bwd_noalloc if name == "noalloc" else lb.libra_attn_pool_bwd
    return f(a["q"], a["k"], a["v"], a["out"], a["lse"], a["dout"], PLAN, a["dq"], a["dk"], a["dv"], **kw)


ENTRY = {"fwd": "libra_attn_pool_fwd", "bwd": "libra_attn_pool_bwd", "noalloc": "libra_attn_pool_bwd_noalloc", "ckpt8": "libra_attn_pool_bwd_ckpt8"}


@pytest.mark.parametrize("name", ENTRY)
def test_right_arguments_reach_the_library(calls, name):
    _call(name, _args())
    assert calls.made[-1] == ENTRY[name]


@pytest.mark.parametrize("name,need", [("bwd", NEED), ("ckpt8", NEED_CKPT)])
def test_a_workspace_that_is_too_small(calls, name, need):
    a = _args()
    for ok in (_t(need, dtype=torch.uint8), _t(need // 4, dtype=torch.float32), _t(need + 7, dtype=torch.uint8)):
        _call(name, a, workspace=ok)
        assert calls.made[-1] == ENTRY[name]
    calls.made.clear()
    strided = _t(2 * need, dtype=torch.uint8)[::2]
    for bad in (_t(need - 1, dtype=torch.uint8), _t(need // 4 - 1, dtype=torch.float32), strided, torch.zeros(need, dtype=torch.uint8)):
        with pytest.raises(AssertionError):
            _call(name, a, workspace=bad)
    assert ENTRY[name] not in calls.made


def test_the_workspace_of_the_plain_backward_is_not_that_of_the_checkpoints(calls):
    with pytest.raises(AssertionError):
        _call("ckpt8", _args(), workspace=_t(NEED, dtype=torch.uint8))


@pytest.mark.parametrize("name,tensors", [
    ("fwd", ("k", "v", "out", "lse")), ("bwd", ("k", "v", "out", "lse", "dout", "dq", "dk", "dv")),
    ("noalloc", ("k", "v", "out", "lse", "dout", "dq", "dk", "dv")), ("ckpt8", ("lse", "dout", "dq", "dk", "dv"))])
def test_tensors_of_another_size_type_or_place(calls, name, tensors):
    for t in tensors:
        a = _args()
        x = a[t]
        other = torch.float32 if x.dtype is torch.bfloat16 else torch.bfloat16
        double = torch.cat([x, x], 1).as_subclass(Dev)[:, ::2]                  # the same shape, not contiguous
        for bad in (x[:-1], torch.zeros(x.shape, dtype=other).as_subclass(Dev), double, x.as_subclass(torch.Tensor)):
            with pytest.raises(AssertionError):
                _call(name, {**a, t: bad})
    assert not any(c in ENTRY.values() for c in calls.made)


@pytest.mark.parametrize("name", ["fwd", "bwd", "ckpt8", "pack", "unpack", "vrsp_work", "vrsp_place"])
def test_what_a_call_on_another_stream_allocates_belongs_to_it(calls, monkeypatch, name):
    """Memory of the current stream that is freed when the call returns would be another tensor's while the kernels still run."""
    now, allocated = [None], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            now.append(self.stream)

        def __exit__(self, *_):
            now.pop()

    def recorded(f):
        def call(*args, **kw):
            allocated.append(now[-1])
            return f(*args, **kw).as_subclass(Dev)
        return call

    a = _args()
    work, offsets = _t(4, dtype=torch.int64), _t(5, dtype=torch.int32)
    run = {"fwd": lambda **kw: lb.libra_attn_pool_fwd(a["q"], a["k"], a["v"], PLAN, **kw),
           "bwd": lambda **kw: lb.libra_attn_pool_bwd(a["q"], a["k"], a["v"], a["out"], a["lse"], a["dout"], PLAN, **kw),
           "ckpt8": lambda **kw: lb.libra_attn_pool_bwd_ckpt8(a["ckpt"], a["lse"], a["dout"], PLAN, **kw),
           "pack": lambda **kw: lb.libra_ckpt8_pack(a["q"], a["k"], a["v"], a["out"], **kw),
           "unpack": lambda **kw: lb.libra_ckpt8_unpack(a["ckpt"], **kw),
           "vrsp_work": lambda **kw: lb.libra_vrsp_work(offsets, offsets, **kw),
           "vrsp_place": lambda **kw: lb.libra_vrsp_place(work, 2, **kw)}[name]
    monkeypatch.setattr(torch, "empty", recorded(torch.empty))
    monkeypatch.setattr(torch, "empty_like", recorded(torch.empty_like))
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda p: ("stream", p))
    run(stream=SimpleNamespace(cuda_stream=77))
    assert allocated and all(s == ("stream", 77) for s in allocated)
    allocated.clear()
    run()
    assert allocated and all(s is None for s in allocated) and now == [None]


@pytest.mark.parametrize("given,passed", [((5, 2), (5, 2)), ((2 ** 40, 2 ** 33), (2 ** 31 - 1, 2 ** 31 - 1)), ((-2 ** 32 + 5, 0), (-1, 0)),
                                          ((7, -2 ** 32 + 3), (7, -1)), ((-2 ** 31 - 1, -2 ** 40), (-1, -1))])
def test_windows_beyond_32_bits_do_not_wrap(monkeypatch, calls, given, passed):
    """A window that is longer than any sample is none; one below zero stays what the library refuses."""
    seen = []
    monkeypatch.setattr(lb, "_lib", SimpleNamespace(libra_plan_tiles_window=lambda *a: seen.append((a[5].value, a[6].value)) or 0,
                                                    libra_plan_destroy=lambda h: 0))
    lb.libra_plan_tiles(_t(2, dtype=torch.int32), 1, 256, window=given[0], sinks=given[1])
    assert seen == [passed]
