"""8-bit checkpoints: the format's pins, and refusals that need no device."""
import ctypes

import numpy as np
import torch

import ckpt_reference as ref


def _bf16(*xs):
    return torch.tensor([*xs] + [0.0] * (32 - len(xs)), dtype=torch.bfloat16)


def test_format_by_hand():
    q, e = ref.held(_bf16(1.0, -1.9921875, 0.0078125, 0.0234375, 0.5))     # 2^0 <= largest < 2^1: steps of 2^-6
    assert e.tolist() == [127] and q[:5].tolist() == [64, -127, 0, 2, 32]   # -127.5 clamps, 0.5 and 1.5 go to even
    assert ref.value(q, e)[:3].tolist() == [1.0, -1.984375, 0.0]
    q, e = ref.held(_bf16(0.0))
    assert e.tolist() == [7] and not q.any()
    q, e = ref.held(_bf16(2.0 ** -130, 2.0 ** -126))                           # below the least step: zero
    assert e.tolist() == [7] and q[:2].tolist() == [0, 1]
    q, e = ref.held(_bf16(float("inf"), 1.0))
    assert e.tolist() == [255] and np.isnan(ref.value(q, e)).all()
    q, e = ref.held(_bf16(3.3895313892515355e38))                              # the largest bf16
    assert e.tolist() == [254] and q[0] == 127 and np.isfinite(ref.value(q, e)).all()


def test_half_a_step():
    g = torch.Generator().manual_seed(3)
    x = torch.randn((50, 3, 64), generator=g) * torch.exp(4 * torch.randn((50, 3, 64), generator=g))
    x = x.to(torch.bfloat16)
    q, e = ref.held(x)
    off = np.abs(ref.value(q, e) - x.double().numpy()).reshape(*e.shape, 32)
    assert (off <= np.ldexp(0.5, e.astype(int) - 133)[..., None]).all()
    back = torch.from_numpy(ref.value(q, e))
    assert torch.equal(back.to(torch.bfloat16).double(), back)                 # exact in bf16
    q2, e2 = ref.held(back.to(torch.bfloat16))                                 # and held without a further loss
    assert np.array_equal(ref.value(q2, e2), ref.value(q, e))


def test_gradients_of_the_layer_on_the_values_read_back():
    """With lse and out of the values read back, dv is the gradient of that forward pass, and dq and dk are as far from it as
    the rounding of out moves the row sums <dout, out>: half a step of each value.  With lse of the values before, rows of P do not
    add up to 1."""
    import window_reference as wref
    T, h, d, window, sinks = 300, 2, 64, 120, 4
    g = torch.Generator().manual_seed(5)
    q, k, v, dout = (torch.randn((T, h, d), generator=g).to(torch.bfloat16) for _ in range(4))
    see = wref.visible([0, T], window, sinks)
    def held(x):
        return torch.from_numpy(ref.value(*ref.held(x)))
    Q, K, V = held(6 * q), held(k), held(v)
    out, lse, *_ = wref.forward(Q, K, V, see)
    given = out.to(torch.bfloat16)
    exact, _ = wref.backward(Q, K, V, out, lse, dout, see)
    got, _ = wref.backward(Q, K, V, held(given), lse, dout, see)
    e = ref.held(given)[1].astype(int)
    step = torch.from_numpy(np.ldexp(0.5, e - 133)).repeat_interleave(32, -1) + out.abs() * 2.0 ** -8     # and out's to bf16
    off = (step * dout.abs().double()).sum(-1).t().unsqueeze(-1)                                          # of <dout, out> [h, T, 1]
    p = torch.exp((Q.transpose(0, 1) @ K.transpose(0, 1).transpose(1, 2)) * d ** -0.5 - lse.unsqueeze(-1)).masked_fill(~see, 0)
    assert torch.allclose(p.sum(-1), torch.ones(h, T, dtype=torch.float64), rtol=0, atol=1e-12)
    bound_q = ((p * off) @ K.abs().transpose(0, 1)).transpose(0, 1) * d ** -0.5
    bound_k = ((p * off).transpose(1, 2) @ Q.abs().transpose(0, 1)).transpose(0, 1) * d ** -0.5
    assert torch.equal(got[2], exact[2])
    assert bool(((got[0] - exact[0]).abs() <= bound_q + 1e-12).all()) and bool(((got[1] - exact[1]).abs() <= bound_k + 1e-12).all())
    _, lse_before, *_ = wref.forward((6 * q), k, v, see)
    assert float((torch.exp(lse - lse_before) - 1).abs().max()) > 0.05


class Dims(ctypes.Structure):
    _fields_ = [("total_tokens", ctypes.c_int64), ("n_samples", ctypes.c_int), ("hq", ctypes.c_int), ("hkv", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("softmax_scale", ctypes.c_float)]


def test_bad_arguments_are_refused_before_any_cuda_call():
    from paper_2607_23250_b200 import build
    lib = ctypes.CDLL(build.build())
    lib.libra_attn_pool_bwd_ckpt8_workspace_bytes.restype = ctypes.c_size_t
    some = ctypes.c_void_p(256)                                                # never dereferenced
    Held = ctypes.c_void_p * 8
    full, dims = Held(*[256] * 8), Dims(10, 1, 2, 1, 64, 0.0)
    args = (None, None, None, None)
    for call in (lambda c, d, x: lib.libra_ckpt8_pack(*x, c, d, None), lambda c, d, x: lib.libra_ckpt8_unpack(c, *x, d, None)):
        x = (some, some, some, some)
        assert call(None, ctypes.byref(dims), x) == -1 and call(full, None, x) == -1
        for bad in (Dims(0, 1, 2, 1, 64, 0), Dims(-4, 1, 2, 1, 64, 0), Dims(10, 1, 0, 1, 64, 0), Dims(10, 1, 2, -1, 64, 0)):
            assert call(full, ctypes.byref(bad), x) == -1
        for d in (0, 32, 96, 192, 512):
            assert call(full, ctypes.byref(Dims(10, 1, 2, 1, d, 0)), x) == -2
        assert call(full, ctypes.byref(Dims(1 << 30, 1, 1 << 10, 1, 64, 0)), x) == -5
        assert call(full, ctypes.byref(dims), args) == 0                       # nothing asked for
        for k in range(8):                                                     # a tensor without its values or exponents
            part = Held(*[0 if i == k else 256 for i in range(8)])
            assert call(part, ctypes.byref(dims), x) == -1
        assert call(Held(264, *[256] * 7), ctypes.byref(dims), x) == -1        # misaligned values, misaligned tensor
        assert call(full, ctypes.byref(dims), (some, ctypes.c_void_p(264), some, some)) == -1
    assert lib.libra_attn_pool_bwd_ckpt8_workspace_bytes(None, ctypes.byref(dims)) == 0
    assert lib.libra_attn_pool_bwd_ckpt8(None, *[some] * 9, None) == -1
    assert lib.libra_attn_pool_bwd_ckpt8(Held(*[256] * 7, 0), *[some] * 8, ctypes.byref(dims), None) == -1


def test_new_entry_points_are_declared_exported_and_bound():
    import os
    import re
    from paper_2607_23250_b200 import build
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "libra.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(libra_[a-z_0-9]+)\s*\(", header))
    lib = ctypes.CDLL(build.build())
    binding = open(os.path.join(root, "paper_2607_23250_b200", "binding.py")).read()
    for name in ("libra_plan_tiles_window", "libra_ckpt8_pack", "libra_ckpt8_unpack", "libra_attn_pool_bwd_ckpt8",
                 "libra_attn_pool_bwd_ckpt8_workspace_bytes"):
        assert name in names and hasattr(lib, name) and f'"{name}"' in binding
