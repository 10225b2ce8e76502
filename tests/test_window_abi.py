"""Windowed plans: refusals that need no device, and the reference's own pins."""
import ctypes

import numpy as np
import torch

import window_reference as ref
from paper_2607_23250_b200 import pools


def test_bad_windows_are_refused_before_any_cuda_call():
    from paper_2607_23250_b200 import build
    lib = ctypes.CDLL(build.build())
    some, h = ctypes.c_void_p(256), ctypes.c_void_p()       # never dereferenced
    for window, sinks in ((0, 0), (-5, 0), (3, -1), (-2 ** 31, 0)):
        assert lib.libra_plan_tiles_window(some, 1, 1, 256, None, window, sinks, None, ctypes.byref(h)) == -1
    assert lib.libra_plan_tiles_window(None, 1, 1, 256, None, 4, 0, None, ctypes.byref(h)) == -1
    assert lib.libra_plan_tiles_window(some, 1, 1, 256, None, 4, 0, None, None) == -1


def test_mask_by_hand():
    see = ref.visible(pools.cu_seqlens([1, 5]), 2, 1)
    assert see.int().tolist() == [[1, 0, 0, 0, 0, 0], [0, 1, 0, 0, 0, 0], [0, 1, 1, 0, 0, 0], [0, 1, 1, 1, 0, 0],
                                  [0, 1, 0, 1, 1, 0], [0, 1, 0, 0, 1, 1]]


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    cu = pools.cu_seqlens([3, 6])
    q, k, v, w = (torch.randn((9, h, 4), generator=g, dtype=torch.float64) for h in (2, 1, 1, 2))
    see = ref.visible(cu, 3, 1)
    out, lse, *_ = ref.forward(q, k, v, see)
    grads, _ = ref.backward(q, k, v, out, lse, w, see)
    for x, dx in zip((q, k, v), grads):
        for at in ((1, 0, 2), (4, 0, 0), (8, 0, 3)):
            eps, old = 1e-6, float(x[at])
            vals = []
            for e in (eps, -eps):
                x[at] = old + e
                vals.append(float((ref.forward(q, k, v, see)[0] * w).sum()))
            x[at] = old
            assert abs((vals[0] - vals[1]) / (2 * eps) - float(dx[at])) < 1e-7 * (1 + abs(float(dx[at])))


def test_weights_by_hand():
    see = ref.visible(pools.cu_seqlens([4, 1, 7]), 2, 1)     # chunks of 4: rows 8-11 see chunk 2, the last of chunk 1, the sink in 1
    assert ref.tile_weights(see, 8, False, 4, 1) == [(8 + 1) + (8 + 1), 8 * 2 + 1]
    assert ref.tile_weights(see, 4, True, 4, 0) == [8, 16, 8]
    assert np.array_equal(ref.visible([0, 12], 12, 0).numpy(), ref.visible([0, 12], 0, 0).numpy())
