"""Attention with a window and sinks from its definition, in 64 bits and on the whole score matrix, with bounds of how far
bf16 kernels may be from it; tile weights and placement by brute force."""
import heapq

import numpy as np
import torch

U = 2.0 ** -8          # half a step of bf16, relative


def visible(cu, window, sinks, device="cpu"):
    """[T, T] truth values: row i sees key k.  window 0: no window."""
    cu = torch.as_tensor(np.asarray(cu), device=device).long()
    t = torch.arange(int(cu[-1]), device=device)
    first = cu[torch.searchsorted(cu, t, right=True) - 1]
    i, k, a = t.unsqueeze(1), t.unsqueeze(0), first.unsqueeze(1)
    see = (k >= a) & (k <= i)
    if window:
        see &= (i - k < window) | (k - a < sinks)
    return see


def _heads(x, hq):
    """[T, h, d] -> fp64 [hq, T, d], kv heads repeated for their query heads."""
    return x.double().transpose(0, 1).repeat_interleave(hq // x.shape[1], 0)


def forward(q, k, v, see, scale=None):
    """-> out, lse, and the bounds of |out - out'| and |lse - lse'|.

    The kernel rounds every P_ik and the result to bf16; its scores and sums are in fp32, a score's sum of d products off by
    at most d 2^-23 of the sum of their magnitudes (tensor cores may truncate), which moves P by that factor and lse by as
    much; the exponential and the logarithm add a few units of 2^-22."""
    T, hq, d = q.shape
    scale = scale or d ** -0.5
    Q, K, V = (_heads(x, hq) for x in (q, k, v))
    s = (Q @ K.transpose(1, 2)) * scale
    off = (d * 2.0 ** -23 * scale) * (Q.abs() @ K.abs().transpose(1, 2)).masked_fill(~see, 0).amax(-1)      # [hq, T]
    s = s.masked_fill(~see, -np.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.unsqueeze(-1))
    out, mass = p @ V, p @ V.abs()
    b_out = mass * (1.02 * U + 2 * off.unsqueeze(-1) + 2.0 ** -18) + out.abs() * U + 1e-30   # (a value of 0: no 0 / 0)
    b_lse = off + 2.0 ** -20 * (lse.abs() + s.masked_fill(~see, 0).abs().amax(-1) + 1)
    return out.transpose(0, 1), lse, b_out.transpose(0, 1), b_lse


def backward(q, k, v, out, lse, dout, see, scale=None):
    """Gradients given out and lse -> (dq, dk, dv), (their bounds).

    P, dP - D and their product are rounded to bf16 by some of the kernels (one rounding by others), the result once more.
    Scores and dP carry the fp32 sums' error as in forward()."""
    T, hq, d = q.shape
    hkv = k.shape[1]
    scale = scale or d ** -0.5
    Q, K, V = (_heads(x, hq) for x in (q, k, v))
    O, G = _heads(out, hq), _heads(dout, hq)
    s = (Q @ K.transpose(1, 2)) * scale
    off = (d * 2.0 ** -23 * scale) * (Q.abs() @ K.abs().transpose(1, 2)) + 2.0 ** -18
    off = off + 2.0 ** -21 * (lse.double().abs().unsqueeze(-1) + s.abs())
    p = torch.exp(s - lse.double().unsqueeze(-1)).masked_fill(~see, 0)
    x = G @ V.transpose(1, 2) - (O * G).sum(-1, keepdim=True)
    x_off = d * 2.0 ** -23 * (G.abs() @ V.abs().transpose(1, 2) + (O.abs() * G.abs()).sum(-1, keepdim=True))
    ds = p * x
    ds_off = ds.abs() * (3.05 * U + off) + 1.02 * p * x_off
    p_off = p * (1.01 * U + off)
    fold = lambda y: y.reshape(hkv, hq // hkv, T, d).sum(1).transpose(0, 1)  # noqa: E731
    dq, dk, dv = (ds @ K).transpose(0, 1) * scale, fold(ds.transpose(1, 2) @ Q) * scale, fold(p.transpose(1, 2) @ G)
    b_dq = (ds_off @ K.abs()).transpose(0, 1) * scale
    b_dk, b_dv = fold(ds_off.transpose(1, 2) @ Q.abs()) * scale, fold(p_off.transpose(1, 2) @ G.abs())
    # fp32 sums of up to T G terms, then the last rounding
    tail = lambda r, b: 1.01 * (b + T * (hq // hkv) * 2.0 ** -24 * b / U) + r.abs() * U * 1.02 + 1e-30  # noqa: E731
    return (dq, dk, dv), (tail(dq, b_dq), tail(dk, b_dk), tail(dv, b_dv))


def worst(got, want, bound):
    """Largest error as a share of its bound; infinite where a value is not finite."""
    r = (got.double() - want).abs() / bound
    return float("inf") if not bool(torch.isfinite(got).all()) else float(r.max()) if r.numel() else 0.0


# ---- planning ---------------------------------------------------------------------------------------------

def tile_weights(see, tile, key_major, cost_block, unit_cost=0):
    """Block-count weights of the blocks of `tile` tokens of one head shard, by counting on the mask."""
    m = see.numpy().T if key_major else see.numpy()
    T = m.shape[0]
    out = []
    for t0 in range(0, T, tile):
        t1 = min(T, t0 + tile)
        w = 0
        for c in range(t0 // cost_block, (t1 - 1) // cost_block + 1):
            rows = m[max(t0, c * cost_block):min(t1, (c + 1) * cost_block)].any(0)
            w += 8 * sum(bool(rows[x:x + cost_block].any()) for x in range(0, T, cost_block)) + unit_cost
        out.append(w)
    return out


def place(weights, n_heads, n_workers):
    """Heaviest first, least-loaded worker, lowest index on ties -> worker of every tile, loads."""
    tiles = sorted(range(len(weights) * n_heads), key=lambda t: (-weights[t // n_heads], t))
    heap = [(0, r) for r in range(n_workers)]
    cta = np.empty(len(tiles), np.int32)
    loads = np.zeros(n_workers, np.int64)
    for t in tiles:
        load, r = heapq.heappop(heap)
        cta[t] = r
        loads[r] = load + weights[t // n_heads]
        heapq.heappush(heap, (int(loads[r]), r))
    return cta, loads


def live_pairs(see, tile, chunk):
    """(chunk, key block, live cells) of every pair-block, chunk by chunk, key blocks ascending."""
    m = see.numpy()
    T = m.shape[0]
    nb = -(-T // tile)
    pad = np.zeros((nb * tile, nb * tile), bool)
    pad[:T, :T] = m
    cells = pad.reshape(nb, tile, nb, tile).any((1, 3))
    R = chunk // tile
    out = []
    for c in range(-(-nb // R)):
        n = cells[c * R:(c + 1) * R].sum(0)
        out += [(c, int(j), int(n[j])) for j in np.flatnonzero(n)]
    return out
