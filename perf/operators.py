"""Windowed pool attention and attention's 8-bit activation checkpoints, as cases that can be timed and checked.

A case is a dict of plain values.  `prepare(case, seed)` makes what a training program holds before the call, `run(state)` is
one pass, `work(case)` the bytes and operations of that pass, `exact(case, seed)` the same results in 64 bits.  With `own`
false a pass is made of elementary torch operations in 32 bits, with `own` true of calls of the public binding.

Kinds of pass:
  fwd    attention forward: a query sees the last `window` positions of its sample, itself among them, and the sample's
         first `sinks` positions
  step   forward and backward of that
  ckpt   q, k, v and out of a layer into an 8-bit checkpoint and back (one layer of the forward pass, and its reading)
  bwd8   backward whose q, k, v and out are in a checkpoint

A checkpoint holds runs of 32 values along the head dimension as eight-bit integers and a power of two: with 2^e the largest
power of two that is not above the largest magnitude of the run (at least 2^-120), x is held as round(x / 2^(e - 6)), ties to
even and at most 127 in magnitude, and stands for that integer times 2^(e - 6), a bf16 number.  The exponent byte is e + 127.
"""
import math

import numpy as np
import torch

own = False

QUERY_BLOCK = 512      # rows that the plain form takes together
DIR_Q, DIR_PAIR = 1, 4


def attention(name, kind, tokens, hq, hkv, d, window, sinks, form="fused", layout="lognormal", param=0.0, draw=0):
    """layout: lognormal (lengths of median 644), short (uniform lengths up to param), frac (one sample of param * tokens
    among lognormal ones).  form: the backward that the plan selects, fused or two-kernel."""
    case = dict(kind=kind, tokens=tokens, hq=hq, hkv=hkv, d=d, window=window, sinks=sinks, form=form, layout=layout,
                param=param, draw=draw)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # a small model's evaluation call on one 4096-token sequence: all latency
        attention("fwd_4k_d64", "fwd", 4096, 4, 4, 64, 512, 4, "two-kernel"),
        # evaluation of the 8B-shaped layer on four packed 32768-token sequences with a 4096-token window
        attention("fwd_131k", "fwd", 131072, 32, 8, 128, 4096, 4),
        # training on a ragged pool of short samples (chat turns), odd token count, a window below most of their lengths
        attention("step_short_10k", "step", 10007, 8, 2, 128, 128, 1, "fused", "short", 400.0),
        # a small model in training on one long document, bit-reproducible backward, an odd window
        attention("step_16k_d64", "step", 16000, 8, 2, 64, 1001, 7, "two-kernel", "frac", 1.0),
        # one training layer of the 8B-shaped pool with a 1024-token window
        attention("step_131k", "step", 131072, 32, 8, 128, 1024, 4),
        # long context: one 65536-token sample, eight query heads per kv head, wide window (largest)
        attention("step_65k_long", "step", 65536, 32, 4, 128, 8192, 64, "fused", "frac", 1.0),
        # wide heads, 32 of them to a kv head
        attention("step_8k_d256", "step", 8192, 32, 1, 256, 777, 5, "fused", "frac", 0.5),
        # checkpoint of a small layer, written and read back
        attention("ckpt_4k_d64", "ckpt", 4096, 4, 4, 64, 0, 0),
        # checkpoint of the 8B-shaped layer
        attention("ckpt_131k", "ckpt", 131072, 32, 8, 128, 0, 0),
        # backward out of the checkpoint, short samples
        attention("bwd8_10k", "bwd8", 10007, 8, 2, 128, 128, 1, "fused", "short", 400.0),
        # backward out of the checkpoint, 8B-shaped layer on an odd number of tokens
        attention("bwd8_33k", "bwd8", 33001, 32, 8, 128, 2048, 4),
        # one rank's slice of the 8B-shaped pool split over 8 GPUs by heads, bit-reproducible backward, no sinks
        attention("bwd8_slice_131k", "bwd8", 131072, 4, 1, 128, 1024, 0, "two-kernel"),
    ]


HEADS = {64: [(4, 4), (8, 2), (16, 4)], 128: [(32, 8), (32, 4), (8, 2), (8, 1), (4, 1)], 256: [(32, 1), (128, 4)]}
MOST_PLAIN_FLOPS = 3.3e13      # the plain form's own operations in step_65k_long
MOST_VALUES = 131072 * 32 * 128


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "step", "step", "step", "ckpt", "bwd8", "bwd8"])
    d = rng.choice([64, 128, 128, 128, 256])
    hq, hkv = rng.choice(HEADS[d])
    layout = rng.choice(["lognormal", "lognormal", "short", "frac"])
    param = {"short": float(_log_int(rng, 2, 2000)), "frac": rng.choice([0.3, 0.5, 1.0])}.get(layout, 0.0)
    form = "two-kernel" if d == 64 else rng.choice(["fused", "fused", "two-kernel"])
    window = 0 if kind == "ckpt" else _log_int(rng, 8, 8192)
    sinks = 0 if kind == "ckpt" else rng.choice([0, 1, 4, _log_int(rng, 1, 300)])
    case = attention(None, kind, _log_int(rng, 300, 131072), hq, hkv, d, window, sinks, form, layout, param,
                     rng.randint(1, 1 << 20))

    def too_much():
        band = _band(case) + QUERY_BLOCK + case["sinks"]
        flops = 0 if kind == "ckpt" else (4 if kind == "fwd" else 14) * d * hq * case["tokens"] * band
        return (flops > MOST_PLAIN_FLOPS or case["tokens"] * hq * d > MOST_VALUES
                or (kind != "ckpt" and case["tokens"] * band * (hq // hkv) > 5.0e9))

    while too_much():
        case["tokens"] = int(case["tokens"] * 0.7)
    return case


# ---- layouts and inputs ---------------------------------------------------------------------------------

def lengths_of(case):
    """Sample lengths; they add up to case["tokens"]."""
    rng = np.random.default_rng([case["draw"], 5])
    total = case["tokens"]
    whole = int(round(case["param"] * total)) if case["layout"] == "frac" else 0
    lengths, left = [], total - whole
    while left > 0:
        if case["layout"] == "short":
            x = int(rng.integers(1, int(case["param"]) + 1))
        else:
            x = int(np.clip(np.rint(np.exp(rng.normal(math.log(644.0), 1.6))), 1, 32768))
        lengths.append(min(x, left))
        left -= lengths[-1]
    if whole:
        lengths.insert(int(rng.integers(0, len(lengths) + 1)), whole)
    return lengths


def _band(case):
    """Positions behind a row that the band of a query block has to reach."""
    return min(case["window"], max(lengths_of(case))) - 1 if case["window"] else 0


def _inputs(case, seed):
    T, hq, hkv, d = case["tokens"], case["hq"], case["hkv"], case["d"]
    lengths = lengths_of(case)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    s = {"case": case, "lengths": lengths, "cu": torch.from_numpy(cu).cuda()}
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1) + case["draw"])
    for name, heads in (("q", hq), ("k", hkv), ("v", hkv), ("dout", hq)):
        if name != "dout" or case["kind"] in ("step", "bwd8"):
            s[name] = torch.randn((T, heads, d), generator=g, device="cuda", dtype=torch.bfloat16)
    if case["kind"] == "ckpt":
        s["out"] = torch.randn((T, hq, d), generator=g, device="cuda", dtype=torch.bfloat16)
    if case["kind"] == "bwd8":                             # what the forward pass has left of the layer
        out, s["lse"] = _plain_fwd(s["q"], s["k"], s["v"], _view(case, s["cu"]))
        s["ckpt"] = {n: _quantise(s.pop(n)) for n in ("q", "k", "v")}
        s["ckpt"]["out"] = _quantise(out.to(torch.bfloat16))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_23250_b200 import binding as lb
        T, hq, hkv, d = case["tokens"], case["hq"], case["hkv"], case["d"]
        if case["kind"] == "bwd8":
            c = s["ckpt"]
            s["ckpt"] = lb.Ckpt8(*(c[n][0] for n in ("q", "k", "v", "out")), *(c[n][1] for n in ("q", "k", "v", "out")))
        if case["kind"] != "ckpt":
            s["plan"] = lb.libra_plan_tiles(s["cu"], hq, 256, directions=DIR_Q | DIR_PAIR if case["form"] == "fused" else 0,
                                            tile_kv=128, n_heads_kv=hkv, total_tokens=T, window=case["window"],
                                            sinks=case["sinks"])
        if case["kind"] in ("fwd", "step"):
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty((hq, T), dtype=torch.float32, device="cuda")
        if case["kind"] in ("step", "bwd8"):
            s["dq"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
            s["dk"], s["dv"] = (torch.empty((T, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            size = (lb.libra_attn_pool_bwd_workspace_bytes(s["plan"], s["q"], s["k"]) if case["kind"] == "step"
                    else lb.libra_attn_pool_bwd_ckpt8_workspace_bytes(s["plan"], s["ckpt"]))
            s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ---- the plain form ---------------------------------------------------------------------------------------

def _view(case, cu):
    """Which keys each block of query rows multiplies with (idx [blocks, keys]) and which of them each row sees."""
    T, B, W, S, back = case["tokens"], QUERY_BLOCK, case["window"], case["sinks"], _band(case)
    nb = -(-T // B)
    tok = torch.arange(nb * B, device="cuda")
    first = cu.long()[torch.searchsorted(cu.long(), tok.clamp(max=T - 1), right=True) - 1]   # start of the row's sample
    b0 = tok[::B].view(nb, 1)
    band = b0 - back + torch.arange(back + B, device="cuda")
    early = first[::B].view(nb, 1) + torch.arange(S, device="cuda")
    idx = torch.cat([torch.where(early < b0 - back, early, -1), band], 1)
    valid = ((idx >= 0) & (idx < T)).view(nb, 1, -1)
    idx = idx.clamp(0, T - 1)
    row, key, start = tok.view(nb, B, 1), idx.view(nb, 1, -1), first.view(nb, B, 1)
    seen = valid & (key >= start) & (key <= row) & ((row - key < W) | (key - start < S)) & (row < T)
    return dict(T=T, idx=idx, unseen=~seen)


def _blocks(x, nb):
    """[T, G, d] of any type -> fp32 [G, blocks, rows, d], the last block filled up with zeros."""
    T, G, d = x.shape
    y = torch.zeros((nb * QUERY_BLOCK, G, d), dtype=torch.float32, device=x.device)
    y[:T] = x
    return y.view(nb, QUERY_BLOCK, G, d).permute(2, 0, 1, 3).contiguous()


def _rows(y, T):
    """[G, blocks, rows, d] -> [T, G, d]."""
    G, nb, B, d = y.shape
    return y.permute(1, 2, 0, 3).reshape(nb * B, G, d)[:T]


def _plain_fwd(q, k, v, view):
    T, hq, d = q.shape
    hkv, (nb, _) = k.shape[1], view["idx"].shape
    G = hq // hkv
    out = torch.empty((T, hq, d), dtype=torch.float32, device=q.device)
    lse = torch.empty((hq, T), dtype=torch.float32, device=q.device)
    for j in range(hkv):                                                   # (one kv head's scores at a time)
        heads = slice(j * G, (j + 1) * G)
        kj, vj = k[:, j].float()[view["idx"]], v[:, j].float()[view["idx"]]
        s = _blocks(q[:, heads], nb) @ kj.transpose(1, 2)
        s.mul_(1.0 / math.sqrt(d)).masked_fill_(view["unseen"], -math.inf)
        m = s.amax(-1, keepdim=True).clamp_(min=-1e30)
        s.sub_(m).exp_()
        l = s.sum(-1, keepdim=True)
        out[:, heads] = _rows((s @ vj) / l, T)
        lse[heads] = (m + l.log()).reshape(G, -1)[:, :T]
    return out, lse


def _plain_bwd(q, k, v, out, lse, dout, view):
    T, hq, d = q.shape
    hkv, (nb, n) = k.shape[1], view["idx"].shape
    G, scale = hq // hkv, 1.0 / math.sqrt(d)
    dq = torch.empty((T, hq, d), dtype=torch.float32, device=q.device)
    dk = torch.zeros((hkv, T, d), dtype=torch.float32, device=q.device)
    dv = torch.zeros_like(dk)
    for j in range(hkv):
        heads = slice(j * G, (j + 1) * G)
        kj, vj = k[:, j].float()[view["idx"]], v[:, j].float()[view["idx"]]
        qj, gj = _blocks(q[:, heads], nb), _blocks(dout[:, heads], nb)
        delta = (_blocks(out[:, heads], nb) * gj).sum(-1, keepdim=True)
        p = qj @ kj.transpose(1, 2)
        p.mul_(scale).sub_(_blocks(lse[heads].t().unsqueeze(-1), nb)).exp_().masked_fill_(view["unseen"], 0.0)
        dv[j].index_add_(0, view["idx"].reshape(-1), (p.transpose(2, 3) @ gj).sum(0).view(nb * n, d))
        p.mul_((gj @ vj.transpose(1, 2)).sub_(delta)).mul_(scale)
        dq[:, heads] = _rows(p @ kj, T)
        dk[j].index_add_(0, view["idx"].reshape(-1), (p.transpose(2, 3) @ qj).sum(0).view(nb * n, d))
    return dq, dk.transpose(0, 1), dv.transpose(0, 1)


def _quantise(x):
    """bf16 [..., d] -> (int8 [..., d], exponent bytes [..., d / 32])."""
    y = x.float().unflatten(-1, (-1, 32))
    e = torch.frexp(y.abs().amax(-1)).exponent.sub(1).clamp(min=-120)
    q = torch.ldexp(y, (6 - e).unsqueeze(-1)).round().clamp(-127, 127)
    return q.flatten(-2).to(torch.int8), (e + 127).to(torch.uint8)


def _restore(held):
    q, e = held
    y = torch.ldexp(q.float().unflatten(-1, (-1, 32)), (e.int() - 133).unsqueeze(-1))
    return y.flatten(-2).to(torch.bfloat16)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2607_23250_b200 import binding as lb
        if kind == "ckpt":
            return tuple(lb.libra_ckpt8_unpack(lb.libra_ckpt8_pack(s["q"], s["k"], s["v"], s["out"])))
        res = {}
        if kind in ("fwd", "step"):
            res["out"], res["lse"] = lb.libra_attn_pool_fwd(s["q"], s["k"], s["v"], s["plan"], out=s["out"], lse=s["lse"])
        grads = dict(dq=s.get("dq"), dk=s.get("dk"), dv=s.get("dv"), workspace=s.get("ws"))
        if kind == "step":
            res["dq"], res["dk"], res["dv"] = lb.libra_attn_pool_bwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"],
                                                                     s["plan"], **grads)
        if kind == "bwd8":
            res["dq"], res["dk"], res["dv"] = lb.libra_attn_pool_bwd_ckpt8(s["ckpt"], s["lse"], s["dout"], s["plan"], **grads)
        return res
    if kind == "ckpt":
        return tuple(_restore(_quantise(s[n])) for n in ("q", "k", "v", "out"))
    view, res, half = _view(case, s["cu"]), {}, torch.bfloat16
    if kind == "bwd8":
        q, k, v, out = (_restore(s["ckpt"][n]) for n in ("q", "k", "v", "out"))
        lse = s["lse"]
    else:
        q, k, v = s["q"], s["k"], s["v"]
        out, lse = _plain_fwd(q, k, v, view)
        res.update(out=out.to(half), lse=lse)
    if kind != "fwd":
        dq, dk, dv = _plain_bwd(q, k, v, out, lse, s["dout"], view)
        res.update(dq=dq.to(half), dk=dk.to(half).contiguous(), dv=dv.to(half).contiguous())
    return res


# ---- the definition in 64 bits, sample by sample ------------------------------------------------------------

def _exact_held(x):
    """The values that a checkpoint of x stands for."""
    y = x.double().reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -120)
    step = torch.exp2(torch.floor(torch.log2(top)) - 6)
    return ((y / step).round().clamp(-127, 127) * step).reshape(x.shape)


def exact(case, seed):
    kind, W, S = case["kind"], case["window"], case["sinks"]
    if kind != "ckpt" and len(lengths_of(case)) > 20000:
        return None                                        # (sample by sample this would take too long)
    s = _inputs(case, seed)
    if kind == "ckpt":
        return tuple(_exact_held(s[n]) for n in ("q", "k", "v", "out"))
    if kind == "bwd8":
        c = {n: s["ckpt"][n][0].double() * torch.exp2(s["ckpt"][n][1].double() - 133).repeat_interleave(32, -1)
             for n in ("q", "k", "v", "out")}
        q, k, v, o_in, lse_in = c["q"], c["k"], c["v"], c["out"], s["lse"].double()
    else:
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    T, hq, d = q.shape
    hkv = k.shape[1]
    G, scale = hq // hkv, d ** -0.5
    dout = s["dout"].double() if kind != "fwd" else None
    out, lse = torch.zeros_like(q), torch.zeros((hq, T), dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    a = 0
    for n in s["lengths"]:
        z = a + n
        step = max(64, min(n, int(1.5e8 // (hq * min(n, W + S + 512)))))
        for r0 in range(a, z, step):
            r1 = min(z, r0 + step)
            lo = max(a, r0 - W + 1)
            keys = torch.cat([torch.arange(a, min(a + S, lo), device="cuda"), torch.arange(lo, r1, device="cuda")])
            rows = torch.arange(r0, r1, device="cuda").unsqueeze(1)
            see = (keys <= rows) & ((rows - keys < W) | (keys < a + S))
            kk, vv = k[keys].transpose(0, 1).unsqueeze(1), v[keys].transpose(0, 1).unsqueeze(1)      # [hkv, 1, keys, d]
            qq = q[r0:r1].transpose(0, 1).reshape(hkv, G, r1 - r0, d)
            x = (qq @ kk.transpose(2, 3)) * scale
            x = x.masked_fill(~see, -math.inf)
            if kind == "bwd8":
                ll = lse_in[:, r0:r1].reshape(hkv, G, r1 - r0, 1)
                oo = o_in[r0:r1].transpose(0, 1).reshape(hkv, G, r1 - r0, d)
                p = torch.exp(x - ll)
            else:
                ll = torch.logsumexp(x, -1, keepdim=True)
                p = torch.exp(x - ll)
                oo = p @ vv
                out[r0:r1] = oo.reshape(hq, r1 - r0, d).transpose(0, 1)
                lse[:, r0:r1] = ll.reshape(hq, r1 - r0)
            if kind == "fwd":
                continue
            gg = dout[r0:r1].transpose(0, 1).reshape(hkv, G, r1 - r0, d)
            ds = p * (gg @ vv.transpose(2, 3) - (oo * gg).sum(-1, keepdim=True)) * scale
            dq[r0:r1] = (ds @ kk).reshape(hq, r1 - r0, d).transpose(0, 1)
            dk[keys] += (ds.transpose(2, 3) @ qq).sum(1).transpose(0, 1)
            dv[keys] += (p.transpose(2, 3) @ gg).sum(1).transpose(0, 1)
        a = z
    if kind == "fwd":
        return dict(out=out, lse=lse)
    grads = dict(dq=dq, dk=dk, dv=dv)
    return grads if kind == "bwd8" else dict(out=out, lse=lse, **grads)


# ---- what a pass cannot do without ----------------------------------------------------------------------------

def work(case):
    T, hq, hkv, d, W, S = case["tokens"], case["hq"], case["hkv"], case["d"], case["window"], case["sinks"]
    held = 33.0 / 32.0                                     # bytes a value in a checkpoint
    q, kv, rows = 2.0 * T * hq * d, 2.0 * T * hkv * d, 4.0 * T * hq
    if case["kind"] == "ckpt":                             # bf16 in and out, the checkpoint out and in
        values = 2.0 * T * (hq + hkv) * d
        return dict(bytes=values * (4 + 2 * held), flops=2 * values)
    pairs = 0.0
    for n in lengths_of(case):
        w = min(W, n)
        pairs += w * (w + 1) / 2 + (n - w) * w
        more = n - w                                       # rows with positions behind the window: 1 .. more of them
        s = min(S, more)
        pairs += s * (s + 1) / 2 + (more - s) * s
    fwd = dict(bytes=2 * q + 2 * kv + rows, flops=4 * d * hq * pairs)                  # q k v in, out lse out
    bwd = dict(bytes=4 * q + 4 * kv + rows, flops=10 * d * hq * pairs)                 # q k v out dout lse in, dq dk dv out
    bwd8 = dict(bytes=held * (q + kv) + 2 * q + 2 * kv + rows, flops=10 * d * hq * pairs)
    parts = {"fwd": [fwd], "step": [fwd, bwd], "bwd8": [bwd8]}[case["kind"]]
    return {key: float(sum(p[key] for p in parts)) for key in ("bytes", "flops")}
