"""8-bit activation checkpoints on the GPU: the format bit for bit, and the backward pass out of them."""
import numpy as np
import pytest
import torch

import ckpt_reference as ref
import window_reference as wref
from paper_2607_23250_b200 import pools

pytestmark = pytest.mark.gpu

# infinities, NaN, zeros, subnormals, ties, runs of one large value, the largest and smallest numbers
def _values(shape, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-20, 20, (*shape[:2], 1), generator=g).float())
    x = x.to(torch.bfloat16)
    flat = x.view(-1, 32)
    odd = [float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 2.0 ** -133, -2.0 ** -127, 3.3895313892515355e38, 127.5, -127.5, 0.5, 1.5, 2.5]
    for i in range(min(len(flat), 4 * len(odd))):
        if i % 4 == 1:
            flat[i, (7 * i) % 32] = odd[i // 4]
        if i % 4 == 2:
            flat[i] = odd[i // 4]
        if i % 4 == 3:                                     # steps of one: ties at .5
            flat[i] = torch.arange(32) * 0.5 + 48
            flat[i, 0] = odd[8 + (i // 4) % 5]
    return x


def _bits(x):
    return x.contiguous().view(torch.int16).cpu()


@pytest.mark.parametrize("T,hq,hkv,d", [(1, 1, 1, 64), (1, 3, 1, 128), (5, 3, 1, 64), (7, 2, 2, 256), (33, 1, 1, 64), (129, 5, 1, 128), (1000, 8, 2, 128)])
def test_pack_and_unpack_match_the_definition(T, hq, hkv, d):
    from paper_2607_23250_b200 import binding as lb
    xs = [_values((T, h, d), 10 * T + i) for i, h in enumerate((hq, hkv, hkv, hq))]
    ckpt = lb.libra_ckpt8_pack(*(x.cuda() for x in xs))
    back = lb.libra_ckpt8_unpack(ckpt)
    for x, q, e, y in zip(xs, ckpt[:4], ckpt[4:], back):
        want_q, want_e = ref.held(x)
        assert np.array_equal(e.cpu().numpy(), want_e)
        fine = np.repeat(want_e != 255, 32, -1)
        assert np.array_equal(q.cpu().numpy()[fine], want_q[fine])
        want = ref.value(want_q, want_e)
        got = y.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[fine], want[fine])


def test_parts_of_a_layer_and_tensors_given():
    from paper_2607_23250_b200 import binding as lb
    k = torch.randn((70, 2, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.randn((70, 6, 64), dtype=torch.bfloat16, device="cuda")
    ckpt = lb.libra_ckpt8_pack(k=k, out=out)
    assert ckpt.q is None and ckpt.v is None and ckpt.k.shape == k.shape and ckpt.out_exp.shape == (70, 6, 2)
    q, k2, v, out2 = lb.libra_ckpt8_unpack(ckpt)
    assert q is None and v is None
    # into memory at hand, whose neighbours stay as they are
    room = torch.full((80, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    held = torch.full((80, 2, 64), 5, dtype=torch.int8, device="cuda")
    exps = torch.full((80, 2, 2), 9, dtype=torch.uint8, device="cuda")
    lb.libra_ckpt8_pack(k=k, ckpt=lb.Ckpt8(k=held[5:75], k_exp=exps[5:75]))
    lb.libra_ckpt8_unpack(lb.Ckpt8(k=held[5:75], k_exp=exps[5:75]), k=room[5:75])
    assert torch.equal(room[5:75], k2) and torch.equal(held[5:75], ckpt.k) and torch.equal(exps[5:75], ckpt.k_exp)
    for x, fill in ((room, 7.0), (held, 5), (exps, 9)):
        assert bool((x[:5] == fill).all()) and bool((x[75:] == fill).all())
    with pytest.raises(AssertionError):
        lb.libra_ckpt8_pack(k=k.transpose(0, 1))
    with pytest.raises(AssertionError):
        lb.libra_ckpt8_pack(k=k.float())
    with pytest.raises(AssertionError):
        lb.libra_ckpt8_pack(k=k, out=out[:60])
    with pytest.raises(lb.LibraError) as err:
        lb.libra_ckpt8_pack(k=torch.zeros((4, 1, 96), dtype=torch.bfloat16, device="cuda"))
    assert err.value.code == lb.ERR_UNSUPPORTED


def test_host_memory_is_refused():
    from paper_2607_23250_b200 import binding as lb
    import ctypes
    x = torch.zeros((8, 1, 64), dtype=torch.bfloat16)
    held, exps = torch.zeros((8, 1, 64), dtype=torch.int8, device="cuda"), torch.zeros((8, 1, 2), dtype=torch.uint8, device="cuda")
    c = lb._Ckpt8Pointers(held.data_ptr(), None, None, None, exps.data_ptr(), None, None, None)
    dims = lb.Dims(8, 0, 1, 1, 64, 0.0)
    null = ctypes.c_void_p(0)
    for call in (lambda p: lb._lib.libra_ckpt8_pack(p, null, null, null, ctypes.byref(c), ctypes.byref(dims), None),
                 lambda p: lb._lib.libra_ckpt8_unpack(ctypes.byref(c), p, null, null, null, ctypes.byref(dims), None)):
        for mem in (x, x.pin_memory()):
            assert call(ctypes.c_void_p(mem.data_ptr())) == lb.ERR_INVALID_ARG


LENGTHS = [150, 1, 700, 33, 260]


def _layer(d, fused, window, sinks, lengths=LENGTHS, hq=4, hkv=2, seed=0, **kw):
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens(lengths)
    t = pools.make_tensors(int(cu[-1]), hq, hkv, d, seed=seed)
    q, k, v, dout = (t[n].cuda() for n in ("q", "k", "v", "dout"))
    directions = lb.LIBRA_DIR_Q | (lb.LIBRA_DIR_PAIR if fused else lb.LIBRA_DIR_KV)
    plan = lb.libra_plan_tiles(torch.from_numpy(cu).cuda(), hq, 256, directions=directions, tile_kv=128, n_heads_kv=hkv,
                               window=window, sinks=sinks, **kw)
    out, lse = lb.libra_attn_pool_fwd(q, k, v, plan)
    return cu, plan, (q, k, v, out), lse, dout


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 0), (130, 5)])
@pytest.mark.parametrize("d,fused", [(64, False), (128, False), (128, True), (256, False), (256, True)])
def test_backward_out_of_a_checkpoint(d, fused, window, sinks):
    """Against the gradients of the tensors that the checkpoint stands for, in 64 bits; in the two-kernel form also the
    same bits as reading it back first."""
    from paper_2607_23250_b200 import binding as lb
    cu, plan, xs, lse, dout = _layer(d, fused, window, sinks, seed=d + window)
    ckpt = lb.libra_ckpt8_pack(*xs)
    grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan)
    torch.cuda.synchronize()
    plan.busy_times(lb.KERNEL_BWD_FUSED if fused and d == 128 else lb.KERNEL_BWD_DQ)
    vals = [torch.from_numpy(ref.value(q.cpu().numpy(), e.cpu().numpy())).cuda() for q, e in zip(ckpt[:4], ckpt[4:])]
    see = wref.visible(cu, window, sinks, "cuda")
    want, bounds = wref.backward(*vals, lse, dout, see)
    for name, g, w, b in zip(("dq", "dk", "dv"), grads, want, bounds):
        assert wref.worst(g, w, b) <= 1, name
    back = lb.libra_ckpt8_unpack(ckpt)
    again = lb.libra_attn_pool_bwd(*back, lse, dout, plan)
    if not fused:
        assert all(torch.equal(x, y) for x, y in zip(grads, again))
    plan.destroy()


@pytest.mark.parametrize("d,fused", [(64, False), (128, False), (128, True), (256, False), (256, True)])
def test_forward_on_the_values_read_back(d, fused):
    """q, k and v packed ahead of a forward pass on what is read back, with scores that are large: against 64 bits, and rows of P
    that add up to 1, so that dv of a sample adds up to its dout.  P and dv are rounded to bf16, half a step each, and lse
    and the scores are off by the bound of lse each."""
    from paper_2607_23250_b200 import binding as lb
    cu, plan, (q, k, v, _), _, dout = _layer(d, fused, 130, 5, seed=d)
    ckpt = lb.libra_ckpt8_pack(6 * q, k, v, torch.zeros_like(q))
    q2, k2, v2, _ = lb.libra_ckpt8_unpack(ckpt)
    out, lse = lb.libra_attn_pool_fwd(q2, k2, v2, plan)
    lb.libra_ckpt8_pack(out=out, ckpt=ckpt)
    grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan)
    vals = [torch.from_numpy(ref.value(x.cpu().numpy(), e.cpu().numpy())).cuda() for x, e in zip(ckpt[:4], ckpt[4:])]
    assert all(torch.equal(x.double(), y) for x, y in zip((q2, k2, v2), vals))
    see = wref.visible(cu, 130, 5, "cuda")
    want, bounds = wref.backward(*vals, lse, dout, see)
    for name, x, w, b in zip(("dq", "dk", "dv"), grads, want, bounds):
        assert wref.worst(x, w, b) <= 1, name
    *_, b_lse = wref.forward(*vals[:3], see)
    heads = q.shape[1] // k.shape[1]
    for a, z in zip(cu[:-1], cu[1:]):
        g = dout[a:z].double()
        total = g.sum(0).view(-1, heads, d).sum(1)
        rows = (g.abs() * (1.01 * wref.U + 2.0 ** -18 + 2 * b_lse[:, a:z].t().unsqueeze(-1))).sum(0).view(-1, heads, d).sum(1)
        room = 1.01 * rows + wref.U * 1.02 * grads[2][a:z].double().abs().sum(0) + 1e-30
        assert bool(((grads[2][a:z].double().sum(0) - total).abs() <= room).all())
    plan.destroy()


@pytest.mark.parametrize("d,fused", [(64, False), (128, False), (128, True), (256, False)])
def test_row_statistics_at_the_ends_of_the_range(d, fused):
    """Gradients near fp32's largest numbers against values of 2^-110, and the other way round: the products are ordinary
    numbers, 127 times such a gradient is not.  Powers of two change no rounding, so dq and dk only scale."""
    from paper_2607_23250_b200 import binding as lb
    cu, plan, (q, k, v, out), lse, dout = _layer(d, fused, 40, 3, seed=d)
    dout = dout.clamp(-3, 3)
    base = lb.libra_attn_pool_bwd_ckpt8(lb.libra_ckpt8_pack(q, k, v, out), lse, dout, plan)
    for down, up in ((110, 121), (-100, -100)):
        v2, out2, dout2 = v * 2.0 ** -down, out * 2.0 ** -down, dout * 2.0 ** up
        ckpt = lb.libra_ckpt8_pack(q, k, v2, out2)
        grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout2, plan)
        again = lb.libra_attn_pool_bwd(*lb.libra_ckpt8_unpack(ckpt), lse, dout2, plan)
        assert all(bool(torch.isfinite(x).all()) for x in grads)
        if not fused:
            assert all(torch.equal(x, y) for x, y in zip(grads, again))
            assert all(torch.equal(x, y * 2.0 ** (up - down)) for x, y in zip(grads[:2], base[:2]))
    plan.destroy()


@pytest.mark.parametrize("sinks", [0, 5, 200])
def test_backward_where_the_library_chose_the_two_kernel_form(sinks):
    """Pair tiles asked for, two kernels taken: statistics, partial sums of sinks' tails and the restored tensors share a workspace
    of exactly the size that is asked for."""
    from paper_2607_23250_b200 import binding as lb
    cu, plan, xs, lse, dout = _layer(128, True, 130, sinks, n_workers=12)
    assert plan.fused_ctas() == 0
    ckpt = lb.libra_ckpt8_pack(*xs)
    size = lb.libra_attn_pool_bwd_ckpt8_workspace_bytes(plan, ckpt)
    room = torch.full((size + 4096,), 171, dtype=torch.uint8, device="cuda")
    grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan, workspace=room[:size])
    again = lb.libra_attn_pool_bwd(*lb.libra_ckpt8_unpack(ckpt), lse, dout, plan)
    torch.cuda.synchronize()
    plan.busy_times(lb.KERNEL_BWD_DQ)
    assert all(torch.equal(x, y) for x, y in zip(grads, again))
    assert bool((room[size:] == 171).all())
    vals = [torch.from_numpy(ref.value(q.cpu().numpy(), e.cpu().numpy())).cuda() for q, e in zip(ckpt[:4], ckpt[4:])]
    want, bounds = wref.backward(*vals, lse, dout, wref.visible(cu, 130, sinks, "cuda"))
    for name, g, w, b in zip(("dq", "dk", "dv"), grads, want, bounds):
        assert wref.worst(g, w, b) <= 1, name
    with pytest.raises(AssertionError):
        lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan, workspace=room[:size - 1])
    plan.destroy()


def test_tensors_of_more_than_two_to_the_31_values():
    """Offsets beyond 32 bits: the far end of a large tensor has the bits that it has by itself, and so have the gradients."""
    from paper_2607_23250_b200 import binding as lb
    T, hq, hkv, d = 70000, 256, 16, 128
    cu = np.arange(0, T + 1, 1000, dtype=np.int32)
    t = pools.make_tensors(T, hq, hkv, d, seed=1, device="cuda")
    assert t["q"].numel() > 2 ** 31
    plan = lb.libra_plan_tiles(torch.from_numpy(cu).cuda(), hq, 256, tile_kv=128, n_heads_kv=hkv, window=60, sinks=2)
    out, lse = lb.libra_attn_pool_fwd(t["q"], t["k"], t["v"], plan)
    xs = (t["q"], t["k"], t["v"], out)
    ckpt = lb.libra_ckpt8_pack(*xs)
    back = lb.libra_ckpt8_unpack(ckpt)
    for part in (slice(0, 300), slice(T - 300, T)):
        mine = lb.libra_ckpt8_pack(*(x[part] for x in xs))
        assert all(torch.equal(a[part], b) for a, b in zip(ckpt, mine))
        assert all(torch.equal(a[part], b) for a, b in zip(back, lb.libra_ckpt8_unpack(mine)))
    grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, t["dout"], plan)
    torch.cuda.synchronize()
    plan.busy_times(lb.KERNEL_BWD_DQ)
    again = lb.libra_attn_pool_bwd(*back, lse, t["dout"], plan)
    assert all(torch.equal(x, y) for x, y in zip(grads, again))
    a = T - 1000                                                # the last sample by itself, against 64 bits
    see = wref.visible([0, 1000], 60, 2, "cuda")
    G = hq // hkv
    for h in (0, hkv - 1):
        heads = slice(h * G, (h + 1) * G)
        vals = [back[0][a:, heads].contiguous(), back[1][a:, h:h + 1].contiguous(), back[2][a:, h:h + 1].contiguous(), back[3][a:, heads].contiguous()]
        want, bounds = wref.backward(*vals, lse[heads, a:], t["dout"][a:, heads], see)
        got = grads[0][a:, heads], grads[1][a:, h:h + 1], grads[2][a:, h:h + 1]
        for name, x, w, b in zip(("dq", "dk", "dv"), got, want, bounds):
            assert wref.worst(x, w, b) <= 1, (name, h)
    plan.destroy()


def test_backward_on_pairs_of_ctas_and_over_dout():
    """The fused form on pairs of CTAs; dq written over dout."""
    from paper_2607_23250_b200 import binding as lb
    cu, plan, xs, lse, dout = _layer(128, True, 0, 0, lengths=[1100], pair_chunk=512)
    assert plan.fused_ctas() == 2
    ckpt = lb.libra_ckpt8_pack(*xs)
    vals = [torch.from_numpy(ref.value(q.cpu().numpy(), e.cpu().numpy())).cuda() for q, e in zip(ckpt[:4], ckpt[4:])]
    want, bounds = wref.backward(*vals, lse, dout, wref.visible(cu, 0, 0, "cuda"))
    for over in (False, True):
        g = dout.clone()
        grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, g, plan, dq=g if over else None)
        for x, w, b in zip(grads, want, bounds):
            assert wref.worst(x, w, b) <= 1
    plan.destroy()


@pytest.mark.parametrize("window,sinks", [(3000, 0), (3500, 4), (4000, 200)])
def test_windowed_backward_on_pairs_of_ctas(window, sinks):
    from paper_2607_23250_b200 import binding as lb
    cu, plan, xs, lse, dout = _layer(128, True, window, sinks, lengths=[100, 7400], hq=2, hkv=1, pair_chunk=512, n_workers=16)
    assert plan.fused_ctas() == 2
    ckpt = lb.libra_ckpt8_pack(*xs)
    grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan)
    torch.cuda.synchronize()
    plan.busy_times(lb.KERNEL_BWD_FUSED)
    vals = [torch.from_numpy(ref.value(q.cpu().numpy(), e.cpu().numpy())).cuda() for q, e in zip(ckpt[:4], ckpt[4:])]
    want, bounds = wref.backward(*vals, lse, dout, wref.visible(cu, window, sinks, "cuda"))
    for name, g, w, b in zip(("dq", "dk", "dv"), grads, want, bounds):
        assert wref.worst(g, w, b) <= 1, name
    plan.destroy()


def test_refusals_and_bad_plans_leave_the_outputs():
    from paper_2607_23250_b200 import binding as lb
    cu, plan, xs, lse, dout = _layer(128, False, 60, 2)
    ckpt = lb.libra_ckpt8_pack(*xs)
    size = lb.libra_attn_pool_bwd_ckpt8_workspace_bytes(plan, ckpt)
    T = int(cu[-1])
    assert size == lb.libra_attn_pool_bwd_workspace_bytes(plan, *xs[:2]) + 256 * (-(-T * 4 * 256 // 256) + 2 * -(-T * 2 * 256 // 256))
    with pytest.raises(AssertionError):
        lb.libra_attn_pool_bwd_ckpt8(ckpt._replace(out=None, out_exp=None), lse, dout, plan)
    with pytest.raises(AssertionError):
        lb.libra_attn_pool_bwd_ckpt8(ckpt, lse[:, :5].contiguous(), dout, plan)
    ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
    with pytest.raises(lb.LibraError) as err:
        lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan, workspace=ws[16:])
    assert err.value.code == lb.ERR_INVALID_ARG
    other = lb.libra_plan_tiles(torch.tensor([0, T - 1], dtype=torch.int32).cuda(), 4, 256, tile_kv=128, n_heads_kv=2)
    with pytest.raises(lb.LibraError) as err:
        lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, other, workspace=ws)
    assert err.value.code == lb.ERR_PLAN_MISMATCH
    bad = lb.libra_plan_tiles(torch.tensor([0, 50, 20, T], dtype=torch.int32).cuda(), 4, 256, tile_kv=128, n_heads_kv=2, total_tokens=T)
    grads = [torch.full(x.shape, 7.0, dtype=torch.bfloat16, device="cuda") for x in xs[:3]]
    lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, bad, *grads)
    assert all(bool((g == 7).all()) for g in grads)
    for p in (plan, other, bad):
        p.destroy()


def test_a_training_layer_captured_on_a_stream():
    """Forward, checkpoint and backward of a windowed layer as one graph, replayed on new inputs."""
    from paper_2607_23250_b200 import binding as lb
    cu, plan, (q, k, v, out), lse, dout = _layer(128, False, 90, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def layer(ws, ckpt, grads):
        lb.libra_attn_pool_fwd(q, k, v, plan, out=out, lse=lse)
        lb.libra_ckpt8_pack(q, k, v, out, ckpt=ckpt)
        lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan, *grads, workspace=ws)

    with torch.cuda.stream(side):
        ckpt = lb.libra_ckpt8_pack(q, k, v, out)
        ws = torch.empty(lb.libra_attn_pool_bwd_ckpt8_workspace_bytes(plan, ckpt), dtype=torch.uint8, device="cuda")
        grads = [torch.empty_like(x) for x in (q, k, v)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer(ws, ckpt, grads)
        for step in range(2):
            q.copy_(torch.roll(q, 1, 0))
            graph.replay()
            got = [x.clone() for x in (out, lse, *grads, *ckpt)]
            layer(ws, ckpt, grads)
            assert all(torch.equal(x, y) for x, y in zip(got, (out, lse, *grads, *ckpt)))
    torch.cuda.synchronize()
    del graph
    plan.destroy()


def test_calls_on_another_stream_keep_their_memory():
    """Checkpoint, its reading and the backward pass on a stream that is behind: what they allocated is not handed to tensors of the
    current stream when they return."""
    from paper_2607_23250_b200 import binding as lb
    cu, plan, xs, lse, dout = _layer(128, False, 130, 5)
    want_ckpt = lb.libra_ckpt8_pack(*xs)
    want_back = lb.libra_ckpt8_unpack(want_ckpt)
    want = lb.libra_attn_pool_bwd_ckpt8(want_ckpt, lse, dout, plan)
    size = lb.libra_attn_pool_bwd_ckpt8_workspace_bytes(plan, want_ckpt)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                          # some 10 ms
    ckpt = lb.libra_ckpt8_pack(*xs, stream=side)
    back = lb.libra_ckpt8_unpack(ckpt, stream=side)
    grads = lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan, stream=side)
    others = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (size, size // 2, 2 * size) for _ in range(2)]
    torch.cuda.synchronize()
    for got, exp in ((ckpt, want_ckpt), (back, want_back), (grads, want)):
        assert all(torch.equal(x, y) for x, y in zip(got, exp))
    assert all(bool((o == 255).all()) for o in others)
    plan.destroy()


def test_kernel_times_and_launch_counts():
    from paper_2607_23250_b200 import binding as lb
    cu, plan, xs, lse, dout = _layer(128, True, 60, 2)
    n0 = lb.launch_count()
    ckpt = lb.libra_ckpt8_pack(*xs)
    assert lb.launch_count() == n0 + 1
    lb.libra_ckpt8_unpack(ckpt)
    assert lb.launch_count() == n0 + 2
    plan.set_timing(True)
    lb.libra_attn_pool_bwd_ckpt8(ckpt, lse, dout, plan)
    assert lb.launch_count() == n0 + 5                     # row statistics and restoring, fused, conversion
    assert plan.kernel_time_ms(lb.KERNEL_BWD_PREP) > 0
    plan.destroy()
