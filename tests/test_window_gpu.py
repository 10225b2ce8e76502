"""Pool attention with a sliding window and sinks: planner, forward and both backward forms against the definition in 64 bits,
with the bounds of window_reference.py."""
import numpy as np
import pytest
import torch

import window_reference as ref
from paper_2607_23250_b200 import pools

pytestmark = pytest.mark.gpu

EDGES = [31, 32, 33, 32, 33, 64, 31, 96, 127, 33, 1, 32, 97, 126, 255, 2, 130]   # starts around words, blocks and tiles


def _tensors(cu, hq, hkv, d, seed):
    t = pools.make_tensors(int(cu[-1]), hq, hkv, d, seed=seed)
    return [t[n].cuda() for n in ("q", "k", "v", "dout")]


def _plan(cu, hq, hkv, fused, window, sinks, **kw):
    from paper_2607_23250_b200 import binding as lb
    directions = lb.LIBRA_DIR_Q | (lb.LIBRA_DIR_PAIR if fused else lb.LIBRA_DIR_KV)
    plan = lb.libra_plan_tiles(torch.from_numpy(cu).cuda(), hq, 256, directions=directions, tile_kv=128, n_heads_kv=hkv,
                               window=window, sinks=sinks, **kw)
    assert plan.status() == 0
    return plan


def _run(plan, q, k, v, dout, fused):
    from paper_2607_23250_b200 import binding as lb
    out, lse = lb.libra_attn_pool_fwd(q, k, v, plan)
    grads = lb.libra_attn_pool_bwd(q, k, v, out, lse, dout, plan)
    torch.cuda.synchronize()
    plan.busy_times(lb.KERNEL_FWD)                                   # raises when a bounded wait gave up
    plan.busy_times(lb.KERNEL_BWD_FUSED if fused and q.shape[2] == 128 else lb.KERNEL_BWD_DQ)
    return out, lse, grads


def _check(cu, q, k, v, dout, got, window, sinks):
    out, lse, grads = got
    see = ref.visible(cu, window, sinks, "cuda")
    o, l, b_o, b_l = ref.forward(q, k, v, see)
    assert ref.worst(out, o, b_o) <= 1
    assert ref.worst(lse, l, b_l) <= 1
    want, bounds = ref.backward(q, k, v, out, lse, dout, see)
    for name, g, w, b in zip(("dq", "dk", "dv"), grads, want, bounds):
        assert ref.worst(g, w, b) <= 1, name


def _case(lengths, hq, hkv, d, fused, window, sinks, seed=0, **kw):
    cu = pools.cu_seqlens(lengths)
    q, k, v, dout = _tensors(cu, hq, hkv, d, seed)
    plan = _plan(cu, hq, hkv, fused, window, sinks, **kw)
    got = _run(plan, q, k, v, dout, fused)
    _check(cu, q, k, v, dout, got, window, sinks)
    plan.destroy()


FORMS = [(64, False), (128, False), (128, True), (256, False), (256, True)]


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 3), (33, 0), (64, 5), (127, 128), (128, 1), (129, 40), (200, 0)])
@pytest.mark.parametrize("d,fused", FORMS)
def test_sample_bounds_at_word_and_block_edges(d, fused, window, sinks):
    _case(EDGES, 2, 1, d, fused, window, sinks, seed=window)


@pytest.mark.parametrize("lengths,window,sinks", [
    ([1], 1, 0), ([1], 5, 5), ([2, 1], 1, 1), ([257], 3, 300), ([1500], 100, 4), ([1500], 500, 0), ([1500], 300, 260),
    ([700, 40, 900], 129, 129), ([100, 1400], 384, 130), ([1000, 600], 640, 1), ([1600], 1599, 0), ([1600], 1, 1599),
    ([130, 1, 1, 1400, 3], 257, 7), ([300, 0, 0, 500, 0, 120], 90, 3)])
@pytest.mark.parametrize("d,fused", FORMS)
def test_long_and_mixed_samples(d, fused, lengths, window, sinks):
    _case(lengths, 4, 2, d, fused, window, sinks, seed=sum(lengths))


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("d,fused", FORMS)
def test_random_pools(d, fused, seed):
    rng = np.random.default_rng([seed, d, fused])
    lengths = pools.random_layout(rng, int(rng.integers(300, 2200)), int(rng.choice([5, 100, 700, 2200])))
    hkv = int(rng.choice([1, 2]))
    hq = hkv * int(rng.choice([1, 2, 3]))
    window = int(np.exp(rng.uniform(0, np.log(1500))))
    sinks = int(rng.choice([0, 1, 4, 128, 300]))
    kw = dict(n_workers=int(rng.choice([0, 5, 36])))
    if fused:
        kw["pair_chunk"] = int(rng.choice([0, 128, 512]))
    _case(lengths, hq, hkv, d, fused, window, sinks, seed=seed, **kw)


@pytest.mark.parametrize("window,sinks", [(3000, 0), (3500, 4), (4000, 200), (3300, 130)])
def test_fused_backward_on_pairs_of_ctas(window, sinks):
    """Query chunks of 512 rows: sinks come as key blocks of their own, apart from the window's, in the later chunks; 130 and
    200 sinks end in the second block of their first pair of key blocks, or fill both."""
    lengths = [100, 7400]
    cu = pools.cu_seqlens(lengths)
    q, k, v, dout = _tensors(cu, 2, 1, 128, 3)
    plan = _plan(cu, 2, 1, True, window, sinks, pair_chunk=512, n_workers=16)
    assert plan.fused_ctas() == 2
    got = _run(plan, q, k, v, dout, True)
    _check(cu, q, k, v, dout, got, window, sinks)
    from paper_2607_23250_b200 import binding as lb
    assert bool((plan.tile_times(lb.KERNEL_BWD_FUSED) > 0).all())      # every pair tile was taken once
    plan.destroy()


def test_the_form_of_the_backward():
    """With few key-major tiles for the workers the fused form, with many the two-kernel one, bit for bit what a plan without
    pair tiles gives; lists that were not asked for stay the library's own."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([900, 300])
    q, k, v, dout = _tensors(cu, 4, 2, 128, 2)
    results = []
    for workers, fused, ctas in ((148, True, 1), (12, True, 0), (12, False, None)):
        plan = _plan(cu, 4, 2, fused, 150, 3, n_workers=workers)
        if fused:
            assert plan.fused_ctas() == ctas
            with pytest.raises(lb.LibraError) as err:
                plan.info(lb.LIBRA_DIR_KV)
            assert err.value.code == lb.ERR_PLAN_MISMATCH
        out, lse = lb.libra_attn_pool_fwd(q, k, v, plan)
        ws = lb.libra_attn_pool_bwd_workspace_bytes(plan, q, k)
        results.append((ws, lb.libra_attn_pool_bwd(q, k, v, out, lse, dout, plan)))
        _check(cu, q, k, v, dout, (out, lse, results[-1][1]), 150, 3)
        plan.destroy()
    assert results[1][0] == results[2][0] < results[0][0]
    q64, k64, v64, g64 = _tensors(cu, 4, 2, 64, 2)              # as without a window, 64-wide heads need key-major lists
    plan = _plan(cu, 4, 2, True, 150, 3, n_workers=12)
    out, lse = lb.libra_attn_pool_fwd(q64, k64, v64, plan)
    with pytest.raises(lb.LibraError) as err:
        lb.libra_attn_pool_bwd(q64, k64, v64, out, lse, g64, plan)
    assert err.value.code == lb.ERR_PLAN_MISMATCH
    plan.destroy()
    assert all(torch.equal(x, y) for x, y in zip(results[1][1], results[2][1]))


@pytest.mark.parametrize("sinks", [0, 3])
def test_busy_times_of_the_form_that_was_chosen(sinks):
    """Of the two kernels where the library took them for a plan with pair tiles, otherwise there is no dK/dV kernel to ask for."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([900, 300])
    q, k, v, dout = _tensors(cu, 4, 2, 128, 2)
    for workers in (12, 148):
        plan = _plan(cu, 4, 2, True, 150, sinks, n_workers=workers)
        out, lse = lb.libra_attn_pool_fwd(q, k, v, plan)
        lb.libra_attn_pool_bwd(q, k, v, out, lse, dout, plan)
        if workers == 12:
            assert plan.fused_ctas() == 0
            for kern in (lb.KERNEL_BWD_DKDV, lb.KERNEL_BWD_DQ):
                busy = plan.busy_times(kern)
                assert len(busy) == 12 and (busy > 0).all()
        else:
            assert plan.fused_ctas() == 1 and plan.busy_times(lb.KERNEL_BWD_FUSED).any()
            with pytest.raises(lb.LibraError) as err:
                plan.busy_times(lb.KERNEL_BWD_DKDV)
            assert err.value.code == lb.ERR_PLAN_MISMATCH
        plan.destroy()


@pytest.mark.parametrize("sinks", [0, 3])
@pytest.mark.parametrize("heads,tile", [(4, 128), (3, 256), (4, 384)])
def test_plans_that_only_the_fused_form_can_take(heads, tile, sinks):
    """A pool for which the two-kernel form would be the faster one, but whose query-major lists its kernels cannot walk: tiles of
    another size, head shards that fit the kv heads in no way.  The fused form needs neither."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([900, 300])
    q, k, v, dout = _tensors(cu, 4, 2, 128, 2)
    first = _plan(cu, 4, 2, True, 150, sinks, n_workers=12)
    assert first.fused_ctas() == 0
    out, lse = lb.libra_attn_pool_fwd(q, k, v, first)
    plan = lb.libra_plan_tiles(torch.from_numpy(cu).cuda(), heads, tile, directions=lb.LIBRA_DIR_Q | lb.LIBRA_DIR_PAIR, tile_kv=128,
                               n_heads_kv=2, window=150, sinks=sinks, n_workers=12)
    assert plan.status() == 0 and plan.fused_ctas() == 1
    assert (lb.libra_attn_pool_bwd_workspace_bytes(plan, q, k) > lb.libra_attn_pool_bwd_workspace_bytes(first, q, k))
    for _ in range(2):
        grads = lb.libra_attn_pool_bwd(q, k, v, out, lse, dout, plan)
        torch.cuda.synchronize()
        plan.busy_times(lb.KERNEL_BWD_FUSED)
        _check(cu, q, k, v, dout, (out, lse, grads), 150, sinks)
    first.destroy()
    plan.destroy()


def test_head_shards_that_do_not_divide_the_heads():
    """Refused by the plan of either form: the pool does not decide what is accepted."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([900, 300])
    q, k, v, dout = _tensors(cu, 4, 2, 128, 2)
    lse = torch.zeros((4, q.shape[0]), device="cuda")
    for workers, ctas in ((12, 0), (148, 1)):
        plan = _plan(cu, 8, 2, True, 150, 3, n_workers=workers)
        assert plan.fused_ctas() == ctas
        launches = lb.launch_count()
        with pytest.raises(lb.LibraError) as err:
            lb.libra_attn_pool_bwd(q, k, v, q, lse, dout, plan)
        assert err.value.code == lb.ERR_INVALID_ARG and lb.launch_count() == launches
        plan.destroy()


@pytest.mark.parametrize("sinks", [0, 4])
def test_plans_of_more_key_blocks_than_the_rank_sort_takes(sinks):
    """65536 key blocks are the most of a key-major list that is asked for; lists of the library's own stay away from longer ones."""
    from paper_2607_23250_b200 import binding as lb
    T = 9_000_000
    cu = torch.arange(0, T + 1, 4500, dtype=torch.int32).cuda()
    plan = lb.libra_plan_tiles(cu, 1, 256, directions=lb.LIBRA_DIR_Q | lb.LIBRA_DIR_PAIR, tile_kv=128, window=100, sinks=sinks)
    assert plan.status() == 0 and plan.fused_ctas() > 0
    plan.destroy()
    with pytest.raises(lb.LibraError) as err:
        lb.libra_plan_tiles(cu, 1, 256, directions=lb.LIBRA_DIR_Q | lb.LIBRA_DIR_KV, tile_kv=128, window=100, sinks=sinks)
    assert err.value.code == lb.ERR_UNSUPPORTED


@pytest.mark.parametrize("window,sinks", [(300, 4), (1500, 200)])
def test_the_longest_pool_of_the_two_kernel_form(window, sinks):
    """65536 key blocks with sinks (no room for lists in which their tails are tiles of their own): 2048 copies of a sample, each of
    which has the gradients of the first, bit for bit."""
    from paper_2607_23250_b200 import binding as lb
    n, copies = 4096, 2048
    t = pools.make_tensors(n, 1, 1, 64, seed=window, device="cuda")
    small = [t[x] for x in ("q", "k", "v", "dout")]
    q, k, v, dout = (x.repeat(copies, 1, 1) for x in small)
    cu = np.arange(0, n * copies + 1, n, dtype=np.int32)
    plan = _plan(cu, 1, 1, False, window, sinks)
    got = _run(plan, q, k, v, dout, False)
    one = (got[0][:n], got[1][:, :n], [g[:n] for g in got[2]])
    _check(np.array([0, n], np.int32), *small, one, window, sinks)
    assert torch.equal(got[0].view(copies, n, 64), one[0].view(1, n, 64).expand(copies, n, 64))
    for g, first in zip(got[2], one[2]):
        assert torch.equal(g.view(copies, n, 64), first.view(1, n, 64).expand(copies, n, 64))
    plan.destroy()


@pytest.mark.parametrize("lengths,window,sinks", [([700, 40, 500], 120, 4), ([9000, 300], 500, 0), ([200, 5000], 900, 140)])
@pytest.mark.parametrize("hq,hkv,shards", [(4, 2, 2), (4, 1, 1), (6, 2, 2)])
@pytest.mark.parametrize("d,fused", FORMS)
def test_several_heads_a_shard(d, fused, hq, hkv, shards, lengths, window, sinks):
    """Query-major tiles of more than one head: few tiles, with a CTA for each half, and many."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens(lengths)
    q, k, v, dout = _tensors(cu, hq, hkv, d, window)
    directions = lb.LIBRA_DIR_Q | (lb.LIBRA_DIR_PAIR if fused else lb.LIBRA_DIR_KV)
    plan = lb.libra_plan_tiles(torch.from_numpy(cu).cuda(), shards, 256, directions=directions, tile_kv=128, n_heads_kv=hkv,
                               window=window, sinks=sinks)
    assert plan.status() == 0
    _check(cu, q, k, v, dout, _run(plan, q, k, v, dout, fused), window, sinks)
    plan.destroy()


@pytest.mark.parametrize("scale", [0.03, 0.4])
@pytest.mark.parametrize("d,fused", FORMS)
def test_a_scale_that_is_given(d, fused, scale):
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([600, 150])
    q, k, v, dout = _tensors(cu, 4, 2, d, 12)
    plan = _plan(cu, 4, 2, fused, 110, 3)
    out, lse = lb.libra_attn_pool_fwd(q, k, v, plan, scale=scale)
    grads = lb.libra_attn_pool_bwd(q, k, v, out, lse, dout, plan, scale=scale)
    see = ref.visible(cu, 110, 3, "cuda")
    o, l, b_o, b_l = ref.forward(q, k, v, see, scale)
    assert ref.worst(out, o, b_o) <= 1 and ref.worst(lse, l, b_l) <= 1
    want, bounds = ref.backward(q, k, v, out, lse, dout, see, scale)
    for name, g, w, b in zip(("dq", "dk", "dv"), grads, want, bounds):
        assert ref.worst(g, w, b) <= 1, name
    plan.destroy()


@pytest.mark.parametrize("over", ["q", "dout"])
@pytest.mark.parametrize("workers", [0, 12])
@pytest.mark.parametrize("d,fused", FORMS)
def test_dq_in_place(d, fused, workers, over):
    """dq written over q or dout: with CTAs for every tile and with few; a fused plan of few workers takes the two-kernel form."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([900, 300])
    q, k, v, dout = _tensors(cu, 4, 2, d, 2)
    plan = _plan(cu, 4, 2, fused, 150, 3, n_workers=workers)
    out, lse = lb.libra_attn_pool_fwd(q, k, v, plan)
    x = {"q": q.clone(), "dout": dout.clone()}
    grads = lb.libra_attn_pool_bwd(x["q"], k, v, out, lse, x["dout"], plan, dq=x[over])
    assert grads[0] is x[over]
    _check(cu, q, k, v, dout, (out, lse, grads), 150, 3)
    plan.destroy()


@pytest.mark.parametrize("sinks", [0, 4])
@pytest.mark.parametrize("d", [64, 256])
def test_a_plan_built_under_capture(d, sinks):
    """The plan holds what the last replay computed, the tails of sinks too."""
    from paper_2607_23250_b200 import binding as lb
    layouts = [pools.cu_seqlens(x) for x in ([700, 500, 1], [1, 1150, 50])]
    q, k, v, dout = _tensors(layouts[0], 2, 1, d, 7)
    cu = torch.from_numpy(layouts[0]).cuda()
    _plan(layouts[0], 2, 1, False, 200, sinks).destroy()            # what a first call sets up is there
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side, capture_error_mode="relaxed"):
        plan = lb.libra_plan_tiles(cu, 2, 256, tile_kv=128, n_heads_kv=1, total_tokens=1201, window=200, sinks=sinks)
    for layout in layouts:
        cu.copy_(torch.from_numpy(layout))
        graph.replay()
        torch.cuda.synchronize()
        assert plan.status() == 0
        _check(layout, q, k, v, dout, _run(plan, q, k, v, dout, False), 200, sinks)
    del graph
    plan.destroy()


@pytest.mark.parametrize("d,fused,window,sinks", [(64, False, 1000, 4), (128, False, 300, 0), (128, True, 5000, 130), (256, False, 2000, 2)])
def test_a_pool_of_twelve_thousand_tokens(d, fused, window, sinks):
    _case([700, 10100, 1200], 2, 1, d, fused, window, sinks, seed=d)


@pytest.mark.parametrize("d,fused", FORMS)
def test_a_window_that_reaches_everything_changes_nothing(d, fused):
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([300, 1, 800, 77])
    q, k, v, dout = _tensors(cu, 4, 2, d, 9)
    full = _plan(cu, 4, 2, fused, 0, 0)
    longest = _plan(cu, 4, 2, fused, 800, 0)
    wide = _plan(cu, 4, 2, fused, int(cu[-1]), 3)
    a, b, c = (_run(p, q, k, v, dout, fused) for p in (full, longest, wide))
    for x in (b, c):
        assert torch.equal(a[0], x[0]) and torch.equal(a[1], x[1])
        if not fused:
            assert all(torch.equal(g, h) for g, h in zip(a[2], x[2]))
    for direction in ((lb.LIBRA_DIR_Q, lb.LIBRA_DIR_PAIR) if fused else (lb.LIBRA_DIR_Q, lb.LIBRA_DIR_KV)):
        x, y = full.export(direction), wide.export(direction)
        assert all(np.array_equal(x[key], y[key]) for key in x)
    for p in (full, longest, wide):
        p.destroy()


@pytest.mark.parametrize("window,sinks", [(200, 1), (130, 130), (90, 300), (1, 128), (2000, 4), (128, 700)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_tails_of_sinks_in_the_two_kernel_form(d, window, sinks):
    """Key blocks with sinks whose row blocks beyond the window are tiles of their own, in one chunk and in several, of samples
    that start in the same key block as others and of one that ends inside a chunk; the same bits twice."""
    cu = pools.cu_seqlens([100, 20, 4500, 40, 2600, 7])
    q, k, v, dout = _tensors(cu, 2, 1, d, window)
    plan = _plan(cu, 2, 1, False, window, sinks)
    got = _run(plan, q, k, v, dout, False)
    _check(cu, q, k, v, dout, got, window, sinks)
    again = _run(plan, q, k, v, dout, False)
    assert all(torch.equal(x, y) for x, y in zip(got[2], again[2]))
    plan.destroy()


@pytest.mark.parametrize("lengths,window,sinks", [([1500], 100, 4), ([1100, 30], 300, 1), ([700], 50, 130), ([40, 900, 3], 1, 128), ([2000], 260, 2)])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 1), (6, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_tails_shared_by_clusters(d, hq, hkv, lengths, window, sinks):
    """Few tiles: clusters of CTAs share the main tiles and the tails."""
    _case(lengths, hq, hkv, d, False, window, sinks, seed=window)


@pytest.mark.parametrize("seed", range(10))
def test_plan_weights_placement_and_pair_tiles(seed):
    from paper_2607_23250_b200 import binding as lb
    rng = np.random.default_rng(70 + seed)
    lengths = pools.random_layout(rng, int(rng.integers(50, 2500)), int(rng.choice([7, 300, 2500])))
    cu = pools.cu_seqlens(lengths)
    window, sinks = int(rng.integers(1, 600)), int(rng.choice([0, 1, 5, 100, 400]))
    see = ref.visible(cu, window, sinks)
    H, Hkv, W = int(rng.integers(1, 4)), int(rng.integers(1, 3)), int(rng.integers(1, 50))
    tile, tile_kv, g = int(rng.choice([16, 100, 256])), int(rng.choice([32, 64, 128])), int(rng.choice([0, 16, 128]))
    chunk = tile_kv * int(rng.choice([1, 3, 8]))
    kw = dict(weight_model=lb.LIBRA_WEIGHT_BLOCKS, cost_block=g, unit_cost_q=5, unit_cost_kv=3) if g else {}
    plan = lb.libra_plan_tiles(torch.from_numpy(cu).cuda(), H, tile, n_workers=W, directions=7, tile_kv=tile_kv,
                               n_heads_kv=Hkv, window=window, sinks=sinks, pair_chunk=chunk, **kw)
    assert plan.status() == 0
    for direction, heads, size, unit in ((lb.LIBRA_DIR_Q, H, tile, 5), (lb.LIBRA_DIR_KV, Hkv, tile_kv, 3)):
        got = plan.export(direction)
        if not g:
            unit = 12 if direction == lb.LIBRA_DIR_Q else 6            # the library's own
        want = ref.tile_weights(see, size, direction == lb.LIBRA_DIR_KV, g or 128, unit)
        assert got["weight"].tolist() == [w for w in want for _ in range(heads)]
        cta, loads = ref.place(want, heads, W)
        assert np.array_equal(got["cta_of_tile"], cta) and np.array_equal(got["loads"], loads)
    want = ref.live_pairs(see, tile_kv, chunk)
    kb, qc, size = plan.export_pairs()
    assert size == chunk
    assert list(zip(qc.tolist(), kb.tolist())) == [(c, j) for c, j, _ in want]
    assert plan.export(lb.LIBRA_DIR_PAIR)["weight"].tolist() == [n for _ in range(Hkv) for *_, n in want]
    plan.destroy()


def test_refusals():
    from paper_2607_23250_b200 import binding as lb
    cu = torch.tensor([0, 300], dtype=torch.int32).cuda()
    for window, sinks in ((-1, 0), (0, 3), (5, -1)):
        with pytest.raises(lb.LibraError) as err:
            lb.libra_plan_tiles(cu, 1, 256, window=window, sinks=sinks)
        assert err.value.code == lb.ERR_INVALID_ARG
    bad = torch.tensor([0, 200, 100, 300], dtype=torch.int32).cuda()
    plan = lb.libra_plan_tiles(bad, 1, 256, directions=7, tile_kv=128, total_tokens=300, window=20, sinks=3)
    assert plan.status() == lb.ERR_BAD_SEQLENS
    t = pools.make_tensors(300, 1, 1, 128, seed=1, device="cuda")
    out = torch.full_like(t["q"], 7.0)
    lb.libra_attn_pool_fwd(t["q"], t["k"], t["v"], plan, out=out)
    assert bool((out == 7).all())
    plan.destroy()


def test_two_kernel_form_is_bit_reproducible_and_captured():
    """Twice the same bits, eagerly and replayed from a graph with other inputs in between; on a stream of its own."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([900, 20, 1100])
    q, k, v, dout = _tensors(cu, 4, 2, 128, 5)
    plan = _plan(cu, 4, 2, False, 250, 6)
    a = _run(plan, q, k, v, dout, False)
    b = _run(plan, q, k, v, dout, False)
    same = lambda x, y: torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and all(torch.equal(g, h) for g, h in zip(x[2], y[2]))  # noqa: E731
    assert same(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = torch.empty_like(q), torch.empty((4, q.shape[0]), device="cuda")
        grads = [torch.empty_like(x) for x in (q, k, v)]
        ws = torch.empty(lb.libra_attn_pool_bwd_workspace_bytes(plan, q, k), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            lb.libra_attn_pool_fwd(q, k, v, plan, out=out, lse=lse)
            lb.libra_attn_pool_bwd(q, k, v, out, lse, dout, plan, *grads, workspace=ws)
        keep = q.clone()
        q.neg_()
        graph.replay()
        q.copy_(keep)
        graph.replay()
    torch.cuda.synchronize()
    assert same(a, (out, lse, grads))
    del graph
    plan.destroy()


@pytest.mark.parametrize("d,fused", FORMS)
def test_two_streams_share_a_plan(d, fused):
    """A layer's passes on two streams at once, each with tensors and a workspace of its own."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([2600, 30, 1500])
    plan = _plan(cu, 4, 2, fused, 300, 5)
    ins = [_tensors(cu, 4, 2, d, seed) for seed in (1, 2)]
    want = [_run(plan, *x, fused) for x in ins]
    streams = [torch.cuda.Stream() for _ in ins]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for x, s, res in zip(ins, streams, got):
            out, lse = lb.libra_attn_pool_fwd(*x[:3], plan, stream=s)
            res.append((out, lse, lb.libra_attn_pool_bwd(*x[:3], out, lse, x[3], plan, stream=s)))
    torch.cuda.synchronize()
    for x, res, w in zip(ins, got, want):
        for out, lse, grads in res:
            assert torch.equal(out, w[0]) and torch.equal(lse, w[1])
            if fused:
                _check(cu, *x, (out, lse, grads), 300, 5)
            else:
                assert all(torch.equal(a, b) for a, b in zip(grads, w[2]))
    plan.destroy()


def test_noalloc_backward_follows_the_plan():
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([500, 300])
    q, k, v, dout = _tensors(cu, 2, 1, 64, 8)
    plan = _plan(cu, 2, 1, False, 90, 3)
    out, lse, grads = _run(plan, q, k, v, dout, False)
    mine = [torch.empty_like(x) for x in (q, k, v)]
    lb.libra_attn_pool_bwd_noalloc(q, k, v, out, lse, dout, plan, *mine)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(grads, mine))
    plan.destroy()


@pytest.mark.parametrize("d,sinks,room", [(64, 4, True), (64, 600, False), (128, 4, False), (128, 600, False), (256, 4, False), (256, 600, False)])
def test_noalloc_backward_without_room_for_the_tails(d, sinks, room):
    """The limit of the allocation-free call is that of the row statistics, whatever the partial sums of a plan with sinks would
    take: with room for them the bits of the other call, without it whole key blocks, twice the same bits."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([2300, 300])
    q, k, v, dout = _tensors(cu, 8, 8, d, 4)
    plan = _plan(cu, 8, 8, False, 100, sinks)
    limit = lb.libra_attn_pool_bwd_noalloc_max_bytes()
    assert (lb.libra_attn_pool_bwd_workspace_bytes(plan, q, k) <= limit) == room
    out, lse, grads = _run(plan, q, k, v, dout, False)
    mine = [[torch.full_like(x, 7.0) for x in (q, k, v)] for _ in range(2)]
    for m in mine:
        lb.libra_attn_pool_bwd_noalloc(q, k, v, out, lse, dout, plan, *m)
    torch.cuda.synchronize()
    for kern in (lb.KERNEL_BWD_DKDV, lb.KERNEL_BWD_DQ):
        plan.busy_times(kern)
    _check(cu, q, k, v, dout, (out, lse, mine[0]), 100, sinks)
    assert all(torch.equal(x, y) for x, y in zip(*mine))
    assert torch.equal(grads[0], mine[0][0])
    if room:
        assert all(torch.equal(x, y) for x, y in zip(grads, mine[0]))
    plan.destroy()


def test_noalloc_backward_refuses_what_only_the_tails_lists_can_do():
    """A plan whose key-major lists are the library's own has no lists of whole key blocks."""
    from paper_2607_23250_b200 import binding as lb
    cu = pools.cu_seqlens([2300, 300])
    q, k, v, dout = _tensors(cu, 8, 8, 128, 4)
    plan = _plan(cu, 8, 8, True, 100, 300, n_workers=12)
    assert plan.fused_ctas() == 0
    out, lse = lb.libra_attn_pool_fwd(q, k, v, plan)
    launches = lb.launch_count()
    with pytest.raises(lb.LibraError) as err:
        lb.libra_attn_pool_bwd_noalloc(q, k, v, out, lse, dout, plan, *[torch.empty_like(x) for x in (q, k, v)])
    assert err.value.code == lb.ERR_SCRATCH_TOO_SMALL and lb.launch_count() == launches
    plan.destroy()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_stalled_producers_give_up_cleanly(d):
    """The bounded waits of the kernels with sinks, as in the tests of the others: no loads are issued, the launch reports a
    timeout and the next one is right."""
    from paper_2607_23250_b200 import binding as lb
    lengths = [1200, 100]
    cu = pools.cu_seqlens(lengths)
    q, k, v, dout = _tensors(cu, 2, 1, d, 4)
    plan = _plan(cu, 2, 1, False, 150, 4)
    good = _run(plan, q, k, v, dout, False)
    plan.set_wait_limit_ns(200_000)
    plan.inject_stall(True)
    lb.libra_attn_pool_fwd(q, k, v, plan)
    with pytest.raises(lb.LibraError) as err:
        plan.busy_times(lb.KERNEL_FWD)
    assert err.value.code == lb.ERR_TIMEOUT
    lb.libra_attn_pool_bwd(q, k, v, *good[:2], dout, plan)
    with pytest.raises(lb.LibraError) as err:
        plan.busy_times(lb.KERNEL_BWD_DQ)
    assert err.value.code == lb.ERR_TIMEOUT
    plan.inject_stall(False)
    plan.set_wait_limit_ns(0)
    again = _run(plan, q, k, v, dout, False)
    assert torch.equal(good[0], again[0]) and all(torch.equal(x, y) for x, y in zip(good[2], again[2]))
    plan.destroy()


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("d,fused", FORMS)
def test_values_that_are_not_finite_stay_near(d, fused, value):
    """Products are taken a block of 128 keys by a tile of 256 rows at a time, masked ones with a weight of 0: a key and a value that are
    not finite reach the tiles of rows that see a key of their block (the block's last key by a window's length), a query
    and its gradient the 256-key tiles of keys that a row of its block sees, the sinks' among them.  Everything else is what it was."""
    T, window, sinks, at = 2300, 300, 4, 900
    cu = pools.cu_seqlens([T])
    q, k, v, dout = _tensors(cu, 2, 1, d, 6)
    plan = _plan(cu, 2, 1, fused, window, sinks)
    out, lse, grads = _run(plan, q, k, v, dout, fused)
    tile = lambda t: t // 256 * 256  # noqa: E731
    block = at // 128 * 128
    near = slice(tile(at), tile(block + 127 + window - 1) + 256)
    k2, v2 = k.clone(), v.clone()
    k2[at], v2[at, 0, 5] = value, value
    out2, lse2, _ = _run(plan, q, k2, v2, dout, fused)
    far = torch.ones(T, dtype=torch.bool, device="cuda")
    far[near] = False
    assert torch.equal(out[far], out2[far]) and torch.equal(lse[:, far], lse2[:, far])
    from paper_2607_23250_b200 import binding as lb
    g2 = dout.clone()
    g2[at] = value
    dq, dk, dv = lb.libra_attn_pool_bwd(q, k, v, out, lse, g2, plan)
    far = torch.ones(T, dtype=torch.bool, device="cuda")
    far[tile(at)] = False
    far[tile(at):tile(at) + 256] = False
    same = torch.equal if not fused else lambda x, y: bool((x - y).abs().max() <= 2.0 ** -6 * y.abs().max())
    assert same(dq[far], grads[0][far])
    far[tile(block - window + 1):tile(at) + 256] = False
    far[:256] = False                                                   # the sinks' tile
    assert same(dk[far], grads[1][far]) and same(dv[far], grads[2][far])
    plan.destroy()


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("d,T,hq", [(64, 2300, 2), (64, 21000, 6), (128, 2300, 2), (128, 21000, 6), (256, 9000, 4)])
def test_a_row_without_a_number_ends_no_launch(d, T, hq, value):
    """Rows that see a key that is not finite are NaN, sinks or not; the worker that met them goes on to its other tiles.  Sizes at
    which a tile has a CTA for each half (2300), one, and a worker several tiles."""
    from paper_2607_23250_b200 import binding as lb
    window, sinks, at = 300, 4, 900
    cu = pools.cu_seqlens([T])
    q, k, v, dout = _tensors(cu, hq, 1, d, 6)
    for fused in (False, True) if d != 64 else (False,):
        plan = _plan(cu, hq, 1, fused, window, sinks)
        want, want_lse = lb.libra_attn_pool_fwd(q, k, v, plan)
        k2 = k.clone()
        k2[at] = value
        out, lse = torch.full_like(want, 7.0), torch.full_like(want_lse, 7.0)
        lb.libra_attn_pool_fwd(q, k2, v, plan, out=out, lse=lse)
        torch.cuda.synchronize()
        plan.busy_times(lb.KERNEL_FWD)                                  # raises where a CTA gave up
        # q has values of either sign in every row: their products with infinities add up to NaN
        assert out[at:at + window].isnan().all() and lse[:, at:at + window].isnan().all()
        far = torch.ones(T, dtype=torch.bool, device="cuda")
        far[at // 256 * 256:(at // 128 * 128 + 127 + window - 1) // 256 * 256 + 256] = False
        assert torch.equal(out[far], want[far]) and torch.equal(lse[:, far], want_lse[:, far])
        grads = lb.libra_attn_pool_bwd(q, k2, v, out, lse, dout, plan)
        torch.cuda.synchronize()
        plan.busy_times(lb.KERNEL_BWD_FUSED if fused and d == 128 and plan.fused_ctas() > 0 else lb.KERNEL_BWD_DQ)
        assert grads[0][at:at + window].isnan().all()
        plan.destroy()
