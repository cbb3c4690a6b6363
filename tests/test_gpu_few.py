"""Chunks of few query rows at head_dim 128 (one launch): what they leave in the cache, replays, two caches at once; against plain 64-bit forms."""
import pytest
import torch

import paper_2601_18383_b200 as D
from tests import extend_reference as R
from tests import tree_reference as TR
from tests.test_gpu_extend import build, chunk
from tests.test_gpu_tree import check, flat

pytestmark = pytest.mark.gpu


def launches(c, call):
    before = D.dynts_cache_launch_count(c.handle)
    call()
    return D.dynts_cache_launch_count(c.handle) - before


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("q_heads,new", [(2, (1, 1, 1)), (4, (9, 0, 16)), (14, (4, 1, 2)), (16, (8, 0, 7)), (2, (64, 33, 31)), (4, (64, 0, 33)), (14, (18, 3, 9))])
@pytest.mark.parametrize("opt", [dict(), dict(window=37, sinks=6), dict(softcap=15.0, slopes=True)], ids=["plain", "sinks", "mods"])
def test_rows_left_and_lengths(dtype, q_heads, new, opt):
    """Tiles that the chunk begins, ends and crosses; groups of 1 to 8 heads; stored rows, then more behind them."""
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = 2.0 ** (-8.0 * torch.arange(1, q_heads + 1) / q_heads) * 0.1
    c, seen = build(dtype=dtype, layers=2, q_heads=q_heads, kv_heads=2, past=(64, 0, 141), cap=400, evict_to=100)
    n_new = list(new)
    for seed in (1, 2):
        check(c, seen, n_new, seed=seed, scale=0.05, stage=False, want_mass=False, by_layer=seed == 2, **opt)
        seen = [s + t for s, t in zip(seen, n_new)]
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_scores_and_a_path(dtype):
    c, seen = build(dtype=dtype, layers=2, q_heads=4, kv_heads=2, past=(90, 0, 33), cap=300)
    n_new, scale = [12, 30, 5], 0.05
    state = R.State(c, scale, scale)
    q, k, v = chunk(c, n_new, 3)
    parents = [[-1, 0, 0, 1, 2, 2, 4, 4, 7, 3, 8, 10], list(range(-1, 29)), [-1, -1, 1, 1, 3]]
    tree, _ = c.tree_plan(flat(parents), n_new)
    s_new = torch.rand(47, device="cuda")
    out = torch.empty_like(q)
    assert launches(c, lambda: c.extend_attn(q, k, v, out, n_new, s_new=s_new, stage=True, tree=tree)) == 1
    paths = [[0, 2, 4, 7], [], [1, 3, 4]]
    path = torch.full((3, 6), -1, dtype=torch.int32, device="cuda")
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    c.extend_commit_path([4, 0, 3], path)
    c.synchronize()
    c.poll_error()
    first = 0
    for b, p in enumerate(paths):
        at = [first + i for i in p]
        first += n_new[b]
        for l in range(2):
            for h in range(2):
                K, V, pos, score = c.export_slab(l, b, h)
                K0, V0, pos0, score0 = state.slab[l, b, h]
                kn, vn = k[l, at, h].cpu(), v[l, at, h].cpu()
                if dtype == "bf16_kv8":
                    kn, vn = R.e4m3(kn, scale).double() * scale, R.e4m3(vn, scale).double() * scale
                assert torch.equal(R.State.value(K, scale), torch.cat([K0, kn.double()])) and torch.equal(R.State.value(V, scale), torch.cat([V0, vn.double()]))
                assert pos.tolist() == pos0.tolist() + list(range(seen[b], seen[b] + len(p)))
                assert torch.equal(score.double(), torch.cat([score0, s_new[at].double().cpu()]))
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_more_query_rows_than_a_cluster_takes(dtype):
    """100 and 128 rows of one sequence, clusters of their own for 32 of them; one of them with values that are not finite beside."""
    for q_heads, kv_heads, new in ((32, 8, 25), (4, 1, 32), (14, 2, 18), (8, 8, 65)):
        c, seen = build(dtype=dtype, q_heads=q_heads, kv_heads=kv_heads, past=(700,), cap=900)
        q, k, v = chunk(c, [new], 7)
        assert launches(c, lambda: c.extend_attn(q, k, v, torch.empty_like(q), [new], stage=True)) == 1
        check(c, seen, [new], want_mass=False, scale=0.05, seed=1)
        check(c, seen, [new], TR.random_trees([new], 3, 6), want_mass=False, scale=0.05, seed=2)
        bad_k, bad_v = k.clone(), v.clone()
        bad_k[:, new - 1] = bad_v[:, new - 1] = float("nan")  # a leaf that the others do not see
        clean, out = torch.empty_like(q), torch.empty_like(q)
        tree, _ = c.tree_plan(torch.tensor([-1] * new, dtype=torch.int32, device="cuda"), [new])
        c.extend_attn(q, k, v, clean, [new], stage=True, tree=tree)
        c.extend_attn(q, bad_k, bad_v, out, [new], tree=tree, stage=True)
        c.synchronize()
        keep = slice(0, new - 1)
        diff = (out[:, keep].double() - clean[:, keep].double()).abs()
        # (rows computed again: a half step of the weights, and one of the output on either side)
        assert (diff <= 2 * 2.0 ** -8 * clean[:, keep].double().abs() + 2.0 ** -8 * v.abs().max().double()).all()
        c.close()


def test_steps_replayed_as_the_sequences_grow():
    """One token per sequence, published: a graph of one step, replayed past tile borders; then it no longer fits."""
    c, seen = build(q_heads=8, kv_heads=2, past=(30, 62, 0), cap=100)
    n_new = [1, 1, 1]
    q, k, v = chunk(c, n_new, 0)
    out = torch.empty_like(q)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    assert launches(c, lambda: c.extend_attn(q, k, v, out, n_new, stage=True, window=40, sinks=3)) == 1
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.set_stream(side)
        with torch.cuda.graph(graph, stream=side):
            c.extend_attn(q, k, v, out, n_new, window=40, sinks=3)
    c.set_stream(torch.cuda.current_stream())
    D.dynts_cache_refresh_lengths(c.handle)  # (what was captured has not run)
    for step in range(38):
        state = R.State(c)
        new = chunk(c, n_new, 10 + step)
        for x, y in zip((q, k, v), new):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        ref, tol, *_ = TR.attend(state, [s + step for s in seen], q, k, v, n_new, None, p_half_step=2.0 ** -8, window=40, sinks=3)
        assert ((out.double().cpu() - ref).abs() <= tol).all()
        D.dynts_cache_refresh_lengths(c.handle)
        assert [c.len(b) for b in range(3)] == [31 + step, 63 + step, 1 + step]
    c.poll_error()
    # the second sequence is full: nothing of it moves, the others go on
    held = out[:, 1].clone()
    graph.replay()
    torch.cuda.synchronize()
    D.dynts_cache_refresh_lengths(c.handle)
    assert [c.len(b) for b in range(3)] == [69, 100, 39] and torch.equal(out[:, 1], held)
    with pytest.raises(D.DyntsError) as e:
        c.poll_error()
    assert e.value.status == D.DYNTS_ERR_DEVICE
    c.close()


def test_two_caches_on_two_streams():
    caches = [build(q_heads=8, kv_heads=2, past=(700, 900), cap=1200, dtype=d)[0] for d in ("bf16", "bf16_kv8")]
    streams = [torch.cuda.Stream() for _ in caches]
    n_new = [6, 3]
    calls = []
    for c, s in zip(caches, streams):
        q, k, v = chunk(c, n_new, 4)
        alone, both = torch.empty_like(q), torch.empty_like(q)
        c.extend_attn(q, k, v, alone, n_new, stage=True)
        c.synchronize()
        s.wait_stream(torch.cuda.current_stream())
        c.set_stream(s)
        calls.append((c, q, k, v, both, alone))
    for _ in range(20):
        for c, q, k, v, both, _alone in calls:
            c.extend_attn(q, k, v, both, n_new, stage=True)
    torch.cuda.synchronize()
    for c, q, k, v, both, alone in calls:
        assert torch.equal(both, alone)
        c.poll_error()
        c.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_hidden_rows_and_stale_ones_may_hold_anything(dtype, bad):
    """What lies behind the window, and behind the chunk's end, where another chunk was staged before, does not reach the answers."""
    c, seen = build(dtype=dtype, q_heads=4, kv_heads=1, past=(50,), cap=256)
    q, k, v = chunk(c, [16], 2)
    c.extend_attn(q, torch.full_like(k, bad), torch.full_like(v, bad), torch.empty_like(q), [16], stage=True)  # 16 rows of nothing good, forgotten
    check(c, seen, [5], want_mass=False, scale=0.05, seed=3)
    k2, v2 = k.clone(), v.clone()
    k2[:, :3], v2[:, :3] = bad, bad
    c.extend_attn(q, k2, v2, torch.empty_like(q), [16])  # held now: positions 50 to 52 hold it
    clean = build(dtype=dtype, q_heads=4, kv_heads=1, past=(50,), cap=256)[0]
    clean.extend_attn(q, k, v, torch.empty_like(q), [16])
    q3, k3, v3 = chunk(c, [2], 5)
    a, b = torch.empty_like(q3), torch.empty_like(q3)
    c.extend_attn(q3, k3, v3, a, [2], window=10, sinks=4, stage=True)
    clean.extend_attn(q3, k3, v3, b, [2], window=10, sinks=4, stage=True)
    c.synchronize(), clean.synchronize()
    # (rows computed again in 32 bits against rows by the tensor cores: a half step of the weights, and one of the output, each)
    assert torch.isfinite(a).all() and ((a.double() - b.double()).abs() <= 2 * 2.0 ** -8 * b.double().abs() + 2 * 2.0 ** -8 * v3.abs().max().double()).all()
    c.close(), clean.close()
