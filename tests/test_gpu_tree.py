"""Trees of drafted tokens: their numbering, attention through the cache with the mask of ancestors, the path of drawn tokens and
its commit; and windows with sinks, for lines and trees.  Against plain 64-bit forms, for every type of row."""
import pytest
import torch

import paper_2601_18383_b200 as D
from tests import extend_reference as R
from tests import tree_reference as TR
from tests.test_gpu_extend import build, chunk

pytestmark = pytest.mark.gpu


def flat(lists):
    return torch.tensor([x for y in lists for x in y], dtype=torch.int32, device="cuda")


def check(c, seen, n_new, trees=None, seed=0, by_layer=False, stage=True, want_mass=True, scale=1.0, sharp=1.0, chunks=None, **opt):
    kv8 = c.dtype_name == "bf16_kv8"
    q, k, v = chunks or chunk(c, n_new, seed, sharp)
    state = R.State(c, scale if kv8 else 1.0, scale if kv8 else 1.0)
    lens = [c.len(b) for b in range(c.batch)]
    half = 0.0 if c.torch_dtype == torch.float32 or c.head_dim != 128 else 2.0 ** -8  # weights rounded to 16 bits before the product
    ref, tol, mass, mass_tol, rows = TR.attend(state, seen, q, k, v, n_new, trees, p_half_step=half, **opt)
    T = sum(n_new)
    pad = torch.full((c.layers * T + 2, c.q_heads, c.head_dim), 7.0, dtype=c.torch_dtype, device="cuda")
    out = pad[: c.layers * T].view(c.layers, T, c.q_heads, c.head_dim)
    buf = torch.full((c.layers, c.batch, c.kv_heads, c.capacity), -3.0, device="cuda") if want_mass else None
    tree = None
    if trees:
        tree, positions = c.tree_plan(flat(trees[0]), n_new)
        assert positions.tolist() == [s + x for s, dep in zip(seen, trees[1]) for x in dep]
    dev_opt = dict(opt, tree=tree, stage=stage)
    if opt.get("slopes") is not None:
        dev_opt["slopes"] = opt["slopes"].cuda()
    if by_layer:
        for l in range(c.layers):
            c.extend_attn_layer(l, q[l], k[l], v[l], out[l], n_new, mass=buf, **dev_opt)
    else:
        c.extend_attn(q, k, v, out, n_new, mass=buf, **dev_opt)
    c.synchronize()
    c.poll_error()
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    bad = (got - ref).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outputs off, worst {((got - ref).abs() / tol).max():.3g} of the bound"
    assert (pad[c.layers * T:] == 7.0).all()
    for (l, b, h), (K, V, pos) in rows.items():
        t, n = int(n_new[b]), lens[b]
        if want_mass:
            m = buf[l, b, h].double().cpu()
            assert (m[n + t if t else 0:] == -3.0).all()
            if t:
                x = (m[: n + t] - mass[l, b, h]).abs()
                assert (x <= mass_tol[l, b, h]).all(), f"mass off by {(x / mass_tol[l, b, h]).max():.3g} of the bound"
        assert c.len(b) == (n if stage else n + t)
        if not stage:
            Kd, Vd, pd, _ = c.export_slab(l, b, h)
            assert torch.equal(R.State.value(Kd, scale), K) and torch.equal(R.State.value(Vd, scale), V) and torch.equal(pd.long(), pos)
    return q, k, v, out, tree


# ---- numbering ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n_new,depth,roots", [([1], 1, 1), ([33, 0, 7], 4, 2), ([64, 1, 200], 9, 1), ([1024], 1024, 1), ([1000], 3, 5), ([31, 32, 96], 2, 40)])
def test_numbering(n_new, depth, roots):
    c, seen = build(past=tuple(5 * (b + 1) for b in range(len(n_new))), cap=1100, q_heads=2, kv_heads=1, d=64, dtype="fp32")
    parents, depths = TR.random_trees(n_new, 3, depth, roots)
    if depth == 1024:  # a line
        parents, depths = [list(range(-1, 1023))], [list(range(1024))]
    tree, positions = c.tree_plan(flat(parents), n_new)
    c.synchronize()
    c.poll_error()
    assert positions.tolist() == [s + x for s, dep in zip(seen, depths) for x in dep]
    first = 0
    for p, dep in zip(parents, depths):
        t = len(p)
        order, size, d, parent = (tree[first:first + t, i].long().cpu() for i in range(4))
        assert d.tolist() == dep and parent.tolist() == p
        below = (order[:, None] - order[None, :] >= 0) & (order[:, None] - order[None, :] < size[None, :])
        assert torch.equal(below, TR.ancestors(p))
        assert sorted(order.tolist()) == list(range(t))
        first += t
    c.close()


def test_a_parent_behind_its_child_is_reported():
    c, seen = build(past=(9, 9), cap=64)
    tree, _ = c.tree_plan(torch.tensor([-1, 0, 5, 1, -1, -7, 1], dtype=torch.int32, device="cuda"), [4, 3])
    c.synchronize()
    assert tree[:, 3].tolist() == [-1, 0, -1, 1, -1, -1, 1]  # it counts as none
    with pytest.raises(D.DyntsError) as e:
        c.poll_error()
    assert e.value.status == D.DYNTS_ERR_DEVICE
    c.close()


# ---- attention ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("q_heads,kv_heads", [(8, 2), (14, 2), (2, 2), (8, 1), (3, 1)])
@pytest.mark.parametrize("past,new", [((0,), (1,)), ((0,), (40,)), ((63,), (5,)), ((64,), (64,)), ((61,), (130,)), ((300,), (25,)), ((1,), (200,))])
def test_tree_bf16_one_sequence(q_heads, kv_heads, past, new):
    c, seen = build(q_heads=q_heads, kv_heads=kv_heads, past=past, cap=384)
    check(c, seen, list(new), TR.random_trees(list(new), past[0]))
    c.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64), ("fp32", 40), ("fp32", 128), ("bf16", 64), ("bf16", 8), ("bf16", 256),
                                     ("bf16_kv8", 48)])
def test_tree_ragged_batch_of_every_type(dtype, d):
    """Sequences without rows, without nodes, cut by an eviction, a forest; two layers in one call, then layer by layer."""
    c, seen = build(dtype=dtype, d=d, layers=2, q_heads=6, kv_heads=2, past=(90, 0, 33, 120, 7), cap=300, evict_to=64)
    n_new = [5, 70, 0, 1, 33]
    trees = TR.random_trees(n_new, 11, 5, 3)
    check(c, seen, n_new, trees, scale=0.05, seed=3)
    check(c, seen, n_new, trees, scale=0.05, seed=4, by_layer=True, want_mass=False)
    c.close()


OPTIONS = [dict(softcap=20.0), dict(slopes=True), dict(window=1), dict(window=3, sinks=2), dict(window=40), dict(window=40, sinks=70),
           dict(softcap=5.0, slopes=True, window=90, sinks=5)]


@pytest.mark.parametrize("opt", OPTIONS, ids=[",".join(o) + str(o.get("window", "")) + "_" + str(o.get("sinks", "")) for o in OPTIONS])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
def test_tree_options(opt, dtype, d):
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = 2.0 ** (-8.0 * torch.arange(1, 9) / 8) * 0.5
    c, seen = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(200, 0, 130), cap=300, evict_to=150)
    n_new = [30, 60, 17]
    check(c, seen, n_new, TR.random_trees(n_new, 5, 7, 2), scale=0.05, **opt)
    c.close()


def test_tree_of_a_line_is_the_chunk():
    """A tree without branches is the staged chunk: the same bits, where the same kernel serves both."""
    c, seen = build(past=(333,), cap=512, q_heads=8, kv_heads=2)
    q, k, v = chunk(c, [50], 1)
    a, b = torch.empty_like(q), torch.empty_like(q)
    c.extend_attn(q, k, v, a, [50], stage=True, softcap=30.0)
    tree, _ = c.tree_plan(torch.arange(-1, 49, dtype=torch.int32, device="cuda"), [50])
    c.extend_attn(q, k, v, b, [50], stage=True, softcap=30.0, tree=tree)
    c.synchronize()
    c.poll_error()
    assert ((a.double() - b.double()).abs() <= 2 * 2.0 ** -8 * a.double().abs() + 2.0 ** -7).all()
    c.close()


def test_hidden_nodes_may_hold_anything():
    """Rows of other branches with infinities and NaN in K and V do not reach a node."""
    for dtype, d in (("bf16", 128), ("fp32", 64), ("bf16", 64)):
        c, seen = build(dtype=dtype, d=d, past=(70,), cap=256, q_heads=4, kv_heads=1)
        parents = [-1, 0, 0, 1, 1, 2, 4, 0]
        depths = [0, 1, 1, 2, 2, 2, 3, 1]
        q, k, v = chunk(c, [8], 2)
        k2, v2 = k.clone(), v.clone()
        for x, bad in ((k2, float("nan")), (v2, float("inf"))):
            x[:, 5] = bad  # node 5: a leaf, seen by itself alone
            x[:, 7] = bad
        out, clean = torch.empty_like(q), torch.empty_like(q)
        tree, _ = c.tree_plan(flat([parents]), [8])
        c.extend_attn(q, k, v, clean, [8], stage=True, tree=tree)
        c.extend_attn(q, k2, v2, out, [8], stage=True, tree=tree)
        c.synchronize()
        keep = [0, 1, 2, 3, 4, 6]
        tol = 2.0 ** -7 * clean[:, keep].double().abs() + 2.0 ** -8 if dtype == "bf16" else 2.0 ** -20
        assert ((out[:, keep].double() - clean[:, keep].double()).abs() <= tol).all()
        c.close()


def test_largest_tree_and_beyond():
    c, seen = build(past=(100,), cap=1200, q_heads=4, kv_heads=1)
    n = [1024]
    check(c, seen, n, TR.random_trees(n, 7, 30, 2))
    big = torch.full((1025,), -1, dtype=torch.int32, device="cuda")
    with pytest.raises(D.DyntsError) as e:
        c.tree_plan(big, [1025])
    assert e.value.status == D.DYNTS_ERR_INVALID_ARG
    c.close()


def test_more_sequences_than_a_launch_takes():
    past = tuple((3 * b) % 50 for b in range(140))
    c, seen = build(past=past, cap=96, q_heads=2, kv_heads=1)
    n_new = [(b * 7) % 12 for b in range(140)]
    check(c, seen, n_new, TR.random_trees(n_new, 1, 4))
    c.close()


def test_replayed_trees_follow_their_parents():
    """Numbering and attention captured once; parents, queries and rows change between replays."""
    c, seen = build(past=(100, 40), cap=256, q_heads=8, kv_heads=2)
    n_new = [12, 9]
    first = TR.random_trees(n_new, 1)
    q, k, v = chunk(c, n_new, 1)
    parents, out = flat(first[0]), torch.empty_like(q)
    tree = torch.empty((21, 4), dtype=torch.int32, device="cuda")
    positions = torch.empty((21,), dtype=torch.int32, device="cuda")

    def call():
        c.tree_plan(parents, n_new, tree=tree, positions=positions)
        c.extend_attn(q, k, v, out, n_new, stage=True, tree=tree)

    call()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.set_stream(side)
        with torch.cuda.graph(graph, stream=side):
            call()
    c.set_stream(torch.cuda.current_stream())
    state = R.State(c)
    for seed in (2, 3):
        trees = TR.random_trees(n_new, seed)
        parents.copy_(flat(trees[0]))
        q2, k2, v2 = chunk(c, n_new, seed)
        q.copy_(q2), k.copy_(k2), v.copy_(v2)
        graph.replay()
        torch.cuda.synchronize()
        ref, tol, *_ = TR.attend(state, seen, q, k, v, n_new, trees, p_half_step=2.0 ** -8)
        assert ((out.double().cpu() - ref).abs() <= tol).all()
    c.poll_error()
    c.close()


# ---- the path of drawn tokens, and its commit --------------------------------------------------------------------------------

def plain_accept(parents, drafted, drawn, n_new, max_path):
    paths, counts, ends, first = [], [], [], 0
    for t in n_new:
        path = [0] if t else []
        while path and len(path) < max_path and drawn[first + path[-1]] >= 0:
            fit = [j for j in range(t) if parents[first + j] == path[-1] and drafted[first + j] == drawn[first + path[-1]]]
            if not fit:
                break
            path.append(fit[0])
        paths.append(path + [-1] * (max_path - len(path)))
        counts.append(len(path))
        ends.append(drawn[first + path[-1]] if t else -1)
        first += t
    return paths, counts, ends


@pytest.mark.parametrize("max_path", [1, 3, 40])
@pytest.mark.parametrize("n_new", [[1], [60, 0, 25, 400], [5] * 150])
def test_accept(n_new, max_path):
    g = torch.Generator().manual_seed(len(n_new) + max_path)
    parents, _ = TR.random_trees(n_new, 2, 30)
    n = sum(n_new)
    drafted = torch.randint(0, 3, (n,), generator=g, dtype=torch.int32)
    drawn = torch.randint(0, 3, (n,), generator=g, dtype=torch.int32)
    drawn[torch.rand(n, generator=g) < 0.05] = -1
    drafted[torch.rand(n, generator=g) < 0.05] = -1  # (no token: never drawn)
    p = flat(parents)
    path, accepted, ends = D.tree_accept(p, drafted.cuda(), drawn.cuda(), n_new, max_path)
    want = plain_accept(p.tolist(), drafted.tolist(), drawn.tolist(), n_new, max_path)
    assert path.tolist() == want[0] and accepted.tolist() == want[1] and ends.tolist() == want[2]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 40), ("bf16", 256)])
def test_commit_of_a_path(dtype, d):
    """The accepted rows lie behind the rows held, bit for bit, with the positions of a line; a chunk behind them attends to them."""
    c, seen = build(dtype=dtype, d=d, layers=2, q_heads=4, kv_heads=2, past=(90, 0, 33, 120), cap=300, evict_to=64)
    n_new = [25, 40, 6, 12]
    trees = TR.random_trees(n_new, 4, 9)
    q, k, v = chunk(c, n_new, 6)
    before = R.State(c, 0.05, 0.05)
    lens = [c.len(b) for b in range(4)]
    tree, _ = c.tree_plan(flat(trees[0]), n_new)
    s_new = torch.rand(sum(n_new), device="cuda")
    c.extend_attn(q, k, v, torch.empty_like(q), n_new, s_new=s_new, stage=True, tree=tree)
    paths = []
    for b, (p, dep) in enumerate(zip(*trees)):
        i, path = max(range(len(p)), key=lambda j: dep[j]), []
        while i >= 0:
            path.append(i)
            i = p[i]
        paths.append(path[::-1])
    paths[2] = []  # nothing of this sequence is taken over
    count = [len(p) for p in paths]
    path = torch.tensor([p + [-1] * (10 - len(p)) for p in paths], dtype=torch.int32, device="cuda")
    with pytest.raises(D.DyntsError) as e:
        c.extend_commit(count)  # the first rows of a tree are no path
    assert e.value.status == D.DYNTS_ERR_STATE
    c.extend_commit_path(count, path)
    c.synchronize()
    c.poll_error()
    first = 0
    for b, t in enumerate(n_new):
        assert c.len(b) == lens[b] + count[b]
        at = [first + i for i in paths[b]]
        first += t
        for l in range(2):
            for h in range(2):
                K, V, pos, score = c.export_slab(l, b, h)
                K0, V0, pos0, score0 = before.slab[l, b, h]
                kn, vn = k[l, at, h].cpu(), v[l, at, h].cpu()
                if dtype == "bf16_kv8":
                    kn, vn = R.e4m3(kn, 0.05).double() * 0.05, R.e4m3(vn, 0.05).double() * 0.05
                assert torch.equal(R.State.value(K, 0.05), torch.cat([K0, kn.double()]))
                assert torch.equal(R.State.value(V, 0.05), torch.cat([V0, vn.double()]))
                assert pos.tolist() == pos0.tolist() + list(range(seen[b], seen[b] + count[b]))
                assert torch.equal(score.double(), torch.cat([score0, s_new[at].double().cpu()]))
    seen = [s + n for s, n in zip(seen, count)]
    check(c, seen, [3, 4, 5, 1], scale=0.05, seed=9)
    with pytest.raises(D.DyntsError) as e:  # what is staged now is a line: its first rows, or a path of it
        c.extend_commit_path([4, 0, 0, 0], path)
    assert e.value.status == D.DYNTS_ERR_INVALID_ARG
    c.extend_commit_path([2, 1, 0, 1], torch.tensor([[0, 2], [3, -1], [-1, -1], [0, -1]], dtype=torch.int32, device="cuda"))
    c.synchronize()
    c.poll_error()
    assert [c.len(b) for b in range(4)] == [lens[b] + count[b] + x for b, x in enumerate([2, 1, 0, 1])]
    c.close()


@pytest.mark.parametrize("bad", [[1, 0], [0, 7], [0, 0], [-1, 2]])
def test_a_path_out_of_order_moves_nothing(bad):
    c, seen = build(past=(20, 20), cap=64)
    n_new = [7, 7]
    q, k, v = chunk(c, n_new, 6)
    c.extend_attn(q, k, v, torch.empty_like(q), n_new, stage=True)
    c.extend_commit_path([2, 2], torch.tensor([[0, 3], bad], dtype=torch.int32, device="cuda"))
    c.synchronize()
    with pytest.raises(D.DyntsError) as e:
        c.poll_error()
    assert e.value.status == D.DYNTS_ERR_DEVICE
    D.dynts_cache_refresh_lengths(c.handle)
    assert c.len(0) == 22 and c.len(1) == 20
    c.close()


# ---- windows with sinks -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64), ("bf16", 64)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (1, 64), (5, 4), (64, 3), (65, 64), (100, 65), (100, 200), (2000, 4), (30, 2 ** 31 - 1), (2 ** 31 - 1, 9), (0, 5)])
def test_sinks(dtype, d, window, sinks):
    """Chunks and single tokens; sinks that end inside a tile, meet the window, or cover everything; sequences shorter than them."""
    c, seen = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(430, 0, 61, 200, 3), cap=640)
    check(c, seen, [70, 130, 1, 0, 1], window=window, sinks=sinks, scale=0.05, seed=1)
    check(c, seen, [1, 1, 1, 1, 1], window=window, sinks=sinks, scale=0.05, seed=2)
    c.close()


def test_sinks_behind_an_eviction():
    """Positions count, not rows: sinks that an eviction has taken are gone, those it left are seen."""
    c, seen = build(q_heads=8, kv_heads=2, past=(400, 300), cap=600, evict_to=64)
    for window, sinks in ((20, 100), (200, 30), (350, 2)):
        check(c, seen, [9, 40], window=window, sinks=sinks, seed=window)
    c.close()


@pytest.mark.parametrize("opt", [dict(softcap=10.0), dict(slopes=True), dict(softcap=30.0, slopes=True)], ids=["cap", "bias", "both"])
@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_sinks_long_ragged(opt, dtype):
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = 2.0 ** (-8.0 * torch.arange(1, 15) / 14) * 0.02
    c, seen = build(dtype=dtype, q_heads=14, kv_heads=2, past=(2100, 900, 1500), cap=2400)
    check(c, seen, [17, 290, 1], window=256, sinks=20, scale=0.05, **opt)
    c.close()


def test_sinks_are_kept_by_the_rows_a_chunk_leaves():
    """Two layers, not staged: the rows stored, the lengths, and a second chunk behind them."""
    c, seen = build(layers=2, q_heads=4, kv_heads=1, past=(150, 20), cap=400)
    n_new = [60, 90]
    check(c, seen, n_new, window=33, sinks=5, stage=False, want_mass=True)
    seen = [s + t for s, t in zip(seen, n_new)]
    check(c, seen, [1, 20], window=33, sinks=5, stage=False, by_layer=True, seed=5)
    c.close()
