"""Chunks of few query rows at head_dim 128 that the cache takes over at once (one launch, scores kept outside): what they leave, growth under replay, a full sequence."""
import pytest
import torch

import paper_2601_18383_b200 as D
from tests import extend_reference as R
from tests import tree_reference as TR
from tests.test_gpu_extend import build, chunk
from tests.test_gpu_few import launches
from tests.test_gpu_speculate import BATCH, L, VOCAB, Small
from tests.test_gpu_tree import check

pytestmark = pytest.mark.gpu

SCALE = 0.05


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
# groups of 1 to 8 heads; sequences without tokens; 8, 16, 32 and 64 query rows in a cluster, and more in clusters of 32
@pytest.mark.parametrize("q_heads,new", [(2, (1, 1, 1)), (4, (9, 0, 16)), (14, (4, 1, 2)), (16, (8, 0, 7)), (2, (64, 33, 31)), (4, (64, 0, 33)), (14, (18, 3, 9)), (8, (0, 0, 30))])
@pytest.mark.parametrize("opt", [dict(), dict(window=37, sinks=6), dict(softcap=15.0, slopes=True), dict(prefix=True)], ids=["plain", "sinks", "mods", "prefix"])
def test_rows_left_and_lengths(dtype, q_heads, new, opt):
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = 2.0 ** (-8.0 * torch.arange(1, q_heads + 1) / q_heads) * 0.1
    if opt.pop("prefix", False):
        return prefixed(dtype, q_heads, list(new))
    c, seen = build(dtype=dtype, layers=2, q_heads=q_heads, kv_heads=2, past=(64, 0, 141), cap=400, evict_to=100, source="external")
    n_new = list(new)
    for seed in (1, 2):
        call = lambda: check(c, seen, n_new, seed=seed, scale=SCALE, stage=False, want_mass=False, by_layer=seed == 2, **opt)
        assert launches(c, call) == (2 if seed == 2 else 1)
        seen = [s + t for s, t in zip(seen, n_new)]
    c.close()


def prefixed(dtype, q_heads, n_new):
    c, seen = build(dtype=dtype, q_heads=q_heads, kv_heads=2, past=(64, 0, 141), cap=400, source="external")
    prefix = [t // 2 for t in n_new]
    q, k, v = chunk(c, n_new, 5)
    state = R.State(c, SCALE, SCALE) if dtype == "bf16_kv8" else R.State(c)
    ref, _, tol, _, rows = R.extend(state, seen, q, k, v, n_new, prefix=prefix, p_half_step=2.0 ** -8)
    out = torch.empty_like(q)
    assert launches(c, lambda: c.extend_attn(q, k, v, out, n_new, prefix=prefix)) == 1
    c.synchronize()
    c.poll_error()
    assert ((out.double().cpu() - ref).abs() <= tol).all()
    for (l, b, h), (K, V, pos) in rows.items():
        Kd, Vd, pd, _ = c.export_slab(l, b, h)
        assert c.len(b) == len(K) and torch.equal(R.State.value(Kd, SCALE), K) and torch.equal(R.State.value(Vd, SCALE), V) and torch.equal(pd.long(), pos)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_scores_of_the_new_rows(dtype):
    """Given, or zero; those of the rows held stay."""
    c, seen = build(dtype=dtype, layers=2, q_heads=8, kv_heads=2, past=(40, 70), cap=200, source="external")
    before = R.State(c)
    n_new = [7, 3]
    s_new = torch.rand(10, device="cuda")
    q, k, v = chunk(c, n_new, 3)
    out = torch.empty_like(q)
    assert launches(c, lambda: c.extend_attn(q, k, v, out, n_new, s_new=s_new)) == 1
    assert launches(c, lambda: c.extend_attn(q, k, v, out, n_new)) == 1
    c.synchronize()
    c.poll_error()
    for l in range(2):
        for h in range(2):
            for b, (first, t) in enumerate(((0, 7), (7, 3))):
                score = c.export_slab(l, b, h)[3].double()
                assert torch.equal(score, torch.cat([before.slab[l, b, h][3], s_new[first:first + t].double().cpu(), torch.zeros(t, dtype=torch.float64)]))
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("q_heads,n_new", [(8, [1, 1, 1]), (8, [9, 2, 0]), (16, [12, 3, 1])])  # 4, 36 (two clusters) and 96 query rows (three)
def test_a_captured_chunk_replayed_as_the_sequences_grow(dtype, q_heads, n_new):
    """The graph's one launch stores, answers and publishes, past tile borders; then one sequence is full: it stays, the others go on."""
    past, room = (30, 62, 0), 38
    cap = max(p + t * room for p, t in zip(past, n_new))
    steps = min((cap - p) // t for p, t in zip(past, n_new) if t)
    full = [b for b, (p, t) in enumerate(zip(past, n_new)) if t and p + t * (steps + 1) > cap]
    c, seen = build(dtype=dtype, q_heads=q_heads, kv_heads=2, past=past, cap=cap, source="external")
    q, k, v = chunk(c, n_new, 0)
    out = torch.empty_like(q)
    c.extend_attn(q, k, v, out, n_new, stage=True, window=40, sinks=3)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.set_stream(side)
        with torch.cuda.graph(graph, stream=side):
            count = launches(c, lambda: c.extend_attn(q, k, v, out, n_new, window=40, sinks=3))
    assert count == 1
    c.set_stream(torch.cuda.current_stream())
    D.dynts_cache_refresh_lengths(c.handle)  # (what was captured has not run)
    for step in range(steps):
        state = R.State(c, SCALE, SCALE) if dtype == "bf16_kv8" else R.State(c)
        for x, y in zip((q, k, v), chunk(c, n_new, 10 + step)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        ref, tol, *_ = TR.attend(state, [s + t * step for s, t in zip(seen, n_new)], q, k, v, n_new, None, p_half_step=2.0 ** -8, window=40, sinks=3)
        assert ((out.double().cpu() - ref).abs() <= tol).all()
        D.dynts_cache_refresh_lengths(c.handle)
        assert [c.len(b) for b in range(3)] == [p + t * (step + 1) for p, t in zip(past, n_new)]
    c.poll_error()
    held, lens, rows = out.clone(), [c.len(b) for b in range(3)], {b: c.export_slab(0, b, 1)[:3] for b in full}
    graph.replay()
    torch.cuda.synchronize()
    D.dynts_cache_refresh_lengths(c.handle)
    assert [c.len(b) for b in range(3)] == [n if b in full else n + t for b, (n, t) in enumerate(zip(lens, n_new))]
    for b in full:
        mine = slice(sum(n_new[:b]), sum(n_new[:b + 1]))
        assert torch.equal(out[:, mine], held[:, mine])
        assert all(torch.equal(x, y) for x, y in zip(rows[b], c.export_slab(0, b, 1)[:3]))
    with pytest.raises(D.DyntsError) as e:
        c.poll_error()
    assert e.value.status == D.DYNTS_ERR_DEVICE
    c.close()


def test_published_and_staged_calls_and_the_commit_of_a_part_share_a_cache():
    """Few query rows and many, staged, committed in part and published, one after another."""
    c, seen = build(layers=2, q_heads=4, kv_heads=2, past=(60, 0, 90), cap=400, source="external")
    for i, (n_new, accept) in enumerate((([5, 1, 8], [3, 0, 8]), ([80, 70, 66], [70, 1, 0]), ([2, 33, 64], [2, 30, 0]))):
        few = max(n_new) * 2 <= 128
        call = lambda: check(c, seen, n_new, seed=i, want_mass=False)  # staged
        assert (launches(c, call) == 1) == few
        c.extend_commit(accept)
        seen = [s + a for s, a in zip(seen, accept)]
        assert [c.len(b) for b in range(3)] == seen
        assert launches(c, lambda: check(c, seen, [4, 1, 1], seed=20 + i, stage=False, want_mass=False)) == 1
        seen = [s + t for s, t in zip(seen, [4, 1, 1])]
    c.close()


def test_a_model_by_staged_trees_by_steps_and_by_the_kernels_of_larger_chunks():
    """Forty tokens as one staged tree whose path is committed, as chunks of five in one launch each, and as chunks of five with the mass (storing,
    tensor-core and mass kernels): every token's logits, and those of a token behind them all."""
    model = Small(4, torch.bfloat16, 128)
    g = torch.Generator(device="cuda").manual_seed(5)
    lens = (60, 70, 50)
    prompts = torch.cat([torch.randint(0, VOCAB, (n,), generator=g, device="cuda") for n in lens])
    line = torch.randint(0, VOCAB, (BATCH, 40), generator=g, device="cuda")
    last = torch.randint(0, VOCAB, (BATCH,), generator=g, device="cuda")
    at = lambda s, t: torch.cat([n + torch.arange(s, s + t, device="cuda", dtype=torch.int32) for n in lens])
    answers = []
    for way in ("tree", "steps", "mass"):
        c = model.cache("bf16")
        if way != "mass":
            c.set_score_source(D.DYNTS_SCORE_EXTERNAL)
        model.logits(c, prompts, torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in lens]), list(lens))
        if way == "tree":
            parents = torch.arange(-1, 39, dtype=torch.int32, device="cuda").repeat(BATCH)
            tree, pos = c.tree_plan(parents, [40] * BATCH)
            assert pos.tolist() == at(0, 40).tolist()
            got = []
            assert launches(c, lambda: got.append(model.logits(c, line.reshape(-1), pos, [40] * BATCH, tree=tree, stage=True))) == L  # 80 query rows: one launch per layer
            x = got[0].view(BATCH, 40, VOCAB)
            path = torch.arange(40, dtype=torch.int32, device="cuda").repeat(BATCH, 1)
            c.extend_commit_path([40] * BATCH, path)
        else:
            parts = []
            for s in range(0, 40, 5):
                call = lambda: parts.append(model.logits(c, line[:, s:s + 5].reshape(-1), at(s, 5), [5] * BATCH).view(BATCH, 5, VOCAB))
                assert (launches(c, call) == L) == (way == "steps")
            x = torch.cat(parts, 1)
        assert [c.len(b) for b in range(BATCH)] == [n + 40 for n in lens]
        behind = model.logits(c, last, at(40, 1), [1] * BATCH)
        c.synchronize()
        c.poll_error()
        answers.append(torch.cat([x, behind.view(BATCH, 1, VOCAB)], 1))
        c.close()
    # outputs of two layers, rounded to bf16 (2^-8) from weights rounded to bf16: a few 2^-8 of a logit's size, 6
    for other in answers[1:]:
        assert (answers[0] - other).abs().max() < 16 * 2.0 ** -8 * 6
