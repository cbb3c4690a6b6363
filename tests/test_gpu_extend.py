"""A chunk of new tokens against the cache (dynts_extend_attn): outputs, stored rows, lengths, scores and
mass against plain 64-bit forms, for every type of row, ragged lengths, rows that lost others to an eviction,
and every option."""
import math

import numpy as np
import pytest
import torch

import paper_2601_18383_b200 as D
from tests import extend_reference as R

pytestmark = pytest.mark.gpu


def make(dtype="bf16", layers=1, q_heads=8, kv_heads=2, d=128, past=(40,), cap=256, evict_to=None, window=8, seed=0, source="attention",
         scale=0.05):
    """A cache with past[b] rows per sequence (evict_to: cut to that many, at random, the positions keep their gaps)."""
    batch = len(past)
    c = D.Cache(layers, batch, q_heads, kv_heads, d, min(cap, 64 if evict_to is None else max(evict_to, 1)), min(window, 8), 1, dtype=dtype,
                capacity=cap)
    c.set_score_source(D.DYNTS_SCORE_ATTENTION if source == "attention" else D.DYNTS_SCORE_EXTERNAL)
    if dtype == "bf16_kv8":
        c.set_kv_scale(scale, scale)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    for b, n in enumerate(past):
        if n:
            k = torch.randn((layers, kv_heads, n, d), generator=g, device="cuda").to(c.torch_dtype)
            v = torch.randn((layers, kv_heads, n, d), generator=g, device="cuda").to(c.torch_dtype)
            c.prefill_seq(b, k, v, n_pinned=0)
    seen = list(past)
    if evict_to is not None:
        sc = c.scores_tensor()
        sc.copy_(torch.rand(sc.shape, generator=g, device="cuda"))
        c.evict(evict_to)
    return c, seen


def chunk(c, n_new, seed=0, sharp=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    T = sum(n_new)
    mk = lambda heads, a=1.0: (a * torch.randn((c.layers, T, heads, c.head_dim), generator=g, device="cuda")).to(c.torch_dtype)
    return mk(c.q_heads, sharp), mk(c.kv_heads), mk(c.kv_heads)


def check(c, seen, n_new, seed=0, by_layer=False, stage=False, want_mass=True, sharp=1.0, scale=1.0, **opt):
    kv8 = c.dtype_name == "bf16_kv8"
    q, k, v = chunk(c, n_new, seed, sharp)
    state = R.State(c, scale if kv8 else 1.0, scale if kv8 else 1.0)
    lens = [c.len(b) for b in range(c.batch)]
    # the weights a tensor-core kernel multiplies are rounded to 16 bits (bf16; f16 beside 8-bit rows)
    half = 0.0 if c.torch_dtype == torch.float32 or c.head_dim != 128 else 2.0 ** -8
    prefix = opt.get("prefix")
    ref, mass, tol, mass_tol, rows = R.extend(state, seen, q, k, v, n_new, p_half_step=half, **opt)
    T = sum(n_new)
    out = torch.full((c.layers, T + 2, c.q_heads, c.head_dim), 7.0, dtype=c.torch_dtype, device="cuda")
    flat = torch.full((c.layers * T + 2, c.q_heads, c.head_dim), 7.0, dtype=c.torch_dtype, device="cuda")
    out = flat[: c.layers * T].view(c.layers, T, c.q_heads, c.head_dim)
    buf = torch.full((c.layers, c.batch, c.kv_heads, c.capacity), -3.0, device="cuda") if want_mass else None
    old = c.scores_tensor().clone()
    dev_opt = dict(opt)
    if opt.get("slopes") is not None:
        dev_opt["slopes"] = opt["slopes"].cuda()
    if by_layer:
        for l in range(c.layers):
            c.extend_attn_layer(l, q[l], k[l], v[l], out[l], n_new, mass=buf, stage=stage, **dev_opt)
    else:
        c.extend_attn(q, k, v, out, n_new, mass=buf, stage=stage, **dev_opt)
    c.synchronize()
    c.poll_error()
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    bad = (got - ref).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outputs off, worst {((got - ref).abs() / tol).max():.3g} of the bound"
    assert (flat[c.layers * T:] == 7.0).all()                      # nothing behind the last token
    accumulate = not stage and c._source == "attention"
    for (l, b, h), (K, V, pos) in rows.items():
        t, n = int(n_new[b]), lens[b]
        if want_mass:
            m = buf[l, b, h].double().cpu()
            assert (m[n + t if t else 0:] == -3.0).all()
            if t:
                x = (m[: n + t] - mass[l, b, h]).abs()
                assert (x <= mass_tol[l, b, h]).all(), f"mass off by {(x / mass_tol[l, b, h]).max():.3g} of the bound"
        if stage:
            assert c.len(b) == n
            continue
        assert c.len(b) == n + t
        Kd, Vd, pd, sd = c.export_slab(l, b, h)
        assert torch.equal(R.State.value(Kd, scale), K) and torch.equal(R.State.value(Vd, scale), V)
        assert torch.equal(pd.long(), pos)
        s0 = torch.cat([state.slab[l, b, h][3], torch.zeros(t, dtype=torch.float64)])
        if accumulate and t:
            want = s0 + mass[l, b, h]
            assert ((sd.double() - want).abs() <= mass_tol[l, b, h] + 2.0 ** -23 * want.abs()).all()
        else:
            assert torch.equal(sd.double(), s0)
    if stage:
        assert torch.equal(torch.stack([c.scores_tensor()[:, b, :, : lens[b]].sum() for b in range(c.batch)]),
                           torch.stack([old[:, b, :, : lens[b]].sum() for b in range(c.batch)]))
    return q, k, v, out, buf


def build(source="attention", **kw):
    c, seen = make(source=source, **kw)
    c._source = source
    return c, seen


SHAPES = [  # q_heads, kv_heads: groups of 4, 7, 1, 8, 3
    (8, 2), (14, 2), (2, 2), (8, 1), (3, 1)]


@pytest.mark.parametrize("q_heads,kv_heads", SHAPES)
@pytest.mark.parametrize("past,new", [((0,), (1,)), ((1,), (1,)), ((63,), (1,)), ((64,), (64,)), ((65,), (130,)), ((200,), (5,)), ((0,), (129,))])
def test_bf16_one_sequence(q_heads, kv_heads, past, new):
    c, seen = build(q_heads=q_heads, kv_heads=kv_heads, past=past, cap=384)
    check(c, seen, list(new))
    c.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64), ("fp32", 40), ("fp32", 128), ("bf16", 64), ("bf16", 8),
                                     ("bf16", 256), ("bf16_kv8", 48)])
@pytest.mark.parametrize("source", ["attention", "external"])
def test_ragged_batch_of_every_type(dtype, d, source):
    """Sequences without rows, without new tokens, cut by an eviction; two layers in one call, then layer by layer."""
    c, seen = build(dtype=dtype, d=d, layers=2, q_heads=6, kv_heads=2, past=(90, 0, 33, 120, 7), cap=300, evict_to=64, source=source)
    assert c.len(0) == 64 and c.len(3) == 64
    n_new = [5, 70, 0, 1, 33]
    check(c, seen, n_new, scale=0.05, seed=3)
    seen = [s + t for s, t in zip(seen, n_new)]
    n_new = [1, 1, 2, 130, 0]
    check(c, seen, n_new, by_layer=True, scale=0.05, seed=4)
    c.close()


OPTIONS = [dict(softcap=20.0), dict(slopes=True), dict(window=1), dict(window=40), dict(prefix=(0, 60, 17)), dict(softcap=5.0, slopes=True, window=90, prefix=(3, 100, 0))]


@pytest.mark.parametrize("opt", OPTIONS, ids=[",".join(o) + str(o.get("window", "")) for o in OPTIONS])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
def test_options(dtype, d, opt):
    opt = dict(opt)
    heads = 8
    if opt.get("slopes"):
        opt["slopes"] = 2.0 ** -torch.arange(1, heads + 1).float()
    c, seen = build(dtype=dtype, d=d, q_heads=heads, kv_heads=2, past=(150, 0, 77), cap=330, evict_to=100)
    n_new = [3, 140, 60]
    if "prefix" in opt:
        opt["prefix"] = list(opt["prefix"])
    check(c, seen, n_new, scale=0.05, seed=9, sharp=2.0, **opt)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("past,new", [((1500, 2050, 700), (1, 1, 1)), ((2000,), (12,)), ((1025, 1900), (300, 17))])
def test_long_caches(dtype, past, new):
    c, seen = build(dtype=dtype, q_heads=14, kv_heads=2, past=past, cap=2304)
    check(c, seen, list(new), scale=0.05, seed=5, sharp=1.5)
    c.close()


@pytest.mark.parametrize("opt", [dict(window=300), dict(softcap=30.0, window=1000), dict(slopes=True)], ids=["window", "cap+window", "bias"])
def test_long_caches_with_options(opt):
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = 2.0 ** -torch.arange(1, 9).float()
    c, seen = build(q_heads=8, kv_heads=2, past=(1700, 2000, 0), cap=2304, evict_to=1500)
    check(c, seen, [1, 130, 500], seed=6, **opt)
    c.close()


def test_logits_that_keep_growing():
    """The running maximum moves in every tile, by far more than any slack a kernel may allow its reference."""
    c, seen = build(q_heads=4, kv_heads=1, past=(300,), cap=512)
    K, V, pos, score = c.export_slab(0, 0, 0)
    K = (K.float() * (1.0 + torch.arange(300) / 24.0)[:, None]).to(torch.bfloat16)
    c.import_slab(0, 0, 0, K, V, pos, score, 0)
    check(c, seen, [100], seed=8, sharp=2.0)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_rows_behind_the_end_do_not_matter(dtype):
    """NaN and infinities in rows that the sequence has lost, behind its end and inside the last tile."""
    c, seen = build(dtype=dtype, q_heads=8, kv_heads=2, past=(190,), cap=256, evict_to=70)
    bad = torch.full((1, 2, 190, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    keep = [c.export_slab(0, 0, h) for h in range(2)]
    bad[..., ::3, :] = float("inf")
    c.prefill_seq(0, bad, bad, n_pinned=0)
    for h in range(2):
        c.import_slab(0, 0, h, *keep[h], 0)
    seen = [int(keep[0][2][-1]) + 1]
    check(c, seen, [5], scale=0.05)
    c.close()


def test_masked_tokens_of_the_chunk_do_not_matter():
    """A later token whose v is not finite leaves the earlier tokens' outputs alone, in the same tile too."""
    c, seen = build(q_heads=8, kv_heads=2, past=(30,), cap=256)
    q, k, v = chunk(c, [80], 3)
    good = torch.empty_like(q)
    c.extend_attn(q, k, v, good, [80], stage=True)
    v2, k2 = v.clone(), k.clone()
    v2[0, 41, 1, 5] = float("nan")
    v2[0, 60, 0, 9] = float("inf")
    k2[0, 70, 0, 3] = float("nan")
    out = torch.empty_like(q)
    c.extend_attn(q, k2, v2, out, [80], stage=True)
    c.synchronize()
    c.poll_error()
    # The columns without such a value keep every bit.  In the others a kernel may compute an element a second way: one
    # way rounds the weights (half a step of bf16, 2^-8) and the output (another), the other at least the output, so the
    # two are at most 3 * 2^-8 * max |v| apart (an output is a mean of v's with weights that sum to one).
    for heads, col, upto in ((slice(0, 4), 9, 60), (slice(4, 8), 5, 41)):
        x, y = out[0, :upto, heads], good[0, :upto, heads]
        rest = torch.arange(128, device="cuda") != col
        assert torch.equal(x[..., rest], y[..., rest])
        assert ((x - y).float().abs() <= 3 * 2.0 ** -8 * v.float().abs().max()).all()
    assert torch.isnan(out[0, 41:, 4:, 5].float()).all() and not torch.isfinite(out[0, 60:70, :4, 9].float()).any()
    assert torch.isnan(out[0, 70:, :4].float()).all()
    c.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
def test_a_chunk_is_as_many_decode_steps(dtype, d):
    """Rows and positions equal bit for bit; outputs and scores within the two kernels' roundings."""
    kw = dict(dtype=dtype, d=d, layers=2, q_heads=8, kv_heads=2, past=(50, 100), cap=200, evict_to=64)
    a, _ = build(**kw)
    b, _ = build(**kw)
    T = 9
    q, k, v = chunk(a, [T, T], 2)
    out = torch.empty_like(q)
    a.extend_attn(q, k, v, out, [T, T])
    o = torch.empty((2, 2, 8, d), dtype=a.torch_dtype, device="cuda")
    steps = []
    for i in range(T):
        pick = lambda x: x.view(2, 2, T, -1, d)[:, :, i].contiguous()
        b.decode_attn(pick(q), pick(k), pick(v), o)
        steps.append(o.clone())
    a.synchronize(), b.synchronize()
    a.poll_error(), b.poll_error()
    want = torch.stack(steps, 2).reshape(2, 2 * T, 8, d).double()
    # each side rounds its weights and its output: two half steps each of values up to the row's largest |v| (< 6)
    assert (out.double() - want).abs().max() <= 4 * R.EPS[a.torch_dtype] * 6 * (1 if dtype != "fp32" else 64)
    for l in range(2):
        for s in range(2):
            for h in range(2):
                x, y = a.export_slab(l, s, h), b.export_slab(l, s, h)
                assert all(torch.equal(x[i], y[i]) for i in range(3))
                assert (x[3] - y[3]).abs().max() <= 1e-4
    a.close(), b.close()


def test_stage_and_commit():
    """Drafted tokens: staged, a part accepted; the cache then equals one that was extended by that part."""
    kw = dict(layers=2, q_heads=8, kv_heads=2, past=(70, 20), cap=128, source="external")
    a, seen = build(**kw)
    b, _ = build(**kw)
    q, k, v, out, _ = check(a, seen, [6, 4], stage=True)
    s_new = torch.rand(10, device="cuda")
    a.extend_attn(q, k, v, out, [6, 4], stage=True, s_new=s_new)
    with pytest.raises(D.DyntsError) as e:
        a.extend_commit([7, 0])
    assert e.value.status == D.DYNTS_ERR_INVALID_ARG
    a.extend_commit([3, 0])
    with pytest.raises(D.DyntsError) as e:
        a.extend_commit([0, 0])                                     # once
    assert e.value.status == D.DYNTS_ERR_STATE
    part = lambda x: x[:, :3].contiguous()
    b.extend_attn(part(q), part(k), part(v), torch.empty_like(part(q)), [3, 0], s_new=s_new[:3].contiguous())
    assert [a.len(0), a.len(1)] == [73, 20] == [b.len(0), b.len(1)]
    for l in range(2):
        for s in range(2):
            for h in range(2):
                assert all(torch.equal(x, y) for x, y in zip(a.export_slab(l, s, h), b.export_slab(l, s, h)))
    # a decode step behind the staged rows overwrites them: nothing left to commit
    a.extend_attn(q, k, v, out, [6, 4], stage=True)
    o = torch.empty((2, 2, 8, 128), dtype=torch.bfloat16, device="cuda")
    a.decode_attn(o.normal_(), torch.randn((2, 2, 2, 128), device="cuda").to(torch.bfloat16), torch.randn((2, 2, 2, 128), device="cuda").to(torch.bfloat16), torch.empty_like(o))
    with pytest.raises(D.DyntsError) as e:
        a.extend_commit([1, 1])
    assert e.value.status == D.DYNTS_ERR_STATE
    a.close(), b.close()


def test_scores_of_the_new_rows_and_a_following_eviction():
    """+inf keeps a question's rows; the eviction ranks the others by what was given."""
    c, seen = build(q_heads=4, kv_heads=1, past=(20,), cap=128, source="external")
    q, k, v = chunk(c, [30], 1)
    s_new = torch.rand(30, device="cuda")
    s_new[4:14] = float("inf")
    c.extend_attn(q, k, v, torch.empty_like(q), [30], s_new=s_new)
    c.evict(24)                                                      # 8 of the window, 10 pinned by their score, 6 by rank
    _, _, pos, score = c.export_slab(0, 0, 0)
    s = torch.cat([torch.zeros(20), s_new.cpu()])
    rest = [j for j in range(42) if not 24 <= j < 34]
    best = sorted(sorted(rest, key=lambda j: (-float(s[j]), j))[:6])
    assert pos.tolist() == sorted(best + list(range(24, 34)) + list(range(42, 50)))
    c.close()


def test_strided_queries_keys_and_values():
    """q, k, v as slices of one fused projection."""
    c, seen = build(q_heads=8, kv_heads=2, past=(70, 3), cap=200, source="external")
    n_new = [40, 31]
    q, k, v = chunk(c, n_new, 4)
    out, out2 = torch.empty_like(q), torch.empty_like(q)
    c.extend_attn(q, k, v, out, n_new, stage=True)
    fused = torch.cat([q[0].reshape(71, -1), k[0].reshape(71, -1), v[0].reshape(71, -1)], 1).contiguous()
    qs, ks, vs = (x.unflatten(1, (-1, 128)) for x in fused.split([1024, 256, 256], 1))
    assert not qs.is_contiguous()
    c.extend_attn_layer(0, qs, ks, vs, out2[0], n_new, stage=True)
    c.synchronize()
    c.poll_error()
    assert torch.equal(out, out2)
    c.close()


def test_more_sequences_than_one_launch_takes():
    past, new = tuple(i % 5 for i in range(150)), [(i * 7) % 4 for i in range(150)]
    c, seen = build(q_heads=4, kv_heads=1, past=past, cap=64)
    check(c, list(seen), new)
    c.close()


def test_captured_chunks_follow_the_lengths():
    """A captured single-token call, replayed: the rows held are read at replay."""
    a, _ = build(q_heads=8, kv_heads=2, past=(60, 5), cap=256)
    b, _ = build(q_heads=8, kv_heads=2, past=(60, 5), cap=256)
    q, k, v = chunk(a, [1, 1], 7)
    out, ref = torch.empty_like(q), torch.empty_like(q)
    run = lambda c, o: c.extend_attn(q, k, v, o, [1, 1], softcap=10.0, window=50)
    run(a, out), run(b, ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        a.set_stream(side)
        with torch.cuda.graph(g, stream=side):
            run(a, out)
    a.set_stream(torch.cuda.current_stream())
    a.refresh_lengths()
    # A capture keeps the cut of the key rows that its lengths suggested, an eager call cuts by the present ones, so the
    # two may round differently: each rounds its weights (half a step of bf16, 2^-8, of at most max |v| in all: the weights
    # sum to one) and its output (the same), so they are at most 4 * 2^-8 * max |v| apart.
    vmax = max(float(a.export_slab(0, s, h)[1].float().abs().max()) for s in range(2) for h in range(2))
    vmax = max(vmax, float(v.float().abs().max()))
    for step in range(70):                                         # across a tile's border
        g.replay()
        run(b, ref)
        torch.cuda.synchronize()
        assert ((out - ref).float().abs() <= 4 * 2.0 ** -8 * vmax).all(), step
    a.refresh_lengths()
    assert a.len(0) == b.len(0) == 131
    for h in range(2):
        x, y = a.export_slab(0, 0, h), b.export_slab(0, 0, h)
        assert all(torch.equal(x[i], y[i]) for i in range(3))
        # each weight within 2 dz + 132 * 2^-23 of its value on either side, dz = (d + 8) 2^-23 sum |q||k| / sqrt(d) with
        # sum |q||k| < 128 (normal values): 2 * 1.9e-4 + 1.6e-5 < 4e-4, so the sums are within 8e-4 of each other
        assert ((x[3] - y[3]).abs() <= 8e-4 * y[3]).all()
    a.poll_error()
    a.close(), b.close()


def test_two_caches_on_two_streams():
    ref = None
    caches = [build(q_heads=8, kv_heads=2, past=(500,), cap=640) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    q, k, v = chunk(caches[0][0], [100], 7)
    outs = [torch.empty_like(q) for _ in range(2)]
    torch.cuda.synchronize()
    for (c, _), st in zip(caches, streams):
        c.set_stream(st)
    for _ in range(5):
        for (c, _), st, o in zip(caches, streams, outs):
            with torch.cuda.stream(st):
                c.extend_attn(q, k, v, o, [100], stage=True)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.isfinite(outs[0].float()).all()
    for c, _ in caches:
        c.poll_error()
        c.close()


def test_refusals_leave_the_cache_unchanged():
    c, seen = build(q_heads=8, kv_heads=2, past=(60, 5), cap=64, layers=2)
    q, k, v = chunk(c, [4, 1], 7)
    out = torch.empty_like(q)
    before = R.State(c).slab

    def refused(status, fn):
        with pytest.raises(D.DyntsError) as e:
            fn()
        assert e.value.status == status, e.value

    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q, k, v, out, [5, 1]))                 # does not add up
    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q.float(), k, v, out, [4, 1]))
    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q, k[..., :64], v, out, [4, 1]))
    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q.cpu(), k, v, out, [4, 1]))
    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q, k, v, out, [4, 1], window=-1))
    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q, k, v, out, [4, 1], softcap=float("nan")))
    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q, k, v, out, [4, 1], prefix=[5, 0]))
    refused(D.DYNTS_ERR_INVALID_ARG, lambda: c.extend_attn(q, k, v, out, [4, 1], mass=torch.zeros(3, device="cuda")))
    big = lambda x: torch.cat([x, x[:, :1]], 1).contiguous()
    refused(D.DYNTS_ERR_CAPACITY, lambda: c.extend_attn(big(q), big(k), big(v), big(out), [5, 1]))
    refused(D.DYNTS_ERR_STATE, lambda: c.extend_commit([0, 0]))
    refused(D.DYNTS_ERR_STATE, lambda: c.extend_attn_layer(1, q[1], k[1], v[1], out[1], [4, 1]))
    c.extend_attn_layer(0, q[0], k[0], v[0], out[0], [4, 1])
    refused(D.DYNTS_ERR_STATE, lambda: c.extend_attn(q, k, v, out, [4, 1]))
    refused(D.DYNTS_ERR_STATE, lambda: c.extend_attn_layer(1, q[1, :, :, :], k[1], v[1], out[1], [3, 2]))
    o = torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    refused(D.DYNTS_ERR_STATE, lambda: c.decode_attn_layer(1, o, o[:, :2].contiguous(), o[:, :2].contiguous(), torch.empty_like(o)))
    assert c.len(0) == 60
    c.extend_attn_layer(1, q[1], k[1], v[1], out[1], [4, 1])
    assert c.len(0) == 64 and c.len(1) == 6
    after = R.State(c).slab
    for s in before:
        n = before[s][0].shape[0]
        assert all(torch.equal(after[s][i][:n], before[s][i]) for i in range(3))
    c.decode_attn_layer
    c.close()


def test_a_reset_sequence_begins_with_its_chunk():
    c, seen = build(q_heads=8, kv_heads=2, past=(60, 30), cap=128)
    c.seq_reset(1)
    check(c, [60, 0], [0, 33])
    check(c, [60, 33], [4, 1], seed=2)
    c.close()
