"""The chunk operators at the borders of what they accept: replayed calls that no longer fit, biases beside rows that lie far
back, windows as wide as an int, logits of minus infinity, old keys far above the newest, slopes below zero, calls back to
back, and the fp32 form at head_dim 128.  Plain 64-bit forms; bounds derived beside each test."""
import math

import pytest
import torch

import paper_2601_18383_b200 as D
from tests import extend_reference as R
from tests.test_gpu_extend import build, check, chunk

pytestmark = pytest.mark.gpu

TYPES = [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)]
SCALE = 0.05                                                         # of the 8-bit rows that `build` makes


def captured(c, call):
    """A graph of `call` on a side stream; the cache is back on the current stream, its lengths are the device's."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        c.set_stream(side)
        with torch.cuda.graph(g, stream=side):
            call()
    c.set_stream(torch.cuda.current_stream())
    c.refresh_lengths()
    return g


@pytest.mark.parametrize("by_layer", [False, True], ids=["one call", "by layers"])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_replayed_chunk_that_does_not_fit(dtype, d, by_layer):
    """The first sequence's chunk no longer fits at the second replay: it keeps its rows, scores and length, its outputs and
    mass are not written, the status says so, and the other sequence's chunk is what it would have been."""
    kw = dict(dtype=dtype, d=d, layers=2, q_heads=8, kv_heads=2, past=(60, 5), cap=64)
    a, _ = build(**kw)
    b, _ = build(**kw)
    q, k, v = chunk(a, [2, 1], 7)
    out, ref = torch.empty_like(q), torch.empty_like(q)
    ma, mb = (torch.full((2, 2, 2, 64), -3.0, device="cuda") for _ in range(2))

    def run(c, o, m):
        if by_layer:
            for l in range(2):
                c.extend_attn_layer(l, q[l], k[l], v[l], o[l], [2, 1], mass=m)
        else:
            c.extend_attn(q, k, v, o, [2, 1], mass=m)

    run(a, out, ma), run(b, ref, mb)
    g = captured(a, lambda: run(a, out, ma))
    g.replay()
    run(b, ref, mb)
    a.refresh_lengths()
    a.poll_error()
    assert a.len(0) == b.len(0) == 64 and a.len(1) == b.len(1) == 7
    before = R.State(a).slab
    out.fill_(7.0), ma.fill_(-3.0), mb.fill_(-3.0)
    torch.cuda.synchronize()
    g.replay()
    one = lambda x: x[:, 2:].contiguous()
    ref1 = torch.empty_like(one(q))
    b.extend_attn(one(q), one(k), one(v), ref1, [0, 1], mass=mb)
    torch.cuda.synchronize()
    with pytest.raises(D.DyntsError) as e:
        a.poll_error()
    assert e.value.status == D.DYNTS_ERR_DEVICE
    a.refresh_lengths()
    assert a.len(0) == 64 and a.len(1) == b.len(1) == 8
    after, want = R.State(a).slab, R.State(b).slab
    for l in range(2):
        for h in range(2):
            assert all(torch.equal(x, y) for x, y in zip(before[l, 0, h], after[l, 0, h]))
            x, y = after[l, 1, h], want[l, 1, h]
            assert all(torch.equal(x[i], y[i]) for i in range(3))
            # (weights within 4e-4 of their value on either side: sum |q||k| < 128, as for captured chunks elsewhere)
            assert ((x[3] - y[3]).abs() <= 8e-4 * y[3]).all()
    assert (out[:, :2] == 7.0).all() and (ma[:, 0] == -3.0).all()
    assert ((ma[:, 1] - mb[:, 1]).abs() <= 8e-4 * mb[:, 1].abs()).all()
    # (each side rounds its weights and its output: half a step of at most max |v| each)
    vmax = max(float(want[l, 1, h][1].abs().max()) for l in range(2) for h in range(2))
    assert ((out[:, 2:].float() - ref1.float()).abs() <= 4 * R.EPS[out.dtype] * vmax * (64 if dtype == "fp32" else 1)).all()
    a.close(), b.close()


@pytest.mark.parametrize("far", [100_000, 1_000_000])
@pytest.mark.parametrize("n,new,prefix", [(30, 5, 0), (30, 5, 3), (30, 90, 0), (66, 1, 0), (66, 40, 7), (104, 5, 0)])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_bias_beside_rows_that_lie_far_back(dtype, d, n, new, prefix, far):
    """Four rows from the beginning beside recent ones.  The bias of a recent row is small, and so has its rounding to be:
    every logit's error is weighed with its weight, not with that of the farthest row."""
    heads, kv_heads = 8, 2
    c, _ = build(dtype=dtype, d=d, q_heads=heads, kv_heads=kv_heads, past=(n,), cap=256)
    G = heads // kv_heads
    pos = torch.cat([torch.arange(4), far + torch.arange(n - 4)]).to(torch.int32)
    for h in range(kv_heads):
        K, V, _, score = c.export_slab(0, 0, h)
        c.import_slab(0, 0, h, K, V, pos, score, 0)
    tot = far + n - 4
    q, k, v = chunk(c, [new], 3)
    slopes = 2.0 ** -torch.arange(1, heads + 1).float()
    state = R.State(c, SCALE, SCALE)
    out, mass = torch.empty_like(q), torch.zeros((1, 1, kv_heads, c.capacity), device="cuda")
    c.extend_attn(q, k, v, out, [new], mass=mass, slopes=slopes.cuda(), prefix=[prefix] if prefix else None, stage=True)
    c.synchronize()
    c.poll_error()
    i, j = torch.arange(new)[:, None], torch.arange(n + new)[None, :]
    visible = (j <= n + i) | (j < n + prefix)
    p_all = torch.cat([pos.long(), tot + torch.arange(new)])
    apart = (p_all[n:, None] - p_all[None, :]).abs().double()
    for h in range(kv_heads):
        K, V, _, _ = state.slab[0, 0, h]
        kn, vn = k[0, :, h].cpu(), v[0, :, h].cpu()
        if dtype == "bf16_kv8":
            kn, vn = R.e4m3(kn, SCALE).double() * SCALE, R.e4m3(vn, SCALE).double() * SCALE
        K, V = torch.cat([K, kn.double()]), torch.cat([V, vn.double()])
        m, mt = torch.zeros(n + new, dtype=torch.float64), torch.zeros(n + new, dtype=torch.float64)
        for x in range(h * G, (h + 1) * G):
            qx = q[0, :, x].cpu().double()
            raw = qx @ K.T / math.sqrt(d)
            z = raw - float(slopes[x]) * apart
            # a dot product's error as in the shared reference; the bias and the logit a few half steps of themselves, the bias
            # of a tile of 64 rows counted from any row of it
            dz = (d + 8) * 2.0 ** -23 * (qx.abs() @ K.abs().T) / math.sqrt(d) + 8 * 2.0 ** -24 * (raw.abs() + z.abs() + float(slopes[x]) * (apart + 64))
            p = torch.softmax(z.masked_fill(~visible, -math.inf), -1)
            dz = dz.masked_fill(~visible, 0.0)
            err = p * (dz + (p * dz).sum(-1, keepdim=True) + 132 * 2.0 ** -23) * 1.01       # its own logit, the sum's, exponentials
            m += p.sum(0)
            mt += err.sum(0)
            o = p @ V
            half = 0.0 if dtype == "fp32" else 2.0 ** -8
            tol = err @ V.abs() + (half + (n + new) / 8 * 2.0 ** -23) * (p @ V.abs()) * 1.01 + R.EPS[q.dtype] * o.abs() * 1.01 + 1e-30
            off = (out[0, :, x].double().cpu() - o).abs()
            assert (off <= tol).all(), f"outputs: {(off / tol).max():.3g} of the bound"
        off, tol = (mass[0, 0, h, : n + new].double().cpu() - m).abs(), mt + (new * G + 8) * 2.0 ** -24 * m + 1e-30
        assert (off <= tol).all(), f"mass: {(off / tol).max():.3g} of the bound"
    c.close()


@pytest.mark.parametrize("q_heads,kv_heads", [(2, 2), (8, 2), (14, 2)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 100])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_windows_as_wide_as_an_int(dtype, d, window, q_heads, kv_heads):
    """2^31 - 1 stands for no window: rows of any distance are seen, and receive their mass."""
    c, seen = build(dtype=dtype, d=d, q_heads=q_heads, kv_heads=kv_heads, past=(150, 0, 333), cap=512, evict_to=200)
    check(c, seen, [70, 33, 1], scale=SCALE, seed=23, window=window)
    c.close()


def test_windows_beyond_an_int_are_refused():
    c, _ = build(q_heads=8, kv_heads=2, past=(60,), cap=128)
    q, k, v = chunk(c, [4], 7)
    for bad in (dict(window=2 ** 31), dict(window=2 ** 32 + 5), dict(prefix=[2 ** 32 + 2])):
        with pytest.raises(D.DyntsError) as e:
            c.extend_attn(q, k, v, torch.empty_like(q), [4], stage=True, **bad)
        assert e.value.status == D.DYNTS_ERR_INVALID_ARG
    c.close()


def test_sections_beyond_an_int_are_refused():
    q = torch.randn((3, 2, 128), device="cuda")
    pos = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    for bad in (dict(sections=[2 ** 32 + 20, 12], rot_dim=64), dict(sections=[2 ** 32 + 20, 12]), dict(sections=[20, 12], rot_dim=2 ** 32 + 64), dict(sections=[-20, 52])):
        with pytest.raises(D.DyntsError) as e:
            D.rope(q, None, pos, **bad)
        assert e.value.status == D.DYNTS_ERR_INVALID_ARG


def plain(state, q, k, v, n, dtype, kv_heads):
    """Outputs of one sequence of one layer in 64 bits, causal: [t, Hq, d]."""
    t, hq, d = q.shape
    G = hq // kv_heads
    i, j = torch.arange(t)[:, None], torch.arange(n + t)[None, :]
    out = torch.empty((t, hq, d), dtype=torch.float64)
    for h in range(kv_heads):
        kn, vn = k[:, h].cpu(), v[:, h].cpu()
        if dtype == "bf16_kv8":
            kn, vn = R.e4m3(kn, SCALE).double() * SCALE, R.e4m3(vn, SCALE).double() * SCALE
        K, V = state.slab[0, 0, h][:2] if n else (torch.zeros((0, d), dtype=torch.float64),) * 2
        K, V = torch.cat([K, kn.double()]), torch.cat([V, vn.double()])
        for x in range(h * G, (h + 1) * G):
            z = (q[:, x].cpu().double() @ K.T / math.sqrt(d)).masked_fill(j > n + i, -math.inf)
            out[:, x] = torch.softmax(z, -1) @ V
    return out


@pytest.mark.parametrize("past,low", [(0, [0]), (40, list(range(40))), (140, list(range(140))), (140, list(range(70, 140))), (2000, list(range(1900))),
                                      (2000, list(range(2000)))])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64), ("bf16", 64)])
def test_logits_of_minus_infinity(dtype, d, past, low):
    """Rows whose key makes every logit -inf (an infinite element against queries of one sign) weigh nothing, whole tiles of
    them too; a token that sees nothing else has no answer: NaN, as its definition has."""
    q_heads, kv_heads, t = 8, 2, 5
    c, _ = build(dtype=dtype, d=d, q_heads=q_heads, kv_heads=kv_heads, past=(past,), cap=max(64, past + 32))
    q, k, v = chunk(c, [t], 29)
    q[..., 3] = -q[..., 3].abs() - 0.5
    if past == 0:
        k[0, 0, :, 3] = math.inf                                     # the first token sees only itself
    else:
        if len(low) == past:
            k[0, :2, :, 3] = math.inf                                # the first two tokens see only such rows
        for h in range(kv_heads):
            K, V, pos, score = c.export_slab(0, 0, h)
            K[low, 3] = math.inf
            c.import_slab(0, 0, h, K, V, pos, score, 0)
    state = R.State(c)
    out = torch.empty_like(q)
    mass = torch.zeros((1, 1, kv_heads, c.capacity), device="cuda")
    c.extend_attn(q, k, v, out, [t], mass=mass, stage=True)
    c.synchronize()
    c.poll_error()
    want, got = plain(state, q[0], k[0], v[0], past, dtype, kv_heads), out[0].double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert fine.any() and (past == 0 or len(low) < past or torch.isnan(want).any())
    # logits off by less than 1e-3 (sum |q||k| < 64 among the finite), weights and outputs rounded: half a step of at most max |v|
    vmax = float(max(v.float().abs().max(), max((s[1].abs().max() for s in state.slab.values() if s[1].numel()), default=0.0)))
    assert ((got - want)[fine].abs() <= (2e-3 + 2 * R.EPS[torch.float32 if dtype == "fp32" else torch.bfloat16]) * vmax).all()
    m = mass[0, 0, 0, : past + t].cpu()
    if past and len(low) < past:
        assert (m[low] == 0).all() and abs(float(m.double().sum()) - t * q_heads // kv_heads) < 1e-3
    elif past:
        assert torch.isnan(m[:past]).all() and torch.isfinite(m[past + 2:]).all()
    else:
        assert torch.isfinite(m[1:]).all()
    c.close()


@pytest.mark.parametrize("past,new", [(2000, 5), (300, 150), (0, 40)], ids=["parts", "more parts", "whole"])
@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_key_that_is_not_a_number(dtype, d, past, new):
    """The tokens that see it have no answer, and nor has the mass of any row they see; the other head keeps its own."""
    at = 3
    c, _ = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(past,), cap=past + new + 20)
    q, k, v = chunk(c, [new], 43)
    out, want = torch.empty_like(q), torch.empty_like(q)
    mass, other = (torch.full((1, 1, 2, c.capacity), -3.0, device="cuda") for _ in range(2))
    c.extend_attn(q, k, v, want, [new], mass=other, stage=True)
    k[0, at, 1, 5] = math.nan
    c.extend_attn(q, k, v, out, [new], mass=mass, stage=True)
    c.synchronize()
    c.poll_error()
    G = 4
    assert torch.equal(out[:, :, :G], want[:, :, :G]) and torch.equal(mass[0, 0, 0], other[0, 0, 0])
    assert torch.equal(out[:, :at, G:], want[:, :at, G:]) and torch.isnan(out[:, at:, G:].float()).all()
    assert torch.isnan(mass[0, 0, 1, : past + new]).all() and (mass[0, 0, 1, past + new:] == -3.0).all()
    c.close()


@pytest.mark.parametrize("dtype,scale", [("bf16", 1.0), ("bf16_kv8", 0.5)])
@pytest.mark.parametrize("past,new,opt", [((2000,), (8,), {}), ((700,), (300,), {}), ((380,) * 33, (20,) * 33, {}), ((900, 300), (40, 1), dict(softcap=1000.0))],
                         ids=["parts", "long", "whole items", "capped"])
def test_old_keys_far_above_the_newest(dtype, scale, past, new, opt):
    """The oldest rows' logits lie hundreds above all newer ones for every query: no reference taken from the newest rows
    holds, every row's answer is finite."""
    c, seen = build(dtype=dtype, q_heads=8, kv_heads=2, past=past, cap=max(p + t for p, t in zip(past, new)) + 20, scale=scale)
    g = torch.Generator(device="cuda").manual_seed(31)
    for b, n in enumerate(past):
        k, v = (torch.randn((1, 2, n, 128), generator=g, device="cuda") for _ in range(2))
        k[:, :, :64] *= 40.0
        c.prefill_seq(b, k.to(torch.bfloat16), v.to(torch.bfloat16), n_pinned=0)
    check(c, list(seen), list(new), scale=scale, seed=31, sharp=2.0, **opt)
    c.close()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("past,new", [((1500,), (30,)), ((64, 0, 500), (7, 120, 1))])
def test_slopes_below_zero(dtype, d, past, new):
    """A bias that grows with the distance: every row's largest logit is its oldest."""
    c, seen = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=past, cap=1600)
    check(c, seen, list(new), scale=SCALE, seed=33, slopes=-2.0 ** -torch.arange(0, 8).float())
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_waits_outlast_rows_computed_again(dtype):
    """Every row is computed again, which takes milliseconds, while the other warps of its CTA may poll a few thousand times."""
    c, seen = build(dtype=dtype, q_heads=8, kv_heads=2, past=(6000,), cap=6400)
    c.set_wait_limit(4096)
    n_new = [300]
    q, k, v = chunk(c, n_new, 37)
    slopes = -2.0 ** -torch.arange(0, 8, device="cuda").float()
    out, again = torch.empty_like(q), torch.empty_like(q)
    c.extend_attn(q, k, v, out, n_new, slopes=slopes, stage=True)
    c.synchronize()
    c.poll_error()
    c.set_wait_limit(1 << 22)
    c.extend_attn(q, k, v, again, n_new, slopes=slopes, stage=True)
    c.synchronize()
    c.poll_error()
    assert torch.isfinite(out.float()).all() and torch.equal(out, again)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16_kv8", "bf16"])
def test_calls_back_to_back_with_other_rows(dtype):
    """Staged calls that overwrite one another's rows, nothing between them, equal the same calls each waited for."""
    n_new = [30, 5, 0, 64]
    kw = dict(dtype=dtype, q_heads=8, kv_heads=2, past=(200, 63, 7, 500), cap=640)
    a, _ = build(**kw)
    b, _ = build(**kw)
    data = [chunk(a, n_new, 40 + i) for i in range(12)]
    res = []
    for c, wait in ((a, False), (b, True)):
        outs = [torch.empty_like(q) for q, _, _ in data]
        mass = [torch.zeros((1, 4, 2, 640), device="cuda") for _ in data]
        torch.cuda.synchronize()
        for (q, k, v), o, m in zip(data, outs, mass):
            c.extend_attn(q, k, v, o, n_new, mass=m, stage=True)
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        c.poll_error()
        res.append((outs, mass))
    for x, y in zip(res[0][0] + res[0][1], res[1][0] + res[1][1]):
        assert torch.equal(x, y)
    a.close(), b.close()


@pytest.mark.parametrize("opt", [dict(), dict(softcap=20.0, slopes=True, window=120, prefix=[3, 50, 0])], ids=["plain", "options"])
@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_the_fp32_form_at_head_dim_128(dtype, opt):
    """Launch variant 1: nothing but the output is rounded to 16 bits."""
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = 2.0 ** -torch.arange(1, 9).float()
    c, seen = build(dtype=dtype, q_heads=8, kv_heads=2, past=(150, 0, 333), cap=512, evict_to=200)
    c.set_launch(0, 1)
    n_new = [6, 90, 33]
    q, k, v = chunk(c, n_new, 35)
    s = SCALE if dtype == "bf16_kv8" else 1.0
    ref, mass, tol, mass_tol, rows = R.extend(R.State(c, s, s), seen, q, k, v, n_new, **opt)
    lens = [c.len(b) for b in range(3)]
    if "slopes" in opt:
        opt["slopes"] = opt["slopes"].cuda()
    out, buf = torch.empty_like(q), torch.zeros((1, 3, 2, 512), device="cuda")
    c.extend_attn(q, k, v, out, n_new, mass=buf, **opt)
    c.synchronize()
    c.poll_error()
    assert ((out.double().cpu() - ref).abs() <= tol).all()
    for (l, b, h), m in mass.items():
        assert ((buf[l, b, h, : lens[b] + n_new[b]].double().cpu() - m).abs() <= mass_tol[l, b, h]).all()
        K, V, pos, _ = c.export_slab(l, b, h)
        assert torch.equal(R.State.value(K, s), rows[l, b, h][0]) and torch.equal(R.State.value(V, s), rows[l, b, h][1])
    c.close()


def test_scales_between_a_staged_chunk_and_its_commit():
    """Rows staged into an empty cache are codes of the scales then set: other scales later forget them; within a chunk that goes
    layer by layer the scales stay."""
    c, _ = build(dtype="bf16_kv8", layers=2, q_heads=8, kv_heads=2, past=(0, 0), cap=64)
    q, k, v = chunk(c, [5, 2], 7)
    out = torch.empty_like(q)
    c.extend_attn(q, k, v, out, [5, 2], stage=True)
    c.set_kv_scale(0.25, 0.25)
    with pytest.raises(D.DyntsError) as e:
        c.extend_commit([5, 2])
    assert e.value.status == D.DYNTS_ERR_STATE and c.len(0) == 0
    c.extend_attn_layer(0, q[0], k[0], v[0], out[0], [5, 2])
    with pytest.raises(D.DyntsError) as e:
        c.set_kv_scale(0.05, 0.05)
    assert e.value.status == D.DYNTS_ERR_STATE
    c.extend_attn_layer(1, q[1], k[1], v[1], out[1], [5, 2])
    for l in range(2):
        K, V, _, _ = c.export_slab(l, 0, 1)
        assert torch.equal(K.view(torch.float8_e4m3fn).float(), R.e4m3(k[l, :5, 1].cpu(), 0.25).float())
    c.close()
