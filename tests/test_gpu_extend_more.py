"""The chunk operators where their work is cut unusually: windows inside a seen prefix, caps that logits reach, one head over
a long cache (parts of many CTAs), group sizes that do not divide a tile, few rows of fp32 over many keys, captured
calls that outgrow their cut, and what the sums of the mass have to be.  The plain 64-bit forms and bounds are those of
the other chunk tests."""
import numpy as np
import pytest
import torch

import paper_2601_18383_b200 as D
from tests import extend_reference as R
from tests.test_gpu_extend import build, check, chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
@pytest.mark.parametrize("window,prefix", [(40, (0, 250, 200)), (1, (3, 300, 260)), (130, (3, 299, 64))])
def test_a_window_inside_a_prefix(dtype, d, window, prefix):
    """The first tokens of a prefix see none of its last rows: what they see lies tiles before the newest."""
    c, seen = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(150, 0, 77), cap=512, evict_to=100)
    check(c, seen, [3, 300, 260], scale=0.05, seed=11, window=window, prefix=list(prefix))
    c.close()


def test_a_window_inside_a_prefix_over_many_parts():
    c, seen = build(q_heads=2, kv_heads=1, past=(900,), cap=3000)
    check(c, seen, [1800], seed=12, window=200, prefix=[1700])
    c.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
@pytest.mark.parametrize("softcap,sharp", [(0.5, 4.0), (3.0, 2.0), (1000.0, 1.0)])
def test_caps_that_logits_reach_and_do_not_reach(dtype, d, softcap, sharp):
    c, seen = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(300, 10), cap=512)
    check(c, seen, [70, 5], scale=0.05, seed=13, sharp=sharp, softcap=softcap)
    c.close()


@pytest.mark.parametrize("q_heads,kv_heads", [(5, 1), (12, 2), (7, 1), (1, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
def test_group_sizes(dtype, q_heads, kv_heads):
    c, seen = build(dtype=dtype, q_heads=q_heads, kv_heads=kv_heads, past=(100, 0, 513), cap=640)
    check(c, seen, [67, 30, 2], scale=0.05, seed=14)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("new", [1, 9])
def test_one_head_over_a_long_cache(dtype, new):
    """An item in more parts than a warp has lanes."""
    c, seen = build(dtype=dtype, q_heads=4, kv_heads=1, past=(20011,), cap=20064)
    check(c, seen, [new], scale=0.05, seed=15)
    c.close()


@pytest.mark.parametrize("dtype,d", [("fp32", 64), ("fp32", 256), ("fp32", 8), ("bf16", 40), ("bf16_kv8", 32)])
@pytest.mark.parametrize("past,new", [((500,), (3,)), ((33, 0), (1, 2)), ((900, 40, 260), (40, 1, 0))])
@pytest.mark.parametrize("opt", [dict(), dict(window=70)], ids=["plain", "window"])
def test_few_rows_over_many_keys(dtype, d, past, new, opt):
    """By FMA: the key tiles of an item dealt to a cluster, some CTAs of which see nothing."""
    c, seen = build(dtype=dtype, d=d, q_heads=4, kv_heads=1, past=past, cap=1024)
    check(c, seen, list(new), scale=0.05, seed=16, **opt)
    c.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
def test_the_mass_of_a_chunk_adds_up(dtype, d):
    """Every query gives away a mass of one.  A query's weights sum to one up to the error of its log-sum-exp (2^-20: a
    logarithm of a sum, in base 2, off by two steps of values below 16) and of each exponential (two steps and a rounding of
    an argument below 32: 2^-19 ln 2); so does the total."""
    c, seen = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(2000, 700), cap=2432)
    n_new = [150, 300]
    q, k, v = chunk(c, n_new, 17)
    mass = torch.zeros((1, 2, 2, c.capacity), device="cuda")
    c.extend_attn(q, k, v, torch.empty_like(q), n_new, mass=mass, stage=True)
    c.synchronize()
    c.poll_error()
    for b in range(2):
        want = n_new[b] * 4
        assert ((mass[0, b].double().sum(-1) - want).abs() <= want * (2.0 ** -20 + 2.0 ** -19)).all()
    c.close()


def test_masked_tokens_with_eight_bit_rows():
    """A NaN is stored as a code; what is hidden behind the causal border changes nothing."""
    c, seen = build(dtype="bf16_kv8", q_heads=8, kv_heads=2, past=(30,), cap=256)
    q, k, v = chunk(c, [80], 3)
    good, out = torch.empty_like(q), torch.empty_like(q)
    c.extend_attn(q, k, v, good, [80], stage=True)
    v2, k2 = v.clone(), k.clone()
    v2[0, 41, 1, 5] = float("nan")
    k2[0, 70, 0, 3] = float("nan")
    c.extend_attn(q, k2, v2, out, [80], stage=True)
    c.synchronize()
    c.poll_error()
    x, y = out[0, :41, 4:], good[0, :41, 4:]
    rest = torch.arange(128, device="cuda") != 5
    assert torch.equal(x[..., rest], y[..., rest]) and torch.equal(out[0, :70, :4], good[0, :70, :4])
    # (two ways to round the weights and the output, as for 16-bit rows: at most 3 * 2^-8 * max |v| apart)
    assert ((x - y).float().abs() <= 3 * 2.0 ** -8 * v.float().abs().max()).all()
    assert torch.isnan(out[0, 41:, 4:, 5].float()).all() and torch.isnan(out[0, 70:, :4].float()).all()
    c.close()


def test_a_captured_chunk_outgrows_its_cut():
    """A captured call whose sequences grow at replay until the mass items are more than the scratch has room for parts of."""
    new = [64] * 16
    kw = dict(q_heads=16, kv_heads=8, past=(10,) * 16, cap=768, source="external")
    a, _ = build(**kw)
    b, _ = build(**kw)
    q, k, v = chunk(a, new, 18)
    out, ref = torch.empty_like(q), torch.empty_like(q)
    ma, mb = (torch.zeros((1, 16, 8, 768), device="cuda") for _ in range(2))
    a.extend_attn(q, k, v, out, new, mass=ma)
    b.extend_attn(q, k, v, ref, new, mass=mb)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        a.set_stream(side)
        with torch.cuda.graph(g, stream=side):
            a.extend_attn(q, k, v, out, new, mass=ma)
    a.set_stream(torch.cuda.current_stream())
    a.refresh_lengths()
    vmax = float(v.float().abs().max()) + 4.0
    for step in range(10):
        g.replay()
        b.extend_attn(q, k, v, ref, new, mass=mb)
        torch.cuda.synchronize()
        # (each side rounds its weights and its output: half a step of at most max |v| each)
        assert ((out - ref).float().abs() <= 4 * 2.0 ** -8 * vmax).all(), step
        # (weights within 4e-4 of their value on either side, as for single tokens)
        assert ((ma - mb).abs() <= 8e-4 * mb).all(), step
    a.poll_error()
    a.refresh_lengths()
    assert a.len(0) == b.len(0) == 10 + 64 * 11
    a.close(), b.close()


def test_counts_as_arrays():
    c, seen = build(q_heads=8, kv_heads=2, past=(60, 5), cap=128)
    q, k, v = chunk(c, [4, 1], 7)
    outs = []
    for n in ([4, 1], (4, 1), np.array([4, 1], dtype=np.int32), np.array([4, 1]), torch.tensor([4, 1], dtype=torch.int32)):
        outs.append(torch.empty_like(q))
        c.extend_attn(q, k, v, outs[-1], n, stage=True)
    c.synchronize()
    assert all(torch.equal(outs[0], o) for o in outs[1:])
    for n in (torch.tensor([4, 1]), torch.tensor([[4], [1]], dtype=torch.int32), torch.tensor([4, 1], dtype=torch.int32, device="cuda")):
        with pytest.raises(D.DyntsError) as e:
            c.extend_attn(q, k, v, outs[0], n, stage=True)
        assert e.value.status == D.DYNTS_ERR_INVALID_ARG
    c.close()


def test_one_scratch_grows_with_the_calls():
    """Small and large calls in turn, eager, on one cache: the scratch of an earlier call may still be in use."""
    c, seen = build(q_heads=8, kv_heads=2, past=(300,), cap=1024)
    outs = []
    for rep in range(2):
        for t in (1, 700, 40, 300):
            q, k, v = chunk(c, [t], t)
            outs.append(torch.empty_like(q))
            c.extend_attn(q, k, v, outs[-1], [t], stage=True)
    c.synchronize()
    c.poll_error()
    assert all(torch.equal(x, y) for x, y in zip(outs[:4], outs[4:]))
    c.close()


def test_scratch_of_another_stream_than_the_current():
    """The cache works on a stream of its own while the current one is busy with memory it has given back."""
    ref, _ = build(q_heads=8, kv_heads=2, past=(300,), cap=1024)
    q, k, v = chunk(ref, [700], 19)
    want, out = torch.empty_like(q), torch.empty_like(q)
    ref.extend_attn(q, k, v, want, [700], stage=True)
    c, _ = build(q_heads=8, kv_heads=2, past=(300,), cap=1024)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c.set_stream(side)
    x = torch.ones((4096, 4096), device="cuda")
    for _ in range(20):
        x = (x @ x).clamp(max=1.0)                                   # keeps the current stream busy ...
    for n in (1 << 22, 1 << 23, 1 << 24):
        y = torch.empty(n, dtype=torch.uint8, device="cuda")
        y.fill_(255)                                                 # ... with writes to blocks it gives back at once
        del y
    c.extend_attn(q, k, v, out, [700], stage=True)
    torch.cuda.synchronize()
    c.poll_error()
    assert torch.equal(out, want)
    c.close(), ref.close()


@pytest.mark.parametrize("d,rot,stride", [(10, 6, 25), (6, 2, 13), (130, 66, 131 * 2 + 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_of_odd_strides(d, rot, stride, dtype, adjacent):
    from tests.test_gpu_rope import plain, tolerance
    n, heads = 37, 2
    base = torch.randn(n * stride + d, device="cuda").to(dtype)
    q = torch.as_strided(base, (n, heads, d), (stride, d, 1))
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 977
    out, _ = D.rope(q, None, pos, theta=5e3, rot_dim=rot, adjacent=adjacent)
    want, raw = plain(q, pos[None], 5e3, [rot // 2], rot, adjacent, False)
    assert ((out.double().cpu() - want).abs() <= tolerance(want, raw, dtype)).all()
    assert torch.equal(out[..., rot:], q[..., rot:])


def test_the_sections_say_how_much_turns():
    q = torch.randn((50, 3, 128), device="cuda")
    pos = torch.arange(100, device="cuda", dtype=torch.int32).view(2, 50)
    a, _ = D.rope(q, None, pos, sections=[20, 12])
    b, _ = D.rope(q, None, pos, sections=[20, 12], rot_dim=64)
    assert torch.equal(a, b) and torch.equal(a[..., 64:], q[..., 64:]) and not torch.equal(a[..., 32:64], q[..., 32:64])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
def test_the_first_call_is_captured(dtype, d):
    """Nothing has run on the cache before the capture: the scratch is taken within it and serves eager calls afterwards."""
    a, _ = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(200, 30), cap=512, source="external")
    b, _ = build(dtype=dtype, d=d, q_heads=8, kv_heads=2, past=(200, 30), cap=512, source="external")
    q, k, v = chunk(a, [20, 3], 21)
    out, want, mass, mass_b = torch.empty_like(q), torch.empty_like(q), *(torch.zeros((1, 2, 2, a.capacity), device="cuda") for _ in range(2))
    b.extend_attn(q, k, v, want, [20, 3], mass=mass_b, stage=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        a.set_stream(side)
        with torch.cuda.graph(g, stream=side):
            a.extend_attn(q, k, v, out, [20, 3], mass=mass, stage=True)
    for _ in range(3):
        out.zero_()
        mass.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(mass, mass_b)
    a.set_stream(torch.cuda.current_stream())
    a.extend_attn(q, k, v, out.zero_(), [20, 3], mass=mass.zero_(), stage=True)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(mass, mass_b)
    a.poll_error()
    del g
    a.close(), b.close()
