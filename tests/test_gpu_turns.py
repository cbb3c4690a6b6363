"""The chunk operators as they are used together: a conversation whose turns are rotated (dynts_rope), attended and scored
(dynts_extend_attn), cut by evictions, with drafted tokens staged and in part taken over, and decode steps in between; and
the presets' extend beside as many of their steps."""
import pytest
import torch

import paper_2601_18383_b200 as D
from paper_2601_18383_b200 import presets as P
from tests import extend_reference as R
from tests.test_gpu_rope import plain, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16_kv8", 128), ("fp32", 64)])
def test_a_conversation(dtype, d):
    L, Nb, Hq, Hkv, theta = 2, 2, 8, 2, 1e4
    c = D.Cache(L, Nb, Hq, Hkv, d, 64, 8, 1, dtype=dtype, capacity=256)
    scale = 1.0
    if dtype == "bf16_kv8":
        scale = 0.05
        c.set_kv_scale(scale, scale)
    g = torch.Generator(device="cuda").manual_seed(5)
    seen = [0, 0]

    def turned(n_new):
        """q, k, v of a chunk for all layers, q and k rotated by the library at the sequences' positions."""
        T = sum(n_new)
        pos = torch.cat([seen[b] + torch.arange(n_new[b]) for b in range(Nb)]).to(torch.int32).cuda()
        mk = lambda heads: torch.randn((L, T, heads, d), generator=g, device="cuda").to(c.torch_dtype)
        q, k, v = mk(Hq), mk(Hkv), mk(Hkv)
        for l in range(L):
            a, b = D.rope(q[l], k[l], pos, theta=theta)
            for x, y in ((q[l], a), (k[l], b)):
                want, raw = plain(x, pos[None], theta, [d // 2], d, False, False)
                assert ((y.double().cpu() - want).abs() <= tolerance(want, raw, x.dtype)).all()
            D.rope(q[l], k[l], pos, q[l], k[l], theta=theta)          # in place
            assert torch.equal(q[l], a) and torch.equal(k[l], b)
        return q, k, v

    def attended(n_new, q, k, v, out, mass=None):
        half = 0.0 if dtype == "fp32" else 2.0 ** -8
        ref, m, tol, mtol, rows = R.extend(R.State(c, scale, scale), seen, q, k, v, n_new, p_half_step=half)

        def compare():
            c.synchronize()
            c.poll_error()
            assert ((out.double().cpu() - ref).abs() <= tol).all()
            if mass is not None:
                for key, want in m.items():
                    assert ((mass[key][: want.shape[0]].double().cpu() - want).abs() <= mtol[key]).all()
            return m, mtol, rows
        return compare

    # the first question and a text behind it, ragged; by layers, as in a model
    mass = torch.zeros((L, Nb, Hkv, c.capacity), device="cuda")
    for n_new in ([90, 33], [41, 70]):
        q, k, v = turned(n_new)
        out = torch.empty_like(q)
        done = attended(n_new, q, k, v, out, mass)
        old = c.scores_tensor().double().cpu().clone()
        for l in range(L):
            c.extend_attn_layer(l, q[l], k[l], v[l], out[l], n_new, mass=mass)
        m, mtol, rows = done()
        for (l, b, h), want in m.items():
            n = want.shape[0] - n_new[b]
            had = torch.cat([old[l, b, h, :n], torch.zeros(n_new[b], dtype=torch.float64)])
            got = c.scores_tensor()[l, b, h, : want.shape[0]].double().cpu()
            assert ((got - had - want).abs() <= mtol[l, b, h] + 2.0 ** -23 * (had + want)).all()
        seen = [s + t for s, t in zip(seen, n_new)]
    # an eviction by those scores: the window and the best of the others, as the oracle's rule has it
    before = R.State(c).slab
    c.evict(64)
    for key, (K, V, pos, score) in R.State(c).slab.items():
        old = before[key]
        n = old[2].shape[0]
        order = sorted(range(n - 8), key=lambda j: (-float(old[3][j]), j))[: 64 - 8]
        keep = sorted(order) + list(range(n - 8, n))
        assert torch.equal(pos, old[2][keep]) and torch.equal(K, old[0][keep]) and torch.equal(V, old[1][keep])
    # drafted tokens: looked at, in part taken over
    q, k, v = turned([5, 4])
    out = torch.empty_like(q)
    done = attended([5, 4], q, k, v, out)
    c.extend_attn(q, k, v, out, [5, 4], stage=True)
    done()
    c.extend_commit([3, 0])
    seen[0] += 3
    assert [c.len(0), c.len(1)] == [67, 64]
    # a decode step, which is a chunk of one token
    q, k, v = turned([1, 1])
    out = torch.empty_like(q)
    done = attended([1, 1], q, k, v, out)
    c.decode_attn(q.view(L, Nb, Hq, d), k.view(L, Nb, Hkv, d), v.view(L, Nb, Hkv, d), out.view(L, Nb, Hq, d))
    _, _, rows = done()
    for (l, b, h), (K, V, pos) in rows.items():
        Kd, Vd, pd, _ = c.export_slab(l, b, h)
        assert torch.equal(R.State.value(Kd, scale), K) and torch.equal(R.State.value(Vd, scale), V) and torch.equal(pd.long(), pos)
    c.close()


@pytest.mark.parametrize("name", ["dynts", "streaming", "t_bottom"])
@pytest.mark.parametrize("T", [7, 90])
def test_a_preset_extends_as_it_steps(name, T):
    """Rows, positions, scores and events of T steps; outputs within the two kernels' roundings."""
    L, Nb, Hq, Hkv, d = 2, 2, 8, 2, 128
    g = torch.Generator(device="cuda").manual_seed(T)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    preset = P.make(name, budget=64, window=8, ratio=0.4, prompt=12)
    kp, vp = mk(L, Nb, Hkv, 20, d), mk(L, Nb, Hkv, 20, d)
    q, k, v = mk(L, Nb, T, Hq, d), mk(L, Nb, T, Hkv, d), mk(L, Nb, T, Hkv, d)
    s = torch.rand((Nb, T), generator=g, device="cuda")
    a, b = (P.PresetRun(preset, L, Nb, Hq, Hkv, d) for _ in range(2))
    for run in (a, b):
        run.prefill(kp, vp)
    out, want = torch.empty_like(q), torch.empty_like(q)
    a.extend(q, k, v, out, predictor_scores=s)
    o = torch.empty((L, Nb, Hq, d), dtype=torch.bfloat16, device="cuda")
    for i in range(T):
        b.step(*(x[:, :, i].contiguous() for x in (q, k, v)), o, predictor_scores=s[:, i].contiguous())
        want[:, :, i] = o
    for run in (a, b):
        run.cache.synchronize()
        run.cache.poll_error()
    assert a.events == b.events and [a.cache.len(x) for x in range(Nb)] == [b.cache.len(x) for x in range(Nb)]
    # each side rounds its weights and its output: two half steps each of values up to the largest |v|
    assert (out.double() - want.double()).abs().max() <= 4 * 2.0 ** -8 * float(max(v.abs().max(), vp.abs().max()))
    for l in range(L):
        for x in range(Nb):
            for h in range(Hkv):
                assert all(torch.equal(y, z) for y, z in zip(a.cache.export_slab(l, x, h), b.cache.export_slab(l, x, h)))
    a.close(), b.close()
