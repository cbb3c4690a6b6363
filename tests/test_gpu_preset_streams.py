"""PresetRun.extend while its cache works on another stream than the current one, which is busy: the pieces it copies, the chunk
calls and what comes back are in order by themselves."""
import pytest
import torch

from paper_2601_18383_b200 import presets as P
from tests import extend_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["dynts", "t_bottom"])
def test_pieces_on_a_stream_of_the_caches_own(name):
    L, Nb, Hq, Hkv, d, T = 2, 2, 8, 2, 128, 150
    g = torch.Generator(device="cuda").manual_seed(5)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    preset = P.make(name, budget=64, window=8, ratio=0.4, prompt=12)
    kp, vp = mk(L, Nb, Hkv, 20, d), mk(L, Nb, Hkv, 20, d)
    q, k, v = mk(L, Nb, T, Hq, d), mk(L, Nb, T, Hkv, d), mk(L, Nb, T, Hkv, d)
    s = torch.rand((Nb, T), generator=g, device="cuda")
    a, b = (P.PresetRun(preset, L, Nb, Hq, Hkv, d) for _ in range(2))
    for run in (a, b):
        run.prefill(kp, vp)
    want = torch.empty_like(q)
    b.extend(q, k, v, want, predictor_scores=s)
    x = torch.ones((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a.cache.set_stream(side)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    for _ in range(30):
        x = (x @ x).clamp(max=1.0)                                   # the current stream is busy; what is queued there comes late
    a.extend(q, k, v, out, predictor_scores=s)
    got = out.clone()                                                # on the current stream, as a caller reads it
    torch.cuda.synchronize()
    for run in (a, b):
        run.cache.poll_error()
    assert torch.equal(got, want)
    assert a.events == b.events > 1
    x, y = R.State(a.cache).slab, R.State(b.cache).slab
    assert all(torch.equal(m, n) for key in x for m, n in zip(x[key], y[key]))
    a.close(), b.close()
