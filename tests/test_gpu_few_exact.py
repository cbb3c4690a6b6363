"""Chunks of few query rows at head_dim 128 where their arithmetic is hardest: against the plain 64-bit form, and never further off than the kernels of larger chunks may be."""
import math

import pytest
import torch

import paper_2601_18383_b200 as D
from tests import extend_reference as R
from tests import tree_reference as TR
from tests.test_gpu_few import launches

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("gap", [8.0, 14.0, 17.0])
@pytest.mark.parametrize("new", [1, 4, 13, 30])
@pytest.mark.parametrize("n", [90, 240, 5000])
def test_small_weights_beside_a_large_one(dtype, gap, new, n):
    """Row 0 takes most of the weight and has the value 0; the answer is what the rows of about e^-gap of its weight give.  (Every warp weighs its
    rows against the largest it has met: in one CTA per slab a quarter of the rows or more are beside row 0.)"""
    scale, G = 0.05, 2
    cap = (n + new + 31) // 32 * 32
    c = D.Cache(1, 1, G, 1, 128, cap, 0, 1, dtype=dtype, capacity=cap)
    if dtype == "bf16_kv8":
        c.set_kv_scale(scale, scale)
    c.set_score_source(D.DYNTS_SCORE_EXTERNAL)
    g = torch.Generator(device="cuda").manual_seed(new)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    u = normal(128)
    u = u / u.norm()
    K, V = 0.2 * normal(1, 1, 1, n, 128), 1.0 + 0.5 * normal(1, 1, 1, n, 128)  # (values of one sign: errors of one sign do not cancel)
    K[0, 0, 0, 0], V[0, 0, 0, 0] = 8.0 * u, 0.0
    q = (gap * math.sqrt(128) / 8.0 * u).expand(1, new, G, 128) + 0.1 * normal(1, new, G, 128)
    k, v = 0.2 * normal(1, new, 1, 128), 1.0 + 0.5 * normal(1, new, 1, 128)
    q, k, v, K, V = (x.bfloat16().contiguous() for x in (q, k, v, K, V))
    c.prefill_seq(0, K[:, 0], V[:, 0], n_pinned=0)
    c.synchronize()
    state = R.State(c, scale, scale) if dtype == "bf16_kv8" else R.State(c)
    # weights rounded to 16 bits of 8 significant ones at the worst
    ref, tol, *_ = TR.attend(state, [n], q, k, v, [new], None, p_half_step=2.0 ** -8)
    out = torch.empty_like(q)
    assert launches(c, lambda: c.extend_attn(q, k, v, out, [new], stage=True)) == 1
    c.synchronize()
    c.poll_error()
    assert ((out.double().cpu() - ref).abs() <= tol).all()
    c.close()
