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


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("cap", [1e5, 1e8, 1e20])
@pytest.mark.parametrize("q_heads,new", [(2, (1, 2)), (8, (4, 1)), (8, (6, 2)), (16, (7, 3)), (16, (14, 9))])  # groups of warps for 8, 16, 32 and 64 rows, and parts
def test_a_cap_far_above_the_logits_is_none(dtype, cap, q_heads, new):
    """c tanh(z / c) is z to within z^3 / 3 c^2, at most 2e-7 of it here: the plain form without a cap is the answer."""
    scale = 0.05
    c = D.Cache(1, 2, q_heads, 2, 128, 320, 0, 1, dtype=dtype, capacity=320)
    if dtype == "bf16_kv8":
        c.set_kv_scale(scale, scale)
    c.set_score_source(D.DYNTS_SCORE_EXTERNAL)
    g = torch.Generator(device="cuda").manual_seed(len(new) + q_heads)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    for b, n in enumerate((200, 77)):
        c.prefill_seq(b, normal(1, 2, n, 128), normal(1, 2, n, 128), n_pinned=0)
    c.synchronize()
    T = sum(new)
    q, k, v = 2 * normal(1, T, q_heads, 128), normal(1, T, 2, 128), normal(1, T, 2, 128)
    state = R.State(c, scale, scale) if dtype == "bf16_kv8" else R.State(c)
    ref, tol, *_ = TR.attend(state, [200, 77], q, k, v, new, None, p_half_step=2.0 ** -8)
    out = torch.empty_like(q)
    assert launches(c, lambda: c.extend_attn(q, k, v, out, list(new), stage=True, softcap=cap)) == 1
    c.synchronize()
    c.poll_error()
    assert ((out.double().cpu() - ref).abs() <= tol).all()
    c.close()
