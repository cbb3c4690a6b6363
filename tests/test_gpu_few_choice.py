"""Which chunks of few query rows go by one launch: few slabs and long ones do, batches of short sequences whose CTAs would take many waves do not."""
import pytest
import torch

import paper_2601_18383_b200 as D
from tests.test_gpu_few import launches

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("batch,held,new,one", [(1, 2048, 5, True), (1, 2048, 25, True), (64, 1500, 1, True), (8, 1000, 8, True),
                                                (33, 48, 32, False), (64, 16, 32, False), (33, 112, 24, False), (64, 48, 24, False)])
def test_launches(dtype, batch, held, new, one):
    cap = (held + new + 31) // 32 * 32
    c = D.Cache(1, batch, 32, 8, 128, cap, 0, 1, dtype=dtype, capacity=cap)
    c.set_score_source(D.DYNTS_SCORE_EXTERNAL)
    K = torch.randn((1, batch, 8, held, 128), device="cuda").bfloat16()
    c.prefill(K, K, n_pinned=0)
    q, k = (torch.randn((1, batch * new, h, 128), device="cuda").bfloat16() for h in (32, 8))
    out = torch.empty_like(q)
    assert (launches(c, lambda: c.extend_attn(q, k, k, out, [new] * batch, stage=True)) == 1) == one
    c.synchronize()
    c.poll_error()
    c.close()
