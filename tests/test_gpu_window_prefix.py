"""Windows beside a prefix that all tokens see, by the tensor-core kernels: borders on both sides of a token, narrow windows and wide ones."""
import pytest
import torch

from tests.test_gpu_extend import build, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("window", [1, 31, 64, 65, 100, 200, 257, 300, 1000])
@pytest.mark.parametrize("past,new,prefix", [((0,), (300,), (300,)), ((130, 0, 64), (200, 150, 260), (200, 40, 129)), ((61, 700), (270, 190), (1, 190)), ((40, 90), (150, 300), (0, 64))])
def test_window_and_prefix(dtype, window, past, new, prefix):
    c, seen = build(dtype=dtype, q_heads=8, kv_heads=2, past=past, cap=1000, source="external")
    check(c, seen, list(new), window=window, prefix=list(prefix), scale=0.05, want_mass=False, seed=window)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "bf16_kv8"])
@pytest.mark.parametrize("window", [64, 200, 257])
def test_window_and_prefix_behind_an_eviction(dtype, window):
    """Positions held with gaps: rows far back, then recent ones."""
    c, seen = build(dtype=dtype, q_heads=14, kv_heads=2, past=(500, 330), cap=700, evict_to=200, source="external")
    check(c, seen, [150, 90], window=window, prefix=[70, 90], scale=0.05, want_mass=False)
    c.close()
