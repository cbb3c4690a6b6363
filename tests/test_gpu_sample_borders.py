"""Sampling where a border is hard to find: fewer tokens than top_k, masks, logits and temperatures at the ends of fp32; against the plain 64-bit form."""
import math

import pytest
import torch

import paper_2601_18383_b200 as D
from tests.test_gpu_sample import check, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 20, 60, 160])  # clusters of eight, four, two CTAs, and single ones
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_fewer_tokens_than_top_k_with_top_p(n, dtype):
    """The histogram of the tokens finds no border, and that of the weights follows at once: the same answer each time."""
    V = 20011
    for finite, where, top_k in ((1200, "spread", 1500), (300, "run", 500), (1100, "run", 5000)):
        x, u = logits(n, V, dtype, finite + n)
        g = torch.Generator(device="cuda").manual_seed(n)
        keep = torch.zeros((n, V), dtype=torch.bool, device="cuda")
        if where == "spread":
            keep.scatter_(1, torch.rand((n, V), generator=g, device="cuda").topk(finite, 1).indices, True)
        else:
            keep[:, 7000:7000 + finite] = True
        x = torch.where(keep, x, torch.full_like(x, -math.inf))
        check(x, u, 0.9, top_k, 0.8)
        first = D.sample(x, u, 1.1, top_k, 0.9, 0.01)
        for _ in range(20):
            again = D.sample(x, u, 1.1, top_k, 0.9, 0.01)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("temperature", [1e37, 1e38, 3e38])
def test_logits_further_apart_than_the_largest_number(temperature):
    """The distance of two fp32 logits overflows; borders by counts of tokens lie on either side of where it does."""
    for n, V in ((3, 5003), (90, 5003), (2, 40009)):
        g = torch.Generator(device="cuda").manual_seed(V + n)
        x = (torch.rand((n, V), generator=g, device="cuda") * 2 - 1) * 3.3e38
        u = torch.rand((n,), generator=g, device="cuda")
        for top_k in (20, 1100, V // 2, V - 1000, V - 3):
            check(x, u, temperature, top_k)
            check(x, u, temperature, top_k, 0.7)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(2, 30011), (100, 9001)])
def test_rows_masked_with_the_lowest_value(dtype, n, V):
    """All but some tokens of a row, whole runs of it, every other one: -inf and the lowest finite value give the same answers."""
    x, u = logits(n, V, dtype, V)
    g = torch.Generator(device="cuda").manual_seed(1)
    masks = [torch.rand((n, V), generator=g, device="cuda") < p for p in (0.99, 0.5)] + [torch.arange(V, device="cuda").expand(n, V) % 2 == 0, torch.arange(V, device="cuda").expand(n, V) > 700]
    for mask in masks:
        low, none = (torch.where(mask, torch.full_like(x, f), x) for f in (torch.finfo(dtype).min, -math.inf))
        for s in (dict(temperature=0.0), dict(temperature=0.7, top_k=50, top_p=0.9), dict(top_k=600), dict(top_k=1500, top_p=0.99), dict(temperature=30.0, top_k=3000), dict(top_p=0.8)):
            a, b = D.sample(low, u, **s), D.sample(none, u, **s)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        check(low[:2], u[:2], 0.7, 50, 0.9)
        check(low[:2], u[:2], 1.0, 1500, 0.99)


def test_the_largest_temperatures():
    """A finite temperature is taken at its value up to the largest number; an infinite one of an array as that."""
    most = torch.finfo(torch.float32).max
    g = torch.Generator(device="cuda").manual_seed(4)
    x = (torch.rand((5, 3001), generator=g, device="cuda") * 2 - 1) * 3.3e38
    u = torch.rand((5,), generator=g, device="cuda")
    for s in (dict(), dict(top_p=0.3), dict(top_k=1200, top_p=0.6), dict(min_p=0.5), dict(top_k=40)):
        check(x, u, most, **s)
        check(x, u, 3.2e38, **s)
        a, b = D.sample(x, u, torch.full((5,), math.inf, device="cuda"), **s), D.sample(x, u, most, **s)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
