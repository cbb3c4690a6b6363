"""Sampling (dynts_sample) against the plain 64-bit form: whole numbers have to be equal."""
import math

import pytest
import torch

import paper_2601_18383_b200 as D
from tests import tree_reference as TR

pytestmark = pytest.mark.gpu


def logits(n, V, dtype, seed, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, V), generator=g, device="cuda") * spread
    few = torch.randint(0, V, (n, min(V, 30)), generator=g, device="cuda")
    x.scatter_(1, few, 3.0 + 3.0 * torch.empty(few.shape, device="cuda").exponential_(1.0, generator=g))
    return x.to(dtype), torch.rand((n,), generator=g, device="cuda")


def check(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    tokens, logprobs = D.sample(x, u, temperature, top_k, top_p, min_p)
    host = lambda s: s.cpu() if torch.is_tensor(s) else s
    want, lp = TR.sample(x, u.cpu(), host(temperature), host(top_k), host(top_p), host(min_p))
    assert tokens.tolist() == want.tolist()
    void = want < 0
    assert torch.isnan(logprobs.cpu()[void]).all()
    got, lp = logprobs.double().cpu()[~void], lp[~void]
    # one rounding to fp32; the sum is within 2^-28 of the exact one, the scaled logit a rounding of a 64-bit quotient
    assert ((got - lp).abs() <= 2.0 ** -24 * lp.abs() + 2.0 ** -26).all()


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.6, top_k=50, top_p=0.9), dict(top_k=1), dict(top_k=7), dict(top_k=500), dict(top_k=700),
            dict(top_p=0.3), dict(top_p=0.95), dict(top_p=0.999), dict(min_p=0.05), dict(min_p=1.0), dict(temperature=1.5, top_p=0.9, min_p=0.02),
            dict(temperature=2.0, top_k=2000, top_p=0.99), dict(temperature=0.05, top_p=0.5), dict(temperature=30.0, top_p=0.7), dict(top_k=10 ** 6, top_p=0.8)]


@pytest.mark.parametrize("s", SETTINGS, ids=[" ".join(f"{k}={v}" for k, v in s.items()) or "uncut" for s in SETTINGS])
@pytest.mark.parametrize("n,V,dtype", [(3, 32003, torch.float32), (2, 128256, torch.bfloat16), (5, 1009, torch.bfloat16), (40, 4099, torch.float32)])
def test_settings(n, V, dtype, s):
    x, u = logits(n, V, dtype, V + n)
    check(x, u, **s)


@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 31, 33, 127, 257, 1000, 8191, 8200])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_small_and_odd_vocabularies(V, dtype):
    x, u = logits(9, V, dtype, V)
    for s in (dict(), dict(top_k=3), dict(top_p=0.6), dict(temperature=0.0), dict(top_k=5, top_p=0.9, min_p=0.1)):
        check(x, u, **s)


@pytest.mark.parametrize("n", [1, 2, 17, 74, 75, 149, 300])
def test_row_counts(n):
    """Every cluster size, and more rows than fit at once."""
    x, u = logits(n, 20011, torch.bfloat16, n)
    check(x, u, 0.8, 40, 0.9)
    check(x[:60], u[:60], 0.8, 0, 0.9)
    check(x[:60], u[:60], 1.2)


def test_settings_of_each_row():
    x, u = logits(64, 5003, torch.float32, 4)
    g = torch.Generator().manual_seed(1)
    pick = lambda v, dt: torch.tensor(v, dtype=dt)[torch.randint(0, len(v), (64,), generator=g)].cuda()
    check(x, u, pick([0.0, 0.5, 1.0, 3.0], torch.float32), pick([0, 1, 20, 600, 9000], torch.int32), pick([1.0, 0.5, 0.9], torch.float32), pick([0.0, 0.1], torch.float32))


def test_values_outside_the_ranges_in_arrays():
    x, u = logits(8, 999, torch.float32, 5)
    t = torch.tensor([-1.0, math.nan, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0], device="cuda")
    k = torch.tensor([0, 0, -5, 0, 0, 0, 0, 0], dtype=torch.int32, device="cuda")
    p = torch.tensor([1.0, 1.0, 1.0, 1.5, math.nan, -0.5, 1.0, 1.0], device="cuda")
    m = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.0, 0.0, -1.0, 1.5], device="cuda")
    same_t, same_k = torch.tensor([0.0, 0.0] + [1.0] * 6), torch.zeros(8, dtype=torch.int32)
    same_p, same_m = torch.tensor([1.0, 1.0, 1.0, 1.0, 1.0, 1e-30, 1.0, 1.0]), torch.tensor([0.0] * 7 + [1.0])
    tokens, _ = D.sample(x, u, t, k, p, m)
    want, _ = TR.sample(x, u.cpu(), same_t, same_k, same_p, same_m)
    assert tokens.tolist() == want.tolist()


def test_ties_go_to_the_lowest_index():
    """Rows of few distinct values: borders inside equal logits, all equal, lists that overflow."""
    g = torch.Generator(device="cuda").manual_seed(9)
    u = torch.rand((6,), generator=g, device="cuda")
    for V in (40, 1003, 33000):
        for levels in (1, 2, 5):
            x = torch.randint(0, levels, (6, V), generator=g, device="cuda").float()
            for dtype in (torch.float32, torch.bfloat16):
                for s in (dict(), dict(top_k=10), dict(top_p=0.5), dict(top_k=300, top_p=0.25), dict(temperature=0.0), dict(min_p=0.5), dict(top_p=0.001)):
                    check(x.to(dtype), u, **s)


def test_the_ends_of_u():
    x, _ = logits(6, 3001, torch.float32, 12)
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, -3.0, math.nan, 7.0], device="cuda")
    check(x, u)
    check(x, u, top_k=5)
    check(x, u, top_p=0.9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_rows(dtype):
    """Logits of -inf, of the type's lowest value, of one finite token; rows without a distribution."""
    x, u = logits(9, 6007, dtype, 3)
    x[0, 100:] = -math.inf
    x[1] = -math.inf
    x[2] = -math.inf
    x[2, 4321] = -5.0
    x[3, 17] = math.nan
    x[4, 6006] = math.inf
    x[5] = torch.finfo(dtype).min
    x[6, ::2] = torch.finfo(dtype).min
    x[7, :6000] = -math.inf
    x[8, 1:] = torch.finfo(dtype).min
    for s in (dict(), dict(top_k=50), dict(top_k=5000), dict(top_p=0.9), dict(temperature=0.0), dict(min_p=0.3), dict(top_k=300, top_p=0.99, temperature=0.3)):
        check(x, u, **s)


def test_zeros_of_both_signs_are_equal():
    x = torch.tensor([[-0.0, 0.0, -0.0, 0.0], [0.0, -0.0, 0.0, -0.0]], device="cuda")
    u = torch.tensor([0.3, 0.9], device="cuda")
    for s in (dict(), dict(top_k=2), dict(top_p=0.5), dict(temperature=0.0)):
        check(x, u, **s)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_any_alignment(dtype):
    """Strided rows that begin at every offset within 16 bytes; what lies between them is not read as logits."""
    wide = torch.full((7, 5000), 100.0, dtype=dtype, device="cuda")
    for off in range(9):
        for V in (4000, 4001, 4006):
            x, u = logits(7, V, dtype, off)
            view = wide[:, off: off + V]
            view.copy_(x)
            check(view, u, 0.9, 30, 0.95)
            check(view, u, 1.0)
            view.fill_(100.0)


def test_large_shifts_and_temperatures():
    x, u = logits(4, 7001, torch.float32, 8)
    check(x + 1000.0, u, top_p=0.9)
    check(x * 1e30, u, top_p=0.9)
    check(x, u, temperature=1e-30, top_p=0.9)
    check(x, u, temperature=1e30)
    check(x, u, temperature=1e30, top_p=0.5)


def test_another_stream_and_a_replay():
    x, u = logits(5, 30000, torch.bfloat16, 2)
    tokens, lp = torch.empty(5, dtype=torch.int32, device="cuda"), torch.empty(5, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    D.sample(x, u, 0.7, 50, 0.9, tokens=tokens, logprobs=lp)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            D.sample(x, u, 0.7, 50, 0.9, tokens=tokens, logprobs=lp)
    for seed in (3, 4):
        x2, u2 = logits(5, 30000, torch.bfloat16, seed)
        x.copy_(x2), u.copy_(u2)
        graph.replay()
        torch.cuda.synchronize()
        assert tokens.tolist() == TR.sample(x, u.cpu(), 0.7, 50, 0.9, 0.0)[0].tolist()


def test_shares_of_many_draws():
    """The drawn tokens' shares are the distribution's: 200000 draws of 5 tokens, each count within 5 standard deviations."""
    p = torch.tensor([0.4, 0.3, 0.15, 0.1, 0.05])
    n = 200000
    x = p.log().expand(n, 5).contiguous().cuda()
    u = torch.rand((n,), generator=torch.Generator(device="cuda").manual_seed(77), device="cuda")
    tokens, _ = D.sample(x, u)
    share = torch.bincount(tokens.cpu().long(), minlength=5) / n
    assert ((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all()


@pytest.mark.parametrize("top_p", [0.99999, 1 - 2.0 ** -23, 1 - 2.0 ** -24, 1e-7, 1e-38])
def test_top_p_near_its_ends(top_p):
    for n, V, dtype in ((4, 128256, torch.float32), (70, 9001, torch.bfloat16)):
        x, u = logits(n, V, dtype, 21)
        check(x, u, top_p=top_p)
        check(x, u, 1.7, top_k=1500, top_p=top_p)
        check(x, u, 0.7, top_k=20, top_p=top_p)


def test_two_streams_at_once():
    """Rows of two calls in flight together; no workspace is shared."""
    sets = [logits(40, 50021, torch.float32, 31), logits(3, 128256, torch.bfloat16, 32)]
    alone = [D.sample(x, u, 0.9, 0, 0.95) for x, u in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    out = []
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (x, u) in zip(streams, sets):
            with torch.cuda.stream(s):
                out.append(D.sample(x, u, 0.9, 0, 0.95))
    torch.cuda.synchronize()
    for i, (tokens, logprobs) in enumerate(out):
        assert torch.equal(tokens, alone[i % 2][0]) and torch.equal(logprobs, alone[i % 2][1])
