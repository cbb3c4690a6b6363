"""Rotary positions (dynts_rope) against the plain 64-bit form: several axes, both pairings, partial rotation, far
positions, strides, in place, odd head sizes; and the host's refusals."""
import math

import pytest
import torch

import paper_2601_18383_b200 as D
from tests.extend_reference import EPS


def plain(x, pos, theta, sections, rot, adjacent, round_robin):
    half = rot // 2
    if not round_robin:
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
    else:
        left, axis = list(sections), []
        while len(axis) < half:
            for a in range(len(left)):
                if left[a]:
                    left[a] -= 1
                    axis.append(a)
    z = x.double().cpu()
    y = z.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        phi = pos.cpu()[axis[i]].double()[:, None] * theta ** (-2.0 * i / rot)
        y[..., a] = z[..., a] * phi.cos() - z[..., b] * phi.sin()
        y[..., b] = z[..., a] * phi.sin() + z[..., b] * phi.cos()
    return y, z


def tolerance(y, z, dtype):
    # cosine and sine: 2^-22 each (the angle's rounding to fp32 and the function), two products and a sum, one rounding of the result
    return EPS[dtype] * y.abs() * 1.01 + 2.0 ** -21 * z.abs().amax(-1, keepdim=True) * 2


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 3, 130, 5000])
@pytest.mark.parametrize("d,rot,sections,adjacent,round_robin", [
    (128, 128, (64,), False, False), (128, 128, (64,), True, False), (128, 128, (16, 24, 24), False, False), (128, 128, (24, 20, 20), False, True),
    (64, 32, (8, 8), True, True), (80, 20, (10,), False, False), (40, 40, (12, 8), False, False), (96, 6, (3,), True, False), (256, 256, (50, 28, 0, 50), False, True)])
def test_matches_the_plain_form(dtype, n, d, rot, sections, adjacent, round_robin):
    g = torch.Generator(device="cuda").manual_seed(n + d)
    q, k = (torch.randn((n, h, d), generator=g, device="cuda").to(dtype) for h in (5, 2))
    pos = torch.randint(0, 1 << 20, (len(sections), n), generator=g, device="cuda", dtype=torch.int32)
    pos[0, 0] = -7
    qo, ko = D.rope(q, k, pos if len(sections) > 1 else pos[0], theta=500000.0, sections=sections, rot_dim=rot, adjacent=adjacent, round_robin=round_robin)
    for x, got in ((q, qo), (k, ko)):
        y, z = plain(x, pos, 500000.0, sections, rot, adjacent, round_robin)
        assert ((got.double().cpu() - y).abs() <= tolerance(y, z, dtype)).all()
        assert torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.gpu
def test_strides_and_in_place():
    n = 70
    fused = torch.randn((n, 8 * 128 + 2 * 2 * 128), device="cuda").to(torch.bfloat16)
    q, k, v = (x.unflatten(1, (-1, 128)) for x in fused.split([1024, 256, 256], 1))
    pos = torch.arange(n, device="cuda", dtype=torch.int32) + 100000
    qo, ko = D.rope(q, k, pos, theta=500000.0)
    keep = v.clone()
    D.rope(q, k, pos, q, k, theta=500000.0)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(v, keep)
    alone, none = D.rope(q, None, pos)
    assert none is None and torch.equal(alone, D.rope(q, k, pos)[0])


@pytest.mark.gpu
def test_no_tokens_and_a_stream_of_its_own():
    q = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    out, _ = D.rope(q, None, torch.empty(0, dtype=torch.int32, device="cuda"))
    assert out.shape == q.shape
    q = torch.randn((300, 4, 128), device="cuda")
    pos = torch.arange(300, device="cuda", dtype=torch.int32)
    want = D.rope(q, None, pos)[0]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = D.rope(q, None, pos)[0]
    st.synchronize()
    assert torch.equal(got, want)


def test_refusals_on_the_host():
    """Refused before anything is launched: needs no GPU."""
    A = 1 << 12  # an address that is never read
    good = dict(q=A, k=A, pos=A, q_out=A, k_out=A, n_tokens=4, q_heads=4, kv_heads=2, head_dim=64, rot_dim=64, n_axes=1, sections=None, flags=0,
                theta=1e4, dtype=D.DYNTS_BF16, strides=None, stream=None)
    for bad in (dict(head_dim=0), dict(head_dim=258), dict(rot_dim=3), dict(rot_dim=66), dict(rot_dim=0), dict(n_axes=2), dict(n_axes=5, sections=[8] * 5),
                dict(sections=[31]), dict(n_axes=2, sections=[40, -8]), dict(flags=4), dict(theta=0.0), dict(theta=float("nan")), dict(theta=float("inf")),
                dict(dtype=D.DYNTS_BF16_KV8), dict(q=None), dict(q_out=None), dict(k_out=None), dict(pos=None), dict(q=A + 2), dict(n_tokens=-1),
                dict(strides=[128, 0, 0, 0]), dict(strides=[0, 0, 0, 64]), dict(q_heads=0)):
        with pytest.raises(D.DyntsError) as e:
            D.dynts_rope(**{**good, **bad})
        assert e.value.status == D.DYNTS_ERR_INVALID_ARG, bad
    D.dynts_rope(**{**good, "n_tokens": 0})


def test_chunk_refusals_on_the_host():
    """A cache without storage yet refuses bad chunks without touching a device."""
    h = D.dynts_cache_create(2, 2, 128, 64, 8)
    D.dynts_cache_set_shape(h, 2, 8, D.DYNTS_BF16, 8)
    A, cap = 1 << 12, D.dynts_cache_capacity(h)

    def opts(**kw):
        o = D.dynts_extend_opts_t()
        for x, y in kw.items():
            setattr(o, x, y)
        return o

    def call(n_new=(3, 2), o=None, q=A, k=A, v=A, out=A, scratch=A, size=1 << 30):
        D.dynts_extend_attn(h, q, k, v, out, list(n_new), o, scratch, size)

    for status, kw in [(D.DYNTS_ERR_INVALID_ARG, dict(n_new=(-1, 2))), (D.DYNTS_ERR_CAPACITY, dict(n_new=(cap + 1, 0))), (D.DYNTS_ERR_INVALID_ARG, dict(q=None)),
                       (D.DYNTS_ERR_INVALID_ARG, dict(k=A + 4)), (D.DYNTS_ERR_INVALID_ARG, dict(out=None)), (D.DYNTS_ERR_INVALID_ARG, dict(scratch=None)),
                       (D.DYNTS_ERR_OOM, dict(size=16)), (D.DYNTS_ERR_INVALID_ARG, dict(o=opts(softcap=-1.0))), (D.DYNTS_ERR_INVALID_ARG, dict(o=opts(softcap=float("inf")))),
                       (D.DYNTS_ERR_INVALID_ARG, dict(o=opts(window=-2))), (D.DYNTS_ERR_INVALID_ARG, dict(o=opts(stage=2))),
                       (D.DYNTS_ERR_INVALID_ARG, dict(o=opts(q_stride=1000))), (D.DYNTS_ERR_INVALID_ARG, dict(o=opts(k_stride=260))), (D.DYNTS_ERR_INVALID_ARG, dict(o=opts(v_stride=128)))]:
        with pytest.raises(D.DyntsError) as e:
            call(**kw)
        assert e.value.status == status, kw
    with pytest.raises(D.DyntsError) as e:
        D.dynts_extend_attn_layer(h, 1, A, A, A, A, [1, 1], None, A, 1 << 30)
    assert e.value.status == D.DYNTS_ERR_STATE
    with pytest.raises(D.DyntsError) as e:
        D.dynts_extend_commit(h, [0, 0])
    assert e.value.status == D.DYNTS_ERR_STATE
    assert D.dynts_extend_scratch_bytes(h, [-1, 0], 1) == 0 and D.dynts_extend_scratch_bytes(h, [1, 0], 3) == 0
    assert D.dynts_extend_scratch_bytes(h, [3, 2], 2) >= 2 * 5 * 8 * 4
    assert D.dynts_cache_len(h, 0) == 0
    D.dynts_cache_destroy(h)
