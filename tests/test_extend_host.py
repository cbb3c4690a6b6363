"""What the chunk operators and dynts_rope refuse on the host, before anything is launched: needs no GPU."""
import pytest

import paper_2601_18383_b200 as D

A = 1 << 12  # an address that is never read


@pytest.mark.parametrize("bad", [dict(head_dim=7, rot_dim=6), dict(head_dim=7, rot_dim=6, flags=D.DYNTS_ROPE_ADJACENT), dict(q_heads=1 << 20),
                                 dict(kv_heads=1 << 20), dict(q_out=A, strides=[320, 0, 0, 0]), dict(k_out=A + 16, k=A + 16, strides=[0, 0, 0, 256])])
def test_rotation(bad):
    good = dict(q=A, k=A, pos=A, q_out=A, k_out=A, n_tokens=4, q_heads=4, kv_heads=2, head_dim=64, rot_dim=64, n_axes=1, sections=None, flags=0,
                theta=1e4, dtype=D.DYNTS_BF16, strides=None, stream=None)
    with pytest.raises(D.DyntsError) as e:
        D.dynts_rope(**{**good, **bad})
    assert e.value.status == D.DYNTS_ERR_INVALID_ARG


@pytest.mark.parametrize("cap", [1e-40, 1e-30, 1e30, float("nan"), -1e-3])
def test_caps_out_of_range(cap):
    h = D.dynts_cache_create(2, 2, 128, 64, 8)
    D.dynts_cache_set_shape(h, 2, 8, D.DYNTS_BF16, 8)
    o = D.dynts_extend_opts_t()
    o.softcap = cap
    with pytest.raises(D.DyntsError) as e:
        D.dynts_extend_attn(h, A, A, A, A, [3, 2], o, A, 1 << 30)
    assert e.value.status == D.DYNTS_ERR_INVALID_ARG
    D.dynts_cache_destroy(h)
