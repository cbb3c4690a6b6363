"""Sizes and refusals of the chunk operators that need no GPU."""
import pytest

import paper_2601_18383_b200 as D

A = 1 << 12  # an address that is never read


def test_scratch_of_a_cache_without_storage_serves_every_device():
    """Before its first call a cache does not know its device: the scratch it asks for has room for the most CTAs a launch may
    have (380: two per SM of 190), each with two parts of 128 query rows of 128 columns and a log-sum-exp."""
    h = D.dynts_cache_create(2, 2, 128, 64, 8)
    D.dynts_cache_set_shape(h, 2, 8, D.DYNTS_BF16, 8)
    assert D.dynts_extend_scratch_bytes(h, [40, 3], 1) >= 2 * 380 * 128 * 129 * 4
    D.dynts_cache_destroy(h)


@pytest.mark.parametrize("counts", [[2 ** 32 + 3, 2], [2 ** 31, 0], [-2 ** 31 - 1, 2]])
def test_counts_beyond_an_int(counts):
    h = D.dynts_cache_create(2, 2, 128, 64, 8)
    D.dynts_cache_set_shape(h, 2, 8, D.DYNTS_BF16, 8)
    for call in (lambda: D.dynts_extend_attn(h, A, A, A, A, counts, None, A, 1 << 30), lambda: D.dynts_extend_attn_layer(h, 0, A, A, A, A, counts, None, A, 1 << 30),
                 lambda: D.dynts_extend_commit(h, counts), lambda: D.dynts_extend_scratch_bytes(h, counts, 1)):
        with pytest.raises(D.DyntsError) as e:
            call()
        assert e.value.status == D.DYNTS_ERR_INVALID_ARG
    D.dynts_cache_destroy(h)
