"""Refusals of sampling, trees and sinks that need no GPU."""
import pytest

import paper_2601_18383_b200 as D

A = 1 << 12  # an address that is never read


def refused(call, status=D.DYNTS_ERR_INVALID_ARG):
    with pytest.raises(D.DyntsError) as e:
        call()
    assert e.value.status == status


def opts(**kw):
    o = D.dynts_sample_opts_t(1.0, 0, 1.0, 0.0, None, None, None, None)
    for k, v in kw.items():
        setattr(o, k, v)
    return o


@pytest.mark.parametrize("kw", [dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.01),
                                dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=float("nan")), dict(temperatures=A + 2)])
def test_sample_settings(kw):
    refused(lambda: D.dynts_sample(A, D.DYNTS_FP32, 2, 100, 0, A, opts(**kw), A, A))


def test_sample_shapes_and_pointers():
    ok = dict(logits=A, dtype=D.DYNTS_BF16, n_rows=2, vocab=100, row_stride=0, u=A, opts=None, tokens=A, logprobs=A)
    for bad in (dict(dtype=D.DYNTS_BF16_KV8), dict(n_rows=-1), dict(vocab=0), dict(vocab=1 << 19), dict(row_stride=99), dict(row_stride=-5), dict(logits=None), dict(u=None),
                dict(tokens=None), dict(logits=A + 1), dict(u=A + 2), dict(tokens=A + 1), dict(logprobs=A + 3), dict(row_stride=1 << 40)):
        refused(lambda: D.dynts_sample(**{**ok, **bad}))
    assert D.dynts_sample(**{**ok, "n_rows": 0, "logits": None}) == D.DYNTS_OK


def cache(batch=2):
    h = D.dynts_cache_create(2, 2, 128, 64, 8)
    D.dynts_cache_set_shape(h, batch, 8, D.DYNTS_BF16, 8)
    return h


def test_tree_plan():
    h = cache()
    refused(lambda: D.dynts_tree_plan(h, A, [3, -1], A, A))
    refused(lambda: D.dynts_tree_plan(h, A, [3, 1025], A, A))
    refused(lambda: D.dynts_tree_plan(h, None, [3, 1], A, A))
    refused(lambda: D.dynts_tree_plan(h, A, [3, 1], None, A))
    refused(lambda: D.dynts_tree_plan(h, A, [3, 1], A + 8, A))
    refused(lambda: D.dynts_tree_plan(h, A + 2, [3, 1], A, A))
    refused(lambda: D.dynts_tree_plan(h, A, [3, 1], A, A + 1))
    refused(lambda: D.dynts_tree_plan(None, A, [3, 1], A, A))
    assert D.dynts_tree_plan(h, None, [0, 0], None) == D.DYNTS_OK
    D.dynts_cache_destroy(h)


def test_tree_accept():
    refused(lambda: D.dynts_tree_accept(A, A, A, [1, 2], 0, A, 4, A, A))
    refused(lambda: D.dynts_tree_accept(A, A, A, [1, 2], 2, A, 0, A, A))
    refused(lambda: D.dynts_tree_accept(A, A, A, [1, -2], 2, A, 4, A, A))
    refused(lambda: D.dynts_tree_accept(A, A, None, [1, 2], 2, A, 4, A, A))
    refused(lambda: D.dynts_tree_accept(A, A, A, [1, 2], 2, None, 4, A, A))
    refused(lambda: D.dynts_tree_accept(A, A, A, [1, 2], 2, A, 4, A, None))


def test_extend_with_more():
    h = cache()
    more, o = D.dynts_extend_more_t(0, None), D.dynts_extend_opts_t()
    call = lambda layer=-1: D.dynts_extend_attn_ex(h, layer, A, A, A, A, [3, 2], o, more, A, 1 << 30)
    refused(lambda: call(-2))
    more.sinks = -1
    refused(call)
    more.sinks, more.tree = 0, A
    refused(call)                # not staged
    o.stage = 1
    more.tree = A + 4
    refused(call)                # misaligned
    more.tree = A
    import ctypes
    prefix = (ctypes.c_int * 2)(1, 0)
    o.prefix = ctypes.addressof(prefix)
    refused(call)                # a tree has no prefix
    refused(lambda: D.dynts_extend_attn_ex(h, -1, A, A, A, A, [1025, 2], o, more, A, 1 << 30), D.DYNTS_ERR_CAPACITY)
    refused(lambda: D.dynts_extend_commit_path(h, [1, 1], A, 4), D.DYNTS_ERR_STATE)
    refused(lambda: D.dynts_extend_commit_path(None, [1, 1], A, 4))
    D.dynts_cache_destroy(h)


@pytest.mark.parametrize("counts", [[2 ** 32 + 3, 2], [2 ** 31, 0]])
def test_counts_beyond_an_int(counts):
    h = cache()
    for call in (lambda: D.dynts_tree_plan(h, A, counts, A, A), lambda: D.dynts_tree_accept(A, A, A, counts, 2, A, 4, A, A),
                 lambda: D.dynts_extend_commit_path(h, counts, A, 4), lambda: D.dynts_extend_attn_ex(h, -1, A, A, A, A, counts, None, None, A, 1 << 30)):
        refused(call)
    D.dynts_cache_destroy(h)
