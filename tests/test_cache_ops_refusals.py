"""Refusals of the cache operators for outputs that share memory.  The checks
run before any CUDA call, on addresses that nothing reads.  (No call here is one
that is accepted: it would be launched where there is a GPU.)"""
import ctypes

import pytest

from test_cache_ops_host import INVALID, P, _call, _evict_args, lib  # noqa: F401 (lib: a fixture)


def _at(base, elements, size=2):
    return ctypes.c_void_p(base.value + elements * size)


HEAD, TREE, LAYER = 6400, 2 * 6400, 4 * 6400  # strides of _evict_args: 100 rows of 64, [3][2][2]


@pytest.mark.parametrize("shift", [HEAD, TREE, LAYER, HEAD + TREE, 2 * LAYER, 2 * LAYER + TREE + HEAD, HEAD - 8, LAYER + 6392])
@pytest.mark.parametrize("sign", [1, -1])
def test_evict_refuses_v_on_other_slices_of_k(lib, shift, sign):  # noqa: F811
    v = _at(P[6], sign * shift)
    # in place, and into caches apart from the sources
    assert _call(lib.adt_kv_evict, _evict_args(), k=P[6], ko=P[6], v=v, vo=v) == INVALID
    assert _call(lib.adt_kv_evict, _evict_args(), ko=P[6], vo=v) == INVALID


def test_evict_refuses_v_in_the_gaps_of_k_where_a_slice_does_not_fit(lib):  # noqa: F811
    wide = dict(ssh=2 * HEAD - 8, ssb=4 * HEAD, sls=8 * HEAD)
    wide |= dict(dsh=wide["ssh"], dsb=wide["ssb"], dls=wide["sls"])
    v = _at(P[6], HEAD)
    assert _call(lib.adt_kv_evict, _evict_args(), k=P[6], ko=P[6], v=v, vo=v, **wide) == INVALID
