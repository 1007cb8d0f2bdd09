"""Refusals of the cache operators for outputs that share memory.  The checks
run before any CUDA call, on addresses that nothing reads.  (No call here is one
that is accepted: it would be launched where there is a GPU.)"""
import ctypes

import pytest

from test_cache_ops_host import INVALID, P, UNSUPPORTED, _call, _evict_args, _score_args, lib  # noqa: F401 (lib: a fixture)


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


ALIASED = [  # (layer, tree, head) strides that pass a slice each and still put two slices on one another
    (2 * 100, 100, 100), (100, 2 * 100, 100), (200, 200, 100), (200, 100, 300), (399, 200, 100), (300, 100, 600), (250, 100, 150)]


@pytest.mark.parametrize("strides", ALIASED)
def test_evict_refuses_destinations_whose_slices_share_rows(lib, strides):  # noqa: F811
    k = dict(zip(("sls", "ssb", "ssh"), (64 * s for s in strides))) | dict(zip(("dls", "dsb", "dsh"), (64 * s for s in strides)))
    assert _call(lib.adt_kv_evict, _evict_args(), **k) == INVALID
    # into other caches, of slices of 50 rows
    half = dict(zip(("dls", "dsb", "dsh"), (32 * s for s in strides)))
    assert _call(lib.adt_kv_evict, _evict_args(), ko=P[6], vo=P[7], **half) == INVALID


@pytest.mark.parametrize("strides", ALIASED)
def test_evict_refuses_scores_whose_slices_share_rows(lib, strides):  # noqa: F811
    c = dict(zip(("cls", "csb", "csh"), strides)) | dict(zip(("ols", "osb", "osh"), strides))
    assert _call(lib.adt_kv_evict, _evict_args(), **c) == INVALID
    half = dict(zip(("ols", "osb", "osh"), (s // 2 for s in strides)))
    assert _call(lib.adt_kv_evict, _evict_args(), so=P[8], **half) == INVALID


@pytest.mark.parametrize("strides", ALIASED)
def test_score_refuses_scores_whose_slices_share_rows(lib, strides):  # noqa: F811
    c = dict(zip(("sls", "ssb", "ssh"), strides))
    assert _call(lib.adt_kv_score, _score_args(), **c) == INVALID
    assert _call(lib.adt_kv_score, _score_args(), **c, so=P[8]) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(qls=2 ** 41), INVALID), (dict(lls=2 ** 40 + 1), INVALID), (dict(lls=2 ** 62), INVALID),
    # 2^20 slices of 2^29 rows, 2^22 passes over each tile of 128: 2^64 in all
    (dict(layers=2 ** 9, B=2 ** 8, H=2 ** 14, Hkv=2 ** 3, max_kv=2 ** 29, max_path=2 ** 18, csh=2 ** 35, csb=2 ** 35, cls=2 ** 35,
          ssh=2 ** 29, ssb=2 ** 32, sls=2 ** 40), UNSUPPORTED),
])
def test_score_refuses_sizes_whose_products_pass_their_types(lib, change, status):  # noqa: F811
    assert _call(lib.adt_kv_score, _score_args(), **change) == status
