"""Refusals of outputs of the 8-bit cache's operators that lie on a call's small inputs (lengths, paths, offsets): no GPU
needed, the checks run before any CUDA call."""
import pytest

from test_cache_ops_host import INVALID, P, _call, lib  # noqa: F401 (lib: a fixture)
from test_q8_host import _at, _compact_args, _read_args


@pytest.mark.parametrize("change", [dict(ko=P[4]), dict(vo=P[4]), dict(ko=_at(P[4], -16)), dict(vo=_at(P[4], -64))])
def test_read_refuses_to_write_its_lengths(lib, change):  # noqa: F811
    assert _call(lib.adt_kv_read_q8, _read_args(), **change) == INVALID

@pytest.mark.parametrize("change", [dict(kvo=P[10]), dict(kvo=_at(P[10], 4)), dict(kvo=P[8]), dict(kvo=_at(P[8], 8)), dict(kvo=P[9]),
                                    dict(kvo=_at(P[9], 60)), dict(kvo=P[0]), dict(kvo=_at(P[1], 6400)), dict(kvo=_at(P[3], 100))])
def test_commit_refuses_new_lengths_on_its_inputs(lib, change):  # noqa: F811
    """accept_len [2], node_offsets [3], path [2][8], which other thread blocks read while the lengths are written; caches and
    scales."""
    assert _call(lib.adt_kv_compact_q8, _compact_args(), **change) == INVALID
