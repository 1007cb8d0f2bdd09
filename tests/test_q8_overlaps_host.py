"""Refusals of outputs of the 8-bit cache's operators that lie on a call's small inputs (lengths, paths, offsets): no GPU
needed, the checks run before any CUDA call."""
import pytest

from test_cache_ops_host import INVALID, P, _call, lib  # noqa: F401 (lib: a fixture)
from test_q8_host import _at, _read_args


@pytest.mark.parametrize("change", [dict(ko=P[4]), dict(vo=P[4]), dict(ko=_at(P[4], -16)), dict(vo=_at(P[4], -64))])
def test_read_refuses_to_write_its_lengths(lib, change):  # noqa: F811
    assert _call(lib.adt_kv_read_q8, _read_args(), **change) == INVALID
