"""Queries that add nothing to adt_kv_score (lse = -inf, or a path entry outside
the tree), where their own values or the cached keys are not finite.  The bound
is that of the score's own parity test."""
import numpy as np
import pytest
import torch

from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from test_parity_kv_score import Case, chain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def oracle_safe(c, absent):
    """The case with the absent queries' values zero: what the oracle is given, which multiplies before it skips."""
    q = c.q.clone()
    q[:, absent] = 0
    return q


@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("H,Hkv,D,kv,path,absent", [
    (4, 2, 64, 100, chain(3), [1]),            # a few queries, masked by eights
    (8, 2, 128, 300, chain(40), [0, 17, 39]),  # more than a pass of them, the first and the last among the absent
    (4, 4, 64, 40, chain(200), [63, 130]),     # a prompt
])
def test_absent_queries_need_not_be_finite(H, Hkv, D, kv, path, absent, garbage):
    c = Case(2, H, Hkv, D, [kv], [path], len(path), seed=kv + H)
    c.lse[:, absent] = -np.inf
    clean = oracle_safe(c, absent)
    c.q[:, absent] = garbage
    got = c.run()
    assert torch.isfinite(got).all()
    c.q = clean
    c.check(got)


@pytest.mark.parametrize("H,Hkv,D,path,absent", [(4, 2, 64, chain(3), [0, 1, 2]), (8, 2, 128, chain(40), chain(40)),
                                                 (4, 4, 64, chain(200), chain(200))])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_absent_queries_leave_scores_of_keys_that_are_not_finite(H, Hkv, D, path, absent, value):
    """Every query absent: no row's score changes, whatever the row holds."""
    c = Case(1, H, Hkv, D, [77], [path], len(path), seed=21)
    c.lse[:, absent] = -np.inf
    c.kc[:, :, :, 5] = value
    got = c.run()
    assert np.array_equal(got[..., :77].cpu().numpy(), c.score[..., :77])
    assert (got[..., 77:77 + len(path)] == 0).all()


def test_path_entries_outside_the_tree_leave_scores_of_keys_that_are_not_finite():
    c = Case(1, 4, 2, 64, [77], [[0, 1, 2]], 3, seed=22)
    c.kc[:, :, :, 5] = float("inf")
    args = list(c.args())
    args[5].fill_(99)
    B.adt_get_device_error()
    B.adt_kv_score(*args, **c.kw())
    assert B.adt_get_device_error() == B.DEVERR_BAD_PATH
    assert np.array_equal(args[-1][..., :77].cpu().numpy(), c.score[..., :77])


def test_absent_queries_among_others_change_no_bit_of_rows_that_are_finite():
    """A query of zeros with lse = -inf and one of NaN give the same bits."""
    c = Case(2, 4, 2, 128, [150, 60], [chain(70), [0, 1]], 70, seed=23)
    c.lse[:, [3, 71]] = -np.inf
    c.q[:, [3, 71]] = 0
    want = c.run()
    c.q[:, [3, 71]] = float("nan")
    assert torch.equal(c.run(), want)


@pytest.mark.parametrize("paths,absent", [([[0, 1, 2]], [1]), ([chain(70)], [3, 64])])
def test_keys_that_are_not_finite_beside_absent_queries_spoil_their_own_score_only(paths, absent):
    """The queries that are there still meet the row; the others' bits do not change."""
    c = Case(2, 4, 2, 64, [150], paths, len(paths[0]), seed=24, lmax=260)
    c.lse[:, absent] = -np.inf
    want = c.run()
    c.kc[0, 0, 1, 40] = float("nan")
    c.kc[:, :, :, 150 + len(paths[0]):] = float("nan")
    got = c.run()
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, 0, 1, 40] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])
