"""adt_tree_attn_q8 where values differ much in size: what a row does not see, or gives no weight, leaves its output as
it is; values near the largest that bf16 holds.  Bounds: those of test_parity_attn_q8 (relative to the weights times
the values of what a row sees)."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import synth
from test_parity_attn_q8 import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


# Items of up to 64 and 128 rows, and small ones; whole ones and ones that several thread blocks share.
MANY = [([40], [300], 2, 2, 64), ([40], [300], 2, 2, 128), ([100], [300], 2, 1, 128), ([33], [5000], 1, 1, 128),
        ([200], [2000], 1, 1, 64)]
FEW = [([3], [300], 2, 2, 64), ([16], [300], 1, 1, 128), ([4], [3000], 4, 1, 64), ([8], [300], 4, 1, 128), ([4], [5000], 4, 1, 128), ([31], [2000], 1, 1, 64)]


def star(case):
    """Every node the root's child, which no other node sees."""
    case.tb.parents[:] = 0
    case.tb.parents[case.tb.node_offsets[:-1]] = -1


def unlike(sizes, kv, H, Hkv, D, apart):
    """A node that no other one sees and cached rows of next to no weight, with values 2^apart of the others'."""
    case = Case(sizes, kv, H, Hkv, D)
    star(case)
    r = synth.rng(apart, "unlike")
    down = 2.0 ** (-min(apart, 80) if apart > 60 else 0)  # (all within bf16)
    case.vs -= int(-math.log2(down))
    case.vt = (case.vt.double() * down).to(torch.bfloat16)
    case.vt[case.n - 1] = (case.vt[case.n - 1].double() * 2.0 ** apart).to(torch.bfloat16)
    # Queries close to one direction, against which the cached rows 3 and the last but one lie: weights of 2^-(apart + 30).
    base = r.standard_normal(D)
    case.q = torch.from_numpy(base + 0.1 * r.standard_normal((case.n, H, D))).to(torch.bfloat16)
    case.kt = (case.kt.double() * 0.2).to(torch.bfloat16)
    case.ks -= 2
    far = -(apart + 30) * math.log(2) / case.scale * base / (base ** 2).sum()
    kc, ks = oracle.q8_rows(far[None])
    for at in (3, kv[0] - 2):
        case.kc[0, :, at], case.ks[0, :, at] = torch.from_numpy(kc[0]).view(torch.float8_e4m3fn), int(ks[0])
        case.vs[0, :, at] += apart
    case.kval = oracle.q8_values(case.kc.view(torch.uint8).numpy(), case.ks.numpy())
    case.vval = oracle.q8_values(case.vc.view(torch.uint8).numpy(), case.vs.numpy())
    return case


def far_apart(sizes, kv, H, Hkv, D, apart):
    case = unlike(sizes, kv, H, Hkv, D, apart)
    g = case.dev()
    case.call(g)
    case.check(g)
    assert B.adt_get_device_error() == 0
    # Nor does it change a bit of the others' outputs whether the unseen node's values are a little larger.
    first = g["out"][:case.n - 1].clone()
    g["vt"][case.n - 1] *= 1.5
    case.call(g)
    assert torch.equal(first, g["out"][:case.n - 1])


@pytest.mark.parametrize("apart", [18, 22, 26, 30, 40, 80])
@pytest.mark.parametrize("sizes,kv,H,Hkv,D", MANY)
def test_values_far_above_those_that_count(sizes, kv, H, Hkv, D, apart):
    far_apart(sizes, kv, H, Hkv, D, apart)


def larger_than_all(sizes, kv, H, Hkv, D):
    case = Case(sizes, kv, H, Hkv, D)
    case.vs += 120  # up to 448 * 2^114
    case.vt = (case.vt.double() * 2.0 ** 114).to(torch.bfloat16)
    case.vval = oracle.q8_values(case.vc.view(torch.uint8).numpy(), case.vs.numpy())
    g = case.dev()
    case.call(g)
    case.check(g)
    assert torch.isfinite(g["out"]).all() and B.adt_get_device_error() == 0


@pytest.mark.parametrize("sizes,kv,H,Hkv,D", MANY)
def test_values_near_the_largest(sizes, kv, H, Hkv, D):
    larger_than_all(sizes, kv, H, Hkv, D)


def rows_of_zeros(sizes, kv, H, Hkv, D, up):
    """A cache of zeros, whose scale is the least there is, and one node with values, 2^up times the usual, which no
    other node sees: outputs of zero, and the scores' sums as ever."""
    case = Case(sizes, kv, H, Hkv, D)
    star(case)
    case.vc.view(torch.uint8)[:], case.vs[:] = 0, 7
    case.vt[:case.n - 1] = 0
    case.vt[case.n - 1] = (case.vt[case.n - 1].double() * 2.0 ** up).to(torch.bfloat16)
    case.vval = oracle.q8_values(case.vc.view(torch.uint8).numpy(), case.vs.numpy())
    g = case.dev()
    case.call(g)
    case.check(g)
    assert (g["out"][:case.n - 1] == 0).all() and B.adt_get_device_error() == 0


@pytest.mark.parametrize("up", [0, 60])
@pytest.mark.parametrize("sizes,kv,H,Hkv,D", MANY)
def test_rows_of_zeros_beside_others(sizes, kv, H, Hkv, D, up):
    rows_of_zeros(sizes, kv, H, Hkv, D, up)


@pytest.mark.parametrize("apart", [18, 26, 40, 60, 80])
@pytest.mark.parametrize("sizes,kv,H,Hkv,D", FEW)
def test_values_far_above_those_that_count_of_few_rows(sizes, kv, H, Hkv, D, apart):
    far_apart(sizes, kv, H, Hkv, D, apart)


@pytest.mark.parametrize("sizes,kv,H,Hkv,D", FEW)
def test_values_near_the_largest_of_few_rows(sizes, kv, H, Hkv, D):
    larger_than_all(sizes, kv, H, Hkv, D)


@pytest.mark.parametrize("up", [0, 60])
@pytest.mark.parametrize("sizes,kv,H,Hkv,D", FEW)
def test_rows_of_zeros_beside_others_of_few_rows(sizes, kv, H, Hkv, D, up):
    rows_of_zeros(sizes, kv, H, Hkv, D, up)
