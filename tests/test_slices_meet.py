"""The check that slices of strided outputs do not share memory, against every
pair of slices compared."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest

from paper_2512_21857_gb300 import build

SOURCE = """
#include "slices.h"
extern "C" int meet(const int64_t* count, const int64_t* stride, int64_t need, int64_t delta) {
  const int64_t c[3] = {count[0], count[1], count[2]}, s[3] = {stride[0], stride[1], stride[2]};
  return adt::slices_meet(c, s, need, delta);
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    d = tmp_path_factory.mktemp("slices")
    (d / "meet.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC, str(d / "meet.cpp"), "-o", str(d / "meet.so")],
                   check=True)
    fn = ctypes.CDLL(os.path.join(d, "meet.so")).meet
    three = ctypes.c_int64 * 3
    return lambda count, stride, need, delta=0: bool(fn(three(*count), three(*stride), ctypes.c_int64(need), ctypes.c_int64(delta)))


def pairs(count, stride, need, delta):
    at = [(i, sum(a * b for a, b in zip(i, stride))) for i in itertools.product(*map(range, count))]
    return any(abs(y + delta - x) < need for i, x in at for j, y in at if delta != 0 or i != j)


def test_every_pair_agrees(meet):
    rng, seen = random.Random(5), [0, 0]
    for _ in range(20000):
        count = [rng.randint(1, 4) for _ in range(3)]
        need = rng.randint(1, 6)
        stride = [need + rng.choice([0, 1, rng.randint(0, 8 * need)]) if n > 1 else rng.randint(0, 9) for n in count]
        delta = rng.choice([0, rng.randint(-60, 60)])
        want = pairs(count, [s if n > 1 else 0 for n, s in zip(count, stride)], need, delta)
        assert meet(count, stride, need, delta) == want, (count, stride, need, delta)
        seen[want] += 1
    assert min(seen) > 2000


@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
def test_packed_dimensions_in_any_order_are_apart(meet, order):
    count, need = [32, 4, 20], 1000
    stride, step = [0] * 3, need
    for k in order:
        stride[k] = step
        step *= count[k]
    assert not meet(count, stride, need)
    stride[order[1]] -= 1
    assert meet(count, stride, need)


def test_large_sizes(meet):
    """Values near the limits of the entry points: no overflow, and at once."""
    assert not meet([65535, 16, 64], [2 ** 40, 2 ** 36, 2 ** 30], 2 ** 30 // 2)
    assert meet([65535, 64, 64], [2 ** 40, 2 ** 40, 2 ** 30], 2 ** 30 // 2)
    # K and V in turn: a slice apart, and shifted by one
    assert not meet([64, 64, 65535], [2 ** 40, 2 ** 38, 2 ** 20], 2 ** 19, 2 ** 19)
    assert meet([64, 64, 65535], [2 ** 40, 2 ** 38, 2 ** 20], 2 ** 19, 2 ** 19 + 1)
    assert meet([64, 64, 65535], [2 ** 40, 2 ** 38, 2 ** 20], 2 ** 19, -(2 ** 38) - 5)


def test_every_pair_agrees_of_dimensions_one_within_the_other(meet):
    """Packed layouts with gaps, and second sets a few strides away."""
    rng, seen = random.Random(6), [0, 0]
    for _ in range(20000):
        count, need = [rng.randint(1, 4) for _ in range(3)], rng.randint(1, 6)
        stride, step = [0] * 3, need
        for k in rng.sample(range(3), 3):
            stride[k] = step + rng.choice([0, 0, need, 2 * need + 1])
            step = stride[k] * count[k] if count[k] > 1 else step
        delta = sum(rng.randint(-2, 2) * s for s in stride) + rng.choice([0, need, -need, need - 1, rng.randint(-9, 9)])
        want = pairs(count, [s if n > 1 else 0 for n, s in zip(count, stride)], need, delta)
        assert meet(count, stride, need, delta) == want, (count, stride, need, delta)
        seen[want] += 1
    assert min(seen) > 2000
