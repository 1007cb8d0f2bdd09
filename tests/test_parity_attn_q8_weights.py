"""adt_tree_attn_q8's weights: one key far above the others, of which there are enough to matter.

All values have one scale and one sign, and the large key's row is zero in all columns but the last, so that weights
that are lost, or rounded the same way for all keys, show.  Bound, per output element, with weights w (sum 1):
  - a weight is rounded to fp16's 11 bits, 2^-11 of it, and ends somewhere: up to FLOOR of the row's largest weight, where
      of up to 16 rows four e4m3 numbers 2^-4 apart end at 2^-21 with the largest at 2^4 or more: half of it, 2^-26;
      of more, fp16 ends at 2^-24 with the largest above 2^6: half of it, 2^-31;
  - scores are within d = 2^-16 S + 2^-17 (1 + T) as in test_parity_attn_q8, so weights over their sum within 4 d;
  - O is a sum in fp32 over at most 2^13 keys, 16 an instruction: 2^-13 of the sum of magnitudes;
  - the output is rounded to bf16, 2^-8 of it.
Weights that end 2^-4 sooner do not fit in it, nor those of bf16: the first tests, which need no GPU."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_cases import ensure_built, i32
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import synth

L, BIG = 4099, 17
HALF = math.log2(1 + 2.0 ** -8)  # a weight of 2^(whole + HALF) lies halfway between two bf16 numbers
FLOOR_FEW, FLOOR = 2.0 ** -26, 2.0 ** -31


def values_of(D, seed):
    """Values [L, D] of one scale and one sign, the large key's only in the last column; their bytes and scales."""
    v = synth.rng(seed, "weights").uniform(0.5, 0.9, size=(503, D))
    v[:, D - 1] = 1.0
    q, s = oracle.q8_rows(v)
    assert (s == s[0]).all()
    q, s = np.tile(q, (9, 1))[:L], np.tile(s, 9)[:L]
    q[BIG, :D - 1] = 0
    return q, s, oracle.q8_values(q, s)


def weights(big, others):
    w = np.full(L, 2.0 ** others)
    w[BIG] = 2.0 ** big
    return w


def bound(w, values, S, T, floor):
    w = w / w.sum()
    A = w @ values
    d = 2.0 ** -16 * S + 2.0 ** -17 * (1 + T)
    return A * (2.0 ** -11 + 4 * d + 2.0 ** -13 + 2.0 ** -8) + floor * w.max() * values.sum(0)


def e4m3_parts(x, parts):
    """x as so many e4m3 numbers, each 16 times what the ones before leave."""
    out, left = 0.0, float(np.float16(x))
    for i in range(parts):
        y = float(torch.tensor(left * 16.0 ** i).to(torch.float8_e4m3fn).float()) / 16.0 ** i
        out, left = out + y, left - y
    return out


def as_bf16(x):
    return float(torch.tensor(x, dtype=torch.float64).to(torch.bfloat16))


# The large key's weight is 2^top where weights are rounded.
@pytest.mark.parametrize("big,others,floor,top,rounded,fits", [
    (23, 0.4, FLOOR_FEW, 4, lambda x: e4m3_parts(x, 3), False), (23, 0.4, FLOOR_FEW, 4, lambda x: e4m3_parts(x, 4), True),
    (18, 0.4, FLOOR_FEW, 4, lambda x: e4m3_parts(x, 2), False), (18, 0.4, FLOOR_FEW, 4, lambda x: e4m3_parts(x, 4), True),
    (12, HALF, FLOOR, 0, as_bf16, False), (12, HALF, FLOOR, 7, np.float16, True),
    (27, 0.3, FLOOR, 0, np.float16, False), (27, 0.3, FLOOR, 7, np.float16, True)])
def test_the_bound_sees_weights_of_fewer_bits(big, others, floor, top, rounded, fits):
    values, w = values_of(64, 1)[2], weights(big, others)
    p = np.where(np.arange(L) == BIG, w, float(rounded(2.0 ** (top - big + others))) * 2.0 ** (big - top))
    got = np.array([as_bf16(x) for x in p @ values / w.sum()])
    over = np.abs(got - w @ values / w.sum()) > bound(w, values, 2 * big, big, floor)
    assert over.any() != fits


def one_key_above(nodes, group, D, big, others, floor):
    """So many kv heads, all alike, that none is cut among thread blocks (a part without the large key would keep all)."""
    ensure_built()
    Hkv = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    H, scale = Hkv * group, 1 / math.sqrt(D)
    unit = scale * math.log2(math.e)  # of a score, in powers of two
    bytes_, s, values = values_of(D, big)
    # Queries of three elements: the large key takes the first, and the second for what bf16 leaves of it, all others the third.
    row = torch.zeros(D, dtype=torch.float64)
    row[0] = float(torch.tensor(big / unit / 16, dtype=torch.float64).to(torch.bfloat16))
    row[1] = big / unit - row[0] * 16
    row[2] = others / unit
    row = row.to(torch.bfloat16)
    key = np.zeros((2, D))
    key[0, 0], key[0, 1], key[1, 2] = 16, 1, 1
    kc, ks = oracle.q8_rows(key)
    assert (oracle.q8_values(kc, ks) == key).all()
    at = (np.arange(L) != BIG).astype(int)

    def heads(x):
        return torch.from_numpy(x).cuda().expand(1, Hkv, *x.shape).contiguous()

    # The tree, a chain: values of 0, and 2^-12 of the others' weights or less, below 2^-20 of the sum in all.
    kt = torch.zeros((nodes, Hkv, D), dtype=torch.bfloat16, device="cuda")
    vt = torch.zeros_like(kt)
    kt[..., 0] = -16.0
    q = row.cuda().expand(nodes, H, D).contiguous()
    out = torch.full_like(q, float("nan"))
    shape = dict(B=1, H=H, Hkv=Hkv, D=D, max_nodes=nodes, max_kv=L)
    B.adt_tree_attn_q8(q, heads(kc[at]).view(torch.float8_e4m3fn), heads(bytes_).view(torch.float8_e4m3fn), heads(ks[at]), heads(s),
                       i32([L]), kt, vt, i32(np.arange(nodes) - 1), i32([0, nodes]), softmax_scale=scale, out=out,
                       workspace=B.zeroed_workspace(B.adt_tree_attn_q8_workspace_size(**shape)), **shape)
    row = row.double().numpy()
    z = unit * (key @ row)
    w = weights(z[0], z[1])
    S = scale * 2 * (16 + 1) * np.abs(row).sum()
    err = np.abs(out.double().cpu().numpy() - w @ values / w.sum())
    limit = bound(w, values, S, big, floor)
    assert (err <= limit).all(), (err / limit).max((0, 1))
    assert B.adt_get_device_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("big,others", [(12, HALF), (18, 0.4), (23, 0.4), (27, 0.3)])
@pytest.mark.parametrize("nodes,group,D", [(64, 1, 64), (33, 1, 128), (100, 1, 128), (1, 40, 64)])
def test_many_small_weights_beside_a_large_one(nodes, group, D, big, others):
    one_key_above(nodes, group, D, big, others, FLOOR)


@pytest.mark.gpu
@pytest.mark.parametrize("big,others", [(12, HALF), (18, 0.4), (23, 0.4), (25, 0.3)])
@pytest.mark.parametrize("nodes,group,D", [(1, 4, 128), (8, 4, 64), (1, 1, 64), (32, 1, 128), (16, 1, 64), (4, 4, 128)])
def test_many_small_weights_beside_a_large_one_of_few_rows(nodes, group, D, big, others):
    one_key_above(nodes, group, D, big, others, FLOOR_FEW)
