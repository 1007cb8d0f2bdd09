"""adt_tree_attn_q8 on the GPU against the fp64 oracle over the values that the 8-bit rows stand for.

Bound, per output element.  A weight may be rounded to bf16 before it meets its
value (2^-8 of it), and its score is off by what the products' operands lose: an
element of q by at most 2^-17 of its row's largest, of a key likewise, and fp32
sums of up to 2^7 products (2^-17 of the sum of magnitudes), so with
  S = scale * max over keys of (max |q| sum |k| + max |k| sum |q|)
a score is within 2^-16 S, the exponential's own error (argument and value)
within 2^-17 of the largest score's size T.  So |out - ref| <= A (2^-8 + 4 (2^-16 S + 2^-17 (1
+ T))) + 2^-8 |ref|, A = sum of weights |value|, the last term the rounding to bf16.
lse: 2 (2^-16 S + 2^-17 (1 + T))."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_cases import ensure_built, i32
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def quantised(shape, seed, name, std=1.0):
    """Random 8-bit rows with scales, some of them far from the others', and their values."""
    r = synth.rng(seed, name)
    q = torch.from_numpy((r.standard_normal(shape) * 100 * std).clip(-448, 448)).to(torch.float8_e4m3fn)
    s = torch.from_numpy((120 + (r.random(shape[:-1]) < 0.1) * r.integers(-6, 2, size=shape[:-1])).astype(np.uint8))
    return q, s, oracle.q8_values(q.view(torch.uint8).numpy(), s.numpy())


class Case:
    def __init__(self, sizes, kv, H, Hkv, D, seed=0, chain=False, spare=5, max_depth=9, max_children=6, qstd=1.0, gap=0):
        self.sizes, self.kv, self.H, self.Hkv, self.D, self.B = sizes, kv, H, Hkv, D, len(kv)
        seed += sum(sizes) + sum(kv) + H + D
        self.tb = synth.tree_batch(sizes, 100, seed, chain=chain, max_depth=max_depth, max_children=max_children)
        self.n = int(self.tb.node_offsets[-1])
        self.rows = max(max(kv) + spare, 1)
        shape = (self.B, Hkv, self.rows, D)
        self.kc, self.ks, self.kval = quantised(shape, seed, "k")
        self.vc, self.vs, self.vval = quantised(shape, seed, "v")
        self.q = synth.bf16_normal((self.n, H, D), seed, "q", std=qstd)
        self.kt = synth.bf16_normal((self.n, Hkv, D), seed, "kt")
        self.vt = synth.bf16_normal((self.n, Hkv, D), seed, "vt")
        self.scale = 1 / math.sqrt(D)

    def dev(self):
        g = {k: getattr(self, k).cuda() for k in ("q", "kc", "vc", "ks", "vs", "kt", "vt")}
        g["kv"], g["parents"], g["offs"] = i32(self.kv), i32(self.tb.parents), i32(self.tb.node_offsets)
        g["out"] = torch.full((self.n, self.H, self.D), float("nan"), dtype=torch.bfloat16, device="cuda")
        g["lse"] = torch.full((self.n, self.H), float("nan"), device="cuda")
        return g

    def shape(self, max_nodes=None, max_kv=None):
        return dict(B=self.B, H=self.H, Hkv=self.Hkv, D=self.D, max_nodes=max_nodes or max(self.sizes),
                    max_kv=max(self.kv) if max_kv is None else max_kv)

    def call(self, g, ws=None, stream=None, lse=True, **shape):
        shape = self.shape(**shape)
        if ws is None:
            ws = B.zeroed_workspace(B.adt_tree_attn_q8_workspace_size(**shape))
        B.adt_tree_attn_q8(g["q"], g["kc"], g["vc"], g["ks"], g["vs"], g["kv"], g["kt"], g["vt"], g["parents"], g["offs"],
                           softmax_scale=self.scale, out=g["out"], lse=g["lse"] if lse else None, workspace=ws, stream=stream,
                           **shape)
        return ws

    def check(self, g, trees=None):
        got, got_lse = g["out"].double().cpu().numpy(), g["lse"].double().cpu().numpy()
        args = (self.kv, self.kt.double().numpy())
        q = self.q.double().numpy()
        vt = self.vt.double().numpy()
        ref, lse = oracle.tree_attention(q, self.kval, self.vval, *args, vt, self.tb.parents, self.tb.node_offsets, self.scale)
        A, _ = oracle.tree_attention(q, self.kval, np.abs(self.vval), *args, np.abs(vt), self.tb.parents, self.tb.node_offsets,
                                     self.scale)
        for b in trees if trees is not None else range(self.B):
            n0, n1 = self.tb.node_offsets[b:b + 2]
            k = np.concatenate([self.kval[b, :, :self.kv[b]], self.kt.double().numpy()[n0:n1].transpose(1, 0, 2)], 1)
            qq = np.abs(q[n0:n1])
            kk = np.repeat(np.abs(k), self.H // self.Hkv, 0)  # [H, keys, D]
            S = self.scale * (qq.max(-1) * kk.sum(-1).max(-1) + qq.sum(-1) * kk.max((-1, -2)))
            T = self.scale * np.sqrt((qq ** 2).sum(-1) * (kk ** 2).sum(-1).max(-1))
            d = 2.0 ** -16 * S + 2.0 ** -17 * (1 + T)
            assert d.max() < 0.05
            err = np.abs(got[n0:n1] - ref[n0:n1])
            bound = A[n0:n1] * (2.0 ** -8 + 4 * d)[..., None] + 2.0 ** -8 * np.abs(ref[n0:n1])
            assert (err <= bound).all(), (b, np.nanmax(err - bound), np.isnan(got[n0:n1]).sum())
            assert (np.abs(got_lse[n0:n1] - lse[n0:n1]) <= 2 * d).all(), (b, np.abs(got_lse[n0:n1] - lse[n0:n1]).max())


@pytest.mark.parametrize("sizes,kv,H,Hkv,D", [
    ([1], [0], 1, 1, 64), ([1], [1], 8, 8, 64), ([1], [127], 4, 1, 128), ([1], [128], 8, 2, 64), ([1], [129], 32, 8, 128),
    ([1], [2400], 32, 32, 128), ([1] * 5, [0, 1, 600, 4097, 128], 8, 2, 128), ([1] * 3, [3000, 17, 64], 20, 5, 64),
    ([26], [512], 8, 8, 64), ([64], [700], 8, 8, 128), ([64, 1, 27, 33], [300, 900, 0, 129], 8, 8, 128),
    ([64, 64, 5], [1000, 0, 513], 8, 2, 128), ([40, 64], [255, 257], 12, 3, 64), ([65], [130], 4, 4, 64),
    ([128, 100], [256, 77], 4, 2, 128), ([129, 3], [1, 300], 3, 1, 64), ([192, 50, 192], [693, 0, 577], 10, 5, 64),
    ([256], [400], 4, 1, 128), ([256, 1], [0, 129], 2, 2, 128), ([200], [300], 7, 1, 64), ([33], [200], 21, 1, 128),
    ([5], [300], 40, 1, 64), ([2, 2], [150, 20], 160, 1, 64), ([3], [1500], 130, 1, 128)])
def test_matches_oracle(sizes, kv, H, Hkv, D):
    case = Case(sizes, kv, H, Hkv, D)
    g = case.dev()
    case.call(g)
    case.check(g)
    assert B.adt_get_device_error() == 0


@pytest.mark.parametrize("n,H,Hkv", [(16, 2, 2), (17, 2, 2), (32, 3, 3), (33, 2, 2), (4, 8, 2), (5, 6, 2), (8, 4, 1), (9, 8, 2),
                                     (1, 16, 1), (1, 17, 1), (1, 32, 1), (1, 33, 1), (64, 1, 1), (13, 5, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_numbers_of_rows_at_which_another_kernel_begins(n, H, Hkv, D):
    case = Case([n, max(n - 1, 1)], [389, 95], H, Hkv, D)
    g = case.dev()
    case.call(g)
    case.check(g)
    assert B.adt_get_device_error() == 0


@pytest.mark.parametrize("sizes,kv,H,Hkv,D", [([64, 9], [512, 100], 8, 4, 64), ([1, 1], [1000, 30], 16, 4, 128)])
def test_longer_caches_and_larger_trees_than_there_are(sizes, kv, H, Hkv, D):
    case = Case(sizes, kv, H, Hkv, D, spare=5000)
    g = case.dev()
    case.call(g, max_nodes=256, max_kv=max(kv) + 4999)
    case.check(g)
    outs = g["out"].clone()
    case.call(g, max_nodes=200, max_kv=max(kv))
    case.check(g)
    assert (outs.double() - g["out"].double()).abs().max() < 0.1


def test_chains_of_256_and_scores_far_apart():
    case = Case([256, 190], [100, 260], 2, 1, 128, chain=True, qstd=6.0)
    g = case.dev()
    case.call(g)
    case.check(g)


def test_one_key_takes_nearly_all_and_the_rest_still_counts():
    """A row of the cache whose key draws e^12 of the others' weight, with values of next to nothing."""
    case = Case([4, 1], [3000, 1500], 4, 2, 64, qstd=0.2)
    for b in range(2):
        big = case.kval[b, :, 3].copy()
        case.q[case.tb.node_offsets[b]:case.tb.node_offsets[b + 1]] += torch.from_numpy(
            np.repeat(big / (big ** 2).sum(-1, keepdims=True) * 12 / case.scale, 2, 0)).to(torch.bfloat16)
        case.vs[b, :, 3] = 90
    case.vval = oracle.q8_values(case.vc.view(torch.uint8).numpy(), case.vs.numpy())
    g = case.dev()
    case.call(g)
    case.check(g)


@pytest.mark.parametrize("H,Hkv,D", [(8, 2, 64), (4, 4, 128)])
def test_rows_behind_the_length_are_not_used(H, Hkv, D):
    case = Case([30, 1, 7], [130, 64, 0], H, Hkv, D, spare=300)
    g = case.dev()
    case.call(g, max_kv=400)
    want = g["out"].clone(), g["lse"].clone()
    for b, L in enumerate(case.kv):
        for c, s in (("kc", "ks"), ("vc", "vs")):
            g[c].view(torch.uint8)[b, :, L:] = 0x7F  # NaN
            g[s][b, :, L:] = 255
    case.call(g, max_kv=400)
    assert torch.equal(g["out"], want[0]) and torch.equal(g["lse"], want[1])
    case.check(g)


def test_strides_offsets_and_an_absent_lse():
    """Caches with K and V in turn and trees apart, scales that start at odd addresses; rows of out behind the last
    node stay as they were."""
    case = Case([9, 20], [77, 203], 6, 2, 128)
    g = case.dev()
    store = torch.zeros((2, 2, 2, case.rows + 9, 128), dtype=torch.uint8, device="cuda")
    flat = torch.zeros(2 * 2 * 2 * (case.rows + 3) + 1, dtype=torch.uint8, device="cuda")[1:].view(2, 2, 2, case.rows + 3)
    for j, (c, s) in enumerate((("kc", "ks"), ("vc", "vs"))):
        store[:, j, :, :case.rows] = g[c].view(torch.uint8)
        flat[:, :, j, :case.rows] = g[s]
        g[c], g[s] = store[:, j].view(torch.float8_e4m3fn), flat[:, :, j]
    out = torch.full((case.n + 4, 6, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    whole, g["out"] = out, out[:case.n]
    case.call(g)
    case.check(g)
    first = g["out"].clone()
    case.call(g, lse=False)
    assert torch.equal(first, g["out"]) and (whole[case.n:] == 9).all()


def test_tree_values_of_other_sizes_than_the_caches():
    """A tree whose keys and values are thousands of times the cache's, or nothing at all."""
    case = Case([12, 12], [90, 300], 4, 2, 64)
    case.vt[:12] *= 3000
    case.kt[3] *= 40
    case.kt[14], case.vt[15], case.q[5] = 0, 0, 0
    g = case.dev()
    case.call(g)
    case.check(g)


def test_values_that_are_not_finite_reach_those_who_see_them_only():
    case = Case([8, 8], [40, 40], 4, 2, 64, chain=True)
    g = case.dev()
    case.call(g)
    clean = g["out"].clone()
    g["kt"][5, 1] = float("nan")     # seen by nodes 5, 6, 7 of tree 0, heads 2 and 3
    g["vt"][2, 0, 7] = float("inf")  # column 7 of heads 0 and 1 of nodes 2 .. 7
    g["ks"][1, 0, 17] = 255          # a cached row of tree 1, heads 0 and 1
    case.call(g)
    bad = ~torch.isfinite(g["out"])
    want = torch.zeros_like(bad)
    want[5:8, 2:] = True
    want[2:8, :2, 7] = True
    want[8:, :2] = True
    assert torch.equal(bad, want)
    assert torch.equal(g["out"][~bad], clean[~bad])
    g["q"][9, 1, 3] = float("nan")
    g["ks"][1, 0, 17] = 120
    case.call(g)
    assert torch.isnan(g["out"][9, 1]).all() and torch.isfinite(g["out"][8]).all() and torch.isfinite(g["out"][9, [0, 2, 3]]).all()


@pytest.mark.parametrize("change,error", [("kv-", B.DEVERR_KV_RANGE), ("kv+", B.DEVERR_KV_RANGE), ("root", B.DEVERR_BAD_TREE),
                                          ("later", B.DEVERR_BAD_TREE), ("orphan", B.DEVERR_BAD_TREE), ("size", B.DEVERR_BAD_TREE)])
@pytest.mark.parametrize("H,Hkv", [(4, 4), (4, 1)])
def test_a_bad_tree_leaves_the_others_right(change, error, H, Hkv):
    case = Case([40, 40, 40], [200, 150, 420], H, Hkv, 64)
    g = case.dev()
    kw = {}
    if change[:2] == "kv":
        g["kv"][1] = -1 if change == "kv-" else 1000
    elif change == "root":
        g["parents"][40] = 0
    elif change == "later":
        g["parents"][40 + 39] = 39
    elif change == "orphan":
        g["parents"][40 + 30] = -1
    else:  # (max_nodes smaller than one of the trees)
        case = Case([40, 41, 40], [200, 150, 420], H, Hkv, 64)
        g, kw = case.dev(), dict(max_nodes=40)
    ws = case.call(g, **kw)
    assert B.adt_get_device_error() == error
    case.check(g, trees=[0, 2])
    ws.zero_()
    if change == "size":
        return
    g["kv"], g["parents"] = i32(case.kv), i32(case.tb.parents)
    case.call(g, ws=ws, **kw)
    case.check(g)
    assert B.adt_get_device_error() == 0


def test_equal_calls_give_equal_bits_and_one_workspace_serves_any_shape():
    cases = [Case([1] * 4, [5000, 30, 700, 64], 8, 2, 128), Case([64], [300], 8, 8, 64), Case([100, 7], [257, 1000], 6, 3, 128)]
    ws = B.zeroed_workspace(max(B.adt_tree_attn_q8_workspace_size(**c.shape()) for c in cases))
    first = []
    for turn in range(3):
        for c in cases:
            g = c.dev()
            c.call(g, ws=ws)
            if turn == 0:
                c.check(g)
                first.append((g["out"], g["lse"]))
            else:
                f = first[cases.index(c)]
                assert torch.equal(f[0], g["out"]) and torch.equal(f[1], g["lse"])
    assert B.adt_get_device_error() == 0


@pytest.mark.parametrize("H,Hkv,D", [(8, 8, 64), (8, 2, 128)])
def test_many_items_of_one_chunk(H, Hkv, D):
    """Trees without a prefix, or with next to none: a thread block has many items, each one or two chunks."""
    case = Case([1, 2, 1, 5] * 18, [0, 3, 0, 130] * 18, H, Hkv, D)
    g = case.dev()
    ws = case.call(g)
    case.check(g)
    first = g["out"].clone()
    for _ in range(5):
        case.call(g, ws=ws)
        assert torch.equal(first, g["out"])
    assert B.adt_get_device_error() == 0


@pytest.mark.parametrize("sizes,kv,H,Hkv,D", [([64, 27, 64, 64], [1300, 900, 1444, 1352], 32, 32, 128),
                                              ([64, 64, 5], [2001, 777, 1500], 32, 8, 128), ([1] * 9, [3000, 1, 900, 128, 5000, 0, 64, 700, 2049], 16, 4, 64)])
def test_calls_whose_inputs_come_from_memory(sizes, kv, H, Hkv, D):
    """The roles of a thread block at other speeds: every call after writes larger than L2, all with equal bits."""
    case = Case(sizes, kv, H, Hkv, D, max_depth=12)
    g = case.dev()
    other = torch.empty(400 << 20, dtype=torch.uint8, device="cuda")
    ws = case.call(g)
    first, lse = g["out"].clone(), g["lse"].clone()
    for i in range(25):
        other.fill_(i)
        g["out"].zero_()
        case.call(g, ws=ws)
        assert torch.equal(first, g["out"]) and torch.equal(lse, g["lse"]), i
    assert B.adt_get_device_error() == 0
    case.check(g)


def test_waits_that_run_out_end_the_call_with_an_error():
    case = Case([64, 9], [900, 300], 8, 4, 128)
    g = case.dev()
    ws = case.call(g)
    case.check(g)
    B.adt_testing_set_wait_limit(1)
    try:
        case.call(g, ws=ws)
        torch.cuda.synchronize()
        assert B.adt_get_device_error() & B.DEVERR_TIMEOUT
    finally:
        B.adt_testing_set_wait_limit(0)
    ws.zero_()
    case.call(g, ws=ws)
    case.check(g)
    assert B.adt_get_device_error() == 0


@pytest.mark.parametrize("H,Hkv,D", [(4, 2, 64), (4, 4, 128), (128, 1, 64)])
def test_cached_bytes_that_are_not_numbers(H, Hkv, D):
    case = Case([3, 1], [200, 77], H, Hkv, D)
    g = case.dev()
    case.call(g)
    clean = g["out"].clone()
    g["vc"].view(torch.uint8)[0, Hkv - 1, 150, 9] = 0xFF  # a column of the last kv head's heads, tree 0
    g["kc"].view(torch.uint8)[1, 0, 60, 5] = 0x7F        # all of the first kv head's, tree 1
    case.call(g)
    want = torch.zeros_like(clean, dtype=torch.bool)
    group = H // Hkv
    want[:3, H - group:, 9] = True
    want[3, :group] = True
    assert torch.equal(torch.isnan(g["out"]), want) and torch.equal(g["out"][~want], clean[~want])


@pytest.mark.parametrize("sizes,kv,H,Hkv,D", [([1, 1, 1], [700, 1000, 300], 8, 2, 128), ([1, 4, 2], [700, 1000, 300], 8, 2, 64),
                                              ([8, 1, 5], [700, 1000, 300], 8, 2, 128), ([40, 9, 64], [700, 1000, 300], 4, 2, 64)])
def test_value_scales_far_apart(sizes, kv, H, Hkv, D):
    """Tree 0: two of three rows next to nothing, or zeros.  Tree 1: scales that rise along the cache.  Tree 2: no value
    but zeros, whose scale is the least there is."""
    case = Case(sizes, kv, H, Hkv, D)
    at = torch.arange(case.rows)
    case.vs[0, :, at % 3 == 0] = 20
    case.vs[0, :, at % 3 == 1] = 7
    case.vc.view(torch.uint8)[0, :, at % 3 == 1] = 0
    case.vs[1] = (30 + at // 130 * 21).clamp(max=200).to(torch.uint8)
    case.vc.view(torch.uint8)[2], case.vs[2] = 0, 7
    case.vt[case.tb.node_offsets[2]:] = 0
    case.vval = oracle.q8_values(case.vc.view(torch.uint8).numpy(), case.vs.numpy())
    g = case.dev()
    case.call(g)
    case.check(g)
    assert (g["out"][case.tb.node_offsets[2]:] == 0).all()
    # A value that is not a number takes its rows' outputs, and leaves the weights' sum.
    want = g["lse"].clone()
    g["vs"][2, 0, 200] = 255
    case.call(g)
    n, group = case.tb.node_offsets[2], H // Hkv
    assert torch.isnan(g["out"][n:, :group]).all() and (g["out"][n:, group:] == 0).all()
    # (Exponents of up to 256, in fp32: 2^-17 of a weight each time, and of the sum's exponent.)
    assert ((g["lse"] - want).abs() <= 2.0 ** -15).all() and B.adt_get_device_error() == 0


@pytest.mark.parametrize("sizes,H,Hkv,D", [([1], 4, 1, 128), ([2], 8, 1, 64), ([8], 4, 1, 128), ([64], 1, 1, 64)])
@pytest.mark.parametrize("step", [5.0, 0.5])
def test_scores_that_grow_along_the_cache(sizes, H, Hkv, D, step):
    """Every chunk's largest score is above all before, by more than what is let pass without scaling O, or less."""
    case = Case(sizes, [2500], H, Hkv, D)
    r = synth.rng(7, "grow")
    base = r.standard_normal(D)
    case.q = torch.from_numpy(np.tile(base, (case.n, H, 1))).to(torch.bfloat16)
    scores = np.arange(case.rows) * (step / 128) + r.standard_normal(case.rows) * 0.3 - step * 19
    keys = scores[:, None] * base / ((base ** 2).sum() * case.scale)
    kc, ks = oracle.q8_rows(keys)
    case.kc[0, 0], case.ks[0, 0] = torch.from_numpy(kc).view(torch.float8_e4m3fn), torch.from_numpy(ks)
    case.kval = oracle.q8_values(case.kc.view(torch.uint8).numpy(), case.ks.numpy())
    g = case.dev()
    ws = case.call(g)
    case.check(g)
    first = g["out"].clone()
    other = torch.empty(400 << 20, dtype=torch.uint8, device="cuda")
    for i in range(10):
        other.fill_(i)
        case.call(g, ws=ws)
        assert torch.equal(first, g["out"])
    assert B.adt_get_device_error() == 0


def test_another_stream_and_two_graphs_with_one_workspace():
    a, b = Case([1, 1], [3000, 700], 8, 2, 128), Case([64, 64], [300, 129], 8, 8, 64)
    ws = B.zeroed_workspace(max(B.adt_tree_attn_q8_workspace_size(**c.shape(max_kv=c.rows)) for c in (a, b)))
    ga, gb = a.dev(), b.dev()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a.call(ga, ws=ws, stream=s, max_kv=a.rows)
    s.synchronize()
    a.check(ga)
    graphs = []
    for c, g in ((a, ga), (b, gb)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.call(g, ws=ws, max_kv=c.rows)
    for _ in range(3):
        for g in (ga, gb):
            g["out"].zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        a.check(ga)
        b.check(gb)
    a.kv = [2999, 703]  # lengths are read at each replay
    ga["kv"].copy_(i32(a.kv))
    graphs[0].replay()
    a.check(ga)
    assert B.adt_get_device_error() == 0


def test_binding_refuses():
    case = Case([2], [5], 2, 1, 64)
    g = case.dev()
    for name, t, err in [("kc", g["kc"].view(torch.uint8), TypeError), ("ks", g["ks"].int(), TypeError), ("q", g["q"].float(), TypeError),
                         ("kc", g["kc"][:, :, :4], ValueError), ("ks", g["ks"][:, :, :4], ValueError),
                         ("kt", g["kt"][:1], ValueError), ("out", g["out"][:1], ValueError), ("parents", g["parents"][:1], ValueError),
                         ("lse", g["lse"][:1], ValueError), ("kv", g["kv"].long(), TypeError), ("vs", g["vs"].cpu(), ValueError)]:
        with pytest.raises(err):
            case.call(dict(g, **{name: t}))
    with pytest.raises(B.AdtError) as e:
        case.call(g, ws=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 5


def test_norm_commit_and_attention_together():
    """As a decoding step uses them: the projection's rows normed and rotated, attention over the 8-bit cache, the
    accepted path committed, the next token's attention; and the cache read back as bf16 gives adt_tree_attn the same."""
    H, Hkv, D, L, n, rows = 8, 2, 128, 300, 12, 330
    r = synth.rng(5, "chain")
    kc, ks, kval = quantised((1, Hkv, rows, D), 5, "k")
    vc, vs, vval = quantised((1, Hkv, rows, D), 5, "v")
    tb = synth.tree_batch([n], 100, 5, max_depth=4, max_children=4)
    proj = torch.from_numpy(r.standard_normal((n, (H + 2 * Hkv) * D)).astype(np.float32)).to(torch.bfloat16).cuda()
    w = torch.from_numpy(1 + 0.1 * r.standard_normal(D).astype(np.float32)).cuda()
    depth = np.array([len(oracle.ancestor_path(tb.parents, t)) - 1 for t in range(n)], np.int32)
    q, k, v = (torch.empty((n, h, D), dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv))
    inv = torch.from_numpy(oracle.rope_freqs(D)[0]).cuda()
    B.adt_norm_rope_qkv(*proj.split([H * D, Hkv * D, Hkv * D], 1), i32(L + depth), inv, H=H, Hkv=Hkv, D=D, q_weight=w, k_weight=w,
                        q_out=q, k_out=k, v_out=v)
    case = Case([n], [L], H, Hkv, D)
    case.tb, case.rows, case.kval, case.vval = tb, rows, kval, vval
    case.kc, case.ks, case.vc, case.vs, case.q, case.kt, case.vt = kc, ks, vc, vs, q.cpu(), k.cpu(), v.cpu()
    g = case.dev()
    case.call(g, max_kv=rows)
    case.check(g)
    path = oracle.ancestor_path(tb.parents, int(depth.argmax()))
    kv_out = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = dict(B=1, Hkv=Hkv, D=D, num_layers=1, max_kv=rows)
    caches = [g[x][None] for x in ("kc", "vc", "ks", "vs")]
    B.adt_kv_compact_q8(*caches, g["kv"], kv_out, k[None], v[None], g["offs"], i32([path]), len(path), i32([len(path) - 1]), **shape)
    nxt = Case([1], [L + len(path)], H, Hkv, D)
    assert kv_out.cpu().tolist() == nxt.kv
    nxt.rows = rows
    nxt.kc, nxt.vc, nxt.ks, nxt.vs = (x[0].cpu() for x in caches)
    nxt.kval, nxt.vval = (oracle.q8_values(c.view(torch.uint8).numpy(), s.numpy()) for c, s in ((nxt.kc, nxt.ks), (nxt.vc, nxt.vs)))
    g = nxt.dev()
    nxt.call(g, max_kv=rows)
    nxt.check(g)
    wide = [torch.zeros((1, 1, Hkv, rows, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.adt_kv_read_q8(*caches, kv_out, *wide, **shape)
    out = torch.empty_like(g["out"])
    B.adt_tree_attn(g["q"], wide[0][0], wide[1][0], g["kv"], g["kt"], g["vt"], g["parents"], g["offs"], B=1, H=H, Hkv=Hkv, D=D,
                    max_nodes=1, max_kv=rows, softmax_scale=nxt.scale, out=out,
                    workspace=B.zeroed_workspace(B.adt_tree_attn_workspace_size(1, H, D, 1, rows)))
    assert (out.double() - g["out"].double()).abs().max() < 2e-2


@pytest.mark.parametrize("n,H,Hkv,D", [(64, 4, 4, 128), (40, 8, 2, 64), (8, 4, 2, 128), (1, 8, 8, 64)])
def test_steps_one_after_the_other_read_what_the_commits_before_wrote(n, H, Hkv, D):
    """Attention, commit, attention, ..., never waited for, equal the same with the device idle before every call."""
    steps, L, take = 30, 200, min(n, 3)
    rows = L + steps * take
    case = Case([n], [L], H, Hkv, D, spare=steps * take, chain=True)
    shape = dict(B=1, Hkv=Hkv, D=D, num_layers=1, max_kv=rows)
    other = torch.empty(300 << 20, dtype=torch.uint8, device="cuda")

    def run(idle):
        g = case.dev()
        ws = B.zeroed_workspace(B.adt_tree_attn_q8_workspace_size(**case.shape(max_kv=rows)))
        kv = [i32([L]) for _ in range(steps + 1)]
        kt, vt = g["kt"].clone(), g["vt"].clone()
        outs = [torch.empty_like(g["out"]) for _ in range(steps)]
        path, alen = i32([list(range(take))]), i32([take - 1])
        for i in range(steps):
            if idle:
                torch.cuda.synchronize()
                other.fill_(i)
                torch.cuda.synchronize()
            g["out"], g["kv"] = outs[i], kv[i]
            case.call(g, ws=ws, lse=False, max_kv=rows)
            if idle:
                torch.cuda.synchronize()
            B.adt_kv_compact_q8(g["kc"][None], g["vc"][None], g["ks"][None], g["vs"][None], kv[i], kv[i + 1], kt[None], vt[None],
                                g["offs"], path, take, alen, **shape)
        assert kv[steps].item() == rows
        return torch.stack(outs)

    want = run(True)
    for _ in range(5):
        assert torch.equal(run(False), want)
    assert B.adt_get_device_error() == 0
