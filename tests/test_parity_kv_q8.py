"""adt_kv_compact_q8 and adt_kv_read_q8 on the GPU: bytes, scales and values equal those of the oracle; all else in
their buffers stays as it was."""
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


def cache_of(layers, nb, Hkv, rows, D, seed):
    """Caches and scales full of what no commit writes there, K and V as views of one allocation."""
    r = synth.rng(seed, "cache")
    kv = torch.from_numpy(r.integers(0, 127, size=(layers, nb, 2, Hkv, rows, D)).astype(np.uint8)).cuda()
    s = torch.from_numpy(r.integers(100, 140, size=(layers, nb, 2, Hkv, rows)).astype(np.uint8)).cuda()
    return kv[:, :, 0].view(torch.float8_e4m3fn), kv[:, :, 1].view(torch.float8_e4m3fn), s[:, :, 0], s[:, :, 1]


def u8(t):
    return t.view(torch.uint8).cpu().numpy()


def case_of(layers, Hkv, D, kv, sizes, paths, max_path, seed):
    nb, offs = len(kv), np.concatenate([[0], np.cumsum(sizes)])
    tree = [synth.bf16_normal((layers, int(offs[-1]) + 3, Hkv, D), seed, n, std=2.0) for n in ("kt", "vt")]
    tree[0][:, ::3] *= 2.0 ** 20
    tree[1][:, ::5] *= 2.0 ** -60
    tree[0][-1, 0, -1, 0], tree[1][0, 0, 0, D - 1], tree[1][0, -1, 0] = float("inf"), float("nan"), 0.0
    p = np.full((nb, max_path), -1, np.int32)
    for b, path in enumerate(paths):
        p[b, :len(path)] = path
    return offs, tree, p


@pytest.mark.parametrize("layers,Hkv,D,kv,sizes,paths,max_path", [
    (1, 8, 64, [5], [26], [[0]], 1),
    (2, 32, 128, [0, 17], [64, 9], [[0, 1, 5, 63], [0]], 8),
    (1, 1, 64, [3], [1], [[0]], 6),
    (3, 5, 128, [9, 0, 30], [40, 70, 33], [list(range(33)), list(range(0, 70, 2)), [0]], 64),
    (2, 20, 64, [0, 1], [300, 257], [list(range(300)), list(range(257))], 300),
    (1, 3, 128, [1], [5], [[0, 4, 4, 2]], 5),  # the same node twice, any order
])
def test_commit_equals_the_oracle(layers, Hkv, D, kv, sizes, paths, max_path):
    nb, rows, max_kv = len(kv), max(kv) + max_path + 3, max(kv) + max_path + 1
    offs, tree, p = case_of(layers, Hkv, D, kv, sizes, paths, max_path, seed=D + Hkv)
    kc, vc, ks, vs = cache_of(layers, nb, Hkv, rows, D, 3)
    want = [u8(t).copy() for t in (kc, vc, ks, vs)]
    for j, t in enumerate(tree):
        q, s = oracle.q8_rows(t.double().numpy())
        for b, path in enumerate(paths):
            for i, node in enumerate(path):
                want[j][:, b, :, kv[b] + i] = q[:, offs[b] + node]
                want[2 + j][:, b, :, kv[b] + i] = s[:, offs[b] + node]
    out = torch.full((nb,), -5, dtype=torch.int32, device="cuda")
    B.adt_kv_compact_q8(kc, vc, ks, vs, i32(kv), out, tree[0].cuda(), tree[1].cuda(), i32(offs), i32(p), max_path,
                        i32([len(x) - 1 for x in paths]), B=nb, Hkv=Hkv, D=D, num_layers=layers, max_kv=max_kv)
    for got, w in zip((kc, vc, ks, vs), want):
        np.testing.assert_array_equal(u8(got), w)
    assert out.cpu().tolist() == [L + len(x) for L, x in zip(kv, paths)]
    assert B.adt_get_device_error() == 0


def test_every_bf16_value_rounds_as_the_oracle_says():
    """Rows that hold all bf16 bit patterns, in order, beside others that shift the scale."""
    D, Hkv = 64, 4
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(1, 256, Hkv, D)
    other = (bits.float().flip(0) * 3).to(torch.bfloat16).roll(7, -1)
    n = bits.shape[1]
    kc, vc, ks, vs = cache_of(1, 1, Hkv, n, D, 4)
    B.adt_kv_compact_q8(kc, vc, ks, vs, i32([0]), None, bits.cuda(), other.cuda(), i32([0, n]), i32(np.arange(n)[None]), n,
                        i32([n - 1]), B=1, Hkv=Hkv, D=D, num_layers=1, max_kv=n)
    for t, c, s in ((bits, kc, ks), (other, vc, vs)):
        q, e = oracle.q8_rows(t.double().numpy()[0])
        np.testing.assert_array_equal(u8(s)[0, 0].T, e)
        np.testing.assert_array_equal(u8(c)[0, 0].transpose(1, 0, 2), q)


@pytest.mark.parametrize("change,error", [
    (dict(alen=[1, -1]), B.DEVERR_KV_RANGE), (dict(alen=[1, 4]), B.DEVERR_KV_RANGE), (dict(kv=[2, -1]), B.DEVERR_KV_RANGE),
    (dict(kv=[2, 9]), B.DEVERR_KV_RANGE), (dict(path=[0, 7]), B.DEVERR_BAD_PATH), (dict(path=[1, 2]), B.DEVERR_BAD_PATH),
    (dict(path=[0, -1]), B.DEVERR_BAD_PATH)])
def test_a_bad_tree_is_skipped_by_itself(change, error):
    D, Hkv, rows = 64, 2, 10
    kv, alen, path = change.get("kv", [2, 3]), change.get("alen", [1, 1]), change.get("path", [0, 2])
    offs, tree, p = case_of(1, Hkv, D, kv, [4, 7], [[0, 3], path], 4, 5)
    kc, vc, ks, vs = cache_of(1, 2, Hkv, rows, D, 6)
    before = [u8(t).copy() for t in (kc, vc, ks, vs)]
    out = torch.full((2,), -5, dtype=torch.int32, device="cuda")
    B.adt_kv_compact_q8(kc, vc, ks, vs, i32(kv), out, tree[0].cuda(), tree[1].cuda(), i32(offs), i32(p), 4, i32(alen), B=2,
                        Hkv=Hkv, D=D, num_layers=1, max_kv=rows)
    assert B.adt_get_device_error() == error
    assert out.cpu().tolist() == [4, kv[1]]
    for got, w in zip((kc, vc, ks, vs), before):
        np.testing.assert_array_equal(u8(got)[:, 1], w[:, 1])
        assert (u8(got)[:, 0, :, 2:4] != w[:, 0, :, 2:4]).any()


@pytest.mark.parametrize("layers,Hkv,D,kv,rows", [(1, 8, 64, [512], 576), (3, 2, 128, [0, 1, 200], 201), (2, 5, 64, [77, 300], 300),
                                                  (1, 1, 128, [1], 1)])
def test_read_equals_the_oracle(layers, Hkv, D, kv, rows):
    nb = len(kv)
    r = synth.rng(D + rows, "cache")
    c = [torch.from_numpy(r.integers(0, 256, size=(layers, nb, Hkv, rows, D)).astype(np.uint8)).cuda() for _ in range(2)]
    s = [torch.from_numpy(r.integers(7, 248, size=(layers, nb, Hkv, rows)).astype(np.uint8)).cuda() for _ in range(2)]
    s[0][0, -1, 0, 0] = 255
    store = torch.full((nb, layers, 2, Hkv, rows + 2, D), 3.0, dtype=torch.bfloat16, device="cuda")  # other strides than the caches'
    out = [store[:, :, j].transpose(0, 1) for j in range(2)]
    B.adt_kv_read_q8(*(x.view(torch.float8_e4m3fn) for x in c), *s, i32(kv), *out, B=nb, Hkv=Hkv, D=D, num_layers=layers,
                     max_kv=rows)
    for x, e, o in zip(c, s, out):
        want = torch.full_like(o, 3.0)
        for b, L in enumerate(kv):
            v = torch.from_numpy(oracle.q8_values(x[:, b, :, :L].cpu().numpy(), e[:, b, :, :L].cpu().numpy()))
            want[:, b, :, :L] = v.to(torch.float64).to(torch.bfloat16).cuda()
        assert torch.equal(o.isnan(), want.isnan()) and torch.equal(o.nan_to_num(5.0), want.nan_to_num(5.0))
    assert B.adt_get_device_error() == 0


def test_read_skips_a_tree_whose_length_is_out_of_range():
    c, s = torch.zeros(1, 3, 2, 8, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.full(
        (1, 3, 2, 8), 127, dtype=torch.uint8, device="cuda")
    out = [torch.full((1, 3, 2, 8, 64), 2.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for bad in (-1, 9):
        B.adt_kv_read_q8(c, c, s, s, i32([3, bad, 8]), *out, B=3, Hkv=2, D=64, num_layers=1, max_kv=8)
        assert B.adt_get_device_error() == B.DEVERR_KV_RANGE
    for o in out:
        assert (o[:, 1] == 2).all() and (o[:, 2] == 0).all() and (o[:, 0, :, :3] == 0).all() and (o[:, 0, :, 3:] == 2).all()


def test_commit_and_read_in_a_graph_and_on_another_stream():
    D, Hkv, layers, n, rows = 128, 4, 2, 6, 40
    offs, tree, p = case_of(layers, Hkv, D, [0], [n], [[0, 2, 5]], 3, 8)
    kc, vc, ks, vs = cache_of(layers, 1, Hkv, rows, D, 9)
    kv, p, kt, vt, offs, alen = i32([4]), i32(p), tree[0].cuda(), tree[1].cuda(), i32(offs), i32([2])
    kv_out = torch.zeros_like(kv)
    out = [torch.zeros((layers, 1, Hkv, rows, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shape = dict(B=1, Hkv=Hkv, D=D, num_layers=layers, max_kv=rows)

    def step(stream=None):
        B.adt_kv_compact_q8(kc, vc, ks, vs, kv, kv_out, kt, vt, offs, p, 3, alen, **shape, stream=stream)
        B.adt_kv_read_q8(kc, vc, ks, vs, kv_out, *out, **shape, stream=stream)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(s)
    s.synchronize()
    first = [o.clone() for o in out]
    q, e = oracle.q8_rows(tree[0].double().numpy())
    want = oracle.q8_values(q, e)[:, [0, 2, 5]].transpose(0, 2, 1, 3)
    np.testing.assert_array_equal(first[0][:, 0, :, 4:7].double().cpu().numpy(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for o in out:
        o.zero_()
    graph.replay()
    for o, f in zip(out, first):
        assert torch.equal(o.nan_to_num(5.0), f.nan_to_num(5.0))
    kv += 9
    graph.replay()
    np.testing.assert_array_equal(out[0][:, 0, :, 13:16].double().cpu().numpy(), want)
    assert int(kv_out) == 16 and B.adt_get_device_error() == 0
