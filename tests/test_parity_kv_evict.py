"""adt_kv_evict on the GPU against the oracle: rows, bytes and indices are equal."""
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


def make_score(kind, shape, seed):
    g = synth.rng(seed, "score")
    if kind == "spread":
        return np.exp(2 * g.standard_normal(shape)).astype(np.float32)
    if kind == "ties":   # few values, zeros of both signs
        return np.array([0.0, -0.0, 0.25, 0.5, 3.0], np.float32)[g.integers(0, 5, shape)]
    if kind == "equal":
        return np.full(shape, 1.5, np.float32)
    if kind == "close":  # apart in the last bits only
        return (1.0 + g.integers(0, 40, shape) * 2.0 ** -23).astype(np.float32)
    odd = np.array([np.nan, -np.nan, np.inf, -np.inf, 3.4e38, -3.4e38, 1e-45, -1e-45, 0.0, 1.0], np.float32)
    return odd[g.integers(0, len(odd), shape)]


class Case:
    def __init__(self, layers, Hkv, D, kv, lmax, kind, seed):
        self.layers, self.Hkv, self.D, self.kv, self.lmax = layers, Hkv, D, kv, lmax
        shape = (layers, len(kv), Hkv, lmax)
        self.kc, self.vc = (synth.bf16_normal(shape + (D,), seed, n) for n in ("kc", "vc"))
        self.score = make_score(kind, shape, seed)

    def kw(self, **more):
        return dict(dict(B=len(self.kv), Hkv=self.Hkv, D=self.D, num_layers=self.layers, max_kv=self.lmax), **more)

    def tensors(self):
        return self.kc.cuda(), self.vc.cuda(), torch.from_numpy(self.score).cuda(), i32(self.kv)

    def outputs(self, budget):
        n = len(self.kv)
        return torch.zeros(n, dtype=torch.int32, device="cuda"), torch.full((self.layers, n, self.Hkv, budget), 99,
                                                                            dtype=torch.int32, device="cuda")

    def oracle(self, budget, sink, recent, **dst):
        return oracle.kv_evict(bits(self.kc), bits(self.vc), self.score, self.kv, budget, sink, recent, **dst)


def bits(t):
    """bf16 or fp32 as integers: equal bytes, NaN among them."""
    return t.cpu().contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).numpy()


def same(got, want):
    k, v, s, n, idx = want
    assert np.array_equal(got[3].cpu().numpy(), n)
    if got[4] is not None:
        assert np.array_equal(got[4].cpu().numpy(), idx)
    assert np.array_equal(bits(got[0]), k) and np.array_equal(bits(got[1]), v)
    if got[2] is not None:
        assert np.array_equal(bits(got[2]), np.ascontiguousarray(s, np.float32).view(np.int32))


SHAPES = [
    # layers, Hkv, D, kv, budget, sink, recent
    (1, 1, 64, [1], 1, 0, 0),
    (1, 1, 128, [2], 1, 0, 0),
    (2, 2, 64, [0, 1, 5], 3, 1, 1),
    (1, 8, 64, [576], 512, 4, 32),
    (2, 3, 128, [31, 32, 33, 64], 32, 2, 8),
    (1, 2, 64, [1000], 1, 0, 1),                     # one row stays
    (1, 2, 64, [1000], 999, 0, 0),                   # one row goes
    (1, 2, 128, [700], 100, 60, 40),                 # nothing by score
    (1, 2, 128, [700, 90], 100, 0, 100),             # a sliding window
    (1, 2, 64, [700], 100, 100, 0),                  # the first rows only
    (2, 2, 128, [4095, 4096, 4097], 2000, 4, 64),    # around a window of rows
    (1, 1, 64, [9000], 8500, 4, 64),
    (1, 2, 128, [12289], 700, 0, 5),
    (40, 5, 64, [130, 60], 64, 1, 16),               # many slices
    (1, 2, 64, [300], 5000, 3, 100),                 # a budget past the capacity
    (3, 1, 128, [257, 1025, 513, 2049], 256, 0, 7),
    (1, 1, 128, [16500, 16384, 3], 9000, 4, 100),    # around a window of the launches for few long slices
]


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "close", "odd"])
@pytest.mark.parametrize("layers,Hkv,D,kv,budget,sink,recent", SHAPES)
def test_evict_in_place_matches_oracle(layers, Hkv, D, kv, budget, sink, recent, kind):
    c = Case(layers, Hkv, D, kv, max(kv) + 3, kind, seed=sum(kv) + budget)
    kc, vc, score, kv_len = c.tensors()
    n, idx = c.outputs(budget)
    B.adt_kv_evict(kc, vc, score, kv_len, n, keep_idx=idx, **c.kw(budget=budget, n_sink=sink, n_recent=recent))
    same((kc, vc, score, n, idx), c.oracle(budget, sink, recent))


@pytest.mark.parametrize("kind", ["spread", "ties"])
@pytest.mark.parametrize("layers,Hkv,D,kv,budget,sink,recent", SHAPES)
def test_evict_into_another_cache_matches_oracle(layers, Hkv, D, kv, budget, sink, recent, kind):
    c = Case(layers, Hkv, D, kv, max(kv) + 3, kind, seed=sum(kv) + budget)
    rows = min(budget, c.lmax) + 2
    shape = (layers, len(kv), Hkv, rows)
    dst = [synth.bf16_normal(shape + (D,), 9, n) for n in ("ko", "vo")] + [torch.rand(shape)]
    src = c.tensors()
    ko, vo, so = (t.cuda() for t in dst)
    n, idx = c.outputs(budget)
    B.adt_kv_evict(*src, n, k_out=ko, v_out=vo, score_out=so, keep_idx=idx,
                   **c.kw(budget=budget, n_sink=sink, n_recent=recent))
    same((ko, vo, so, n, idx), c.oracle(budget, sink, recent, k_dst=bits(dst[0]), v_dst=bits(dst[1]), score_dst=dst[2].numpy()))
    assert np.array_equal(bits(src[0]), bits(c.kc)) and np.array_equal(bits(src[2]), c.score.view(np.int32))


def test_evict_outputs_are_optional():
    c = Case(2, 2, 64, [300, 50], 310, "spread", 5)
    want = c.oracle(100, 4, 16)
    kc, vc, score, kv_len = c.tensors()
    B.adt_kv_evict(kc, vc, score, kv_len, **c.kw(budget=100, n_sink=4, n_recent=16), move_scores=False)
    assert np.array_equal(bits(kc), want[0]) and np.array_equal(bits(vc), want[1])
    assert np.array_equal(bits(score), c.score.view(np.int32))


def test_evict_scores_into_a_second_buffer():
    """Caches in place, scores to a buffer with strides of its own: the call can be made again with equal results."""
    c = Case(2, 2, 128, [300, 50], 310, "ties", 6)
    want = c.oracle(100, 4, 16, score_dst=np.zeros((2, 2, 2, 120), np.float32))
    for _ in range(2):
        kc, vc, score, kv_len = c.tensors()
        n, idx = c.outputs(100)
        so = torch.zeros((2, 2, 2, 120), device="cuda")
        B.adt_kv_evict(kc, vc, score, kv_len, n, score_out=so, keep_idx=idx, **c.kw(budget=100, n_sink=4, n_recent=16))
        same((kc, vc, so, n, idx), want)


def test_evict_with_strides_of_larger_caches():
    c = Case(2, 2, 64, [140, 60], 150, "spread", 7)
    kc, vc, score, kv_len = c.tensors()
    big = [torch.full((2, 3, 4, 160, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bs = torch.full((2, 4, 3, 170), 5.0, device="cuda")
    for x, t in zip(big, (kc, vc)):
        x[:, 1:, :2, :150] = t
    bs[:, 1:3, 1:, :150] = score
    n, idx = c.outputs(64)
    B.adt_kv_evict(big[0][:, 1:, :2], big[1][:, 1:, :2], bs[:, 1:3, 1:], kv_len, n, keep_idx=idx,
                   **c.kw(budget=64, n_sink=2, n_recent=9))
    same((big[0][:, 1:, :2, :150], big[1][:, 1:, :2, :150], bs[:, 1:3, 1:, :150], n, idx), c.oracle(64, 2, 9))
    for x in big:
        x[:, 1:, :2, :150] = 5.0
        assert (x == 5.0).all()
    bs[:, 1:3, 1:, :150] = 5.0
    assert (bs == 5.0).all()


def test_evict_flags_bad_lengths():
    c = Case(2, 2, 64, [140, 60, 90], 150, "spread", 8)
    want = c.oracle(64, 2, 9)
    for bad in (-1, 151, 2 ** 31 - 1, -2 ** 31):
        kc, vc, score, _ = c.tensors()
        n, idx = c.outputs(64)
        B.adt_get_device_error()
        B.adt_kv_evict(kc, vc, score, i32([140, bad, 90]), n, keep_idx=idx, **c.kw(budget=64, n_sink=2, n_recent=9))
        assert B.adt_get_device_error() == B.DEVERR_KV_RANGE
        assert n.tolist() == [64, bad, 64]
        assert np.array_equal(bits(kc[:, [0, 2]]), want[0][:, [0, 2]]) and np.array_equal(bits(kc[:, 1]), bits(c.kc[:, 1]))
        assert np.array_equal(bits(score[:, 1]), c.score[:, 1].view(np.int32)) and (idx[:, 1] == 99).all()


def test_evict_in_a_graph_on_another_stream():
    c = Case(3, 2, 64, [500, 130], 512, "spread", 9)
    want = c.oracle(128, 4, 32)
    kc, vc, score, kv_len = c.tensors()
    first = [t.clone() for t in (kc, vc, score)]
    n, idx = c.outputs(128)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    B.adt_kv_evict(kc, vc, score, kv_len, n, keep_idx=idx, **c.kw(budget=128, n_sink=4, n_recent=32), stream=s)
    s.synchronize()
    same((kc, vc, score, n, idx), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.adt_kv_evict(kc, vc, score, kv_len, n, keep_idx=idx, **c.kw(budget=128, n_sink=4, n_recent=32))
    for _ in range(2):
        for t, f in zip((kc, vc, score), first):
            t.copy_(f)
        idx.fill_(0)
        graph.replay()
        same((kc, vc, score, n, idx), want)


def test_evict_the_longest_cache():
    """2^20 rows of one head, nearly all distinct scores: against torch's stable sort."""
    L, budget = 1 << 20, 300001
    g = torch.Generator(device="cuda").manual_seed(1)
    score = torch.rand((1, 1, 1, L), generator=g, device="cuda")
    kc = torch.arange(L, device="cuda", dtype=torch.int32)[None, None, None, :, None].expand(1, 1, 1, L, 32).contiguous()
    kc = kc.view(torch.bfloat16)  # 64 bf16 values a row: its number, 32 times
    vc = kc.clone()
    idx = torch.zeros((1, 1, 1, budget), dtype=torch.int32, device="cuda")
    key = score.clone()
    key[..., :3] = key[..., -1000:] = 2.0
    rows = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget].sort(-1).values
    want = torch.gather(score, 3, rows)
    B.adt_kv_evict(kc, vc, score, i32([L]), keep_idx=idx, B=1, Hkv=1, D=64, num_layers=1, max_kv=L, budget=budget, n_sink=3,
                   n_recent=1000)
    assert torch.equal(idx.long(), rows) and torch.equal(score[..., :budget], want)
    for x in (kc, vc):
        assert torch.equal(x.view(torch.int32)[0, 0, 0, :budget], rows.to(torch.int32)[0, 0, 0, :, None].expand(budget, 32))


def test_evict_binding_checks_what_it_is_given():
    c = Case(2, 2, 64, [140, 60], 150, "spread", 10)
    kc, vc, score, kv = c.tensors()
    n, idx = c.outputs(64)
    other = [torch.zeros((2, 2, 2, 64, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    small = torch.zeros((2, 2, 2, 64), device="cuda")
    for args, more, err in [
            ((kc.half(), vc, score, kv), {}, TypeError), ((kc, vc[:1], score, kv), {}, ValueError),
            ((kc, vc, score[..., :149], kv), {}, ValueError), ((kc, vc, score.double(), kv), {}, TypeError),
            ((kc, vc, score, kv.long()), {}, TypeError), ((kc, vc, score, kv[:1]), {}, ValueError),
            ((kc, vc, score, kv, kv), {}, B.AdtError), ((kc, vc, score, kv, n), dict(keep_idx=idx[:1]), ValueError),
            ((kc, vc, score, kv, n), dict(k_out=other[0]), ValueError), ((kc, vc, score, kv, n), dict(k_out=other[0], v_out=other[1]), ValueError),
            ((kc, vc, score, kv, n), dict(k_out=other[0], v_out=other[0][:, :, :, :63], score_out=small), ValueError),
            ((kc, vc, score, kv, n), dict(k_out=other[0], v_out=vc, score_out=small), B.AdtError),
            ((kc, vc, score, kv, n), dict(score_out=small[..., :63]), ValueError),
            ((kc, vc.transpose(1, 2).contiguous().transpose(1, 2), score, kv, n), {}, ValueError),
            ((kc, vc, score, kv, n), dict(n_sink=60, n_recent=5), B.AdtError)]:
        with pytest.raises(err):
            B.adt_kv_evict(*args, **c.kw(budget=64, **more))
    assert np.array_equal(bits(kc), bits(c.kc)) and np.array_equal(bits(vc), bits(c.vc))


@pytest.mark.parametrize("max_more", [0, 5])
def test_evict_of_caches_in_one_allocation(max_more):
    # [layers, B, Hkv, K and V, rows, D]: the spans of K and V overlap, their slices do not.
    c = Case(2, 3, 64, [300, 80], 300, "spread", 17)
    both = torch.zeros(2, 2, 3, 2, 300 + max_more, 64, dtype=torch.bfloat16, device="cuda")
    both[:, :, :, 0, :300], both[:, :, :, 1, :300] = c.kc.cuda(), c.vc.cuda()
    kc, vc = both[:, :, :, 0], both[:, :, :, 1]
    _, _, score, kv_len = c.tensors()
    n, idx = c.outputs(100)
    B.adt_kv_evict(kc, vc, score, kv_len, n, keep_idx=idx, **c.kw(budget=100, n_sink=4, n_recent=16))
    same((kc[..., :300, :], vc[..., :300, :], score, n, idx), c.oracle(100, 4, 16))
    assert not both[:, :, :, :, 300:].any()
