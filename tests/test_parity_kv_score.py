"""adt_kv_score on the GPU against the fp64 oracle.

Bound, per row, from the oracle's sums over the queries that reach it: a
product of D bf16 pairs is exact before it is summed in fp32, whose order and
rounding (truncation at worst) cost up to 2 D 2^-24 of sum |q_d k_d|, times the
scale; scaling and subtracting lse round twice (2^-23 of |scale s| + |lse|,
below 2^-22 (|scale s - lse| + 2 |lse|)); the conversion to base two and the
exponential cost 2^-21 of the argument's size and of the value; the sum of the
weights one rounding a term."""
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


class Case:
    def __init__(self, layers, H, Hkv, D, kv, paths, nodes, seed, lmax=None, decay=1.0, qscale=1.0):
        self.layers, self.H, self.Hkv, self.D, self.kv, self.paths, self.decay = layers, H, Hkv, D, kv, paths, decay
        self.B, self.nodes = len(kv), nodes
        self.offs = np.arange(self.B + 1) * nodes
        self.lmax = lmax or max(L + len(p) for L, p in zip(kv, paths)) + 5
        self.scale = D ** -0.5
        self.q = synth.bf16_normal((layers, self.B * nodes, H, D), seed, "q", std=qscale)
        self.kc = synth.bf16_normal((layers, self.B, Hkv, self.lmax, D), seed, "kc")
        self.score = synth.rng(seed, "score").random((layers, self.B, Hkv, self.lmax)).astype(np.float32)
        # lse of each accepted query over the rows it sees (other nodes' values are never read)
        self.lse = np.full((layers, self.B * nodes, H), 1e30, np.float32)
        q, k = self.q.double(), self.kc.double()
        for b, (L, path) in enumerate(zip(kv, paths)):
            at = [b * nodes + t for t in path]
            s = torch.einsum("lihd,lhjd->lhij", q[:, at], k[:, b].repeat_interleave(H // Hkv, 1)) * self.scale
            see = torch.arange(self.lmax)[None] <= L + torch.arange(len(path))[:, None]
            self.lse[:, at] = s.masked_fill(~see, -np.inf).logsumexp(-1).transpose(1, 2).float().numpy()

    def padded_path(self, max_path):
        out = np.full((self.B, max_path), -1, np.int32)
        for b, p in enumerate(self.paths):
            out[b, :len(p)] = p
        return i32(out)

    def args(self, max_path=None):
        max_path = max_path or max(len(p) for p in self.paths)
        return (self.q.cuda(), torch.from_numpy(self.lse).cuda(), self.kc.cuda(), i32(self.kv), i32(self.offs),
                self.padded_path(max_path), max_path, i32([len(p) - 1 for p in self.paths]), torch.from_numpy(self.score).cuda())

    def kw(self):
        return dict(B=self.B, H=self.H, Hkv=self.Hkv, D=self.D, num_layers=self.layers, max_kv=self.lmax,
                    softmax_scale=self.scale, decay=self.decay)

    def run(self, **kw):
        args = self.args()
        B.adt_kv_score(*args, **self.kw(), **kw)
        return args[-1]

    def check(self, got):
        ref, terms = oracle.kv_score(self.q.double().numpy(), self.lse, self.kc.double().numpy(), self.kv, self.offs, self.paths,
                                     self.score, self.scale, self.decay)
        w, wqk, wt = terms
        used = self.lse[np.isfinite(self.lse) & (self.lse < 1e29)]
        big = np.abs(used).max() if used.size else 0.0
        rel = 2 * self.D * 2.0 ** -24 * self.scale * wqk + 2.0 ** -20 * wt + 2.0 ** -21 * (1 + big) * w
        count = max(len(p) for p in self.paths) * (self.H // self.Hkv) + 1
        bound = rel * 1.01 + count * 2.0 ** -24 * np.abs(ref) + 2.0 ** -140
        err = np.abs(got.double().cpu().numpy() - ref)
        assert (err <= bound).all(), (err / np.maximum(bound, 1e-300)).max()
        for b, (L, p) in enumerate(zip(self.kv, self.paths)):  # rows behind the last token
            assert np.array_equal(got[:, b, :, L + len(p):].cpu().numpy(), self.score[:, b, :, L + len(p):])


def chain(n):
    return list(range(n))


@pytest.mark.parametrize("layers,H,Hkv,D,kv,paths,nodes", [
    (1, 1, 1, 64, [0], [[0]], 1),                             # the first token of all
    (1, 8, 8, 64, [512], [[0]], 26),                          # one decoded token
    (2, 4, 4, 128, [0, 1], [[0], [0, 3]], 8),
    (3, 4, 2, 64, [127, 128, 129], [[0, 2], [0], [0, 1, 5]], 9),      # around a tile of keys
    (2, 8, 2, 128, [126, 255, 300], [[0, 4, 7], [0, 1, 2, 3, 4, 5], [0]], 12),
    (1, 20, 5, 64, [700], [[0, 9, 10, 22, 40, 63]], 64),
    (2, 3, 1, 128, [77], [chain(13)], 13),                    # an odd group
    (1, 32, 2, 64, [400, 3], [chain(33), chain(9)], 33),      # 16 heads a group: more queries than a tile
    (1, 4, 4, 128, [0, 40], [chain(256), chain(200)], 256),   # prompts
    (1, 4, 1, 64, [5], [chain(129)], 129),
    (1, 65, 1, 64, [200], [chain(4)], 4),
    (40, 4, 4, 64, [90, 40, 1, 0, 300], [[0], [0, 1], [0, 2, 3], [0], [0, 1]], 5),  # more slices than processors
    (2, 2, 2, 128, [3100], [[0, 1, 2]], 3),
])
def test_score_matches_oracle(layers, H, Hkv, D, kv, paths, nodes):
    c = Case(layers, H, Hkv, D, kv, paths, nodes, seed=layers + H + D + sum(kv))
    c.check(c.run())


@pytest.mark.parametrize("decay", [0.0, 0.9])
def test_score_decays(decay):
    c = Case(2, 4, 2, 64, [200, 64], [[0, 1], [0]], 4, seed=4, decay=decay)
    c.check(c.run())


def test_score_without_decay_reads_no_old_score():
    c = Case(1, 4, 2, 64, [200], [[0, 1]], 4, seed=4, decay=0.0)
    c.score[..., :202] = np.nan
    args = c.args()
    B.adt_kv_score(*args, **c.kw())
    assert torch.isfinite(args[-1]).all()


def test_score_of_sharp_attention():
    """Scores of +-60: weights from 1 to nothing."""
    c = Case(1, 4, 4, 128, [700], [[0, 1, 2, 3, 4]], 5, seed=8, qscale=6.0)
    c.check(c.run())


def test_score_into_another_buffer_and_repeated():
    c = Case(2, 8, 2, 64, [333, 90], [[0, 3, 4], [0]], 6, seed=11)
    args = c.args()
    out = args[-1].clone()
    B.adt_kv_score(*args, **c.kw(), score_out=out)
    assert torch.equal(args[-1].cpu(), torch.from_numpy(c.score))
    c.check(out)
    for _ in range(3):
        again = args[-1].clone()
        B.adt_kv_score(*args, **c.kw(), score_out=again)
        assert torch.equal(again, out)
    B.adt_kv_score(*args, **c.kw())
    assert torch.equal(args[-1], out)


def test_score_with_strides_of_larger_buffers():
    """Layers, trees and heads of larger caches, queries and scores; a capacity (max_kv) below the rows there are."""
    c = Case(2, 4, 2, 64, [130, 60], [[0, 2], [0, 1, 3]], 5, seed=12, lmax=140)
    q, lse, kc, kv, offs, path, max_path, alen, score = c.args(max_path=7)
    bq = torch.full((2, 3) + q.shape[1:], 5.0, dtype=q.dtype, device="cuda")
    bl = torch.full((2, 3) + lse.shape[1:], 5.0, device="cuda")
    bk = torch.full((2, 3, 4, 150, 64), float("nan"), dtype=kc.dtype, device="cuda")
    bs = torch.full((2, 3, 4, 155), 3.0, device="cuda")
    bq[:, 1], bl[:, 2] = q, lse
    bk[:, :2, 1:3, :140], bs[:, 1:, :2, :140] = kc, score
    B.adt_kv_score(bq[:, 1], bl[:, 2], bk[:, :2, 1:3], kv, offs, path, max_path, alen, bs[:, 1:, :2], **c.kw())
    c.check(bs[:, 1:, :2, :140])
    rest = torch.ones_like(bs, dtype=torch.bool)
    rest[:, 1:, :2, :140] = False
    assert (bs[rest] == 3.0).all()


def test_score_ignores_what_lies_behind_the_cache():
    """Infinities and NaN in rows behind the last token change nothing; a poisoned row within it spoils its own score."""
    c = Case(1, 4, 2, 128, [150], [[0, 1]], 3, seed=13, lmax=260)
    want = c.run()
    c.kc[:, :, :, 152:] = float("nan")
    c.kc[:, :, :, 170:] = float("inf")
    assert torch.equal(c.run(), want)
    c.kc[0, 0, 1, 40, 7] = float("nan")
    got = c.run()
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, 0, 1, 40] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])


def test_score_of_queries_that_saw_nothing():
    c = Case(1, 4, 2, 64, [100], [[0, 1, 2]], 3, seed=14)
    c.lse[0, 1] = -np.inf
    got = c.run()
    assert torch.isfinite(got).all()
    c.check(got)


def test_score_flags_bad_input():
    c = Case(2, 4, 2, 64, [100, 50, 70], [[0, 1], [0, 2], [0, 1, 3]], 5, seed=15)
    want = c.run()
    for kv, alen in (([100, -1, 70], None), ([100, c.lmax, 70], None), ([100, 50, 70], [1, -1, 2]), ([100, 50, 70], [1, 3, 2])):
        args = list(c.args())
        args[3] = i32(kv)
        args[7] = i32(alen) if alen else args[7]
        B.adt_get_device_error()
        B.adt_kv_score(*args, **c.kw())
        assert B.adt_get_device_error() == B.DEVERR_KV_RANGE
        assert torch.equal(args[-1][:, 1].cpu(), torch.from_numpy(c.score[:, 1]))
        assert torch.equal(args[-1][:, [0, 2]], want[:, [0, 2]])
    for node in (-1, 5, 2 ** 30):  # an entry outside the tree adds nothing
        args = list(c.args())
        args[5][2, 1] = node
        B.adt_kv_score(*args, **c.kw())
        assert B.adt_get_device_error() == B.DEVERR_BAD_PATH
        assert torch.equal(args[-1][:, :2], want[:, :2])
        d = Case(2, 4, 2, 64, [100, 50, 70], [[0, 1], [0, 2], [0, 1, 3]], 5, seed=15)
        d.lse[:, 10 + 1] = -np.inf
        assert torch.equal(args[-1][:, 2], d.run()[:, 2])


def test_score_in_a_graph_on_another_stream():
    c = Case(2, 8, 8, 64, [300], [[0, 1, 4]], 6, seed=16)
    args = c.args()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.from_numpy(c.score).cuda()
    torch.cuda.current_stream().synchronize()
    B.adt_kv_score(*args, **c.kw(), score_out=out, stream=s)
    s.synchronize()
    c.check(out)
    graph, replayed = torch.cuda.CUDAGraph(), torch.from_numpy(c.score).cuda()
    with torch.cuda.graph(graph):
        B.adt_kv_score(*args, **c.kw(), score_out=replayed)
    for _ in range(2):
        graph.replay()
        assert torch.equal(replayed, out)


@pytest.mark.parametrize("D,paths", [(64, [[0, 1], [0]]), (128, [chain(130), chain(40)])])
def test_score_wait_that_runs_out_is_reported(D, paths):
    """Waits limited to one poll give up, the kernel leaves in order, and the next call is right."""
    c = Case(6, 4, 2, D, [700, 1300], paths, 140, seed=17)
    args = c.args()
    B.adt_get_device_error()
    B.adt_testing_set_wait_limit(1)
    try:
        B.adt_kv_score(*args, **c.kw())
        assert B.adt_get_device_error() & B.DEVERR_TIMEOUT
    finally:
        B.adt_testing_set_wait_limit(0)
    c.check(c.run())
    assert B.adt_get_device_error() == 0


@pytest.mark.parametrize("kv,paths", [
    ([0, 2000, 1, 5, 900, 0, 129, 40], [chain(n) for n in (1, 3, 1, 130, 2, 1, 1, 9)]),    # short trees beside long ones
    ([37] * 70, [chain(1 + b % 4) for b in range(70)]),                                    # more trees than a warp has lanes
])
def test_score_deals_uneven_trees(kv, paths):
    c = Case(3, 4, 2, 64, kv, paths, 140, seed=18)
    c.check(c.run())


def test_score_binding_checks_what_it_is_given():
    """Dimensions of one may have any stride; wrong shapes, types and strides are refused."""
    c = Case(1, 1, 1, 64, [70], [[0]], 1, seed=19)
    args = list(c.args())
    args[0] = args[0].as_strided((1, 1, 1, 64), (8, 8, 8, 1))
    args[1] = args[1].as_strided((1, 1, 1), (3, 5, 7))
    B.adt_kv_score(*args, **c.kw())
    c.check(args[-1])
    c = Case(2, 4, 2, 64, [100, 50], [[0, 1], [0, 2]], 5, seed=20)
    good = list(c.args())
    for i, bad, err in [(0, good[0].float(), TypeError), (0, good[0][:1], ValueError), (0, good[0].transpose(1, 2), ValueError),
                        (0, good[0][..., ::2], ValueError), (1, good[1][:, :9], ValueError), (1, good[1].double(), TypeError),
                        (2, good[2][:, :, :1], ValueError), (2, good[2][:, :, :, :90], ValueError), (2, good[2].half(), TypeError),
                        (2, good[2].transpose(3, 4).contiguous().transpose(3, 4), ValueError), (3, good[3][:1], ValueError),
                        (3, good[3].long(), TypeError), (4, good[4][:2], ValueError), (5, good[5][:1], ValueError),
                        (7, good[7].cpu(), ValueError), (8, good[8][..., ::2], ValueError), (8, good[8].cpu(), ValueError)]:
        args = list(good)
        args[i] = bad
        with pytest.raises(err):
            B.adt_kv_score(*args, **c.kw())
    with pytest.raises(ValueError, match="share strides"):
        B.adt_kv_score(*good, **c.kw(), score_out=torch.zeros((2, 2, 2, c.lmax + 1), device="cuda"))
