"""The cache operators as they are used: the verify step and the decode loop
with a bounded cache, and the decode loop with the library's rotation.  Scores
that the device made decide the evictions, so each eviction is compared with
the oracle's on the device's own scores (bit for bit), and each score with the
oracle's on the device's own queries, lse and cache."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_cases import ensure_built
from oracle.step import draft_tree, verify_step
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import decode, synth
from paper_2512_21857_gb300.decode import Decoder, ModelShape, RopeShape
from paper_2512_21857_gb300.verify_step import StepShape, TreeVerifyStep
from test_decode_e2e import NEAR_TIE_BF16, SMALL, _check, _prompt, _reference

pytestmark = pytest.mark.gpu

# A score is a sum of weights, each made in fp32: the terms of the bound in the score's own parity test come to less
# than 2^-14 of it for scores up to 30 and lse up to 20 (D = 128: 2 D 2^-24 sum |q k| scale < 2^-16 * 30 ...).
SCORE_RTOL = 2.0 ** -14


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def bits(t):
    return t.cpu().contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).numpy()


def score_oracle(q, lse, kc, kv, offs, path, alen, score, scale):
    kv, offs, alen, path = (t.cpu().numpy() for t in (kv, offs, alen, path))
    paths = [path.reshape(len(kv), -1)[b, :alen[b] + 1].tolist() for b in range(len(kv))]
    return oracle.kv_score(q.double().cpu().numpy(), lse.double().cpu().numpy(), kc.double().cpu().numpy(), kv, offs, paths,
                           score.double().cpu().numpy(), scale)[0]


@pytest.mark.parametrize("graph", [False, True])
def test_verify_steps_with_a_bounded_cache(graph):
    """Three turns of two images: the step's own outputs equal the unbounded step's, then scores and evictions."""
    layers, H, Hkv, D, V, depth, width, nmax = 2, 4, 2, 64, 4096, 3, 3, 16
    shape = StepShape(layers=layers, H=H, Hkv=Hkv, D=D, V=V, kv_len=[90, 41], depth=[depth] * 2, width=[width] * 2,
                      max_nodes=nmax, lmax=120, kv_budget=64, kv_sink=2, kv_recent=12)
    step = TreeVerifyStep(shape, keep_layer_outputs=True)
    inp = synth.step_inputs(layers, H, Hkv, D, V, [90, 41], [depth] * 2, [width] * 2, step.n, step.lmax, seed=77)
    trees = [draft_tree(inp["draft_rows"][b], width, depth, int(inp["root_token"][b]), nmax) for b in range(2)]
    offs = np.concatenate([[0], np.cumsum(step.n)])
    for b, t in enumerate(trees):
        deepest = int(np.argmax(t["depth"]))
        synth.plant_path(inp["target"][offs[b]:offs[b + 1]], t["parents"], t["tokens"],
                         oracle.ancestor_path(t["parents"], deepest)[:2 + b])
    step.load_inputs(inp)
    kv = [90, 41]
    if graph:  # captured with the caches as they are; the replays below do the work
        step.launch()
        torch.cuda.synchronize()
        step.load_inputs(inp)
        step.score.zero_()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step.launch()
    for turn in range(3):
        before = [t.clone() for t in (step.k_cache, step.v_cache, step.score)]
        step.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        if graph:
            g.replay()
        else:
            step.launch()
        assert B.adt_get_device_error() == 0
        ref = verify_step(inp["draft_rows"], [width] * 2, [depth] * 2, inp["root_token"].tolist(), nmax,
                          inp["q"].double().numpy(), before[0].double().cpu().numpy(), before[1].double().cpu().numpy(), kv,
                          inp["k_tree"].double().numpy(), inp["v_tree"].double().numpy(), inp["target"], inp["u_accept"],
                          inp["u_sample"], B.ACCEPT_GREEDY)
        for layer in range(layers):
            assert np.abs(step.attn_out[layer].double().cpu().numpy() - ref["attn"][layer][0]).max() <= 1.8e-2
        lens = [int(n) for n in ref["kv_len"]]
        assert step.kv_len_out.tolist() == lens and step.accept_len.tolist() == [1, 2]
        # scores: over the committed cache, which the eviction has moved since
        kc = torch.as_tensor(ref["k_cache"])
        want = score_oracle(step.q, step.lse, kc, step.kv_len, step.node_offsets, step.path, step.accept_len, before[2], D ** -0.5)
        got = step.score.double().cpu().numpy()
        for b, n in enumerate(lens):
            m = min(n, 64)
            for layer in range(layers):
                for h in range(Hkv):
                    rows = oracle.cache_ops.kept_rows(want[layer, b, h, :n].tolist(), 64, 2, 12)
                    mine = got[layer, b, h, :m]
                    # the kept rows' scores are the oracle's, up to rows whose scores are nearly the threshold's
                    np.testing.assert_allclose(np.sort(mine), np.sort(want[layer, b, h, rows]), rtol=2 * SCORE_RTOL, atol=1e-9)
                    # and K and V of every kept row are those of a committed row with that score, in order
                    at = [int(np.abs(want[layer, b, h, :n] - x).argmin()) for x in mine]
                    assert at == sorted(at)
                    assert np.array_equal(step.k_cache[layer, b, h, :m].double().cpu().numpy(), ref["k_cache"][layer, b, h, at])
                    assert np.array_equal(step.v_cache[layer, b, h, :m].double().cpu().numpy(), ref["v_cache"][layer, b, h, at])
        kv = [min(n, 64) for n in lens]
        assert step.kv_len_kept.tolist() == kv


class Watch:
    """Stands before the decode loop's calls and compares each with the oracle."""

    def __init__(self, monkeypatch):
        self.scores = self.evictions = 0
        self.real_score, self.real_evict = B.adt_kv_score, B.adt_kv_evict
        monkeypatch.setattr(decode.B, "adt_kv_score", self.score)
        monkeypatch.setattr(decode.B, "adt_kv_evict", self.evict)

    def score(self, q, lse, kc, kv, offs, path, max_path, alen, score, **kw):
        want = score_oracle(q, lse, kc, kv, offs, path, alen, score, kw["softmax_scale"])
        weights = want.sum()
        self.real_score(q, lse, kc, kv, offs, path, max_path, alen, score, **kw)
        np.testing.assert_allclose(score.double().cpu().numpy(), want, rtol=SCORE_RTOL, atol=1e-9)
        # each committed token spreads a weight of one over the rows for every layer and head
        self.scores += 1
        self.total = weights

    def evict(self, kc, vc, score, kv, kv_out=None, **kw):
        want = oracle.kv_evict(bits(kc), bits(vc), score.cpu().numpy(), kv.cpu().numpy(), kw["budget"], kw["n_sink"],
                               kw["n_recent"])
        self.real_evict(kc, vc, score, kv, kv_out, **kw)
        assert np.array_equal(bits(kc), want[0]) and np.array_equal(bits(vc), want[1])
        assert np.array_equal(bits(score), want[2].view(np.int32))
        self.evictions += 1


@pytest.mark.parametrize("batch,graphs,rope", [(1, False, None), (2, True, None), (2, False, RopeShape(rotary_dim=64, interleaved=True))])
def test_decode_with_a_bounded_cache(monkeypatch, batch, graphs, rope):
    shape = ModelShape(**{**SMALL.__dict__, "rope": rope})
    dec = Decoder(shape, batch=batch, grid=(8, 8), prompt_len=8, seed=7, max_nodes=32, graphs=graphs, kv_budget=24, kv_slack=8,
                  kv_sink=2, kv_recent=8)
    assert dec.target.lmax == 24 + 8 + 9 + 1
    watch = Watch(monkeypatch)
    out, stats = dec.generate(_prompt(shape.vocab, 8, 1))
    assert B.adt_get_device_error() == 0
    assert all(len(o) == 64 for o in out) and watch.scores == stats.steps + 1 and watch.evictions >= 3
    assert math.isfinite(watch.total)


@pytest.mark.parametrize("graphs", [False, True])
def test_decode_with_a_budget_that_is_never_reached_is_the_same(graphs):
    kw = dict(batch=2, grid=(6, 8), prompt_len=8, seed=7, max_nodes=32, graphs=graphs)
    prompt = _prompt(SMALL.vocab, 8, 1)
    plain = Decoder(SMALL, **kw).generate(prompt)
    bounded = Decoder(SMALL, **kw, kv_budget=500)
    assert bounded.generate(prompt)[0] == plain[0]
    assert bounded.generate(prompt)[0] == plain[0]  # scores and caches start anew


def test_decode_with_a_bounded_cache_counts_positions_apart():
    """The positions that the target is given go on counting while its cache stays short."""
    dec = Decoder(SMALL, batch=1, grid=(8, 8), prompt_len=8, seed=7, max_nodes=32, kv_budget=16, kv_slack=0, kv_sink=1,
                  kv_recent=4)
    seen, run = [], dec.target.run

    def watched(x, pos, parents, offs, kv, batch, image=None):
        seen.append((int(pos[0]), int(kv[0])))
        return run(x, pos, parents, offs, kv, batch, image)

    dec.target.run = watched
    dec.generate(_prompt(SMALL.vocab, 8, 1))
    first = [p for p, _ in seen[1:]]
    assert first[0] == 7 and all(b > a for a, b in zip(first, first[1:])) and first[-1] >= 7 + 64 - 10
    assert max(k for _, k in seen) <= 16 and seen[-1][1] == 16


def test_decoder_refuses_bad_budgets():
    with pytest.raises(ValueError):
        Decoder(SMALL, grid=(2, 2), kv_budget=-1)
    with pytest.raises(ValueError):
        Decoder(SMALL, grid=(2, 2), kv_budget=8, kv_slack=-1)
    dec = Decoder(SMALL, grid=(2, 2), prompt_len=8, kv_budget=8)
    with pytest.raises(ValueError, match="deepest"):
        dec.generate(_prompt(SMALL.vocab, 8, 1), ctrl_params=dict(d_hi=20))


@pytest.mark.parametrize("rope", [
    RopeShape(), RopeShape(interleaved=True, rotary_dim=64),
    RopeShape(rotary_dim=48, scaling=B.ROPE_LINEAR, factor=2.0),
    RopeShape(scaling=B.ROPE_BY_PARTS, factor=4.0, orig_len=512.0), RopeShape(interleaved=True, scaling=B.ROPE_NTK, factor=8.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_decode_with_the_librarys_rotation_equals_greedy(rope, dtype):
    """As the decode loop's own test: every token is the choice of a reference that rotates in torch, but for near ties."""
    shape = ModelShape(**{**SMALL.__dict__, "rope": rope, "dtype": dtype})
    dec = Decoder(shape, batch=2, grid=(6, 8), prompt_len=8, seed=7, max_nodes=64, graphs=dtype == torch.bfloat16)
    prompt = _prompt(shape.vocab, 8, 1)
    out, _ = dec.generate(prompt)
    choice, margins = _reference(shape, dec.target_w, prompt, out)
    for b in range(2):
        _check(out[b], choice[b], margins[b], max_ties=3, near_tie=NEAR_TIE_BF16)
    assert B.adt_get_device_error() == 0


def _calls(seed, H=4, Hkv=2, D=64, L=300, rows=360):
    """Inputs of a score and an eviction of their own, on the device."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    q, lse = rnd(2, 6, H, D).bfloat16(), rnd(2, 6, H).abs() + 5
    kc, vc, score = rnd(2, 2, Hkv, rows, D).bfloat16(), rnd(2, 2, Hkv, rows, D).bfloat16(), rnd(2, 2, Hkv, rows).exp()
    i = dict(dtype=torch.int32, device="cuda")
    return dict(q=q, lse=lse, kc=kc, vc=vc, score=score, kv=torch.tensor([L, 40 + seed], **i), offs=torch.tensor([0, 3, 6], **i),
                path=torch.tensor([[0, 2], [0, 1]], **i), alen=torch.tensor([1, 1], **i), out=torch.tensor([L + 2, 42 + seed], **i))


def _turn(c, stream=None, D=64):
    kw = dict(B=2, Hkv=2, D=D, num_layers=2, max_kv=c["kc"].shape[3], stream=stream)
    B.adt_kv_score(c["q"], c["lse"], c["kc"], c["kv"], c["offs"], c["path"], 2, c["alen"], c["score"], H=4, softmax_scale=0.125, **kw)
    B.adt_kv_evict(c["kc"], c["vc"], c["score"], c["out"], budget=100, n_sink=2, n_recent=20, **kw)


def test_turns_on_two_streams_at_once():
    """Neither call keeps a workspace: turns that overlap on the device do not meet."""
    alone = [_calls(s) for s in range(6)]
    for c in alone:
        _turn(c)
    both = [_calls(s) for s in range(6)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for k, c in enumerate(both):
        _turn(c, streams[k % 3])
    torch.cuda.synchronize()
    for a, c in zip(alone, both):
        for name in ("kc", "vc", "score"):
            assert torch.equal(a[name], c[name])


def test_offsets_past_32_bits():
    """Layers, heads and rows of projections that lie more than 2^32 bytes and 2^31 elements apart."""
    c = _calls(3)
    want = {k: v.clone() for k, v in c.items()}
    _turn(want)
    far = (1 << 31) + 64
    big = torch.empty(far + (1 << 26), dtype=torch.bfloat16, device="cuda")
    wide = torch.empty(far + (1 << 20), device="cuda")
    shape, rows = c["kc"].shape, c["kc"].shape[3]
    stride = (far, 1 << 18, 1 << 16, 64, 1)
    kc, vc = big.as_strided(shape, stride), big.as_strided(shape, stride, 1 << 22)
    score = wide.as_strided(shape[:4], (far, 4 * rows, rows, 1))
    for t, s in ((kc, "kc"), (vc, "vc"), (score, "score")):
        t.copy_(c[s])
    _turn(dict(c, kc=kc, vc=vc, score=score))
    assert B.adt_get_device_error() == 0
    for t, s in ((kc, "kc"), (vc, "vc"), (score, "score")):
        assert torch.equal(t, want[s])
    x = torch.randn((3, 2 * 64), device="cuda").bfloat16()
    ld = 1 << 30
    y = big.as_strided((3, 2 * 64), (ld + 8, 1))
    y.copy_(x)
    pos, inv = torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    out = [torch.empty((3, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for src, o in zip((x, y), out):
        B.adt_rope_qkv(src, None, None, pos, inv, H=2, Hkv=1, D=64, q_out=o)
    assert torch.equal(*out)
