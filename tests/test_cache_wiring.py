"""What the verify step and the decode loop hand the cache operators: scores that
start anew with another sequence, and the lse and queries of the attention that
was paid."""
import numpy as np
import pytest
import torch

import oracle
from gpu_cases import LSE_ATOL, ensure_built
from oracle.step import draft_tree, verify_step
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import synth
from paper_2512_21857_gb300.decode import Decoder, ModelShape, RopeShape
from paper_2512_21857_gb300.verify_step import StepShape, TreeVerifyStep
from test_decode_e2e import SMALL, _prompt

LAYERS, H, HKV, D, V, NMAX = 2, 4, 2, 64, 4096, 16
KV, DEPTH, WIDTH = [90, 41], [3, 3], [3, 3]


def make_step(**kw):
    ensure_built()
    shape = StepShape(layers=LAYERS, H=H, Hkv=HKV, D=D, V=V, kv_len=KV, depth=DEPTH, width=WIDTH, max_nodes=NMAX, lmax=120,
                      kv_budget=64, kv_sink=2, kv_recent=12)
    return TreeVerifyStep(shape, **kw)


def inputs(step, seed):
    return synth.step_inputs(LAYERS, H, HKV, D, V, KV, DEPTH, WIDTH, step.n, step.lmax, seed=seed)


def bits(t):
    return t.cpu().contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).numpy()


@pytest.mark.gpu
def test_another_sequence_starts_with_scores_of_its_own():
    used, fresh = make_step(), make_step()
    used.load_inputs(inputs(used, 1))
    for _ in range(3):  # (the caches' rows move; the scores go on)
        used.launch()
    assert (used.score > 0).any()
    second = inputs(used, 2)
    for step in (used, fresh):
        step.load_inputs(second)
        step.launch()
    assert B.adt_get_device_error() == 0
    assert used.kv_len_kept.tolist() == fresh.kv_len_kept.tolist() == [64, 42]
    for b, n in enumerate(fresh.kv_len_kept.tolist()):
        for name in ("score", "k_cache", "v_cache"):
            assert np.array_equal(bits(getattr(used, name)[:, b, :, :n]), bits(getattr(fresh, name)[:, b, :, :n]))


@pytest.mark.gpu
def test_a_sequence_may_bring_its_scores():
    step = make_step()
    inp = inputs(step, 3)
    score = torch.rand(step.score.shape, generator=torch.Generator().manual_seed(4))
    step.load_inputs(dict(inp, score=score))
    assert torch.equal(step.score.cpu(), score)
    step.load_inputs(dict(q=inp["q"]))  # the same sequence's next tree: the scores stay
    assert torch.equal(step.score.cpu(), score)
    step.load_inputs(inp)
    assert not step.score.any()


# The weights that a committed token and head pay to the rows they see sum to one.  On the device each is off by the
# error of lse (LSE_ATOL, the attention tests' bound) and that of the score's fp32 (2^-14 relative, the turns' tests' bound).
def mass_error(before, after, kv, alen, group):
    """[layers, B, Hkv]: (what a call with decay 1 added to the live rows) / (heads of the group x tokens committed) - 1, and
    the bound of its size."""
    added, size = np.zeros(before.shape[:3]), np.zeros(before.shape[:3])
    for b, (L, a) in enumerate(zip(kv, alen)):
        new = after[:, b, :, :L + a + 1].sum(-1)
        added[:, b] = (new - before[:, b, :, :L].sum(-1)) / (group * (a + 1)) - 1
        size[:, b] = np.expm1(LSE_ATOL) + 2.0 ** -14 + 2.0 ** -23 * new / (group * (a + 1))  # (one rounding a row's score)
    return added, size


def test_the_sum_of_the_weights_sees_another_layers_lse_and_stale_queries():
    g = np.random.default_rng(6)
    layers, kv, paths, offs = 3, [30, 9], [[0, 2], [0]], [0, 3, 6]
    q, k = g.standard_normal((layers, 6, 4, 16)), g.standard_normal((layers, 2, 2, 40, 16))
    score = g.random((layers, 2, 2, 40))
    lse = np.full((layers, 6, 4), np.inf)
    for b in range(2):
        for i, node in enumerate(paths[b]):
            s = 0.25 * np.einsum("lhd,lhjd->lhj", q[:, offs[b] + node], k[:, b, :, :kv[b] + i + 1].repeat(2, 1))
            lse[:, offs[b] + node] = np.log(np.exp(s).sum(-1))
    for qq, zz, right in ((q, lse, True), (q, np.roll(lse, 1, 0), False), (np.roll(q, 1, 0), lse, False)):
        after = oracle.kv_score(qq, zz, k, kv, offs, paths, score, 0.25)[0]
        err, bound = mass_error(score, after, kv, [1, 0], 2)
        assert (np.abs(err) <= bound).all() == right and (right or (np.abs(err) > 2 * bound).mean() > 0.5)


def watch_scores(monkeypatch, group):
    """Checks the sums of every call of adt_kv_score; returns the list of the calls' lengths and accepted nodes."""
    real, calls = B.adt_kv_score, []

    def watched(q, lse, kc, kv, offs, path, max_path, alen, score, **kw):
        before = score.double().cpu().numpy()
        real(q, lse, kc, kv, offs, path, max_path, alen, score, **kw)
        err, bound = mass_error(before, score.double().cpu().numpy(), kv.tolist(), alen.tolist(), group)
        assert (np.abs(err) <= bound).all(), np.abs(err / bound).max()
        calls.append((kv.tolist(), alen.tolist()))

    monkeypatch.setattr(B, "adt_kv_score", watched)
    return calls


@pytest.mark.gpu
def test_verify_step_scores_by_its_own_attention(monkeypatch):
    step = make_step(keep_layer_outputs=True)
    inp = inputs(step, 77)
    trees = [draft_tree(inp["draft_rows"][b], WIDTH[b], DEPTH[b], int(inp["root_token"][b]), NMAX) for b in range(2)]
    offs = np.concatenate([[0], np.cumsum(step.n)])
    for b, t in enumerate(trees):
        synth.plant_path(inp["target"][offs[b]:offs[b + 1]], t["parents"], t["tokens"],
                         oracle.ancestor_path(t["parents"], int(np.argmax(t["depth"])))[:2 + b])
    step.load_inputs(inp)
    calls = watch_scores(monkeypatch, H // HKV)
    step.launch()
    ref = verify_step(inp["draft_rows"], WIDTH, DEPTH, inp["root_token"].tolist(), NMAX, inp["q"].double().numpy(),
                      inp["k_cache"].double().numpy(), inp["v_cache"].double().numpy(), KV, inp["k_tree"].double().numpy(),
                      inp["v_tree"].double().numpy(), inp["target"], inp["u_accept"], inp["u_sample"], B.ACCEPT_GREEDY)
    want = np.stack([ref["attn"][layer][1] for layer in range(LAYERS)])
    assert np.abs(step.lse.double().cpu().numpy() - want).max() < LSE_ATOL
    assert np.abs(want[0] - want[1]).mean() > 10 * LSE_ATOL  # (else layers could be exchanged unseen)
    assert calls == [(KV, [1, 2])] and step.accept_len.tolist() == [1, 2]
    assert B.adt_get_device_error() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("batch,graphs,rope", [(1, False, None), (2, True, RopeShape()), (2, False, RopeShape(interleaved=True))])
def test_decode_scores_by_its_own_attention(monkeypatch, batch, graphs, rope):
    """Prompt, growing cache and turns: each call adds one for every token committed, layer and head."""
    ensure_built()
    shape = ModelShape(**{**SMALL.__dict__, "rope": rope})
    dec = Decoder(shape, batch=batch, grid=(8, 8), prompt_len=8, seed=7, max_nodes=32, graphs=graphs, kv_budget=24, kv_slack=8,
                  kv_sink=2, kv_recent=8)
    calls = watch_scores(monkeypatch, shape.heads // shape.kv_heads)
    _, stats = dec.generate(_prompt(shape.vocab, 8, 1))
    assert B.adt_get_device_error() == 0
    lens = [max(kv) for kv, _ in calls]
    assert len(calls) == stats.steps + 1 and lens[0] == 0 and max(lens) > 24 and any(b < a for a, b in zip(lens, lens[1:]))
