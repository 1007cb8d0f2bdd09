"""What the verify step and the decode loop hand the cache operators: scores that
start anew with another sequence, and the lse and queries of the attention that
was paid."""
import numpy as np
import pytest
import torch

from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import synth
from paper_2512_21857_gb300.verify_step import StepShape, TreeVerifyStep

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
