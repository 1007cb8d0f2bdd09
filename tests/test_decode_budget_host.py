"""Refusals of the decode loop and the verify step with a bounded cache that need no GPU."""
import pytest
import torch

from paper_2512_21857_gb300.decode import Decoder, ModelShape
from paper_2512_21857_gb300.verify_step import StepShape, TreeVerifyStep

TINY = ModelShape(layers=1, hidden=128, heads=2, kv_heads=2, head_dim=64, ffn=256, vocab=512)


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2512_21857_gb300 import build
    build.build()
    threads = torch.get_num_threads()
    torch.set_num_threads(1)  # (no thread pool: tests that follow fork this process)
    yield
    torch.set_num_threads(threads)


@pytest.mark.parametrize("length,refused", [(8, False), (17, False), (33, False), (34, True), (60, True)])
def test_prompts_that_a_bounded_cache_does_not_hold_are_refused(length, refused):
    """A cache of 24 + 8 rows and a path of 10: the prompt but its last token, and a first path, have to fit."""
    dec = Decoder(TINY, device="cpu", grid=(8, 8), prompt_len=8, kv_budget=24, kv_slack=8)
    assert dec.target.lmax == 42
    # (what is taken goes on to the attention, which has no GPU here)
    with pytest.raises(ValueError, match="prompt_len = 8" if refused else "CUDA"):
        dec.prefill(list(range(length)))


@pytest.mark.parametrize("kw", [dict(kv_budget=-1), dict(kv_budget=8, kv_sink=5, kv_recent=4), dict(kv_budget=8, kv_sink=-1),
                                dict(kv_budget=8, kv_recent=-1)])
def test_budgets_that_no_eviction_takes_are_refused_before_a_step(kw):
    shape = StepShape(layers=1, H=2, Hkv=2, D=64, V=256, kv_len=[20], depth=[2], width=[2], max_nodes=8, **kw)
    with pytest.raises(ValueError, match="kv_budget"):
        TreeVerifyStep(shape, device="cpu")


@pytest.mark.parametrize("kw", [dict(kv_sink=-1), dict(kv_recent=-1), dict(kv_slack=-1)])
def test_decoder_refuses_negative_parts_of_a_budget(kw):
    with pytest.raises(ValueError, match="kv_sink"):
        Decoder(TINY, device="cpu", grid=(2, 2), prompt_len=8, kv_budget=8, **kw)
