"""The decode loop's refusals with a bounded cache that need no GPU."""
import pytest
import torch

from paper_2512_21857_gb300.decode import Decoder, ModelShape

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
