"""The largest elements that a commit into the 8-bit cache takes, and what reading them back gives."""
import pytest
import torch

from gpu_cases import ensure_built, i32
from paper_2512_21857_gb300 import binding as B

pytestmark = pytest.mark.gpu


def test_elements_that_round_past_bf16_read_back_as_infinity():
    """Of a row's scale 2^120: 240 is a value, 248 lies halfway to 256, which is 2^128."""
    ensure_built()
    D = 64
    row = torch.tensor([240.0, 247.0, 248.0, 255.0, -248.0, -240.0, 1.0, 0.0] * 8, dtype=torch.float64) * 2.0 ** 120
    x = row.to(torch.bfloat16).view(1, 1, 1, D).cuda()
    c = [torch.zeros((1, 1, 1, 1, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    s = [torch.zeros((1, 1, 1, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
    shape = dict(B=1, Hkv=1, D=D, num_layers=1, max_kv=1)
    B.adt_kv_compact_q8(*c, *s, i32([0]), None, x, x, i32([0, 1]), i32([[0]]), 1, i32([0]), **shape)
    out = [torch.zeros((1, 1, 1, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.adt_kv_read_q8(*c, *s, i32([1]), *out, **shape)
    inf = float("inf")
    want = torch.tensor([240.0 * 2.0 ** 120, 240.0 * 2.0 ** 120, inf, inf, -inf, -240.0 * 2.0 ** 120, 2.0 ** 120, 0.0] * 8)
    for o, scale in zip(out, s):
        assert int(scale) == 247 and torch.equal(o.float().cpu().flatten(), want)
