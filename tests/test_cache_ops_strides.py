"""Strides of dimensions of one: they say nothing, and two tensors of one shape
need not agree on them."""
import pytest
import torch

from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from test_parity_kv_evict import Case as EvictCase
from test_parity_kv_evict import bits, same
from test_parity_kv_score import Case as ScoreCase


def test_strides_of_dimensions_of_one_are_left_out():
    wide = torch.empty(4, 3, 5, 7, 64, dtype=torch.bfloat16)
    assert B._strides3(wide[:1, 1:2, :1], 1, 1, 1, 7, 64, "k") == (0, 0, 0)
    assert B._strides3(wide[:, 1:2], 4, 1, 5, 7, 64, "k") == (3 * 5 * 7 * 64, 0, 7 * 64)
    assert B._strides3(torch.empty(4, 1, 5, 9), 4, 1, 5, 7, 0, "score") == (45, 0, 9)


@pytest.fixture
def built():
    ensure_built()


@pytest.mark.gpu
@pytest.mark.parametrize("layers,Hkv,kv", [(2, 2, [140]), (1, 2, [140, 60]), (2, 1, [140, 60]), (1, 1, [140])])
def test_evict_where_only_strides_of_one_differ(built, layers, Hkv, kv):
    """K a slice of a larger cache, V one of its own; the same for the destinations."""
    c = EvictCase(layers, Hkv, 64, kv, 150, "spread", 31)
    kc, vc, score, kv_len = c.tensors()
    n, idx = c.outputs(64)

    def as_slice(t):  # dimensions of one from a larger tensor
        s = list(t.stride())
        for d in range(3):
            if t.shape[d] == 1:
                s[d] = 7 * t.numel() + 3  # (no multiple of a vector)
        return t.as_strided(t.shape, s)

    k2, s2 = as_slice(kc), as_slice(score)
    assert k2.stride() != vc.stride()
    B.adt_kv_evict(k2, vc, s2, kv_len, n, keep_idx=idx, **c.kw(budget=64, n_sink=2, n_recent=9))
    same((kc, vc, score, n, idx), c.oracle(64, 2, 9))
    src = c.tensors()
    ko, vo = (torch.zeros((layers, len(kv), Hkv, 64, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    so = torch.zeros((layers, len(kv), Hkv, 64), device="cuda")
    B.adt_kv_evict(src[0], as_slice(src[1]), src[2], src[3], n, k_out=ko, v_out=as_slice(vo), score_out=as_slice(so), keep_idx=idx,
                   **c.kw(budget=64, n_sink=2, n_recent=9))
    zero = torch.zeros_like(ko)
    same((ko, vo, so, n, idx), c.oracle(64, 2, 9, k_dst=bits(zero), v_dst=bits(zero), score_dst=torch.zeros_like(so).cpu().numpy()))


@pytest.mark.gpu
@pytest.mark.parametrize("layers,Hkv,kv,paths", [(1, 2, [140, 60], [[0, 1], [0]]), (2, 2, [140], [[0, 1]]), (2, 1, [140], [[0]])])
def test_score_where_only_strides_of_one_differ(built, layers, Hkv, kv, paths):
    c = ScoreCase(layers, 2 * Hkv, Hkv, 64, kv, paths, 3, seed=32)
    args = list(c.args())

    def as_slice(t, dims):
        return t.as_strided(t.shape, [3 + 7 * t.numel() if d < dims and t.shape[d] == 1 else s for d, s in enumerate(t.stride())])

    out = torch.from_numpy(c.score).cuda()
    args[0], args[1], args[2] = as_slice(args[0], 1), as_slice(args[1], 1), as_slice(args[2], 3)
    B.adt_kv_score(*args, **c.kw(), score_out=as_slice(out, 3))
    c.check(out)
