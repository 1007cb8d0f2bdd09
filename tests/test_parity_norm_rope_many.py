"""adt_norm_rope_qkv of so many tokens that a thread block takes several, one after the other (from 2432 on, where one
fills it), against the fp64 oracle with the bounds of test_parity_norm_rope."""
import numpy as np
import pytest
import torch

import oracle
from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import synth
from test_parity_norm_rope import check, params_of, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


# (One token a turn and two or four turns; several tokens a turn; heads that are not a power of two of lanes.)
@pytest.mark.parametrize("N,H,Hkv,D,R", [
    (2500, 32, 8, 128, 128), (5003, 32, 8, 128, 128), (5003, 32, 8, 128, 36), (2500, 32, 8, 128, 10), (5003, 32, 8, 128, 0),
    (20011, 2, 1, 64, 64), (40003, 3, 1, 64, 10), (10007, 10, 5, 80, 48), (5003, 8, 16, 128, 90)])
@pytest.mark.parametrize("layer,interleaved,dtype,wtype", [(False, False, torch.bfloat16, torch.bfloat16),
                                                           (True, True, torch.bfloat16, torch.float32),
                                                           (True, False, torch.float32, torch.float32)])
def test_several_tokens_a_thread_block(N, H, Hkv, D, R, layer, interleaved, dtype, wtype):
    seed = N + R
    q, k, v = rows_of(N, (H + 2 * Hkv) * D, dtype, seed, "rows", shift=0.4).split([H * D, Hkv * D, Hkv * D], 1)
    pos = synth.rng(seed, "pos").integers(0, 5000, size=N).astype(np.int32)
    inv = oracle.rope_freqs(R)[0] if R else np.zeros(0)
    qw, qb = params_of(H, D, False, wtype, seed, "q", True)
    kw, kb = params_of(Hkv, D, True, wtype, seed, "k", layer)
    whole = [torch.full((N + 2, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv)]
    out = [w[:N] for w in whole]
    B.adt_norm_rope_qkv(q, k, v, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), H=H, Hkv=Hkv, D=D,
                        norm=B.NORM_LAYER if layer else B.NORM_RMS, eps=1e-5, q_weight=qw, q_bias=qb, k_weight=kw, k_bias=kb,
                        layout=B.ROPE_INTERLEAVED if interleaved else B.ROPE_HALF, magnitude=1.25, q_out=out[0], k_out=out[1],
                        v_out=out[2])
    check(out[0], q, layer, 1e-5, qw, qb, pos, inv, 1.25, interleaved)
    check(out[1], k, layer, 1e-5, kw, kb, pos, inv, 1.25, interleaved)
    assert torch.equal(out[2].flatten(), v.to(torch.bfloat16).flatten())
    assert all((w[N:] == 7).all() for w in whole)


@pytest.mark.parametrize("R", [128, 36])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_equals_out_of_place(R, interleaved):
    N, H, Hkv, D = 5003, 32, 8, 128
    q, k, v = (rows_of(N, h * D, torch.bfloat16, 1, n).contiguous() for h, n in ((H, "q"), (Hkv, "k"), (Hkv, "v")))
    pos, inv = torch.arange(N, dtype=torch.int32, device="cuda"), torch.from_numpy(oracle.rope_freqs(R)[0]).cuda()
    kw = dict(H=H, Hkv=Hkv, D=D, layout=int(interleaved), norm=B.NORM_LAYER)
    out = [torch.empty((N, h, D), dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv)]
    B.adt_norm_rope_qkv(q, k, v, pos, inv, q_out=out[0], k_out=out[1], v_out=out[2], **kw)
    check(out[0], q, True, 1e-6, None, None, pos.cpu().numpy(), inv.cpu().numpy(), 1.0, interleaved)
    B.adt_norm_rope_qkv(q, k, v, pos, inv, q_out=q, k_out=k, v_out=v, **kw)
    for a, o in zip((q, k, v), out):
        assert torch.equal(a.view(N, -1, D), o)
