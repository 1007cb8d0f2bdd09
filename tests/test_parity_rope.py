"""adt_rope_qkv on the GPU against the fp64 oracle.

Bound: the result is rounded to bf16 once, half a step of which is 2^-8 of the
value; before that it is made in fp32 from a cosine and a sine whose angle is
exact to 2^-23 rad (a fraction of a turn below 1/2 rounded to fp32: 2^-26
turns), that are within two units in the last place (2^-22) and take one more
rounding for the magnitude, then two products and a sum (2^-23 of |a| + |b|):
less than 2^-20 (|a| + |b|) magnitude in all.  Far positions add the fp64
angle's own rounding, in both: t f 2^-51 rad."""
import numpy as np
import pytest
import torch

import oracle
from gpu_cases import ensure_built
from paper_2512_21857_gb300 import binding as B
from paper_2512_21857_gb300 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()


def rows_of(N, width, dtype, seed, name, pad=0):
    x = synth.f32_normal((N, width + pad), seed, name, std=1.5)
    return torch.from_numpy(x).to(dtype).cuda()[:, :width]


def pair_sums(x, R, interleaved):
    """|a| + |b| of the pair that each element belongs to (0 where it is copied)."""
    s = np.zeros(x.shape)
    i = np.arange(R // 2)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    s[..., ia] = s[..., ib] = np.abs(x[..., ia]) + np.abs(x[..., ib])
    return s


def check(got, x, pos, inv, magnitude, interleaved):
    x = x.double().cpu().numpy().reshape(got.shape)
    ref = oracle.rope_rows(x, pos, inv, magnitude, interleaved)
    far = np.abs(np.asarray(pos, np.float64)).max() * (inv.max() if len(inv) else 0.0) * 2.0 ** -51
    slack = pair_sums(x, 2 * len(inv), interleaved) * abs(magnitude) * (2.0 ** -20 + far)
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= slack + 2.0 ** -8 * (np.abs(ref) + slack)).all(), (err - slack - 2.0 ** -8 * np.abs(ref)).max()


@pytest.mark.parametrize("N,H,Hkv,D,R", [
    (1, 32, 32, 128, 128), (1, 1, 1, 64, 64), (64, 32, 8, 128, 64), (5, 20, 20, 64, 64), (333, 8, 2, 128, 128),
    (3, 7, 1, 80, 80), (3, 5, 5, 80, 48), (2, 3, 3, 6, 2), (9, 4, 2, 64, 16), (4, 4, 4, 128, 0), (2, 2, 1, 33, 20),
    (3, 3, 2, 96, 90), (2, 2, 2, 256, 256), (1, 2, 1, 1500, 1024), (700, 40, 10, 128, 32)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("packed", [True, False])
def test_rope_matches_oracle(N, H, Hkv, D, R, interleaved, dtype, packed):
    seed = N + H + D + R
    if packed:
        rows = rows_of(N, (H + 2 * Hkv) * D, dtype, seed, "rows")
        q, k, v = rows.split([H * D, Hkv * D, Hkv * D], 1)
    else:  # rows of their own, with strides of their own (odd ones among them)
        q, k, v = (rows_of(N, h * D, dtype, seed, n, pad) for h, n, pad in ((H, "q", 0), (Hkv, "k", 8), (Hkv, "v", 3)))
    pos = synth.rng(seed, "pos").integers(0, 5000, size=N).astype(np.int32)
    inv = oracle.rope_freqs(R)[0] if R else np.zeros(0)
    out = [torch.full((N, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv)]
    B.adt_rope_qkv(q, k, v, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), H=H, Hkv=Hkv, D=D,
                   layout=B.ROPE_INTERLEAVED if interleaved else B.ROPE_HALF, magnitude=1.25, q_out=out[0], k_out=out[1],
                   v_out=out[2])
    check(out[0], q, pos, inv, 1.25, interleaved)
    check(out[1], k, pos, inv, 1.25, interleaved)
    assert torch.equal(out[2].flatten(), v.to(torch.bfloat16).flatten())


@pytest.mark.parametrize("D,R", [(128, 128), (80, 50)])
def test_rope_at_far_and_negative_positions(D, R):
    pos = np.array([0, 1, -1, 99999, 1 << 20, (1 << 20) + 1, 2 ** 31 - 1, -2 ** 31, 123456789], np.int32)
    N = len(pos)
    q = rows_of(N, 2 * D, torch.float32, 5, "q")
    inv = oracle.rope_freqs(R, 500000.0)[0]
    out = torch.empty((N, 2, D), dtype=torch.bfloat16, device="cuda")
    B.adt_rope_qkv(q, None, None, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), H=2, Hkv=1, D=D, q_out=out)
    check(out, q, pos, inv, 1.0, False)


@pytest.mark.parametrize("D,R", [(128, 128), (128, 64), (64, 10)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_in_place_equals_out_of_place(D, R, interleaved):
    N, H, Hkv = 37, 8, 2
    q, k = rows_of(N, H * D, torch.bfloat16, 1, "q"), rows_of(N, Hkv * D, torch.bfloat16, 1, "k")
    pos, inv = torch.arange(N, dtype=torch.int32, device="cuda"), torch.from_numpy(oracle.rope_freqs(R)[0]).cuda()
    kw = dict(H=H, Hkv=Hkv, D=D, layout=int(interleaved))
    qo, ko = (torch.empty((N, h, D), dtype=torch.bfloat16, device="cuda") for h in (H, Hkv))
    B.adt_rope_qkv(q, k, None, pos, inv, q_out=qo, k_out=ko, **kw)
    q, k = q.contiguous(), k.contiguous()
    B.adt_rope_qkv(q, k, None, pos, inv, q_out=q, k_out=k, **kw)
    assert torch.equal(q.view(N, H, D), qo) and torch.equal(k.view(N, Hkv, D), ko)


@pytest.mark.parametrize("D,R", [(64, 64), (64, 32), (80, 50)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_keeps_odd_values_to_their_pairs(D, R, interleaved):
    """An infinity or a NaN shows up in its own pair only; a position turns its own row only."""
    N, H = 3, 2
    x = rows_of(N, H * D, torch.float32, 2, "x")
    y = x.clone()
    bad = (1, D + 3)  # row 1, head 1, element 3
    y[bad] = float("nan")
    y[2, 0] = float("inf")
    pos, inv = torch.tensor([4, 5, 6], dtype=torch.int32, device="cuda"), torch.from_numpy(oracle.rope_freqs(R)[0]).cuda()
    out = [torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for src, o in zip((x, y), out):
        B.adt_rope_qkv(src, None, None, pos, inv, H=H, Hkv=1, D=D, layout=int(interleaved), q_out=o)
    odd = ~torch.isfinite(out[1])
    i, j = (2, 3) if interleaved else (3, 3 + R // 2)
    want = torch.zeros_like(odd)
    want[1, 1, [i, j]] = True
    want[2, 0, [0, 1 if interleaved else R // 2]] = True
    assert torch.equal(odd, want)
    assert torch.equal(out[0][~odd], out[1][~odd])


def test_rope_of_no_rows():
    e = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda")
    pos, inv = torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    B.adt_rope_qkv(e, None, None, pos, inv, H=2, Hkv=1, D=64, q_out=torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"))


def test_rope_on_another_stream_and_in_a_graph():
    N, H, D = 64, 8, 128
    q, pos = rows_of(N, H * D, torch.bfloat16, 3, "q"), torch.arange(N, dtype=torch.int32, device="cuda")
    inv = torch.from_numpy(oracle.rope_freqs(D)[0]).cuda()
    out = torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.adt_rope_qkv(q, None, None, pos, inv, H=H, Hkv=1, D=D, q_out=out, stream=s)
    s.synchronize()
    eager = out.clone()
    check(eager, q, pos.cpu().numpy(), inv.cpu().numpy(), 1.0, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.adt_rope_qkv(q, None, None, pos, inv, H=H, Hkv=1, D=D, q_out=out)
    out.zero_()
    graph.replay()
    assert torch.equal(out, eager)
    pos += 9
    graph.replay()
    check(out, q, pos.cpu().numpy(), inv.cpu().numpy(), 1.0, False)


def test_rope_binding_refuses():
    q, pos = torch.zeros((2, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    inv, out = torch.ones(32, dtype=torch.float64, device="cuda"), torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    ok = dict(H=2, Hkv=1, D=64, q_out=out)
    for args, kw, err in [((q, None, None, pos, inv), dict(q_out=None), ValueError), ((q, None, None, pos, inv), dict(H=3), ValueError),
                          ((q.half(), None, None, pos, inv), {}, TypeError), ((q, None, None, pos.long(), inv), {}, TypeError),
                          ((q, None, None, pos, inv.float()), {}, TypeError), ((q.t(), None, None, pos, inv), {}, ValueError),
                          ((q, None, None, pos, inv), dict(q_out=out.float()), TypeError),
                          ((q, q.float()[:, :64], None, pos, inv), dict(k_out=out[:, :1].contiguous()), TypeError),
                          ((q, None, None, pos, torch.ones(33, dtype=torch.float64, device="cuda")), {}, B.AdtError)]:
        with pytest.raises(err):
            B.adt_rope_qkv(*args, **dict(ok, **kw))
