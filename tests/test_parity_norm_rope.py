"""adt_norm_rope_qkv on the GPU against the fp64 oracle.

Bound.  Sums of D values are made by lanes in turn and then across lanes: at most
D / 16 + 5 <= 261 roundings of 2^-24 one after the other, so a mean is within
2^-16 of the mean magnitude and a variance within 2^-15 of its value, beside
what the centred values carry.  With z the normed element, A = mean |x| / sqrt(mean
square + eps) and the root within 2^-15: z is within 2^-15 (1 + |z|) (1 + A).
Times the weight (one rounding), plus the bias (one more): within
|w| 2^-15 (1 + |z|) (1 + A) + 2^-22 (|w z| + |b|).  The rotation adds the
slack of both elements of a pair, and 2^-20 of their sizes (as adt_rope_qkv),
and the result is rounded to bf16 once: 2^-8 of it."""
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


def rows_of(N, width, dtype, seed, name, pad=0, shift=0.0):
    x = synth.f32_normal((N, width + pad), seed, name, std=1.5) + np.float32(shift)
    x[:, ::37] *= 8
    return torch.from_numpy(x).to(dtype).cuda()[:, :width]


def params_of(h, D, per_head, dtype, seed, name, bias):
    shape = (h, D) if per_head else (D,)
    w = torch.from_numpy(1 + synth.f32_normal(shape, seed, name + "w", std=0.3)).to(dtype).cuda()
    return w, torch.from_numpy(synth.f32_normal(shape, seed, name + "b", std=0.2)).to(dtype).cuda() if bias else None


def check(got, x, layer, eps, w, b, pos, inv, magnitude, interleaved):
    N, h, D = got.shape
    x = x.double().cpu().numpy().reshape(N, h, D)
    w = np.ones(D) if w is None else w.double().cpu().numpy()
    b = np.zeros(D) if b is None else b.double().cpu().numpy()
    y, z, spread = oracle.norm_rows(x, layer, eps, w, b)
    slack = np.abs(w) * 2.0 ** -15 * (1 + np.abs(z)) * (1 + spread) + 2.0 ** -22 * (np.abs(w * z) + np.abs(b))
    slack += 2.0 ** -20 * np.abs(y)
    far = np.abs(np.asarray(pos, np.float64)).max() * (inv.max() if len(inv) else 0.0) * 2.0 ** -51
    R = 2 * len(inv)
    i = np.arange(R // 2)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    slack[..., ia] = slack[..., ib] = abs(magnitude) * (slack[..., ia] + slack[..., ib] +
                                                        far * (np.abs(y[..., ia]) + np.abs(y[..., ib])))
    ref = oracle.rope_rows(y, pos, inv, magnitude, interleaved)
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= slack + 2.0 ** -8 * (np.abs(ref) + slack)).all(), (err - slack - 2.0 ** -8 * np.abs(ref)).max()


@pytest.mark.parametrize("N,H,Hkv,D,R", [
    (1, 32, 32, 128, 128), (1, 1, 1, 64, 64), (64, 32, 8, 128, 64), (5, 20, 20, 64, 64), (333, 8, 2, 128, 128),
    (3, 7, 1, 80, 80), (3, 5, 5, 80, 48), (2, 3, 3, 6, 2), (9, 4, 2, 64, 16), (4, 4, 4, 128, 0), (2, 2, 1, 33, 20),
    (3, 3, 2, 96, 90), (2, 2, 2, 256, 256), (6, 3, 1, 512, 32), (1, 2, 1, 1500, 1024), (2, 1, 1, 4096, 64), (700, 40, 10, 128, 32),
    (3, 2, 2, 1, 0), (2000, 8, 8, 64, 64), (1500, 5, 1, 72, 30), (1100, 40, 10, 128, 36), (9, 4, 2, 64, 10),
    (3, 2, 2, 256, 250), (6, 3, 1, 512, 30), (1300, 1, 1, 48, 2)])
@pytest.mark.parametrize("layer,interleaved", [(False, False), (True, True), (False, True), (True, False)])
@pytest.mark.parametrize("dtype,wtype", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16),
                                         (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("packed", [True, False])
def test_norm_rope_matches_oracle(N, H, Hkv, D, R, layer, interleaved, dtype, wtype, packed):
    seed = N + H + D + R
    if packed:
        rows = rows_of(N, (H + 2 * Hkv) * D, dtype, seed, "rows", shift=0.4)
        q, k, v = rows.split([H * D, Hkv * D, Hkv * D], 1)
    else:  # rows of their own, with strides of their own (odd ones among them)
        q, k, v = (rows_of(N, h * D, dtype, seed, n, pad) for h, n, pad in ((H, "q", 0), (Hkv, "k", 8), (Hkv, "v", 3)))
    pos = synth.rng(seed, "pos").integers(0, 5000, size=N).astype(np.int32)
    inv = oracle.rope_freqs(R)[0] if R else np.zeros(0)
    qw, qb = params_of(H, D, packed, wtype, seed, "q", layer)
    kw, kb = params_of(Hkv, D, not packed, wtype, seed, "k", not interleaved)
    out = [torch.full((N, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv)]
    B.adt_norm_rope_qkv(q, k, v, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), H=H, Hkv=Hkv, D=D,
                        norm=B.NORM_LAYER if layer else B.NORM_RMS, eps=1e-5, q_weight=qw, q_bias=qb, k_weight=kw, k_bias=kb,
                        layout=B.ROPE_INTERLEAVED if interleaved else B.ROPE_HALF, magnitude=1.25, q_out=out[0], k_out=out[1],
                        v_out=out[2])
    check(out[0], q, layer, 1e-5, qw, qb, pos, inv, 1.25, interleaved)
    check(out[1], k, layer, 1e-5, kw, kb, pos, inv, 1.25, interleaved)
    assert torch.equal(out[2].flatten(), v.to(torch.bfloat16).flatten())


@pytest.mark.parametrize("D,R", [(128, 128), (80, 50), (33, 0)])
@pytest.mark.parametrize("layer", [False, True])
def test_large_means_small_rows_and_absent_weights(D, R, layer):
    """Rows whose mean is 30 times their spread, tiny rows that eps decides, rows of zeros; no weights; k only."""
    N, H = 5, 3
    x = rows_of(N, H * D, torch.float32, 9, "x")
    x[0] = x[0] / 40 + 50.0
    x[1] *= 1e-4
    x[2] = 0
    x[3] *= 1e6
    pos, inv = np.arange(N, dtype=np.int32), oracle.rope_freqs(R)[0] if R else np.zeros(0)
    out = torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda")
    B.adt_norm_rope_qkv(None, x, None, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), H=1, Hkv=H, D=D,
                        norm=B.NORM_LAYER if layer else B.NORM_RMS, eps=1e-6, k_out=out)
    check(out, x, layer, 1e-6, None, None, pos, inv, 1.0, False)
    assert not out[2].any()


def test_many_tokens_of_one_large_head():
    """A thread block's tokens are as many as the angles leave room for."""
    N, D = 40000, 512
    q = rows_of(N, D, torch.bfloat16, 4, "q")
    pos, inv = np.arange(N, dtype=np.int32), oracle.rope_freqs(D)[0]
    out = torch.empty((N, 1, D), dtype=torch.bfloat16, device="cuda")
    B.adt_norm_rope_qkv(q, None, None, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), H=1, Hkv=1, D=D, q_out=out)
    check(out, q, False, 1e-6, None, None, pos, inv, 1.0, False)


def test_far_and_negative_positions():
    pos = np.array([0, 1, -1, 99999, 1 << 20, (1 << 20) + 1, 2 ** 31 - 1, -2 ** 31, 123456789], np.int32)
    q = rows_of(len(pos), 2 * 128, torch.float32, 5, "q")
    inv = oracle.rope_freqs(128, 500000.0)[0]
    out = torch.empty((len(pos), 2, 128), dtype=torch.bfloat16, device="cuda")
    B.adt_norm_rope_qkv(q, None, None, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda(), H=2, Hkv=1, D=128, q_out=out)
    check(out, q, False, 1e-6, None, None, pos, inv, 1.0, False)


@pytest.mark.parametrize("D,R", [(128, 128), (128, 64), (64, 10)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_equals_out_of_place(D, R, interleaved):
    N, H, Hkv = 37, 8, 2
    q, k = rows_of(N, H * D, torch.bfloat16, 1, "q"), rows_of(N, Hkv * D, torch.bfloat16, 1, "k")
    pos, inv = torch.arange(N, dtype=torch.int32, device="cuda"), torch.from_numpy(oracle.rope_freqs(R)[0]).cuda()
    kw = dict(H=H, Hkv=Hkv, D=D, layout=int(interleaved), norm=B.NORM_LAYER)
    qo, ko = (torch.empty((N, h, D), dtype=torch.bfloat16, device="cuda") for h in (H, Hkv))
    B.adt_norm_rope_qkv(q, k, None, pos, inv, q_out=qo, k_out=ko, **kw)
    q, k = q.contiguous(), k.contiguous()
    B.adt_norm_rope_qkv(q, k, None, pos, inv, q_out=q, k_out=k, **kw)
    assert torch.equal(q.view(N, H, D), qo) and torch.equal(k.view(N, Hkv, D), ko)


@pytest.mark.parametrize("D,R", [(64, 64), (128, 32), (80, 50)])
def test_odd_values_stay_in_their_heads(D, R):
    N, H = 3, 4
    x = rows_of(N, H * D, torch.float32, 2, "x")
    y = x.clone()
    y[1, D + 3] = float("nan")
    y[2, 3 * D] = float("inf")
    pos, inv = torch.tensor([4, 5, 6], dtype=torch.int32, device="cuda"), torch.from_numpy(oracle.rope_freqs(R)[0]).cuda()
    out = [torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for src, o in zip((x, y), out):
        B.adt_norm_rope_qkv(src, None, None, pos, inv, H=H, Hkv=1, D=D, norm=B.NORM_LAYER, q_out=o)
    same = torch.ones(N, H, dtype=torch.bool, device="cuda")
    same[1, 1] = same[2, 3] = False
    assert torch.equal(out[0][same], out[1][same]) and torch.isnan(out[1][1, 1]).all() and torch.isnan(out[1][2, 3]).all()


def test_no_rows_another_stream_and_a_graph():
    N, H, D = 64, 8, 128
    inv = torch.from_numpy(oracle.rope_freqs(D)[0]).cuda()
    e = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda")
    B.adt_norm_rope_qkv(e, None, None, torch.empty(0, dtype=torch.int32, device="cuda"), inv, H=1, Hkv=1, D=128,
                        q_out=torch.empty((0, 1, 128), dtype=torch.bfloat16, device="cuda"))
    q, pos = rows_of(N, H * D, torch.bfloat16, 3, "q"), torch.arange(N, dtype=torch.int32, device="cuda")
    w, b = params_of(H, D, True, torch.float32, 3, "q", True)
    out = torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda")
    kw = dict(H=H, Hkv=1, D=D, q_weight=w, q_bias=b, q_out=out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.adt_norm_rope_qkv(q, None, None, pos, inv, stream=s, **kw)
    s.synchronize()
    eager = out.clone()
    check(eager, q, False, 1e-6, w, b, pos.cpu().numpy(), inv.cpu().numpy(), 1.0, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.adt_norm_rope_qkv(q, None, None, pos, inv, **kw)
    out.zero_()
    graph.replay()
    assert torch.equal(out, eager)
    pos += 9
    graph.replay()
    check(out, q, False, 1e-6, w, b, pos.cpu().numpy(), inv.cpu().numpy(), 1.0, False)


def test_binding_refuses():
    q, pos = torch.zeros((2, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    inv, out = torch.ones(32, dtype=torch.float64, device="cuda"), torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    ok = dict(H=2, Hkv=1, D=64, q_out=out)
    for kw, err in [(dict(q_out=None), ValueError), (dict(H=3), ValueError), (dict(q_weight=w[:63]), ValueError),
                    (dict(q_weight=w.half()), TypeError), (dict(q_weight=w, q_bias=w.bfloat16()), TypeError),
                    (dict(q_weight=w, q_bias=w.expand(2, 64).contiguous()), ValueError),
                    (dict(q_weight=w.expand(2, 64)), ValueError), (dict(q_weight=w.cpu()), ValueError),
                    (dict(k_weight=w, q_weight=w.double()), TypeError), (dict(eps=-1.0), B.AdtError), (dict(norm=2), B.AdtError),
                    (dict(q_out=out.float()), TypeError)]:
        with pytest.raises(err):
            B.adt_norm_rope_qkv(q, None, None, pos, inv, **dict(ok, **kw))
