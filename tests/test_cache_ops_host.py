"""Host parts of the cache operators: the frequencies, and every refusal that
needs no GPU (the checks run before any CUDA call)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2512_21857_gb300 import binding as B

INVALID, UNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2512_21857_gb300 import build
    build.build()
    return B.lib()


@pytest.mark.parametrize("R", [2, 6, 64, 128])
@pytest.mark.parametrize("name,code,kw", [
    ("none", B.ROPE_NONE, {}), ("linear", B.ROPE_LINEAR, dict(factor=4.0)), ("ntk", B.ROPE_NTK, dict(factor=8.0)),
    ("by_parts", B.ROPE_BY_PARTS, dict(factor=4.0, orig_len=8192.0)),
    ("by_parts", B.ROPE_BY_PARTS, dict(factor=32.0, orig_len=2048.0, turns_lo=2.0, turns_hi=20.0))])
def test_frequencies_match_oracle(lib, R, name, code, kw):
    if name == "ntk" and R == 2:
        with pytest.raises(B.AdtError):
            B.adt_rope_freqs(R, scaling=code, **kw)
        return
    for theta in (10000.0, 500000.0, 1.0):
        inv, mag = B.adt_rope_freqs(R, theta=theta, scaling=code, **kw)
        want, wmag = oracle.rope_freqs(R, theta, name, **kw)
        # a power and a few products in fp64: 2^-53 each, the exponent (up to 2 ln 5e5 times an error of 2^-53) most of it
        np.testing.assert_allclose(inv.numpy(), want, rtol=64 * 2.0 ** -53)
        assert abs(mag - wmag) <= 2.0 ** -23 * wmag


@pytest.mark.parametrize("kw", [dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=1026), dict(theta=0.5),
                                dict(theta=math.inf), dict(theta=math.nan), dict(scaling=4), dict(scaling=-1),
                                dict(scaling=B.ROPE_LINEAR, factor=0.5), dict(scaling=B.ROPE_NTK, factor=math.nan),
                                dict(scaling=B.ROPE_BY_PARTS, factor=2.0, orig_len=0.0),
                                dict(scaling=B.ROPE_BY_PARTS, factor=2.0, orig_len=100.0, turns_lo=3.0, turns_hi=3.0)])
def test_frequencies_refuse(lib, kw):
    kw = dict(dict(rotary_dim=64), **kw)
    with pytest.raises(B.AdtError) as e:
        B.adt_rope_freqs(kw.pop("rotary_dim"), **kw)
    assert e.value.status == INVALID


def _call(fn, base, **change):
    args = dict(base, **change)
    return fn(*args.values())


P = [ctypes.c_void_p(1 << 20 << i) for i in range(12)]  # far apart, 16-byte aligned, never read: the checks fail first


def _rope_args():
    return dict(q=P[0], ldq=384, k=P[1], ldk=384, v=P[2], ldv=384, typ=0, pos=P[3], inv=P[4], mag=1.0, layout=0, N=4, H=1,
                Hkv=1, D=128, rot=128, qo=P[5], ko=P[6], vo=P[7], stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(typ=2), INVALID), (dict(layout=2), INVALID), (dict(N=-1), INVALID), (dict(D=0), INVALID), (dict(D=5000), INVALID),
    (dict(rot=7), INVALID), (dict(rot=130), INVALID), (dict(rot=-2), INVALID), (dict(mag=math.inf), INVALID),
    (dict(mag=math.nan), INVALID), (dict(q=None), INVALID), (dict(ko=None), INVALID), (dict(pos=None), INVALID),
    (dict(inv=None), INVALID), (dict(H=0), INVALID), (dict(Hkv=0), INVALID), (dict(ldq=127), INVALID),
    (dict(ldv=127), INVALID), (dict(ldk=2 ** 41), INVALID),
    (dict(q=None, k=None, v=None, qo=None, ko=None, vo=None), INVALID),
    (dict(D=2048, rot=1026, ldq=2048, ldk=2048, ldv=2048), UNSUPPORTED),
    (dict(q=ctypes.c_void_p((1 << 20) + 1)), INVALID), (dict(typ=1, q=ctypes.c_void_p((1 << 20) + 2)), INVALID),
    (dict(qo=P[0]), INVALID),                             # in place needs packed rows
    (dict(qo=P[0], ldq=128, typ=1), INVALID),             # ... and bf16 rows
    (dict(qo=P[1], ldk=128), INVALID),                    # an output over another input
    (dict(qo=P[6]), INVALID),                             # two outputs in one place
    (dict(qo=ctypes.c_void_p((1 << 20) + 16), ldq=128), INVALID),  # shifted against its input
])
def test_rope_refuses(lib, change, status):
    assert _call(lib.adt_rope_qkv, _rope_args(), **change) == status


def test_rope_refuses_more_rows_than_its_indexes_take(lib):
    one = dict(q=P[0], qo=P[5], k=None, ko=None, v=None, vo=None)
    assert _call(lib.adt_rope_qkv, _rope_args(), **dict(one, D=8, rot=8, ldq=8, qo=ctypes.c_void_p(1 << 50)),
                 N=2 ** 31 - 1) == INVALID
    # rows whose bytes pass 64 bits
    assert _call(lib.adt_rope_qkv, _rope_args(), **dict(one, ldq=2 ** 40, N=2 ** 29, qo=ctypes.c_void_p(1 << 50))) == INVALID


def test_rope_of_no_rows_is_done(lib):
    assert _call(lib.adt_rope_qkv, _rope_args(), N=0, q=None, qo=None, pos=None) == 0


def _score_args():
    return dict(q=P[0], lse=P[1], kc=P[2], kv=P[3], offs=P[4], path=P[5], max_path=8, alen=P[6], B=2, H=4, Hkv=2, D=64,
                layers=3, max_kv=100, qls=64 * 4 * 10, lls=40, cls=4 * 6400, csb=2 * 6400, csh=6400, scale=0.1, decay=1.0,
                si=P[7], so=P[7], sls=400, ssb=200, ssh=100, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(lse=None), INVALID), (dict(kc=None), INVALID), (dict(kv=None), INVALID),
    (dict(offs=None), INVALID), (dict(path=None), INVALID), (dict(alen=None), INVALID), (dict(si=None), INVALID),
    (dict(so=None), INVALID), (dict(B=0), INVALID), (dict(H=5), INVALID), (dict(H=0, Hkv=0), INVALID),
    (dict(layers=0), INVALID), (dict(max_path=0), INVALID), (dict(max_kv=0), INVALID), (dict(max_kv=1 << 30), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=math.nan), INVALID), (dict(decay=-0.1), INVALID), (dict(decay=1.1), INVALID),
    (dict(decay=math.nan), INVALID), (dict(csh=6392), INVALID), (dict(csb=6404), INVALID), (dict(cls=-8), INVALID),
    (dict(ssh=99), INVALID), (dict(ssb=-1), INVALID), (dict(qls=4), INVALID), (dict(q=ctypes.c_void_p(24)), INVALID),
    (dict(kc=ctypes.c_void_p(8)), INVALID), (dict(D=96), UNSUPPORTED), (dict(D=32), UNSUPPORTED),
    (dict(layers=4000, B=2000, cls=1 << 30, csb=1 << 20, sls=1 << 30, ssb=1 << 20), UNSUPPORTED),
    (dict(sls=2 ** 41), INVALID), (dict(max_path=1 << 20, H=2048, Hkv=2), INVALID),
    (dict(so=ctypes.c_void_p(P[7].value + 4)), INVALID),  # neither the same buffer nor apart
])
def test_score_refuses(lib, change, status):
    assert _call(lib.adt_kv_score, _score_args(), **change) == status


def _evict_args():
    return dict(k=P[0], v=P[1], sls=4 * 6400, ssb=2 * 6400, ssh=6400, score=P[2], cls=400, csb=200, csh=100, kv=P[3],
                kvo=P[4], ko=P[0], vo=P[1], dls=4 * 6400, dsb=2 * 6400, dsh=6400, so=P[2], ols=400, osb=200, osh=100,
                idx=P[5], B=2, Hkv=2, D=64, layers=3, max_kv=100, budget=50, sink=4, recent=8, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(score=None), INVALID), (dict(kv=None), INVALID),
    (dict(ko=None), INVALID), (dict(vo=None), INVALID), (dict(kvo=P[3]), INVALID), (dict(B=0), INVALID),
    (dict(Hkv=0), INVALID), (dict(layers=0), INVALID), (dict(max_kv=0), INVALID), (dict(budget=0), INVALID),
    (dict(sink=-1), INVALID), (dict(recent=-1), INVALID), (dict(sink=30, recent=21), INVALID),
    (dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID), (dict(D=80), UNSUPPORTED),
    (dict(max_kv=1 << 30, budget=50), INVALID), (dict(budget=1 << 30), INVALID),
    (dict(cls=2 ** 41), INVALID), (dict(ko=P[6], vo=P[7], dls=2 ** 41), INVALID), (dict(ssh=6399), INVALID), (dict(ssh=6300), INVALID),
    (dict(csh=99), INVALID), (dict(ko=P[6], vo=P[7], dsh=3199), INVALID), (dict(ko=P[6], vo=P[7], osh=49), INVALID),
    (dict(k=ctypes.c_void_p(8)), INVALID),
    (dict(ko=P[6]), INVALID),                              # K elsewhere, V in place
    (dict(dsh=6408), INVALID),                             # in place with other strides
    (dict(ko=ctypes.c_void_p(P[0].value + 16), vo=P[7]), INVALID),
    (dict(ko=P[1], vo=P[0]), INVALID),                     # K into V
    (dict(so=ctypes.c_void_p(P[2].value + 4)), INVALID),
    (dict(osh=104), INVALID),                              # scores in place with other strides
])
def test_evict_refuses(lib, change, status):
    assert _call(lib.adt_kv_evict, _evict_args(), **change) == status


def test_evict_refuses_one_destination_for_both_and_lengths_that_overlap(lib):
    # K and V onto one another: in place, and from caches of their own
    assert _call(lib.adt_kv_evict, _evict_args(), k=P[0], v=P[0], ko=P[0], vo=P[0]) == INVALID
    assert _call(lib.adt_kv_evict, _evict_args(), ko=P[6], vo=P[6]) == INVALID
    # tree 1's length read where tree 0's new one is written, and the other way round
    for shift in (4, -4):
        assert _call(lib.adt_kv_evict, _evict_args(), kvo=ctypes.c_void_p(P[3].value + shift)) == INVALID


def test_bindings_refuse_cpu_tensors_and_wrong_types(lib):
    bf, f32, i32 = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, 64), torch.zeros(2, dtype=torch.int32)
    inv = torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="CUDA"):
        B.adt_rope_qkv(bf, None, None, i32, inv, H=1, Hkv=1, D=64, q_out=bf)
    cache, score = torch.zeros(1, 1, 1, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 1, 4)
    with pytest.raises(ValueError, match="CUDA"):
        B.adt_kv_evict(cache, cache, score, i32, B=1, Hkv=1, D=64, num_layers=1, max_kv=4, budget=2)
    with pytest.raises(ValueError, match="CUDA"):
        B.adt_kv_score(bf.view(1, 2, 1, 64), torch.zeros(1, 2, 1), cache, i32, i32, i32, 1, i32, score, B=1, H=1, Hkv=1, D=64,
                       num_layers=1, max_kv=4, softmax_scale=1.0)
    with pytest.raises(ValueError, match="both or neither"):
        B.adt_kv_evict(cache, cache, score, i32, k_out=cache, B=1, Hkv=1, D=64, num_layers=1, max_kv=4, budget=2)
    with pytest.raises(ValueError, match="without moving"):
        B.adt_kv_evict(cache, cache, score, i32, score_out=score, move_scores=False, B=1, Hkv=1, D=64, num_layers=1,
                       max_kv=4, budget=2)
