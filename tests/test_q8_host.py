"""Refusals of the head norms and of the 8-bit cache that need no GPU: the checks run before any CUDA call, on
addresses that nothing reads.  (No call here is one that is accepted: it would be launched where there is a GPU.)"""
import ctypes
import math

import pytest
import torch

from paper_2512_21857_gb300 import binding as B
from test_cache_ops_host import INVALID, P, UNSUPPORTED, _call, lib  # noqa: F401 (lib: a fixture)

WORKSPACE = 5


def _at(base, shift):
    return ctypes.c_void_p(base.value + shift)


def _norm_args():
    return dict(q=P[0], ldq=384, k=P[1], ldk=384, v=P[2], ldv=384, typ=0, norm=0, eps=1e-6, qw=P[8], qb=None, qws=0, kw=P[9],
                kb=None, kws=0, wtyp=1, pos=P[3], inv=P[4], mag=1.0, layout=0, N=4, H=1, Hkv=1, D=128, rot=128, qo=P[5],
                ko=P[6], vo=P[7], stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(typ=2), INVALID), (dict(wtyp=2), INVALID), (dict(wtyp=-1), INVALID), (dict(norm=2), INVALID), (dict(norm=-1), INVALID),
    (dict(eps=-1e-9), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(layout=2), INVALID),
    (dict(N=-1), INVALID), (dict(N=2 ** 31 - 1), INVALID), (dict(D=0), INVALID), (dict(D=5000), INVALID), (dict(rot=7), INVALID),
    (dict(rot=130), INVALID), (dict(rot=-2), INVALID), (dict(mag=math.nan), INVALID), (dict(q=None), INVALID),
    (dict(ko=None), INVALID), (dict(pos=None), INVALID), (dict(inv=None), INVALID), (dict(H=0), INVALID), (dict(Hkv=0), INVALID),
    (dict(ldq=127), INVALID), (dict(ldk=2 ** 41), INVALID), (dict(qws=127), INVALID), (dict(kws=-128), INVALID),
    (dict(qw=_at(P[8], 2)), INVALID), (dict(wtyp=0, kb=_at(P[9], 1)), INVALID), (dict(q=_at(P[0], 1)), INVALID),
    (dict(D=2048, rot=1026, ldq=2048, ldk=2048, ldv=2048), UNSUPPORTED),
    (dict(q=None, k=None, v=None, qo=None, ko=None, vo=None), INVALID),
    (dict(qo=P[0]), INVALID), (dict(qo=P[0], ldq=128, typ=1), INVALID), (dict(qo=P[1], ldk=128), INVALID),
    (dict(qo=P[6]), INVALID), (dict(qo=_at(P[0], 16), ldq=128), INVALID),
    (dict(qo=P[8]), INVALID), (dict(vo=_at(P[9], -1008)), INVALID),  # an output over the weights
])
def test_norm_refuses(lib, change, status):  # noqa: F811
    assert _call(lib.adt_norm_rope_qkv, _norm_args(), **change) == status


def test_norm_of_no_rows_is_done(lib):  # noqa: F811
    assert _call(lib.adt_norm_rope_qkv, _norm_args(), N=0, q=None, qo=None, pos=None) == 0


ROWS, HEAD, TREE, LAYER = 100, 6400, 2 * 6400, 4 * 6400  # [3][2][2] slices of 100 rows of 64


def _compact_args():
    return dict(kc=P[0], vc=P[1], ks=P[2], vs=P[3], kv=P[4], kvo=P[5], kt=P[6], vt=P[7], offs=P[8], path=P[9], max_path=8,
                alen=P[10], B=2, Hkv=2, D=64, layers=3, max_kv=ROWS, cls=LAYER, csb=TREE, csh=HEAD, sls=400, ssb=200, ssh=100,
                tls=64 * 2 * 20, stream=None)


def _read_args():
    return dict(kc=P[0], vc=P[1], ks=P[2], vs=P[3], kv=P[4], ko=P[6], vo=P[7], B=2, Hkv=2, D=64, layers=3, max_kv=ROWS,
                cls=LAYER, csb=TREE, csh=HEAD, sls=400, ssb=200, ssh=100, ols=LAYER, osb=TREE, osh=HEAD, stream=None)


def _attn_args():
    return dict(q=P[5], kc=P[0], vc=P[1], ks=P[2], vs=P[3], kv=P[4], csb=TREE, csh=HEAD, ssb=200, ssh=100, kt=P[6], vt=P[7],
                par=P[8], offs=P[9], B=2, H=4, Hkv=2, D=64, max_nodes=8, max_kv=ROWS, scale=0.125, out=P[10], lse=None, ws=P[11],
                bytes=1 << 40, stream=None)


CACHE = [  # refused by all three
    (dict(kc=None), INVALID), (dict(vc=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID),
    (dict(kv=None), INVALID), (dict(B=0), INVALID), (dict(B=65536), INVALID), (dict(Hkv=0), INVALID), (dict(D=96), UNSUPPORTED),
    (dict(D=32), UNSUPPORTED), (dict(max_kv=1 << 30), INVALID), (dict(csh=HEAD - 16), INVALID), (dict(csh=HEAD + 8), INVALID),
    (dict(csb=-TREE), INVALID), (dict(csb=2 ** 41), INVALID), (dict(ssh=99), INVALID), (dict(ssb=-200), INVALID),
    (dict(ssb=2 ** 41), INVALID), (dict(kc=_at(P[0], 8)), INVALID), (dict(vc=_at(P[1], 1)), INVALID),
    (dict(ks=P[0]), INVALID), (dict(vs=_at(P[1], 6000)), INVALID),  # scales within a cache
]


@pytest.mark.parametrize("change,status", CACHE + [
    (dict(kt=None), INVALID), (dict(vt=None), INVALID), (dict(offs=None), INVALID), (dict(path=None), INVALID),
    (dict(alen=None), INVALID), (dict(layers=0), INVALID), (dict(layers=65536), INVALID), (dict(max_path=0), INVALID),
    (dict(max_path=(1 << 20) + 1), INVALID), (dict(max_kv=0), INVALID), (dict(kvo=P[4]), INVALID),
    (dict(kvo=_at(P[4], 4)), INVALID), (dict(tls=-8), INVALID), (dict(tls=4), INVALID), (dict(kt=_at(P[6], 8)), INVALID),
    (dict(vc=P[0]), INVALID), (dict(vs=P[2]), INVALID),                             # K and V in one place
    (dict(vc=_at(P[0], HEAD)), INVALID), (dict(vc=_at(P[0], -LAYER)), INVALID),     # V on other slices of K
    (dict(vs=_at(P[2], 100)), INVALID), (dict(vs=_at(P[2], -299)), INVALID),
    (dict(csb=HEAD), INVALID), (dict(cls=TREE + HEAD), INVALID), (dict(ssb=100), INVALID), (dict(sls=300), INVALID),
])
def test_compact_refuses(lib, change, status):  # noqa: F811
    assert _call(lib.adt_kv_compact_q8, _compact_args(), **change) == status


@pytest.mark.parametrize("change,status", CACHE + [
    (dict(ko=None), INVALID), (dict(vo=None), INVALID), (dict(layers=0), INVALID), (dict(max_kv=0), INVALID),
    (dict(osh=HEAD - 8), INVALID), (dict(osb=TREE + 4), INVALID), (dict(ols=2 ** 41), INVALID), (dict(ko=_at(P[6], 2)), INVALID),
    (dict(vo=P[6]), INVALID), (dict(vo=_at(P[6], 2 * HEAD)), INVALID), (dict(osb=HEAD), INVALID),
    (dict(ko=P[0]), INVALID), (dict(vo=P[2]), INVALID), (dict(ko=_at(P[3], 320)), INVALID),  # over an input
    (dict(B=60000, Hkv=60000, layers=60000, csh=HEAD, csb=HEAD, cls=HEAD, ssh=100, ssb=100, sls=100), INVALID),
])
def test_read_refuses(lib, change, status):  # noqa: F811
    assert _call(lib.adt_kv_read_q8, _read_args(), **change) == status


@pytest.mark.parametrize("change,status", CACHE + [
    (dict(q=None), INVALID), (dict(kt=None), INVALID), (dict(vt=None), INVALID), (dict(par=None), INVALID),
    (dict(offs=None), INVALID), (dict(out=None), INVALID), (dict(H=5), INVALID), (dict(H=0), INVALID),
    (dict(max_nodes=0), INVALID), (dict(max_nodes=257), UNSUPPORTED), (dict(max_kv=-1), INVALID), (dict(scale=0.0), INVALID),
    (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(q=_at(P[5], 8)), INVALID),
    (dict(kt=_at(P[6], 8)), INVALID), (dict(out=_at(P[10], 8)), INVALID),
    (dict(B=60000, H=400, Hkv=2, max_nodes=64), INVALID),  # more query rows than a call takes
])
def test_attention_refuses(lib, change, status):  # noqa: F811
    assert _call(lib.adt_tree_attn_q8, _attn_args(), **change) == status


def test_attention_workspace_of_refused_shapes_is_nothing(lib):  # noqa: F811
    ok = dict(B=2, H=4, Hkv=2, D=64, max_nodes=8, max_kv=100)
    for change in (dict(B=0), dict(H=3), dict(Hkv=0), dict(D=96), dict(max_nodes=0), dict(max_nodes=257), dict(max_kv=-1),
                   dict(B=60000, H=400, max_nodes=64)):
        assert B.adt_tree_attn_q8_workspace_size(**dict(ok, **change)) == 0


def test_bindings_refuse_cpu_tensors(lib):  # noqa: F811
    bf, i32 = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    c, s = torch.zeros(1, 1, 1, 4, 64).to(torch.float8_e4m3fn), torch.zeros(1, 1, 1, 4, dtype=torch.uint8)
    tree = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        B.adt_norm_rope_qkv(bf, None, None, i32, torch.zeros(32, dtype=torch.float64), H=1, Hkv=1, D=64, q_out=bf)
    with pytest.raises(ValueError, match="CUDA"):
        B.adt_kv_compact_q8(c, c, s, s, i32, None, tree, tree, i32, i32, 1, i32, B=1, Hkv=1, D=64, num_layers=1, max_kv=4)
    with pytest.raises(ValueError, match="CUDA"):
        B.adt_kv_read_q8(c, c, s, s, i32, c.bfloat16(), c.bfloat16(), B=1, Hkv=1, D=64, num_layers=1, max_kv=4)
    with pytest.raises(ValueError, match="CUDA"):
        B.adt_tree_attn_q8(bf.view(2, 1, 64), c[0], c[0], s[0], s[0], i32, tree[0], tree[0], i32, i32, B=1, H=1, Hkv=1, D=64,
                           max_nodes=2, max_kv=4, softmax_scale=1.0, out=bf, workspace=torch.zeros(16, dtype=torch.uint8))
