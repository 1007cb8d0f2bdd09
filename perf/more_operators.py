"""The 8-bit cache and what stands before it, as measurable cases: head norms with rotation, quantised commit, reading back, attention.

  norm    ``adt_norm_rope_qkv``: queries and keys of a projection normalised head by head and rotated, one pass;
  write   ``adt_kv_compact_q8``: the accepted path's K/V committed to a cache of 8-bit values with a scale for each row;
  read    ``adt_kv_read_q8``: rows of that cache as bf16 again;
  attn    ``adt_tree_attn_q8``: tree attention, and single tokens, over that cache.

A cached row (one kv head of one token) is D e4m3 values and one scale byte s: value = e4m3 * 2^(s - 127).  Caches are
[layers][trees][kv heads][rows][D], scales the same without D.  Lists of per-tree numbers are texts ("600,1337").
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
E4M3 = torch.float8_e4m3fn


def _ints(text):
    return [int(x) for x in str(text).split(",")]


def _text(values):
    return ",".join(str(int(v)) for v in values)


# ------------------------------------------------------------------ the cases

def _norm(**kw):
    return dict(dict(kind="norm", norm="rms", layout="half", dtype="bf16", per_head=False, bias=False, weight="f32"), **kw)


def _write(**kw):
    return dict(dict(kind="write"), **kw)


def _read(**kw):
    return dict(dict(kind="read"), **kw)


def _attn(**kw):
    return dict(dict(kind="attn", lse=False), **kw)


def listed():
    return [
        # One token of a 7B decoder on its way into attention: the smallest call, bound by its launch.
        _norm(name="norm_token_7b", N=1, H=32, Hkv=32, D=128, rot=128, pos=2399),
        # Eight images' draft trees of a target with grouped heads and a LayerNorm of its own for each head, fp32 residual
        # stream, half of each head rotated, pairs side by side.
        _norm(name="norm_trees_layer_f32", N=501, H=32, Hkv=8, D=128, rot=64, pos=5000, norm="layer", layout="interleaved",
              dtype="f32", per_head=True, bias=True),
        # A prompt of 16384 tokens at the 7B shape, weights as the model holds them: bound by memory.
        _norm(name="norm_prompt_7b", N=16384, H=32, Hkv=32, D=128, rot=128, pos=16383, weight="bf16"),
        # One layer after a single decoded token (8 heads x 64).
        _write(name="write_token", layers=1, Hkv=8, D=64, kv="512", path="1", nodes=26, lmax=576),
        # All 32 layers of the 7B verify step, eight tokens committed.
        _write(name="write_step_7b", layers=32, Hkv=32, D=128, kv="2400", path="8", nodes=64, lmax=2464),
        # The prompts of two guided branches as chains, all layers of a LlamaGen-XL-shaped target.
        _write(name="write_prompt_guided", layers=36, Hkv=20, D=64, kv="0,0", path="2048,1931", nodes=2048, lmax=2700),
        # One small layer back as bf16.
        _read(name="read_layer", layers=1, Hkv=8, D=64, kv="512", lmax=576),
        # Grouped heads, four images, eight layers: what an engine does that hands a cache over to bf16 operators.
        _read(name="read_grouped_ragged", layers=8, Hkv=8, D=128, kv="6001,1777,3500,5120", lmax=6144),
        # One token over a short cache, one layer, called by itself: latency.
        _attn(name="attn_token", kv="512", nodes="1", max_nodes=1, H=8, Hkv=8, D=64, lmax=576, lse=True),
        # Plain decoding of a ragged batch with grouped heads, long contexts.
        _attn(name="attn_tokens_grouped", kv="30011,905,12000,7777,20480,16384,2049,4097,9001,25000,1,6144,14333,3333,11111,8192",
              nodes="1," * 15 + "1", max_nodes=1, H=32, Hkv=8, D=128, lmax=30080),
        # A layer of the 7B verify step, four images with trees of 64 nodes and fewer.
        _attn(name="attn_trees_7b", kv="2400,2113,1444,2352", nodes="64,64,27,64", max_nodes=64, H=32, Hkv=32, D=128, lmax=2464),
        # Grouped heads, trees over long ragged prefixes.
        _attn(name="attn_trees_grouped", kv="6001,4777,3500,5120", nodes="64,64,64,64", max_nodes=64, H=32, Hkv=8, D=128,
              lmax=6144, lse=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "write", "read", "attn", "attn"])
    H, D = rng.choice([8, 20, 32, 40]), rng.choice([64, 128])
    Hkv = rng.choice([H, H, H // 4])
    if kind == "norm":
        D = rng.choice([64, 128, 128, 80, 256])
        rot = rng.choice([D, D, D // 2, 2 * rng.randint(0, D // 2)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        N = _log_int(rng, 1, min(16384, 300e6 / ((H + 2 * Hkv) * D * (4 if dtype == "bf16" else 6))))
        norm = rng.choice(["rms", "rms", "layer"])
        return _norm(N=N, H=H, Hkv=Hkv, D=D, rot=rot, pos=N - 1 + _log_int(rng, 1, 1000000), dtype=dtype, norm=norm,
                     layout=rng.choice(["half", "half", "interleaved"]), per_head=rng.random() < 0.3,
                     bias=norm == "layer" and rng.random() < 0.7, weight=rng.choice(["f32", "bf16"]))
    nb = rng.choice([1, 1, 2, 3, 4, 8])
    if kind == "attn":
        nb = rng.choice([1, 2, 4, 8, 16])
        most = rng.choice([1, 1, 8, 26, 64, 64, 192])
        kv = [_log_int(rng, 1, 30000) for _ in range(nb)]
        cap = 4e9 / (H * D * 4)  # flops of the largest listed case, over those of a (row, key)
        while sum(kv) * most > cap / 2 or max(kv) * nb * (Hkv * D * 8 + most * H * 8) > 8e9:
            kv = [max(1, L // 2) for L in kv]
        nodes = [rng.randint(max(1, most // 4), most) for _ in range(nb)]
        return _attn(kv=_text(kv), nodes=_text(nodes), max_nodes=most, H=H, Hkv=Hkv, D=D, lmax=max(kv) + most + rng.randint(0, 64),
                     lse=rng.random() < 0.5)
    kv = [_log_int(rng, 1, 8000) for _ in range(nb)]
    layers = max(1, min(rng.choice([1, 8, 32]), int(3e8 // (2 * sum(kv) * Hkv * D))))
    if kind == "read":
        return _read(layers=layers, Hkv=Hkv, D=D, kv=_text(kv), lmax=max(kv) + rng.randint(0, 64))
    cap = rng.choice([1, 6, 16, 64, 2048])
    path = [rng.randint(1, cap) for _ in range(nb)]
    nodes = max(rng.choice([26, 64]), cap)
    layers = max(1, min(layers, int(3e8 // (2 * nb * nodes * Hkv * D))))
    return _write(layers=layers, Hkv=Hkv, D=D, kv=_text(kv), path=_text(path), nodes=nodes, lmax=max(kv) + cap + rng.randint(0, 64))


def _own_keys(nodes):
    """(row, key) pairs of a tree that sit in the tree: the depths of `_parents`, whose node t has parent (t - 1) // 3."""
    depth = [1] * nodes
    for t in range(1, nodes):
        depth[t] = depth[(t - 1) // 3] + 1
    return sum(depth)


def work(case):
    if case["kind"] == "norm":
        vals = case["N"] * (case["H"] + 2 * case["Hkv"]) * case["D"]
        normed = case["N"] * (case["H"] + case["Hkv"]) * case["D"]
        heads = case["H"] + case["Hkv"] if case["per_head"] else 2
        weights = heads * case["D"] * (4 if case["weight"] == "f32" else 2) * (2 if case["bias"] else 1)
        return {"bytes": vals * ((2 if case["dtype"] == "bf16" else 4) + 2) + 4 * case["N"] + weights, "flops": 8 * normed}
    D, Hkv, kv = case["D"], case["Hkv"], _ints(case["kv"])
    if case["kind"] == "attn":
        H, nodes = case["H"], _ints(case["nodes"])
        pairs = sum(n * L + _own_keys(n) for L, n in zip(kv, nodes))
        return {"bytes": sum(kv) * Hkv * (2 * D + 2) + sum(nodes) * (4 * Hkv * D + 4 * H * D + 4 * H * case["lse"]),
                "flops": 4 * D * H * pairs}
    rows = case["layers"] * Hkv * (sum(kv) if case["kind"] == "read" else sum(_ints(case["path"])))
    return {"bytes": rows * 2 * (3 * D + 1), "flops": 0}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rand(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _bf16(g, *shape):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    for part in out:
        part.copy_(_rand(g, *shape[1:]))
    return out


def _i32(x):
    return torch.as_tensor(list(x), dtype=torch.int32, device=DEV)


def _norm_state(case, seed):
    g = _gen(seed)
    N, H, Hkv, D, R = (case[k] for k in ("N", "H", "Hkv", "D", "rot"))
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    rows = _rand(g, N, (H + 2 * Hkv) * D) * 1.7 + (0.3 if case["norm"] == "layer" else 0.0)
    rows[:, ::37] *= 8  # channels that stand out, as trained projections have
    q, k, v = rows.to(t).split([H * D, Hkv * D, Hkv * D], 1)  # one packed projection
    pos = torch.arange(case["pos"] - N + 1, case["pos"] + 1, device=DEV, dtype=torch.int32)
    if N <= 512:  # the nodes of trees: siblings share a position
        pos = (pos - torch.randint(0, 6, (N,), generator=g, device=DEV, dtype=torch.int32)).clamp_min(0)
    wt = torch.float32 if case["weight"] == "f32" else torch.bfloat16
    par = {}
    for x, h in (("q", H), ("k", Hkv)):
        shape = (h, D) if case["per_head"] else (D,)
        par[x + "_weight"] = (1 + 0.2 * _rand(g, *shape)).to(wt)
        par[x + "_bias"] = (0.1 * _rand(g, *shape)).to(wt) if case["bias"] else None
    inv = torch.tensor([10000.0 ** (-2.0 * p / R) for p in range(R // 2)], dtype=torch.float64, device=DEV)
    out = [torch.empty((N, h, D), dtype=torch.bfloat16, device=DEV) for h in (H, Hkv, Hkv)]
    return dict(q=q, k=k, v=v, pos=pos, inv=inv, par=par, out=out)


def _power(e):
    """2^e in fp32 for whole numbers e from -126 to 127, by its bits: exact."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantised(x):
    """(bytes as e4m3, scale bytes) of rows x in fp32: the least power of two with max |x| <= 448 times it, 2^-120 at least."""
    most = x.abs().amax(-1)
    e = (torch.frexp(most).exponent - 9).clamp(min=-120)  # most < 2^(e + 9) = 512 * 2^e
    e = e + (most > 448 * _power(e)).to(e.dtype)
    return (x * _power(-e)[..., None]).to(E4M3), (e + 127).to(torch.uint8)


def _cache(g, *shape):
    """A cache of 8-bit rows and its scales, some rows larger than others."""
    values, scales = torch.empty(shape, dtype=E4M3, device=DEV), torch.empty(shape[:-1], dtype=torch.uint8, device=DEV)
    for v, s in zip(values, scales):
        x = _rand(g, *shape[1:])
        x *= 1 + (torch.rand((*shape[1:-1], 1), generator=g, device=DEV) < 0.1)
        x, e = _quantised(x)
        v.copy_(x)
        s.copy_(e)
    return values, scales


def _write_state(case, seed):
    g = _gen(seed)
    layers, Hkv, D, lmax, n = (case[k] for k in ("layers", "Hkv", "D", "lmax", "nodes"))
    kv, path = _i32(_ints(case["kv"])), _i32(_ints(case["path"]))
    nb, R = len(kv), int(path.max())
    kt, vt = _bf16(g, layers, nb * n, Hkv, D), _bf16(g, layers, nb * n, Hkv, D)
    kt[..., 1::29] *= 6  # key channels that stand out
    nodes = torch.rand((nb, n - 1), generator=g, device=DEV).argsort(1)[:, :R - 1].sort(1).values + 1
    paths = torch.cat([torch.zeros((nb, 1), dtype=torch.int64, device=DEV), nodes], 1).to(torch.int32)
    paths = torch.where(torch.arange(R, device=DEV)[None] < path[:, None], paths, -1).contiguous()
    cache = [torch.zeros((layers, nb, Hkv, lmax, D), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2)]
    scale = [torch.zeros((layers, nb, Hkv, lmax), dtype=torch.uint8, device=DEV) for _ in range(2)]
    return dict(kt=kt, vt=vt, kv=kv, kv_out=torch.zeros_like(kv), paths=paths, R=R, alen=path - 1, nb=nb,
                offs=_i32(n * b for b in range(nb + 1)), kc=cache[0], vc=cache[1], ks=scale[0], vs=scale[1])


def _read_state(case, seed):
    g = _gen(seed)
    kv = _i32(_ints(case["kv"]))
    shape = (case["layers"], len(kv), case["Hkv"], case["lmax"], case["D"])
    (kc, ks), (vc, vs) = _cache(g, *shape), _cache(g, *shape)
    out = [torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    return dict(kc=kc, vc=vc, ks=ks, vs=vs, kv=kv, nb=len(kv), ko=out[0], vo=out[1])


def _parents(nodes):
    """A drafted tree in layers: node t hangs below node (t - 1) // 3."""
    return [-1] + [(t - 1) // 3 for t in range(1, nodes)]


def _attn_state(case, seed):
    g = _gen(seed)
    H, Hkv, D, lmax, most = (case[k] for k in ("H", "Hkv", "D", "lmax", "max_nodes"))
    kv, nodes = _i32(_ints(case["kv"])), _ints(case["nodes"])
    nb, total = len(kv), sum(nodes)
    (kc, ks), (vc, vs) = _cache(g, nb, Hkv, lmax, D), _cache(g, nb, Hkv, lmax, D)
    q, kt, vt = _bf16(g, total, H, D), _bf16(g, total, Hkv, D), _bf16(g, total, Hkv, D)
    offs = [sum(nodes[:b]) for b in range(nb + 1)]
    st = dict(kc=kc, vc=vc, ks=ks, vs=vs, kv=kv, q=q, kt=kt, vt=vt, nb=nb, offs=_i32(offs),
              parents=_i32(x for n in nodes for x in _parents(n)), out=torch.empty((total, H, D), dtype=torch.bfloat16, device=DEV),
              lse_out=torch.empty((total, H), device=DEV) if case["lse"] else None, ws={})
    # which node sits in slot t of tree b, and which slots of the tree a slot sees
    st["at"] = torch.tensor([[offs[b] + min(t, n - 1) for t in range(most)] for b, n in enumerate(nodes)], device=DEV)
    st["there"] = torch.tensor([[t < n for t in range(most)] for n in nodes], device=DEV)
    see = torch.eye(most, dtype=torch.bool)
    for t, p in enumerate(_parents(most)):
        if p >= 0:
            see[t] |= see[p]
    st["see"] = see.to(DEV)
    return st


def prepare(case, seed):
    make = {"norm": _norm_state, "write": _write_state, "read": _read_state, "attn": _attn_state}[case["kind"]]
    return dict(make(case, seed), case=case)


# ------------------------------------------------------------------ plain forms

def _turn(x, c, s, rot, layout):
    """Rows x [N, heads, D] in fp32 with the first `rot` values of each head rotated."""
    head, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        return torch.cat([a * c - b * s, b * c + a * s, rest], -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), rest], -1)


def _norm_plain(st):
    case = st["case"]
    N, D, par = case["N"], case["D"], st["par"]
    angle = st["pos"].double()[:, None] * st["inv"]
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def one(name):
        x = st[name].float().view(N, -1, D)
        if case["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * par[name + "_weight"].float()
        if case["bias"]:
            x = x + par[name + "_bias"].float()
        return _turn(x, c, s, case["rot"], case["layout"]).to(torch.bfloat16)

    return [one("q"), one("k"), st["v"].to(torch.bfloat16).view(N, -1, D)]


def _values(cache, scale):
    """What 8-bit rows stand for, in fp32."""
    return cache.float() * _power(scale.to(torch.int32) - 127)[..., None]


def _write_plain(st):
    """Every path entry quantised, and put where it goes in the cache."""
    layers, lmax, R = st["case"]["layers"], st["case"]["lmax"], st["R"]
    there = (torch.arange(R, device=DEV)[None] < st["alen"][:, None] + 1).nonzero()  # (tree, entry)
    b, i = there[:, 0], there[:, 1]
    at, row = (st["offs"][b] + st["paths"][b, i]).long(), (st["kv"][b] + i).long()
    for tree, cache, scale in ((st["kt"], st["kc"], st["ks"]), (st["vt"], st["vc"], st["vs"])):
        x, e = _quantised(tree[:, at].float())  # [layers, entries, Hkv, D]
        cache.view(torch.uint8)[:, b, :, row] = x.view(torch.uint8).transpose(0, 1)
        scale[:, b, :, row] = e.transpose(0, 1)
    st["kv_out"].copy_(st["kv"] + st["alen"] + 1)
    return st["kc"], st["vc"], st["ks"], st["vs"], st["kv_out"]


def _read_plain(st):
    there = (torch.arange(st["case"]["lmax"], device=DEV) < st["kv"][:, None])[None, :, None, :, None]
    for cache, scale, out in ((st["kc"], st["ks"], st["ko"]), (st["vc"], st["vs"], st["vo"])):
        out.copy_(torch.where(there, _values(cache, scale).to(torch.bfloat16), out))
    return st["ko"], st["vo"]


def _attn_plain(st):
    case = st["case"]
    H, Hkv, D, lmax, most = (case[k] for k in ("H", "Hkv", "D", "lmax", "max_nodes"))
    nb, G = st["nb"], H // Hkv
    keys = torch.cat([_values(st["kc"], st["ks"]), st["kt"].float()[st["at"]].transpose(1, 2)], 2)
    vals = torch.cat([_values(st["vc"], st["vs"]), st["vt"].float()[st["at"]].transpose(1, 2)], 2)
    q = st["q"].float()[st["at"]].view(nb, most, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(nb, Hkv, G * most, D)
    s = (q @ keys.transpose(2, 3) * D ** -0.5).view(nb, Hkv, G, most, lmax + most)
    prefix = (torch.arange(lmax, device=DEV) < st["kv"][:, None])[:, None].expand(nb, most, lmax)
    see = torch.cat([prefix, (st["see"] & st["there"][:, None]) | torch.eye(most, dtype=torch.bool, device=DEV)], 2)[:, None, None]
    s = torch.where(see, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    w = torch.exp(s - top)
    total = w.sum(-1, keepdim=True)
    o = (w / total).view(nb, Hkv, G * most, lmax + most) @ vals
    o = o.view(nb, Hkv, G, most, D).permute(0, 3, 1, 2, 4).reshape(nb, most, H, D)
    st["out"].copy_(o[st["there"]])
    if st["lse_out"] is None:
        return st["out"]
    lse = (top + torch.log(total)).view(nb, H, most).transpose(1, 2)
    st["lse_out"].copy_(lse[st["there"]])
    return st["out"], st["lse_out"]


def run(st):
    case = st["case"]
    if not own:
        return {"norm": _norm_plain, "write": _write_plain, "read": _read_plain, "attn": _attn_plain}[case["kind"]](st)
    from paper_2512_21857_gb300 import binding as B
    if case["kind"] == "norm":
        q, k, v = st["out"]
        B.adt_norm_rope_qkv(st["q"], st["k"], st["v"], st["pos"], st["inv"], H=case["H"], Hkv=case["Hkv"], D=case["D"],
                            norm=B.NORM_LAYER if case["norm"] == "layer" else B.NORM_RMS, eps=1e-6,
                            layout=B.ROPE_HALF if case["layout"] == "half" else B.ROPE_INTERLEAVED, q_out=q, k_out=k, v_out=v,
                            **st["par"])
        return [q, k, v]
    if case["kind"] == "write":
        B.adt_kv_compact_q8(st["kc"], st["vc"], st["ks"], st["vs"], st["kv"], st["kv_out"], st["kt"], st["vt"], st["offs"],
                            st["paths"], st["R"], st["alen"], B=st["nb"], Hkv=case["Hkv"], D=case["D"],
                            num_layers=case["layers"], max_kv=case["lmax"])
        return st["kc"], st["vc"], st["ks"], st["vs"], st["kv_out"]
    if case["kind"] == "read":
        B.adt_kv_read_q8(st["kc"], st["vc"], st["ks"], st["vs"], st["kv"], st["ko"], st["vo"], B=st["nb"], Hkv=case["Hkv"],
                         D=case["D"], num_layers=case["layers"], max_kv=case["lmax"])
        return st["ko"], st["vo"]
    shape = dict(B=st["nb"], H=case["H"], Hkv=case["Hkv"], D=case["D"], max_nodes=case["max_nodes"], max_kv=case["lmax"])
    if "own" not in st["ws"]:  # the workspace that a user's program keeps
        st["ws"]["own"] = B.zeroed_workspace(B.adt_tree_attn_q8_workspace_size(**shape))
    B.adt_tree_attn_q8(st["q"], st["kc"], st["vc"], st["ks"], st["vs"], st["kv"], st["kt"], st["vt"], st["parents"], st["offs"],
                       softmax_scale=case["D"] ** -0.5, out=st["out"], lse=st["lse_out"], workspace=st["ws"]["own"], **shape)
    return st["out"] if st["lse_out"] is None else (st["out"], st["lse_out"])


# ------------------------------------------------------------------ exact values

def _norm_exact(case, st):
    N, H, Hkv, D, R = (case[k] for k in ("N", "H", "Hkv", "D", "rot"))
    unit = torch.polar(torch.ones((N, R // 2), dtype=torch.float64, device=DEV), torch.outer(st["pos"].double(), st["inv"]))
    out = []
    for x, h in (("q", H), ("k", Hkv)):
        y = st[x].double().reshape(N, h, D)
        if case["norm"] == "layer":
            y = (y - y.sum(-1, keepdim=True) / D) / torch.sqrt(y.var(-1, unbiased=False, keepdim=True) + 1e-6)
        else:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / D + 1e-6)
        y = y * st["par"][x + "_weight"].double()
        if case["bias"]:
            y = y + st["par"][x + "_bias"].double()
        i = torch.arange(R // 2, device=DEV)
        re, im = (i, i + R // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(y[:, :, re], y[:, :, im]) * unit[:, None, :]
        y[:, :, re], y[:, :, im] = z.real, z.imag
        out.append(y)
    return out + [st["v"].double().reshape(N, Hkv, D)]


def _e4m3_exact(y):
    """y in 64 bits to the nearest e4m3 value, halves to even: steps of an eighth of its power of two, of 2^-9 at least."""
    step = _power64(torch.frexp(y.abs().clamp_min(2.0 ** -6)).exponent - 4)
    return torch.round(y / step) * step


def _power64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _write_exact(case, st):
    out = [x.double() for x in (st["kc"], st["vc"])] + [x.clone() for x in (st["ks"], st["vs"])] + [torch.zeros_like(st["kv"])]
    for b, (L, n) in enumerate(zip(_ints(case["kv"]), _ints(case["path"]))):
        at = b * case["nodes"] + st["paths"][b, :n].long()
        for j, tree in enumerate((st["kt"], st["vt"])):
            for layer in range(case["layers"]):
                x = tree[layer, at].double().transpose(0, 1)
                most = x.abs().max(-1).values
                e = torch.ceil(torch.log2(most.clamp_min(1e-300) / 448)).clamp_min(-120)
                e = torch.where(most <= 448 * _power64(e - 1), e - 1, torch.where(most > 448 * _power64(e), e + 1, e)).clamp_min(-120)
                out[j][layer, b, :, L:L + n] = _e4m3_exact(x / _power64(e)[..., None])
                out[2 + j][layer, b, :, L:L + n] = (e + 127).to(torch.uint8)
        out[4][b] = L + n
    return tuple(out)


def _read_exact(case, st):
    out = [st["ko"].double(), st["vo"].double()]
    for o, x, s in zip(out, (st["kc"], st["vc"]), (st["ks"], st["vs"])):
        for b, L in enumerate(_ints(case["kv"])):
            o[:, b, :, :L] = x[:, b, :, :L].double() * _power64(s[:, b, :, :L].long() - 127)[..., None]
    return tuple(out)


def _attn_exact(case, st):
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    if work(case)["flops"] > 2e12:
        return None
    out = torch.empty((st["q"].shape[0], H, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((st["q"].shape[0], H), dtype=torch.float64, device=DEV)
    n0 = 0
    for b, (L, n) in enumerate(zip(_ints(case["kv"]), _ints(case["nodes"]))):
        up = _parents(n)
        mask = torch.full((n, n), -math.inf, dtype=torch.float64)
        for t in range(n):
            a = t
            while a >= 0:
                mask[t, a] = 0.0
                a = up[a]
        for h in range(H):
            g = h // (H // Hkv)
            k = torch.cat([st["kc"][b, g, :L].double() * _power64(st["ks"][b, g, :L].long() - 127)[:, None], st["kt"][n0:n0 + n, g].double()])
            v = torch.cat([st["vc"][b, g, :L].double() * _power64(st["vs"][b, g, :L].long() - 127)[:, None], st["vt"][n0:n0 + n, g].double()])
            s = torch.matmul(st["q"][n0:n0 + n, h].double(), k.T) / math.sqrt(D)
            s[:, L:] += mask.to(DEV)
            lse[n0:n0 + n, h] = torch.logsumexp(s, 1)
            out[n0:n0 + n, h] = torch.softmax(s, 1) @ v
        n0 += n
    return (out, lse) if case["lse"] else out


def exact(case, seed):
    return {"norm": _norm_exact, "write": _write_exact, "read": _read_exact, "attn": _attn_exact}[case["kind"]](case, prepare(case, seed))
