"""The cache operators, as measurable cases: rotary positions, accumulated attention weight, eviction.

  rope    ``adt_rope_qkv``: the rows of a Q/K/V projection rotated to their positions, as they enter attention and cache;
  score   ``adt_kv_score``: the attention weight that every cached row got from the tokens just committed, added up;
  evict   ``adt_kv_evict``: the cache cut down to the rows with the most of it.

Lists of per-tree numbers are texts ("600,1337").  Caches are [layers][trees][kv heads][rows][D], as the library's are.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"


def _ints(text):
    return [int(x) for x in str(text).split(",")]


def _text(values):
    return ",".join(str(int(v)) for v in values)


# ------------------------------------------------------------------ the cases

def _rope(**kw):
    return dict(dict(kind="rope", layout="half", dtype="bf16", scaling="none", factor=1.0, theta=10000.0, packed=True), **kw)


def _score(**kw):
    return dict(dict(kind="score", decay=1.0), **kw)


def _evict(**kw):
    return dict(dict(kind="evict", inplace=True, sink=4, recent=64), **kw)


def listed():
    return [
        # One token of a 7B decoder, rotated on its way into attention: the smallest call, bound by its launch.
        _rope(name="rope_token_7b", N=1, H=32, Hkv=32, D=128, rot=128, pos=2399),
        # A 64-node draft tree of a target with grouped heads; half of each head rotated, pairs side by side, far into a
        # context four times the trained one (frequencies scaled by parts).
        _rope(name="rope_tree_partial", N=64, H=32, Hkv=8, D=128, rot=64, pos=120000, layout="interleaved",
              scaling="by_parts", factor=4.0, theta=500000.0),
        # fp32 residual stream (the decode loop's --decode-fp32), LlamaGen-XL heads, eight images' trees at once.
        _rope(name="rope_llamagen_f32", N=501, H=20, Hkv=20, D=64, rot=64, pos=575, dtype="f32"),
        # A prompt of 16384 tokens at the 7B shape: the largest, bound by memory.
        _rope(name="rope_prompt_7b", N=16384, H=32, Hkv=32, D=128, rot=128, pos=16383, scaling="linear", factor=4.0),
        # One layer after a single decoded token (8 heads x 64, KV 512).
        _score(name="score_token", layers=1, H=8, Hkv=8, D=64, kv="512", path="1", nodes=26, lmax=576),
        # All 32 layers of the 7B verify step after eight tokens were committed.
        _score(name="score_step_7b", layers=32, H=32, Hkv=32, D=128, kv="2400", path="8", nodes=64, lmax=2464),
        # Grouped heads over long ragged prefixes, four images, old weight fading.
        _score(name="score_grouped_ragged", layers=8, H=32, Hkv=8, D=128, kv="6001,4777,3500,5120", path="9,1,4,2", nodes=64,
               lmax=6144, decay=0.9),
        # A prompt of 256 tokens as one chain (the two branches of guidance) after 693 and 577 cached ones: every
        # token's weight counts, so the products and exponentials do too.
        _score(name="score_prompt_guided", layers=36, H=20, Hkv=20, D=64, kv="693,577", path="256,256", nodes=256, lmax=960),
        # One small layer, a few rows over its budget.
        _evict(name="evict_layer", layers=1, Hkv=8, D=64, kv="576", budget=512, lmax=576, recent=32),
        # All 32 layers of the 7B loop, 96 rows over the budget, in place: the turn that a bounded decode loop takes
        # every few steps.
        _evict(name="evict_step_7b", layers=32, Hkv=32, D=128, kv="2400", budget=2304, lmax=2464),
        # Prefill caches of two guided branches cut down into the smaller caches that decode on.
        _evict(name="evict_prompt_guided", layers=36, Hkv=20, D=64, kv="1693,1577", budget=512, lmax=1700, inplace=False),
        # Grouped heads, four images, one of them within its budget.
        _evict(name="evict_grouped_ragged", layers=8, Hkv=8, D=128, kv="6001,1777,3500,5120", budget=2048, lmax=6144,
               recent=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "score", "evict"])
    H, D = rng.choice([8, 20, 32, 40]), rng.choice([64, 128])
    Hkv = rng.choice([H, H, H // 4])
    if kind == "rope":
        D = rng.choice([64, 128, 128, 80])
        rot = rng.choice([D, D, D // 2, 2 * rng.randint(1, D // 2)])
        scaling = rng.choice(["none", "none", "linear", "ntk", "by_parts"]) if rot > 2 else "none"
        dtype = rng.choice(["bf16", "bf16", "f32"])
        N = _log_int(rng, 1, min(16384, 300e6 / ((H + 2 * Hkv) * D * (4 if dtype == "bf16" else 6))))
        return _rope(N=N, H=H, Hkv=Hkv, D=D, rot=rot, pos=N - 1 + _log_int(rng, 1, 1000000), dtype=dtype,
                     layout=rng.choice(["half", "half", "interleaved"]), scaling=scaling,
                     factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                     theta=rng.choice([10000.0, 500000.0]), packed=rng.random() < 0.7)
    nb = rng.choice([1, 1, 2, 3, 4, 8])
    kv = [_log_int(rng, 1, 8000) for _ in range(nb)]
    layers = max(1, min(rng.choice([1, 8, 32]), int(4e8 // (2 * sum(kv) * Hkv * D))))
    lmax = max(kv) + 256 + rng.randint(0, 64)
    if kind == "score":
        cap = rng.choice([1, 6, 16, 16, 64, 256])
        path = [rng.randint(1, cap) for _ in range(nb)]
        nb = max(1, min(nb, int(3e8 // (max(path) * H * lmax))))  # long paths of many heads: fewer images, fewer layers
        kv, path = kv[:nb], path[:nb]
        lmax = min(lmax, max(kv) + 300)
        layers = max(1, min(layers, int(3e8 // (nb * max(path) * H * lmax)), int(3e10 // (2 * D * H * sum(n * (L + n) for L, n in zip(kv, path))))))
        return _score(layers=layers, H=H, Hkv=Hkv, D=D, kv=_text(kv), path=_text(path), nodes=max(rng.choice([26, 64, 64]), cap),
                      lmax=lmax, decay=rng.choice([1.0, 1.0, 0.95, 0.0]))
    budget = _log_int(rng, 1, max(kv) * 1.1 + 1)
    recent = rng.randint(0, budget // 2)
    return _evict(layers=layers, Hkv=Hkv, D=D, kv=_text(kv), budget=budget, lmax=lmax, inplace=rng.random() < 0.6,
                  sink=rng.randint(0, min(4, budget - recent)), recent=recent)


def work(case):
    if case["kind"] == "rope":
        vals = case["N"] * (case["H"] + 2 * case["Hkv"]) * case["D"]
        pairs = case["N"] * (case["H"] + case["Hkv"]) * case["rot"] // 2
        return {"bytes": vals * ((2 if case["dtype"] == "bf16" else 4) + 2) + 4 * case["N"], "flops": 6 * pairs}
    layers, Hkv, D, kv = case["layers"], case["Hkv"], case["D"], _ints(case["kv"])
    if case["kind"] == "score":
        H, path = case["H"], _ints(case["path"])
        rows = sum(L + n for L, n in zip(kv, path))
        pairs = sum(n * L + n * (n + 1) // 2 for L, n in zip(kv, path))
        return {"bytes": layers * (rows * Hkv * (2 * D + 4) + sum(kv) * Hkv * 4 * (case["decay"] != 0) + sum(path) * H * (2 * D + 4)),
                "flops": layers * H * pairs * (2 * D + 3)}
    keep = [min(L, case["budget"]) for L in kv]
    # in place the sinks stay where they are, and so does a cache within its budget
    moved = sum(n - case["sink"] if L > n else 0 for L, n in zip(kv, keep)) if case["inplace"] else sum(keep)
    return {"bytes": layers * Hkv * (8 * D * moved + 4 * sum(kv) + 4 * sum(keep) + 4 * len(kv) * case["budget"]), "flops": 0}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _rand(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _bf16(g, *shape):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    for layer in out:
        layer.copy_(_rand(g, *shape[1:]))
    return out


def _i32(x):
    return torch.as_tensor(list(x), dtype=torch.int32, device=DEV)


def _frequencies(case):
    """Radians a position for each pair of a head, in 64 bits (a model's configuration fixes them once)."""
    R, theta, s = case["rot"], case["theta"], case["factor"]
    if case["scaling"] == "ntk":
        theta = theta * s ** (R / (R - 2))
    inv = [theta ** (-2.0 * p / R) for p in range(R // 2)]
    if case["scaling"] == "linear":
        inv = [f / s for f in inv]
    if case["scaling"] == "by_parts":  # trained on 8192 positions: what turns under once there is stretched, over 32 times is kept
        ramp = [min(1.0, max(0.0, (8192 * f / (2 * math.pi) - 1.0) / 31.0)) for f in inv]
        inv = [f * (g + (1.0 - g) / s) for f, g in zip(inv, ramp)]
    return inv, 0.1 * math.log(s) + 1.0 if case["scaling"] == "by_parts" else 1.0


def _rope_state(case, seed):
    g = _gen(seed)
    N, H, Hkv, D = (case[k] for k in ("N", "H", "Hkv", "D"))
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    rows = _rand(g, N, (H + 2 * Hkv) * D).to(t)  # a projection's output
    q, k, v = rows.split([H * D, Hkv * D, Hkv * D], 1)
    if not case["packed"]:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pos = torch.arange(case["pos"] - N + 1, case["pos"] + 1, device=DEV, dtype=torch.int32)
    if N <= 512:  # the nodes of trees: siblings share a position
        pos = (pos - torch.randint(0, 6, (N,), generator=g, device=DEV, dtype=torch.int32)).clamp_min(0)
    inv, magnitude = _frequencies(case)
    out = [torch.empty((N, h, D), dtype=torch.bfloat16, device=DEV) for h in (H, Hkv, Hkv)]
    return dict(q=q, k=k, v=v, pos=pos, inv=torch.tensor(inv, dtype=torch.float64, device=DEV), magnitude=magnitude, out=out)


def _chain_mask(kv, path, R, lmax):
    """[trees, R, lmax]: whether path entry i of a tree is there and sees cache row j (causal after the prefix)."""
    i = torch.arange(R, device=DEV)[None, :, None]
    j = torch.arange(lmax, device=DEV)[None, None, :]
    return (i < path[:, None, None]) & (j <= kv[:, None, None] + i)


def _score_state(case, seed):
    g = _gen(seed)
    layers, H, Hkv, D, lmax, n = (case[k] for k in ("layers", "H", "Hkv", "D", "lmax", "nodes"))
    kv, path = _i32(_ints(case["kv"])), _i32(_ints(case["path"]))
    nb, R, G = len(kv), int(path.max()), H // Hkv
    kc = _bf16(g, layers, nb, Hkv, lmax, D)
    # a few rows draw much of the attention, as the first tokens and other anchors do
    kc[:, :, :, :2] *= 2
    kc *= 1 + (torch.rand((layers, nb, Hkv, lmax, 1), generator=g, device=DEV) < 0.03).to(torch.bfloat16)
    q = _bf16(g, layers, nb * n, H, D)
    # the accepted path: nodes of the tree in ascending order, the root first; a chain takes them all
    nodes = torch.rand((nb, n - 1), generator=g, device=DEV).argsort(1)[:, :R - 1].sort(1).values + 1
    paths = torch.cat([torch.zeros((nb, 1), dtype=torch.int64, device=DEV), nodes], 1).to(torch.int32)
    paths = torch.where(torch.arange(R, device=DEV)[None] < path[:, None], paths, -1).contiguous()
    offs = _i32(n * b for b in range(nb + 1))
    # what attention returned for these rows
    lse = torch.zeros((layers, nb * n, H), device=DEV)
    at = (offs[:-1, None] + paths.clamp_min(0)).long()
    see = _chain_mask(kv, path, R, lmax)[:, None, :, None, :]
    for layer in range(layers):
        rows = q[layer][at].float().view(nb, R, Hkv, G, D).transpose(1, 2)
        s = (rows.reshape(nb, Hkv, R * G, D) @ kc[layer].float().transpose(2, 3)).view(nb, Hkv, R, G, lmax) * D ** -0.5
        z = torch.where(see, s, -math.inf).logsumexp(-1).transpose(1, 2).reshape(nb, R, H)
        there = torch.arange(R, device=DEV)[None] < path[:, None]
        lse[layer][at[there]] = z[there]
    score = torch.rand((layers, nb, Hkv, lmax), generator=g, device=DEV) * 3
    return dict(q=q, lse=lse, kc=kc, kv=kv, offs=offs, paths=paths, R=R, alen=path - 1, score=score, out=score.clone(), nb=nb)


def _evict_state(case, seed):
    g = _gen(seed)
    layers, Hkv, D, lmax, budget = (case[k] for k in ("layers", "Hkv", "D", "lmax", "budget"))
    kv = _i32(_ints(case["kv"]))
    nb = len(kv)
    kc, vc = _bf16(g, layers, nb, Hkv, lmax, D), _bf16(g, layers, nb, Hkv, lmax, D)
    # accumulated weight is spread over orders of magnitude; rows that nothing looked at share a score of zero
    score = torch.exp(1.5 * _rand(g, layers, nb, Hkv, lmax))
    score *= torch.rand(score.shape, generator=g, device=DEV) > 0.02
    st = dict(kc=kc, vc=vc, score=score, kv=kv, nb=nb, kv_out=torch.zeros_like(kv),
              idx=torch.empty((layers, nb, Hkv, budget), dtype=torch.int32, device=DEV))
    if case["inplace"]:  # scores go to a second buffer that the next turn reads, caches stay where they are
        st.update(ko=kc, vo=vc, so=torch.zeros_like(score))
    else:
        shape = (layers, nb, Hkv, budget + 64)
        st.update(ko=torch.zeros(shape + (D,), dtype=torch.bfloat16, device=DEV),
                  vo=torch.zeros(shape + (D,), dtype=torch.bfloat16, device=DEV), so=torch.zeros(shape, device=DEV))
    return st


def prepare(case, seed):
    make = {"rope": _rope_state, "score": _score_state, "evict": _evict_state}[case["kind"]]
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


def _rope_plain(st):
    case = st["case"]
    N, D = case["N"], case["D"]
    angle = st["pos"].double()[:, None] * st["inv"]
    c, s = (torch.cos(angle) * st["magnitude"]).float()[:, None], (torch.sin(angle) * st["magnitude"]).float()[:, None]
    q, k = (_turn(st[x].float().view(N, -1, D), c, s, case["rot"], case["layout"]).to(torch.bfloat16) for x in ("q", "k"))
    return [q, k, st["v"].to(torch.bfloat16).view(N, -1, D)]


def _score_plain(st):
    case = st["case"]
    layers, H, Hkv, D, lmax = (case[k] for k in ("layers", "H", "Hkv", "D", "lmax"))
    nb, R, G = st["nb"], st["R"], H // Hkv
    at = (st["offs"][:-1, None] + st["paths"].clamp_min(0)).long()
    q = st["q"][:, at].float().view(layers, nb, R, Hkv, G, D).transpose(2, 3).reshape(layers, nb, Hkv, R * G, D)
    lse = st["lse"][:, at].view(layers, nb, R, Hkv, G).transpose(2, 3).reshape(layers, nb, Hkv, R * G, 1)
    w = torch.exp(q @ st["kc"].float().transpose(3, 4) * D ** -0.5 - lse)
    see = _chain_mask(st["kv"], st["alen"] + 1, R, lmax)[:, None, :, None, :].expand(nb, 1, R, G, lmax).reshape(nb, 1, R * G, lmax)
    new = torch.where(see, w, 0.0).sum(3)
    j = torch.arange(lmax, device=DEV)[None, None, :]
    L = st["kv"][:, None, None]
    old = torch.where(j < L, st["score"] * case["decay"], 0.0)
    st["out"].copy_(torch.where(j <= L + st["alen"][:, None, None], old + new, st["out"]))
    return st["out"]


def _evict_plain(st):
    case = st["case"]
    budget, D, lmax = case["budget"], case["D"], case["lmax"]
    j = torch.arange(lmax, device=DEV)[None, None, None, :]
    L = st["kv"][None, :, None, None]
    n = L.clamp(max=budget)
    # rank: what has to stay first, then by score; a stable sort breaks ties by index
    key = torch.where((j < case["sink"]) | (j >= L - case["recent"]), math.inf, st["score"])
    key = torch.where(j < L, key, -math.inf)
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices
    kept = torch.where(torch.arange(lmax, device=DEV) < n, best, lmax).sort(-1).values[..., :budget]
    there = kept < lmax
    kept = kept.clamp(max=lmax - 1)
    rows = min(budget, lmax)
    for src, dst in ((st["kc"], st["ko"]), (st["vc"], st["vo"])):
        moved = torch.gather(src, 3, kept[..., None].expand(*kept.shape, D))
        dst[:, :, :, :rows] = torch.where(there[..., None], moved, dst[:, :, :, :rows])
    st["so"][..., :rows] = torch.where(there, torch.gather(st["score"], 3, kept), st["so"][..., :rows])
    st["kv_out"].copy_(st["kv"].clamp(max=budget))
    st["idx"].fill_(-1)
    st["idx"][..., :rows] = torch.where(there, kept, -1).to(torch.int32)
    return st["ko"], st["vo"], st["so"], st["kv_out"], st["idx"]


def run(st):
    case = st["case"]
    if not own:
        return {"rope": _rope_plain, "score": _score_plain, "evict": _evict_plain}[case["kind"]](st)
    from paper_2512_21857_gb300 import binding as B
    if case["kind"] == "rope":
        q, k, v = st["out"]
        B.adt_rope_qkv(st["q"], st["k"], st["v"], st["pos"], st["inv"], H=case["H"], Hkv=case["Hkv"], D=case["D"],
                       layout=B.ROPE_HALF if case["layout"] == "half" else B.ROPE_INTERLEAVED, magnitude=st["magnitude"],
                       q_out=q, k_out=k, v_out=v)
        return [q, k, v]
    if case["kind"] == "score":
        B.adt_kv_score(st["q"], st["lse"], st["kc"], st["kv"], st["offs"], st["paths"], st["R"], st["alen"], st["score"],
                       score_out=st["out"], B=st["nb"], H=case["H"], Hkv=case["Hkv"], D=case["D"], num_layers=case["layers"],
                       max_kv=case["lmax"], softmax_scale=case["D"] ** -0.5, decay=case["decay"])
        return st["out"]
    B.adt_kv_evict(st["kc"], st["vc"], st["score"], st["kv"], st["kv_out"], k_out=st["ko"], v_out=st["vo"], score_out=st["so"],
                   keep_idx=st["idx"], B=st["nb"], Hkv=case["Hkv"], D=case["D"], num_layers=case["layers"],
                   max_kv=case["lmax"], budget=case["budget"], n_sink=case["sink"], n_recent=case["recent"])
    return st["ko"], st["vo"], st["so"], st["kv_out"], st["idx"]


# ------------------------------------------------------------------ exact values

def _rope_exact(case, st):
    N, H, Hkv, D, R = (case[k] for k in ("N", "H", "Hkv", "D", "rot"))
    unit = torch.polar(torch.full((N, R // 2), st["magnitude"], dtype=torch.float64, device=DEV), torch.outer(st["pos"].double(), st["inv"]))
    out = []
    for x, h in ((st["q"], H), (st["k"], Hkv)):
        y = x.double().reshape(N, h, D)
        i = torch.arange(R // 2, device=DEV)
        re, im = (i, i + R // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(y[:, :, re], y[:, :, im]) * unit[:, None, :]
        y[:, :, re], y[:, :, im] = z.real, z.imag
        out.append(y)
    return out + [st["v"].double().reshape(N, Hkv, D)]


def _score_exact(case, st):
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    kv, path, out = _ints(case["kv"]), _ints(case["path"]), st["out"].double()
    for b, (L, n) in enumerate(zip(kv, path)):
        keys = st["kc"][:, b, :, :L + n].double()
        total = torch.zeros(keys.shape[:3], dtype=torch.float64, device=DEV)
        total[..., :L] = st["score"][:, b, :, :L].double() * case["decay"]
        for i in range(n):
            node = b * case["nodes"] + int(st["paths"][b, i])
            q = st["q"][:, node].double().view(case["layers"], Hkv, H // Hkv, D)
            lse = st["lse"][:, node].double().view(case["layers"], Hkv, H // Hkv, 1)
            w = torch.exp(torch.matmul(q, keys[:, :, :L + i + 1].transpose(2, 3)) / math.sqrt(D) - lse)
            total[..., :L + i + 1] += w.sum(2)
        out[:, b, :, :L + n] = total
    return out


def _evict_exact(case, st):
    out = [st[x].double().clone() for x in ("ko", "vo", "so")] + [torch.zeros_like(st["kv"]), torch.full_like(st["idx"], -1)]
    for b, L in enumerate(_ints(case["kv"])):
        n, lo, hi = min(L, case["budget"]), min(L, case["sink"]), max(0, L - case["recent"])
        out[3][b] = n
        stay = torch.zeros(st["score"].shape[0], st["score"].shape[2], L, dtype=torch.bool, device=DEV)
        stay[..., :lo], stay[..., hi:] = True, True
        if L == n:
            stay[:] = True
        else:
            mid = st["score"][:, b, :, lo:hi].double()
            want = n - int(stay[0, 0].sum())
            # the want-th largest, all above it, and the first of those equal to it
            cut = mid.topk(want, dim=-1).values[..., -1:] if want else torch.full_like(mid[..., :1], math.inf)
            above, equal = mid > cut, mid == cut
            stay[..., lo:hi] = above | (equal & (equal.cumsum(-1) <= want - above.sum(-1, keepdim=True)))
        rows = stay.nonzero()[:, 2].view(*stay.shape[:2], n)
        for x, dst in (("kc", out[0]), ("vc", out[1])):
            dst[:, b, :, :n] = torch.take_along_dim(st[x][:, b], rows[..., None], 2).double()
        out[2][:, b, :, :n] = torch.take_along_dim(st["score"][:, b], rows, 2).double()
        out[4][:, b, :, :n] = rows.to(torch.int32)
    return tuple(out)


def exact(case, seed):
    return {"rope": _rope_exact, "score": _score_exact, "evict": _evict_exact}[case["kind"]](case, prepare(case, seed))
