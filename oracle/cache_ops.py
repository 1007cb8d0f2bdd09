"""Plain CPU oracle of the cache operators: rotary positions (with head norms
before them), the attention weight added up per cached row, the eviction that
goes by it, and the 8-bit cache.

TEST INFRASTRUCTURE, like the rest of ``oracle/``: fp64 throughout, one row at
a time, no code shared with the library.
"""
from __future__ import annotations

import math

import numpy as np


def rope_freqs(rotary_dim, theta=10000.0, scaling="none", factor=1.0, orig_len=0.0, turns_lo=1.0, turns_hi=32.0):
    """(radians a position for each pair, magnitude of cosine and sine)."""
    inv = []
    for p in range(rotary_dim // 2):
        base = theta * factor ** (rotary_dim / (rotary_dim - 2)) if scaling == "ntk" else theta
        f = math.exp(-2.0 * p / rotary_dim * math.log(base))
        if scaling == "linear":
            f = f / factor
        elif scaling == "by_parts":
            turns = orig_len * f / (2 * math.pi)
            if turns >= turns_hi:
                pass
            elif turns <= turns_lo:
                f = f / factor
            else:
                keep = (turns - turns_lo) / (turns_hi - turns_lo)
                f = keep * f + (1 - keep) * f / factor
        inv.append(f)
    return np.array(inv), 0.1 * math.log(factor) + 1.0 if scaling == "by_parts" else 1.0


def rope_rows(x, positions, inv_freq, magnitude=1.0, interleaved=False):
    """x [N, heads, D] rotated: pair p of every head times the complex number
    magnitude * e^(i t inv_freq[p]); elements past 2 * len(inv_freq) unchanged."""
    y = np.array(x, dtype=np.float64)
    R = 2 * len(inv_freq)
    for n, t in enumerate(positions):
        for p, f in enumerate(inv_freq):
            ia, ib = (2 * p, 2 * p + 1) if interleaved else (p, p + R // 2)
            z = (y[n, :, ia] + 1j * y[n, :, ib]) * (magnitude * np.exp(1j * np.remainder(float(t) * f, 2 * math.pi)))
            y[n, :, ia], y[n, :, ib] = z.real, z.imag
    return y


def kv_score(q, lse, k_cache, kv_len, node_offsets, paths, score, scale, decay=1.0):
    """q [layers, nodes, H, D]; lse [layers, nodes, H]; k_cache [layers, B, Hkv,
    rows, D]; paths: each tree's accepted nodes (tree-local), the tokens in
    cache rows kv_len[b] + i.  Returns the new scores (rows behind the last
    token as they were) and, for error bounds, per row the sums over queries of
    w, w * sum_d |q_d k_d|, and w * |scale q.k - lse|."""
    q, k = np.asarray(q, np.float64), np.asarray(k_cache, np.float64)
    out = np.array(score, np.float64)
    terms = np.zeros((3,) + out.shape)
    layers, B, Hkv = k.shape[:3]
    group = q.shape[2] // Hkv
    for b in range(B):
        L, path = int(kv_len[b]), list(paths[b])
        out[:, b, :, :L] *= decay
        out[:, b, :, L:L + len(path)] = 0.0
        for i, node in enumerate(path):
            for h in range(group * Hkv):
                keys = k[:, b, h // group, :L + i + 1]
                qq = q[:, int(node_offsets[b]) + node, h]
                z = np.asarray(lse, np.float64)[:, int(node_offsets[b]) + node, h]
                if np.isneginf(z).all():
                    continue
                t = scale * np.einsum("ljd,ld->lj", keys, qq) - z[:, None]
                w = np.exp(t)
                out[:, b, h // group, :L + i + 1] += w
                terms[0, :, b, h // group, :L + i + 1] += w
                terms[1, :, b, h // group, :L + i + 1] += w * np.einsum("ljd,ld->lj", np.abs(keys), np.abs(qq))
                terms[2, :, b, h // group, :L + i + 1] += w * np.abs(t)
    return out, terms


def kept_rows(score, budget, n_sink, n_recent):
    """The rows of one slice that stay, ascending: all within the budget, else
    the first n_sink, the last n_recent and the best between (sorted by score,
    NaN first, then by row)."""
    L = len(score)
    if L <= budget:
        return list(range(L))
    middle = range(n_sink, L - n_recent)
    rank = sorted(middle, key=lambda j: (0 if math.isnan(score[j]) else 1, 0.0 if math.isnan(score[j]) else -score[j], j))
    return sorted(list(range(n_sink)) + rank[:budget - n_sink - n_recent] + list(range(L - n_recent, L)))


def kv_evict(k_cache, v_cache, score, kv_len, budget, n_sink=0, n_recent=0, k_dst=None, v_dst=None, score_dst=None):
    """Returns (k, v, score, kv_len, keep_idx) after the eviction; the
    destinations default to the sources (in place)."""
    src = [np.asarray(x) for x in (k_cache, v_cache, score)]
    dst = [np.array(s if d is None else d) for s, d in zip(src, (k_dst, v_dst, score_dst))]
    layers, B, Hkv = src[0].shape[:3]
    idx = np.full((layers, B, Hkv, budget), -1, np.int32)
    for l in range(layers):
        for b in range(B):
            for g in range(Hkv):
                rows = kept_rows([float(s) for s in src[2][l, b, g, :int(kv_len[b])]], budget, n_sink, n_recent)
                idx[l, b, g, :len(rows)] = rows
                for s, d in zip(src, dst):
                    d[l, b, g, :len(rows)] = s[l, b, g, rows]
    return dst[0], dst[1], dst[2], np.minimum(np.asarray(kv_len), budget), idx


def norm_rows(x, layer, eps, weight=None, bias=None):
    """x [N, heads, D] normed head by head; weight and bias [D] or [heads, D].  Returns the result and, for error
    bounds, the normed rows before weight and bias and each head's mean |x| / sqrt(mean square + eps)."""
    x = np.asarray(x, np.float64)
    y = x - x.mean(-1, keepdims=True) if layer else x
    root = np.sqrt((y * y).mean(-1, keepdims=True) + eps)
    hat = y / root
    out = hat if weight is None else hat * np.asarray(weight, np.float64)
    if bias is not None:
        out = out + np.asarray(bias, np.float64)
    return out, hat, np.abs(x).mean(-1, keepdims=True) / root


def e4m3_values():
    """The value of every e4m3 byte, by its bits (NaN for 0x7f and 0xff)."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = math.nan if b & 127 == 127 else -v if b & 128 else v
    return out


def q8_rows(x):
    """Rows x [..., D] as (e4m3 bytes [..., D], scale bytes [...]): the least power of two 2^(s - 127), s >= 7, with
    max |x| <= 448 times it; elements to the nearest value, halves to the even byte."""
    x = np.asarray(x, np.float64)
    table = e4m3_values()[:127]  # the values that are not negative, ascending
    q, s = np.zeros(x.shape, np.uint8), np.zeros(x.shape[:-1], np.uint8)
    for at in np.ndindex(x.shape[:-1]):
        row = x[at]
        if not np.isfinite(row).all():
            s[at] = 255
            continue
        e = -120
        while np.abs(row).max() > 448 * 2.0 ** e:
            e += 1
        y = np.abs(row) / 2.0 ** e
        hi = np.searchsorted(table, y).clip(1, 126)  # table[hi - 1] <= y <= table[hi]
        up, down = table[hi] - y, y - table[hi - 1]
        pick = np.where(up < down, hi, np.where(up > down, hi - 1, np.where(hi % 2 == 0, hi, hi - 1)))
        q[at] = pick + np.where(np.signbit(row), 128, 0)
        s[at] = e + 127
    return q, s


def q8_values(q, s):
    """What rows of an 8-bit cache stand for."""
    s = np.asarray(s).astype(np.int64)
    scale = np.where(s == 255, math.nan, np.exp2(np.where(s == 255, 0, s) - 127.0))
    return e4m3_values()[np.asarray(q)] * scale[..., None]
