"""Plain 64-bit implementations of the cache operators (attention weight of
cached keys, eviction, decoding behind a shared prefix), for their tests.
They share nothing with the HIP path; bf16 inputs are raw bits (uint16)."""
from __future__ import annotations

import math

import numpy as np

import oracle
import synth


def f64(bits):
    return synth.f32_from_bf16_bits(np.asarray(bits).reshape(-1)).reshape(
        np.shape(bits)).astype(np.float64)


def scores_of(q, k, rows, cu, n_rows_of, *, scale=0.0, lse=None):
    """sum of the softmax weights that rows ``rows`` (packed tokens, sequence
    by sequence) give their sequence's keys up to themselves: [Hkv, N], and the
    largest sum_c |q_c k_c| of a score in the exp2 domain (the size that its
    rounding errors go by).  lse: base-2 log-sum-exps [Hq, len(rows)] in place
    of the exact ones."""
    q, k = f64(q), f64(k)
    N, hkv, d = k.shape
    hq = q.shape[1]
    G = hq // hkv
    c = (scale if scale > 0 else 1.0 / math.sqrt(d)) * math.log2(math.e)
    out = np.zeros((hkv, N))
    size = 0.0
    r = 0
    for b in range(len(cu) - 1):
        for _ in range(n_rows_of[b]):
            i = int(rows[r])
            keys = slice(int(cu[b]), i + 1)
            for h in range(hq):
                x = c * (k[keys, h // G] @ q[i, h])
                size = max(size, float((c * (np.abs(k[keys, h // G]) @ np.abs(q[i, h]))).max()))
                z = lse[h, r] if lse is not None else x.max() + np.log2(np.exp2(x - x.max()).sum())
                out[h // G, keys] += np.exp2(x - z)
            r += 1
    return out, size


def score_tolerance(total, rows, d, size):
    """Bound on the fp32 result's error: every term is 2^x with x a sum of d
    products, scaled, less a log-sum-exp of the same size (each operation off
    by 2^-24 of sum |q k|, the exponential and the logarithm by 2^-22), and
    the terms are added to each other one after the other."""
    rel = math.log(2.0) * (2 * d + 8) * size * 2.0 ** -24 + (rows + 16) * 2.0 ** -24
    return rel * np.abs(total) + 1e-30


def step_scores(q, k, cu, z, *, scale=0.0):
    """One decoding step: sequence b's token gives its weights to all its keys
    where z[b]; as ``scores_of``."""
    q, k = f64(q), f64(k)
    N, hkv, d = k.shape
    hq = q.shape[1]
    G = hq // hkv
    c = (scale if scale > 0 else 1.0 / math.sqrt(d)) * math.log2(math.e)
    out = np.zeros((hkv, N))
    size = 0.0
    for b in range(len(cu) - 1):
        if not z[b]:
            continue
        keys = slice(int(cu[b]), int(cu[b + 1]))
        for h in range(hq):
            x = c * (k[keys, h // G] @ q[b, h])
            size = max(size, float((c * (np.abs(k[keys, h // G]) @ np.abs(q[b, h]))).max()))
            w = np.exp2(x - x.max())
            out[h // G, keys] += w / w.sum()
    return out, size


def evict(score, cu, budget, recent):
    """(kept packed rows [Hkv, kept], cu_keep): the last min(recent, n) rows
    and the n - recent others of the largest scores, ascending."""
    hkv = score.shape[0]
    kept = [[] for _ in range(hkv)]
    cu_keep = [0]
    for b in range(len(cu) - 1):
        L = int(cu[b + 1] - cu[b])
        n = min(L, budget)
        rec = min(recent, n)
        cu_keep.append(cu_keep[-1] + n)
        for h in range(hkv):
            x = score[h, cu[b]:cu[b] + L - rec].astype(np.float64) + 0.0
            x = np.where(np.isnan(x), -np.inf, x), ~np.isnan(x)
            # largest first, numbers before NaN, lowest index first
            order = sorted(range(L - rec), key=lambda i: (not x[1][i], -x[0][i], i))
            rows = sorted(order[:n - rec]) + list(range(L - rec, L))
            kept[h] += [int(cu[b]) + i for i in rows]
    return np.array(kept, np.int64).reshape(hkv, -1), np.array(cu_keep, np.int32)


def whole_caches(pre, own, cu_pre, cu_grp, cu):
    """[prefix ; own rows] of every sequence, packed, and its cu_seqlens."""
    parts, lens = [], []
    for r in range(len(cu_pre) - 1):
        for b in range(int(cu_grp[r]), int(cu_grp[r + 1])):
            parts += [pre[cu_pre[r]:cu_pre[r + 1]], own[cu[b]:cu[b + 1]]]
            lens.append(int(cu_pre[r + 1] - cu_pre[r] + cu[b + 1] - cu[b]))
    return np.concatenate(parts), np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def decode_prefix(x, cu_pre, cu_grp, cu, window, threshold, *, gain_local=None, gain_global=None):
    """The decoding oracle on every sequence's whole cache.  x: q, k, v, k_pre,
    v_pre, gate and any of their _g forms."""
    k, whole = whole_caches(x["k_pre"], x["k"], cu_pre, cu_grp, cu)
    v, _ = whole_caches(x["v_pre"], x["v"], cu_pre, cu_grp, cu)
    kg = vg = None
    if "k_g" in x:
        kg, _ = whole_caches(x["k_pre_g"], x["k_g"], cu_pre, cu_grp, cu)
        vg, _ = whole_caches(x["v_pre_g"], x["v_g"], cu_pre, cu_grp, cu)
    return oracle.decode(x["q"], k, v, x["gate"], whole, window, threshold,
                         q_g_new=x.get("q_g"), k_g=kg, v_g=vg, gain_local=gain_local,
                         gain_global=gain_global)
