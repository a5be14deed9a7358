"""64-bit statements of the cache operators for the tests: attention weights per position, the kept set of an
eviction, and paged problems whose requests share prefixes.  Plain numpy over the host arrays of
tests.helpers.make_problem; no code of the library."""
from __future__ import annotations

import numpy as np

from paper_2609_20734_b200 import synth
from tests.helpers import dense_kv


def dense_unit(prob, cache, kv_layer, b, g):
    """[t, D] fp64 rows of one (cache slice, request, kv head), gathered at once."""
    lay, P, D, t = prob["layout"], prob["P"], prob["D"], int(prob["seq_lens"][b])
    j = np.arange(t)
    base = (kv_layer * lay.layer_stride + prob["table"][b, j // P].astype(np.int64) * lay.block_stride
            + (j % P) * lay.token_stride + g * lay.head_stride)
    return synth.bf16_bits_to_f32(cache[base[:, None] + np.arange(D)]).astype(np.float64)


def softmax_rows(prob, l, b, h, kv_layer=None, sm_scale=None):
    """(weights [t], out [D], lse) of one query head over its whole history."""
    g = h // (prob["Hq"] // prob["Hkv"])
    kvl = l if kv_layer is None else kv_layer
    K, V = dense_unit(prob, prob["k"], kvl, b, g), dense_unit(prob, prob["v"], kvl, b, g)
    q = synth.bf16_bits_to_f32(prob["q"][l, b, h]).astype(np.float64)
    z = (K @ q) * (1.0 / np.sqrt(prob["D"]) if sm_scale is None else sm_scale)
    m = z.max()
    e = np.exp(z - m)
    return e / e.sum(), (e @ V) / e.sum(), m + np.log(e.sum())


def full_reference(prob, kv_index=None, sm_scale=None):
    """out [L,B,Hq,D], lse [L,B,Hq] and per (layer, request, kv head) the summed weights of the Full pass."""
    L, B, Hq, Hkv, D = (prob[x] for x in ("L", "B", "Hq", "Hkv", "D"))
    out, lse, wts = np.full((L, B, Hq, D), np.nan), np.full((L, B, Hq), np.nan), {}
    for l in range(L):
        for b in range(B):
            if prob["seq_lens"][b] < 1:
                continue
            for h in range(Hq):
                w, o, e = softmax_rows(prob, l, b, h, None if kv_index is None else kv_index[l], sm_scale)
                out[l, b, h], lse[l, b, h] = o, e
                key = (l, b, h // (Hq // Hkv))
                wts[key] = wts.get(key, 0) + w
    return out, lse, wts


def kept_positions(weights, t, budget, sinks, recent):
    """The kept set of one (slice, request, kv head), in order of position (weights: fp32 array)."""
    if t <= budget:
        return np.arange(t)
    w = np.asarray(weights[:t], dtype=np.float64) + 0.0
    key = np.where(np.isnan(w), np.inf, w)
    nan = np.isnan(w)
    mid = np.arange(sinks, t - recent)
    order = sorted(mid.tolist(), key=lambda i: (not nan[i], -key[i], i))[: budget - sinks - recent]
    return np.array(sorted(list(range(sinks)) + order + list(range(t - recent, t))), dtype=np.int64)


def evict_reference(prob, weights, budget, sinks, recent, mask=None):
    """(k, v, weights, seq_lens, kept) after the eviction; inputs are not changed."""
    lay, P, D, B, Hkv = prob["layout"], prob["P"], prob["D"], prob["B"], prob["Hkv"]
    S = weights.shape[0]
    k, v, w, lens = prob["k"].copy(), prob["v"].copy(), weights.copy(), prob["seq_lens"].copy()
    kept = np.full((S, B, Hkv, budget), -7, np.int32)
    for b in range(B):
        t = int(prob["seq_lens"][b])
        if t < 1 or (mask is not None and not mask[b]):
            continue
        lens[b] = min(t, budget)

        def rows(s, g, pos):
            return (s * lay.layer_stride + prob["table"][b, pos // P].astype(np.int64) * lay.block_stride
                    + (pos % P) * lay.token_stride + g * lay.head_stride)[:, None] + np.arange(D)

        for s in range(S):
            for g in range(Hkv):
                keep = kept_positions(weights[s, b, g], t, budget, sinks, recent)
                kept[s, b, g, :len(keep)], kept[s, b, g, len(keep):] = keep, -1
                if t <= budget:
                    continue
                dst = rows(s, g, np.arange(budget))
                k[dst], v[dst] = prob["k"][rows(s, g, keep)], prob["v"][rows(s, g, keep)]
                w[s, b, g, :budget], w[s, b, g, budget:t] = weights[s, b, g, keep], 0
    return k, v, w, lens, kept


def share_prefixes(prob, groups, prefix, copy_pages=()):
    """Makes requests groups[i] .. groups[i+1]-1 of a problem share their first prefix[i] positions: whole pages
    through the table (or, for requests in copy_pages, as copies in their own pages), the rest as copies."""
    lay, P, D = prob["layout"], prob["P"], prob["D"]
    for i, n in enumerate(prefix):
        lead = groups[i]
        for b in range(groups[i] + 1, groups[i + 1]):
            m = min(n, int(prob["seq_lens"][b]), int(prob["seq_lens"][lead]))
            whole = m // P if b not in copy_pages else 0
            for s in range(prob["kv_layers"]):
                for g in range(prob["Hkv"]):
                    pos = np.arange(whole * P, m)
                    for c in ("k", "v"):
                        at = [(s * lay.layer_stride + prob["table"][r, pos // P].astype(np.int64) * lay.block_stride
                               + (pos % P) * lay.token_stride + g * lay.head_stride)[:, None] + np.arange(D) for r in (lead, b)]
                        prob[c][at[1]] = prob[c][at[0]]
            prob["table"][b, :whole] = prob["table"][lead, :whole]
    return prob
