"""CPU oracle of the paged K/V cache: appending with rotation, and attention over the pages.  TEST INFRASTRUCTURE ONLY, like
bsfa_oracle; nothing here imports the HIP binding.

Plain loops over batch elements and heads in fp64, on tensors whose values are the 16-bit ones.  Beside its results,
`attend` returns what their error is measured in: `spread`, the attention's mean of |v|, which a rounding of the
probabilities is relative to, and `score`, the largest sum of |q_i k_i| / sqrt(d) of a row, which rounding in a score's sum is.
"""
from __future__ import annotations

import math

import torch


def places(table_row, n, page, n_pages):
    """Page and place of tokens 0 .. n - 1, and which of them lie in a page of the cache."""
    t = torch.arange(n)
    ids = table_row.long()[t // page]
    return ids, t % page, (ids >= 0) & (ids < n_pages)


def append(k, v, k_cache, v_cache, table, start, cos_sin=None, q=None, seqlens=None, interleaved=False):
    """The caches after the call, and q and k rotated (rows that are left alone: NaN), all fp64."""
    B, N = k.shape[:2]
    page, n_pages = k_cache.shape[1], k_cache.shape[0]
    kc, vc = k_cache.double().clone(), v_cache.double().clone()
    ko = torch.full(k.shape, math.nan, dtype=torch.float64)
    qo = None if q is None else torch.full(q.shape, math.nan, dtype=torch.float64)
    for b in range(B):
        for i in range(N if seqlens is None else min(N, max(0, int(seqlens[b])))):
            pos = int(start[b]) + i
            if not 0 <= pos < table.shape[1] * page:
                continue
            ko[b, i] = _turn(k[b, i].double(), cos_sin, pos, interleaved)
            if q is not None:
                qo[b, i] = _turn(q[b, i].double(), cos_sin, pos, interleaved)
            at = int(table[b, pos // page])
            if 0 <= at < n_pages:
                kc[at, pos % page] = ko[b, i]
                vc[at, pos % page] = v[b, i].double()
    return kc, vc, qo, ko


def _turn(x, cos_sin, pos, interleaved):
    if cos_sin is None:
        return x
    rot = cos_sin.shape[1]
    y = x.clone()
    for e in range(rot // 2):
        a, b = (2 * e, 2 * e + 1) if interleaved else (e, e + rot // 2)
        c, s = float(cos_sin[pos, e]), float(cos_sin[pos, rot // 2 + e])
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def attend(q, k_cache, v_cache, table, lens, q_lens=None, causal=True, prefix_table=None, prefix_len=0):
    """out, lse, spread, score (rows that are left alone: NaN), fp64."""
    B, N, hq, d = q.shape
    n_pages, page, hkv, _ = k_cache.shape
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    spread = out.clone()
    lse = torch.full(q.shape[:3], math.nan, dtype=torch.float64)
    score = lse.clone()
    flat = [x.reshape(n_pages * page, hkv, d) for x in (k_cache, v_cache)]
    for b in range(B):
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        m = N if q_lens is None else min(max(int(q_lens[b]), 0), N)
        ids, at, there = places(table[b], n, page, n_pages)
        place = torch.arange(n)
        if prefix_table is not None:
            pids, pat, pthere = places(prefix_table, prefix_len, page, n_pages)
            ids, at, there = torch.cat([pids, ids]), torch.cat([pat, at]), torch.cat([pthere, there])
            place = torch.cat([torch.full((prefix_len,), -(1 << 40)), place])           # before everything
        where = (ids * page + at)[there]
        place = place[there]
        for h in range(hq):
            k, v = (x[where, h // (hq // hkv)].double() for x in flat)
            rows = q[b, :m, h].double()
            s = rows @ k.t() / math.sqrt(d)
            hidden = place[None, :] > (n - m + torch.arange(m))[:, None] if causal else torch.zeros(m, len(where), dtype=torch.bool)
            s = s.masked_fill(hidden, -math.inf)
            z = torch.logsumexp(s, dim=1) if len(where) else torch.full((m,), -math.inf, dtype=torch.float64)
            p = torch.where(hidden, 0.0, (s - torch.where(z == -math.inf, 0.0, z)[:, None]).exp())
            out[b, :m, h], lse[b, :m, h] = p @ v, z
            spread[b, :m, h] = p @ v.abs()
            size = (rows.abs() @ k.abs().t() / math.sqrt(d)).masked_fill(hidden, 0.0)
            score[b, :m, h] = size.amax(dim=1) if len(where) else 0.0
    return out, lse, spread, score
