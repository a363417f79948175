"""fp64 definitions of the calls on packed sequences and on a paged key-value cache (test infrastructure only).

Plain numpy over the tensors' exact values; nothing here is shared with the CUDA path. Attention functions return, beside the
outputs, what a test needs to bound a kernel's error: sum_j p_ij |v_j| and sum_d |q_id k_jd| * scale.
"""
from __future__ import annotations

import math
from typing import Optional

import numpy as np


def attend(q, k, v, seen, scale: Optional[float] = None):
    """One head. q [n, d], k, v [m, d], seen [n, m] bool. Returns (o, lse, absolute, weights, spread): a row that sees nothing
    has o = 0, lse = -inf; what is not seen does not count, whatever it holds. absolute = sum_j p |v|; weights = p;
    spread [n] = the largest sum_d |q k| * scale of the row."""
    scale = 1.0 / math.sqrt(q.shape[1]) if scale is None else scale
    n, d = q.shape
    o, absolute = np.zeros((n, d)), np.zeros((n, d))
    lse, weights, spread = np.full(n, -np.inf), np.zeros(seen.shape), np.zeros(n)
    for i in range(n):
        at = np.nonzero(seen[i])[0]
        if len(at) == 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            x = (k[at] @ q[i]) * scale
            top = x.max()
            p = np.exp(x - top)
            total = p.sum()
            lse[i] = top + np.log(total)
            p = p / total
            weights[i, at] = p
            o[i] = p @ v[at]
            absolute[i] = p @ np.abs(v[at])
            spread[i] = (np.abs(k[at]) @ np.abs(q[i])).max() * scale
    return o, lse, absolute, weights, spread


def attn_packed(q, k, v, cu_q, cu_k, causal: bool, scale: Optional[float] = None):
    """q [total_q, heads_q, d], k, v [total_k, heads_kv, d]. Returns o, lse [heads_q, total_q], absolute, spread [heads_q,
    total_q]; rows behind the last sequence are NaN."""
    heads_q, group = q.shape[1], q.shape[1] // k.shape[1]
    o, absolute = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, spread = np.full((heads_q, q.shape[0]), np.nan), np.full((heads_q, q.shape[0]), np.nan)
    for b in range(len(cu_q) - 1):
        rows, keys = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        seen = np.ones((n, m), bool)
        if causal:
            seen = np.arange(m)[None, :] <= np.arange(n)[:, None] + m - n
        for h in range(heads_q):
            o[rows, h], lse[h, rows], absolute[rows, h], _, spread[h, rows] = attend(
                q[rows, h], k[keys, h // group], v[keys, h // group], seen, scale)
    return o, lse, absolute, spread


def positions(table_row, length, page_size, num_pages):
    """(position, page, place) of the cached positions whose page exists."""
    out = []
    for j in range(min(max(length, 0), len(table_row) * page_size)):
        page = int(table_row[j // page_size])
        if 0 <= page < num_pages:
            out.append((j, page, j % page_size))
    return out


def attn_paged(q, k, v, table, lens, mass_in=None, scale: Optional[float] = None):
    """q [batch, heads_q, d], k, v [pages, page_size, heads_kv, d]. Returns o, lse [batch, heads_q], absolute, spread [batch,
    heads_q], mass [batch, heads_kv, max_pages * page_size] (NaN behind a sequence's length)."""
    batch, heads_q, _ = q.shape
    num_pages, page_size, heads_kv, _ = k.shape
    group = heads_q // heads_kv
    room = table.shape[1] * page_size
    o, absolute, lse, spread = np.zeros(q.shape), np.zeros(q.shape), np.full((batch, heads_q), -np.inf), np.zeros((batch, heads_q))
    mass = np.full((batch, heads_kv, room), np.nan)
    for b in range(batch):
        at = positions(table[b], int(lens[b]), page_size, num_pages)
        j, page, place = (np.array([x[i] for x in at], dtype=np.int64) for i in range(3))
        length = min(max(int(lens[b]), 0), room)
        mass[b, :, :length] = 0.0 if mass_in is None else mass_in[b, :, :length]
        for h in range(heads_q):
            g = h // group
            o[b, h], lse[b, h], absolute[b, h], w, spread[b, h] = (
                x[0] for x in attend(q[b, h][None], k[page, place, g], v[page, place, g], np.ones((1, len(j)), bool), scale))
            mass[b, g, j] += w
    return o, lse, absolute, spread, mass


def kept_positions(mass_row, length, keep, recent):
    """Ascending positions that stay: all if they fit, else the `recent` last ones and those of the others with the largest
    mass (ties to the lower position, NaN lowest)."""
    if length <= keep:
        return list(range(length))
    order = sorted(range(length - recent), key=lambda j: (math.inf if math.isnan(mass_row[j]) else -float(mass_row[j]), j))
    finite_last = [j for j in order if not math.isnan(mass_row[j])] + [j for j in order if math.isnan(mass_row[j])]
    return sorted(finite_last[:keep - recent]) + list(range(length - recent, length))
