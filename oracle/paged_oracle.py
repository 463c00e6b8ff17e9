"""Double-precision definitions of the rotary and paged-cache operators (numpy, host): rotation of pairs, rows of a
paged cache, attention of one token over them with the per-row weights, and the rows that eviction keeps."""
from __future__ import annotations

import math

import numpy as np


def rope_table(rot_dim, base, scaling="plain", factor=1.0, original_len=0.0, low_freq=1.0, high_freq=4.0, beta_fast=32.0,
               beta_slow=1.0):
    """Radians per position of each pair, one pair at a time."""
    out = []
    for i in range(rot_dim // 2):
        f = 1.0 / base ** (2.0 * i / rot_dim)
        if scaling == "linear":
            f = f / factor
        elif scaling == "llama3":
            wavelength = 2.0 * math.pi / f
            if wavelength > original_len / low_freq:
                f = f / factor
            elif wavelength >= original_len / high_freq:
                s = (original_len / wavelength - low_freq) / (high_freq - low_freq)
                f = (1.0 - s) * f / factor + s * f
        elif scaling == "yarn":
            def pair_of(turns):
                return rot_dim * math.log(original_len / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))
            lo, hi = max(math.floor(pair_of(beta_fast)), 0), min(math.ceil(pair_of(beta_slow)), rot_dim - 1)
            r = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = (1.0 - r) * f + r * f / factor
        out.append(f)
    return np.array(out)


def rotate(x, positions, freqs, rot_dim, rot_offset=0, interleaved=False, magnitude=1.0, inverse=False):
    """x [T, H, d]; the dims [rot_offset, rot_offset + rot_dim) of every head turned by positions x freqs."""
    y = np.array(x, dtype=np.float64)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(freqs, dtype=np.float64)
    c, s = np.cos(angle)[:, None], (-1.0 if inverse else 1.0) * np.sin(angle)[:, None]
    i = np.arange(rot_dim // 2)
    a, b = (rot_offset + 2 * i, rot_offset + 2 * i + 1) if interleaved else (rot_offset + i, rot_offset + rot_dim // 2 + i)
    xa, xb = y[..., a].copy(), y[..., b].copy()
    y[..., a] = magnitude * (xa * c - xb * s)
    y[..., b] = magnitude * (xb * c + xa * s)
    return y


def cache_rows(pages, table_row, length):
    """pages [n_pages, Hkv, page, d] -> [length, Hkv, d]: the first rows of one sequence; rows on a page number out of range
    are left out.  Also returns which rows those are."""
    page, rows, there = pages.shape[2], [], []
    for r in range(length):
        p = int(table_row[r // page])
        if 0 <= p < pages.shape[0]:
            rows.append(pages[p, :, r % page])
            there.append(r)
    return np.stack(rows) if rows else np.zeros((0,) + (pages.shape[1], pages.shape[3])), np.array(there, dtype=np.int64)


def decode(q, k, v, scale):
    """q [Hq, d], k [n, Hkv, d], v [n, Hkv, dv] -> (out [Hq, dv], weights [Hkv, n] summed over a KV head's query heads,
    and per head the sums sum_r p_r |v_r| and max_r sum_c |q_c k_rc| that error bounds are made of)."""
    hq, hkv, n = q.shape[0], k.shape[1], k.shape[0]
    g = hq // hkv
    out, w = np.zeros((hq, v.shape[2])), np.zeros((hkv, n))
    mass, reach = np.zeros((hq, v.shape[2])), np.zeros(hq)
    if n == 0:
        return out, w, mass, reach
    for h in range(hq):
        x = (k[:, h // g] @ q[h]) * scale
        p = np.exp(x - x.max())
        p /= p.sum()
        out[h] = p @ v[:, h // g]
        mass[h] = p @ np.abs(v[:, h // g])
        reach[h] = (np.abs(k[:, h // g]) @ np.abs(q[h])).max() * scale
        w[h // g] += p
    return out, w, mass, reach


def kept_rows(weights, length, sink, recent, topk):
    """Rows of one (sequence, KV head) that eviction keeps, ascending; weights [>= length]."""
    if length <= sink + recent + topk:
        return np.arange(length)
    middle = np.arange(sink, length - recent)
    w = np.asarray(weights, dtype=np.float64)[middle]
    w = np.where(np.isnan(w), -np.inf, w)
    nan = np.isnan(np.asarray(weights, dtype=np.float64)[middle])
    best = sorted(range(len(middle)), key=lambda j: (nan[j], -w[j], j))[:topk]
    return np.concatenate([np.arange(sink), np.sort(middle[best]) if topk else middle[:0], np.arange(length - recent, length)])
