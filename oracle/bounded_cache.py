"""fp64 oracle of the operators for windows, prompts, attention weights and
eviction (test infrastructure only): numpy over the same bit patterns, strides
and block tables as oracle.PagedInputs, written from the formulas and sharing
no code with the CUDA path.

A query at position i of its sequence sees position t when t <= i and
(window == 0 or i - t < window or t < sinks).
"""
from __future__ import annotations

import numpy as np

from . import PagedInputs, decode_bits, default_scale


def seen(i, t, window: int, sinks: int):
    """Broadcast: does the query at position i see position t?"""
    m = t <= i
    if window > 0:
        m = m & ((i - t < window) | (t < sinks))
    return m


def rows_of(inp: PagedInputs, b: int, positions, which: str) -> np.ndarray:
    """K ("k") or V ("v") rows of the logical positions of sequence b, fp64 [n, Hkv, D]."""
    s = inp.shape
    pool = (inp.k if which == "k" else inp.v).ravel()
    sp, st, sh = ((s.k_stride_page, s.k_stride_token, s.k_stride_head) if which == "k"
                  else (s.v_stride_page, s.v_stride_token, s.v_stride_head))
    t = np.asarray(positions, dtype=np.int64)
    page = inp.block_table[b, t // inp.P].astype(np.int64)
    assert (page >= 0).all(), "a visible position has no page"
    at = page * sp + (t % inp.P) * st
    at = at[:, None, None] + np.arange(inp.Hkv)[None, :, None] * sh + np.arange(inp.D)[None, None, :]
    bits = pool[at]
    return decode_bits(bits, bool(s.in_fp16)).reshape(bits.shape)


def attention(inp: PagedInputs, new_lens, window: int = 0, sinks: int = 0, scale=None, run_mask=None, absolute=False):
    """inp.q holds the rows of all sequences' last new_lens[b] positions, one sequence behind the other.
    Returns out [rows, Hq, D], lse [rows, Hq] and, per sequence, the attention weight of every position summed
    over its queries and over the query heads of a KV head: [Hkv, seq_len].  absolute: out from |V| (what relative
    errors of the weights are multiplied with)."""
    G = inp.Hq // inp.Hkv
    scale = default_scale(inp.D) if scale is None else scale
    q = decode_bits(inp.q, bool(inp.shape.in_fp16)).reshape(inp.q.shape)
    out = np.zeros(q.shape)
    lse = np.full(q.shape[:2], -np.inf)
    weights = []
    row = 0
    for b, n_new in enumerate(new_lens):
        L = int(inp.seq_lens[b])
        w = np.zeros((inp.Hkv, L))
        weights.append(w)
        if n_new == 0 or L == 0 or (run_mask is not None and not run_mask[b]):
            row += n_new
            continue
        i = np.arange(L - n_new, L)[:, None]
        t = np.arange(L)
        m = seen(i, t[None, :], window, sinks)
        used = m.any(0)
        t, m = t[used], m[:, used]
        k, v = rows_of(inp, b, t, "k"), rows_of(inp, b, t, "v")
        v = np.abs(v) if absolute else v
        for g in range(inp.Hkv):
            for h in range(g * G, (g + 1) * G):
                with np.errstate(invalid="ignore"):
                    x = (q[row:row + n_new, h] @ k[:, g].T) * scale
                x = np.where(m, x, -np.inf)
                top = x.max(1, keepdims=True)
                e = np.where(m, np.exp(x - top), 0.0)
                total = e.sum(1, keepdims=True)
                p = e / total
                out[row:row + n_new, h] = np.where(used_rows(m), p @ v[:, g], 0.0)
                lse[row:row + n_new, h] = (top + np.log(total))[:, 0]
                w[g, used] += p.sum(0)
        row += n_new
    return out, lse, weights


def used_rows(m):
    return m.any(1)[:, None]


def kept_positions(weights, length: int, budget: int, sinks: int, recent: int) -> np.ndarray:
    """Positions that stay of one (sequence, KV head): all of them up to the budget; else the first `sinks`, the last
    `recent` and the rest of the budget by weight, the lowest position first among equals (NaN counts as -inf)."""
    if length <= budget:
        return np.arange(length)
    w = np.asarray(weights[:length], dtype=np.float64)
    w = np.where(np.isnan(w), -np.inf, w)
    sure = np.zeros(length, dtype=bool)
    sure[:sinks] = True
    sure[length - recent:] = True
    rest = np.flatnonzero(~sure)
    order = sorted(rest.tolist(), key=lambda t: (-w[t], t))
    sure[order[:budget - sinks - recent]] = True
    return np.flatnonzero(sure)
