"""CPU oracle of rotary positions and of the paged latent cache (numpy, float64), from the definitions in
include/bdrotary.h, without the library's code: angles in exact rational arithmetic, pairs one by one as complex numbers,
the softmax in 64 bits.
"""

from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

from .cache_oracle import visible

# pi to 60 digits: positions up to 2^31 times frequencies of 53 bits leave 30 digits behind the point
PI = Fraction(3141592653589793238462643383279502884197169399375105820974945, 10 ** 60)


def angles(positions, frequencies) -> np.ndarray:
    """position * frequency modulo 2 pi, [positions, frequencies]: reduced exactly, then rounded to float64."""
    turns = [Fraction(float(f)) / (2 * PI) for f in frequencies]
    at = {int(p): [float(int(p) * t % 1) * 2 * math.pi for t in turns] for p in np.unique(positions)}
    return np.array([at[int(p)] for p in positions]).reshape(len(positions), len(turns))


def rotate(x, positions, frequencies, scale=1.0, interleaved=False, inverse=False) -> np.ndarray:
    """x float64 [tokens, heads, dim]; the first 2 len(frequencies) elements of each head turned."""
    x = np.array(x, dtype=np.float64)
    n = 2 * len(frequencies)
    by = scale * np.exp((-1j if inverse else 1j) * angles(positions, frequencies))
    first, second = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    with np.errstate(invalid="ignore"):
        a, b = x[..., first].copy(), x[..., second].copy()
        c, s = by.real[:, None], by.imag[:, None]
        x[..., first], x[..., second] = a * c - b * s, a * s + b * c
    return x


def latent_write(latent, rope, slots, held_latent, held_rope):
    """Rows of latents and (turned) key parts into [pages, page, dim] arrays; returns both afterwards."""
    out_l, out_r = np.array(held_latent), np.array(held_rope)
    page = out_l.shape[1]
    for i, slot in enumerate(slots):
        if 0 <= slot < out_l.shape[0] * page:
            fine = np.isfinite(latent[i]).all()
            out_l[slot // page, slot % page] = latent[i] if fine else 0.0
            out_r[slot // page, slot % page] = rope[i] if fine else np.nan
    return out_l, out_r


def latent_attention(q, latent, rope, block_table, kv_lens, query_start, scale, mask_block):
    """q float64 [tokens, heads, latent_dim + rope_dim]; returns (out, lse, spread, work) as cache_oracle.attention does.
    Pages outside the cache are zeros."""
    n_tok, heads, _ = q.shape
    n_pages, page, dim = latent.shape
    out, spread = np.zeros((n_tok, heads, dim)), np.zeros((n_tok, heads, dim))
    lse, work = np.full((n_tok, heads), -np.inf), np.zeros((n_tok, heads))
    none = np.zeros((1, page, dim + rope.shape[2]))
    rows = np.concatenate([np.concatenate([latent, rope], 2), none])
    for s in range(len(kv_lens)):
        n, q0 = max(int(kv_lens[s]), 0), int(query_start[s])
        q_len = int(query_start[s + 1]) - q0
        pages = np.asarray(block_table[s][:-(-n // page)], dtype=np.int64)
        pages = np.where((pages >= 0) & (pages < n_pages), pages, n_pages)
        key = rows[pages].reshape(-1, rows.shape[2])[:n]
        for i in range(q_len):
            see = visible(n, q_len, i, mask_block)
            if see == 0:
                continue
            k, v, qq = key[:see], key[:see, :dim], q[q0 + i]
            with np.errstate(invalid="ignore"):
                x = qq @ k.T * scale
                top = np.where(np.isfinite(x).any(1), np.max(np.where(np.isfinite(x), x, -np.inf), 1), 0.0)[:, None]
                w = np.exp(x - top)
                total = w.sum(1, keepdims=True)
                out[q0 + i] = w @ v / total
                spread[q0 + i] = w @ np.abs(v) / total
            lse[q0 + i] = (top + np.log(total))[:, 0]
            work[q0 + i] = np.max(np.abs(qq) @ np.abs(k).T, 1) * abs(scale)
    return out, lse, spread, work
