"""Seeded synthetic inputs for the paged 8-bit key/value cache. Holds no step of its operators.

Pages are handed out in random order. Everything that no call may read is set to what would show: codes and scales of
unused pages and of a page's tail are NaN, table entries behind a request's pages are out of range.
"""

from __future__ import annotations

from dataclasses import dataclass

import numpy as np

NAN_CODE, NAN_SCALE, BAD_PAGE = 0x7F, 0xFF, 0x7FFFFFF0


@dataclass
class CacheInputs:
    k: np.ndarray        # uint8 [pages, page, heads, dim]
    v: np.ndarray
    k_scale: np.ndarray  # uint8 [pages, heads]
    v_scale: np.ndarray
    table: np.ndarray    # int32 [n_seq, blocks]
    kv_lens: np.ndarray  # int32 [n_seq]


def random_cache(kv_lens, page: int, n_kv: int, dim: int, *, seed: int = 0, k_exp=(-9, -5), v_exp=(-9, -5),
                 extra_cols: int = 2) -> CacheInputs:
    """Codes of about N(0, 64^2) (every seventh page's last head: subnormal codes) with scale exponents drawn from the
    two ranges: keys and values of order 1 with the default ones."""
    rng = np.random.default_rng(seed)
    lens = np.maximum(np.asarray(kv_lens, dtype=np.int64), 0)
    held = -(-lens // page)
    n_pages = int(held.sum()) + 3
    order = rng.permutation(n_pages)
    table = np.full((len(lens), int(held.max(initial=0)) + extra_cols), BAD_PAGE, dtype=np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += int(h)

    def codes(exp):
        from oracle.cache_oracle import e4m3_encode

        x = np.clip(rng.normal(0, 64, (n_pages, page, n_kv, dim)), -448, 448)
        x[::7, :, -1] *= 2.0 ** -13
        c, e = e4m3_encode(x), (rng.integers(exp[0], exp[1] + 1, (n_pages, n_kv)) + 127).astype(np.uint8)
        used = np.zeros((n_pages, page), dtype=bool)
        for s, n in enumerate(lens):
            for j in range(int(held[s])):
                used[table[s, j], :max(0, min(page, int(n) - j * page))] = True
        c[~used] = NAN_CODE
        e[~used.any(1)] = NAN_SCALE
        return c, e

    k, ks = codes(k_exp)
    v, vs = codes(v_exp)
    return CacheInputs(k, v, ks, vs, table, np.asarray(kv_lens, dtype=np.int32))


def random_tables(n_seq: int, page: int, *, seed: int = 0, max_len: int = 400, max_new: int = 70, spare: int = 5,
                  cols=None, give: float = 0.3) -> dict:
    """Requests with lengths 0..max_len that add or (a share of `give`) give back tokens; `spare` pages more in the pool
    than they need (negative: too few), which wrap around the ring's end."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, max_len + 1, n_seq)
    lens[rng.random(n_seq) < 0.1] = 0
    new = rng.integers(0, max_new + 1, n_seq)
    back = rng.random(n_seq) < give
    new[back] = -rng.integers(0, 2 * max_new + 1, int(back.sum()))
    held, want = -(-lens // page), -(-np.maximum(lens + new, 0) // page)
    cols = int(max(held.max(initial=0), want.max(initial=0))) if cols is None else cols
    free = max(0, int(np.maximum(want - held, 0).sum()) + spare)
    n_pages = int(held.sum()) + free
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((n_seq, max(cols, int(held.max(initial=0)))), BAD_PAGE, dtype=np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += int(h)
    R = max(n_pages, 1)
    ring = np.full(R, -1, dtype=np.int32)
    head = R * 3 + R - free // 2
    ring[(head + np.arange(free)) % R] = order[at:]
    return {"lens": lens.astype(np.int32), "new": new.astype(np.int32), "table": table[:, :max(cols, 0)].copy(),
            "ring": ring, "pool": np.array([head, head + free], np.int64),
            "max_tokens": int(np.maximum(new, 0).sum()) + 3}
