"""CPU oracle of the paged 8-bit key/value cache (numpy, float64): page tables, quantising writes, attention.

Written from the definitions in include/bdcache.h, without the library's code: integer bookkeeping request by request,
E4M3 by its table of 256 values, the softmax in 64 bits.
"""

from __future__ import annotations

import numpy as np

E_MIN, E_MAX = 27, 247


def e4m3_values() -> np.ndarray:
    """The 256 E4M3 values in float64 (codes 0x7f and 0xff: NaN)."""
    code = np.arange(256)
    exp, man = (code >> 3) & 15, code & 7
    mag = np.where(exp == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (exp.astype(float) - 10))
    mag[(code & 127) == 127] = np.nan
    return np.where(code & 128, -mag, mag)


E4M3 = e4m3_values()


def e4m3_encode(x: np.ndarray) -> np.ndarray:
    """Nearest E4M3 code of float64 values (ties to even, |x| <= 448 expected, saturating); NaN -> 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    mag = np.minimum(np.abs(x), 448.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        exp = np.where(mag > 0, np.floor(np.log2(np.where(mag > 0, mag, 1.0))), -9.0)
    step = 2.0 ** (np.maximum(exp, -6.0) - 3.0)
    q = np.rint(mag / step) * step  # np.rint: ties to even multiples of the step, which are even codes
    q = np.minimum(q, 448.0)
    code = np.searchsorted(E4M3[:127], q).astype(np.uint8)
    code = np.where(np.signbit(x), code | 128, code).astype(np.uint8)
    return np.where(np.isnan(x), np.uint8(0x7F), code)


def scale_byte(amax: np.ndarray) -> np.ndarray:
    """E8M0 byte of the smallest power of two that brings amax to at most 448."""
    m, e = np.frexp(np.asarray(amax, dtype=np.float64))  # m in [0.5, 1), 448 = 0.875 * 2^9
    b = e - 9 + (m > 0.875) + 127
    return np.where(np.asarray(amax) > 0, np.clip(b, E_MIN, E_MAX), E_MIN).astype(np.int64)


def pow2(byte) -> np.ndarray:
    return np.ldexp(1.0, np.asarray(byte, dtype=np.int64) - 127)


def tables(lens, new, block_table, free_pages, pool, page_size: int, max_tokens: int) -> dict:
    table, ring = np.array(block_table), np.array(free_pages)
    before, R = ring.copy(), len(ring)
    head, tail = int(pool[0]), int(pool[1])
    taken = given = wanted = 0
    kv, status, starts, slots, positions = [], [], [0], [], []
    for s in range(len(lens)):
        old, n = max(int(lens[s]), 0), int(new[s])
        want = max(old + n, 0)
        had, has = -(-old // page_size), -(-want // page_size)
        code = 2 if max(had, has) > table.shape[1] else 0
        if code == 0 and has > had:
            wanted += has - had
            if wanted > tail - head:
                code = 1
        if code == 0:
            for j in range(had, has):
                table[s, j] = before[(head + taken) % R]
                taken += 1
            for j in range(has, had):
                ring[(tail + given) % R] = table[s, j]
                given += 1
        for p in range(old, old + max(n, 0)):
            positions.append(p)
            slots.append(-1 if code else int(table[s, p // page_size]) * page_size + p % page_size)
        starts.append(len(positions))
        kv.append(old if code else want)
        status.append(code)
    pad = [-1] * max(0, max_tokens - len(slots))
    return {"kv_lens": np.array(kv, np.int32), "query_start": np.array(starts, np.int32),
            "slot_map": np.array((slots + pad)[:max_tokens], np.int64),
            "positions": np.array((positions + pad)[:max_tokens], np.int32), "status": np.array(status, np.int32),
            "pool": np.array([head + taken, tail + given], np.int64), "block_table": table, "free_pages": ring}


def write(k, v, slots, k_codes, v_codes, k_scale, v_scale):
    """k, v float64 [tokens, heads, dim]; codes uint8 [pages, page, heads, dim]; returns the four arrays afterwards."""
    kc, vc, ks, vs = (np.array(a) for a in (k_codes, v_codes, k_scale, v_scale))
    n_pages, page = kc.shape[:2]
    slots = np.asarray(slots, dtype=np.int64)
    ok = (slots >= 0) & (slots < n_pages * page)
    i = 0
    while i < len(slots):
        if not ok[i]:
            i += 1
            continue
        p, a = int(slots[i]) // page, int(slots[i]) % page
        there = [t for t in range(min(page - a, len(slots) - i)) if ok[i + t] and slots[i + t] == slots[i] + t]
        rows, at = [i + t for t in there], [a + t for t in there]
        for h in range(kc.shape[2]):
            x, y = np.array(k[rows, h], np.float64), np.array(v[rows, h], np.float64)
            bad = ~(np.isfinite(x).all(1) & np.isfinite(y).all(1))
            for new, codes, scale, fill in ((x, kc, ks, 0x7F), (y, vc, vs, 0)):
                good = np.where(bad[:, None], 0.0, new)
                e = int(scale_byte(np.abs(good).max()))
                if a:
                    e = max(e, int(scale[p, h]))
                    if e > int(scale[p, h]):
                        held = E4M3[codes[p, :a, h]] * np.ldexp(1.0, int(scale[p, h]) - e)
                        codes[p, :a, h] = e4m3_encode(held)
                scale[p, h] = e
                codes[p, at, h] = np.where(bad[:, None], np.uint8(fill), e4m3_encode(good * pow2(254 - e)))
        i = rows[-1] + 1
    return kc, vc, ks, vs


def visible(kv_len: int, q_len: int, i: int, mask_block: int) -> int:
    if mask_block == 0:
        return kv_len
    return min(max(kv_len - q_len + min(q_len, (i // mask_block + 1) * mask_block), 0), kv_len)


def attention(q, k_codes, v_codes, k_scale, v_scale, block_table, kv_lens, query_start, scale, mask_block):
    """q float64 [tokens, heads, dim]; returns (out, lse, spread, work): the attention in float64, its log-sum-exp, the
    weighted mean of |v| and the largest sum of |q k| scale of a row (what rounding errors are proportional to)."""
    n_tok, n_q, dim = q.shape
    n_pages, page, n_kv = k_codes.shape[:3]
    g = n_q // n_kv
    out, spread = np.zeros((n_tok, n_q, dim)), np.zeros((n_tok, n_q, dim))
    lse, work = np.full((n_tok, n_q), -np.inf), np.zeros((n_tok, n_q))
    for s in range(len(kv_lens)):
        n, q0 = max(int(kv_lens[s]), 0), int(query_start[s])
        q_len = int(query_start[s + 1]) - q0
        pages = np.asarray(block_table[s][:-(-n // page)], dtype=np.int64)
        k = (E4M3[k_codes[pages]] * pow2(k_scale[pages])[:, None, :, None]).reshape(-1, n_kv, dim)[:n]
        v = (E4M3[v_codes[pages]] * pow2(v_scale[pages])[:, None, :, None]).reshape(-1, n_kv, dim)[:n]
        for i in range(q_len):
            see = visible(n, q_len, i, mask_block)
            if see == 0:
                continue
            for h in range(n_q):
                kk, vv, qq = k[:see, h // g], v[:see, h // g], q[q0 + i, h]
                x = kk @ qq * scale
                top = np.nanmax(x) if np.isfinite(x).any() else 0.0
                w = np.exp(x - top)
                total = w.sum()
                out[q0 + i, h] = w @ vv / total
                spread[q0 + i, h] = w @ np.abs(vv) / total
                lse[q0 + i, h] = top + np.log(total)
                work[q0 + i, h] = np.max(np.abs(kk) @ np.abs(qq)) * abs(scale)
    return out, lse, spread, work


def attention_largest_term(q, k_codes, v_codes, k_scale, v_scale, block_table, kv_lens, query_start, scale, mask_block):
    """[tokens, heads, dim]: the largest p_t 2^(value exponent) of the tokens that a row sees, p its softmax, times the sum
    of their value codes' magnitudes: what absolute errors of weights too small for their format are proportional to."""
    n_tok, n_q, dim = q.shape
    n_kv = k_codes.shape[2]
    g = n_q // n_kv
    out = np.zeros((n_tok, n_q, dim))
    for s in range(len(kv_lens)):
        n, q0 = max(int(kv_lens[s]), 0), int(query_start[s])
        q_len = int(query_start[s + 1]) - q0
        pages = np.asarray(block_table[s][:-(-n // k_codes.shape[1])], dtype=np.int64)
        k = (E4M3[k_codes[pages]] * pow2(k_scale[pages])[:, None, :, None]).reshape(-1, n_kv, dim)[:n]
        codes = np.abs(E4M3[v_codes[pages]]).reshape(-1, n_kv, dim)[:n]
        ve = np.repeat(pow2(v_scale[pages]), k_codes.shape[1], axis=0)[:n]
        for i in range(q_len):
            see = visible(n, q_len, i, mask_block)
            for h in range(n_q if see else 0):
                x = k[:see, h // g] @ q[q0 + i, h] * scale
                w = np.exp(x - np.max(x))
                out[q0 + i, h] = np.max(w * ve[:see, h // g]) / w.sum() * codes[:see, h // g].sum(0)
    return out


def attention_best_token(q, k_codes, v_codes, k_scale, v_scale, block_table, kv_lens, query_start, scale, mask_block):
    """For each row: the value of the token with the best score [tokens, heads, dim], by how much that score is above
    the next [tokens, heads] (infinite for one token), and the largest |value| it sees [tokens, heads, dim]."""
    n_tok, n_q, dim = q.shape
    n_kv = k_codes.shape[2]
    g = n_q // n_kv
    value, most, gap = np.zeros((n_tok, n_q, dim)), np.zeros((n_tok, n_q, dim)), np.full((n_tok, n_q), np.inf)
    for s in range(len(kv_lens)):
        n, q0 = max(int(kv_lens[s]), 0), int(query_start[s])
        q_len = int(query_start[s + 1]) - q0
        pages = np.asarray(block_table[s][:-(-n // k_codes.shape[1])], dtype=np.int64)
        k = (E4M3[k_codes[pages]] * pow2(k_scale[pages])[:, None, :, None]).reshape(-1, n_kv, dim)[:n]
        v = (E4M3[v_codes[pages]] * pow2(v_scale[pages])[:, None, :, None]).reshape(-1, n_kv, dim)[:n]
        for i in range(q_len):
            see = visible(n, q_len, i, mask_block)
            for h in range(n_q if see else 0):
                x = k[:see, h // g] @ q[q0 + i, h] * scale
                t = int(np.argmax(x))
                value[q0 + i, h], most[q0 + i, h] = v[t, h // g], np.abs(v[:see, h // g]).max(0)
                if see > 1:
                    gap[q0 + i, h] = x[t] - np.max(np.delete(x, t))
    return value, gap, most
