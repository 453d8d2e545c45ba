"""Rotary positions and the paged latent cache of a serving program: what each call is given, what it returns, and how
much of it there is, as cases that can be timed and compared.

Four operators, as one forward of a batch of requests uses them:

  rotate        kv_rotate: queries (or keys) turned by their positions, or back by them (the adjoint)
  append        kv_write_rotated: keys turned and stored with the values in the paged 8-bit cache, queries turned in the
                same call
  latent_write  kv_latent_write: one latent vector and one turned key part for each token into the paged 16-bit cache
  latent_attn   kv_latent_attention: attention of all heads over that cache, single tokens, drafts, prompts

Inputs: queries, keys, values and latents N(0, 1) times an amplitude for each head (2^-2 to 2^2) where they have heads,
keys with a few strong channels, as projected states have them. Lengths are spread evenly over the case's range, in an
order of the seed; pages are handed out in an order of the seed. Rotation tables have the frequencies of base^(-2p/dim),
stretched for long contexts where a case says so.
"""

import math

import numpy as np
import torch

own = False

E_MIN, E_MAX = 27, 247  # the exponents a write stores: scales 2^-100 to 2^120


# ------------------------------------------------------------------------------------------------------------ cases --
def _rotate(name, n_seq, lo, hi, add, heads, dim, rot, inter=False, factor=1.0, back=False, dtype="bf16"):
    """`add` new tokens of each of n_seq requests behind lo..hi others; the first `rot` of `dim` elements of each head are
    turned, pairs next to each other (`inter`) or half of them apart; contexts stretched by `factor`."""
    c = {"op": "rotate", "n_seq": n_seq, "lo": lo, "hi": hi, "add": add, "heads": heads, "dim": dim, "rot": rot,
         "inter": inter, "factor": factor, "back": back, "dtype": dtype}
    return dict(c, name=name) if name else c


def _append(name, n_seq, lo, hi, add, page, n_q, n_kv, dim, rot, inter=False, factor=1.0, dtype="bf16"):
    """`add` new tokens of each of n_seq requests into the 8-bit cache; n_q 0: keys and values alone."""
    c = {"op": "append", "n_seq": n_seq, "lo": lo, "hi": hi, "add": add, "page": page, "n_q": n_q, "n_kv": n_kv,
         "dim": dim, "rot": rot, "inter": inter, "factor": factor, "dtype": dtype}
    return dict(c, name=name) if name else c


def _latent_write(name, n_seq, lo, hi, add, page, dim, rot, inter=True, factor=1.0, dtype="bf16"):
    c = {"op": "latent_write", "n_seq": n_seq, "lo": lo, "hi": hi, "add": add, "page": page, "dim": dim, "rot": rot,
         "inter": inter, "factor": factor, "dtype": dtype}
    return dict(c, name=name) if name else c


def _latent_attn(name, n_seq, lo, hi, q_len, block, page, heads, dim, rot, dtype="bf16", lse=False):
    """n_seq requests of lo..hi tokens in the latent cache, the last q_len of them this forward's; `block`: 0 no mask, 1
    causal, else causal by blocks."""
    c = {"op": "latent_attn", "n_seq": n_seq, "lo": lo, "hi": hi, "q_len": q_len, "block": block, "page": page,
         "heads": heads, "dim": dim, "rot": rot, "dtype": dtype, "lse": lse}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the queries of one token of each request of a serving batch: a call's latency
        _rotate("rotate_64x1", 64, 50, 8000, 1, 32, 128, 128),
        # back from the largest window's turned queries, far into long documents: the adjoint; bands of frequencies
        _rotate("rotate_back_256x8x64", 256, 1000, 900000, 512, 32, 128, 128, True, 32.0, True),
        # one token of each request of a serving batch: queries, keys and values
        _append("append_64x1", 64, 50, 8000, 1, 64, 32, 8, 128, 128),
        # windows of 3 blocks of 20 in pages of 32, heads of 80 of which 48 are turned
        _append("append_48x3x20_d80", 48, 33, 2001, 60, 32, 10, 5, 80, 48, True),
        # the largest window
        _append("append_256x8x64", 256, 64, 1024, 512, 64, 32, 8, 128, 128, False, 8.0),
        # one token of each request of a serving batch: a call's latency
        _latent_write("latent_write_64x1", 64, 50, 8000, 1, 64, 512, 64),
        # the largest window's tokens
        _latent_write("latent_write_256x8x64", 256, 64, 1024, 512, 64, 512, 64, True, 32.0),
        # one request alone, one token: a call's latency
        _latent_attn("latent_token_1", 1, 1531, 1531, 1, 0, 32, 16, 512, 64),
        # one token of each request of a serving batch, lengths as they fall
        _latent_attn("latent_token_64", 64, 57, 8189, 1, 0, 64, 16, 512, 64),
        # two long documents, f16, an odd number of heads: work split along the cache
        _latent_attn("latent_token_2_long_f16", 2, 110001, 131071, 1, 0, 64, 20, 512, 64, "f16"),
        # speculative decoding, all heads on one GPU: 32 requests x (4 drafts + 1), causal, with the log-sum-exp
        _latent_attn("latent_verify_32x5", 32, 300, 4001, 5, 1, 64, 128, 512, 64, lse=True),
        # prompts of 1025 tokens behind what is cached, two at a time, f16, a smaller latent, small pages
        _latent_attn("latent_prompt_2x1025_f16", 2, 1025, 3333, 1025, 1, 16, 16, 256, 32, "f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "latent_write", "latent_attn", "latent_attn", "latent_attn"])
    page = rng.choice([16, 32, 32, 64, 64, 128, 256])
    n_seq = _log(rng, 1, 256)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16"])
    inter, factor = rng.random() < 0.5, rng.choice([1.0, 1.0, 8.0, 32.0])
    dim = rng.choice([64, 80, 96, 128, 128, 128])
    rot = rng.choice([dim, dim, dim // 32 * 16, 16])
    add = rng.choice([1, _log(rng, 1, 512)])
    if op == "rotate":
        hi = _log(rng, 16, 900000)
        return _rotate(None, n_seq, rng.randint(0, hi), hi, add, rng.choice([1, 5, 8, 12, 28, 32]), dim, rot, inter, factor,
                       rng.random() < 0.5, dtype)
    if op == "append":
        n_kv, hi = rng.choice([1, 2, 4, 5, 8]), _log(rng, 16, 1024)
        return _append(None, n_seq, rng.randint(0, hi), hi, add, page, n_kv * rng.choice([0, 1, 2, 3, 4]), n_kv, dim, rot,
                       inter, factor, dtype)
    dim, rot = rng.choice([(512, 64), (512, 64), (512, 64), (256, 32), (128, 64), (448, 48), (96, 16)])
    if op == "latent_write":
        hi = _log(rng, 16, 1024)
        return _latent_write(None, n_seq, rng.randint(0, hi), hi, add, page, dim, rot, inter, factor, dtype)
    heads = rng.choice([1, 5, 8, 16, 16, 20, 32, 64, 128])
    q_len = rng.choice([1, 1, 1, rng.randint(2, 9), _log(rng, 8, 512), _log(rng, 8, 1025)])
    block = rng.choice([0, 1, rng.choice([8, 20, 32, 64])]) if q_len > 1 else rng.choice([0, 1])
    hi = max(q_len, _log(rng, 100, 131071 if q_len == 1 else 8192))
    lo = max(q_len, rng.randint(hi // 8, hi))
    while n_seq > 1 and (n_seq * q_len * heads * hi > 32 * 5 * 128 * 2100 or n_seq * hi > 64 * 4100):
        n_seq //= 2
    q_len = max(1, min(q_len, 32 * 5 * 128 * 2100 // (heads * hi)))
    return _latent_attn(None, n_seq, lo, hi, q_len, block, page, heads, dim, rot, dtype, rng.random() < 0.3)


# ----------------------------------------------------------------------------------------------------------- inputs --
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _lens(c):
    """n_seq lengths spread over lo..hi."""
    n = c["n_seq"]
    return [c["lo"] + (c["hi"] - c["lo"]) * (2 * s + 1) // (2 * n) if n > 1 else c["hi"] for s in range(n)]


def _pages(n, page):
    return -(-n // page)


def _frequencies(c):
    """Radians a position for each pair, float64 [rot / 2]. Where the context is stretched, frequencies that turn once or
    less in 4096 positions are divided by the factor, those with 32 turns or more are kept."""
    f = 10000.0 ** (-np.arange(0, c["rot"], 2, dtype=np.float64) / c["rot"])
    keep = np.clip((4096 * f / (2 * math.pi) - 1) / 31, 0, 1) if c["factor"] != 1 else 1.0
    return f * keep + f / c["factor"] * (1 - keep)


def _amplitude(c):
    return 1 + 0.1 * math.log(c["factor"])


def _turns(c):
    """The same as fractions of a turn times 2^64, as the calls take them: a position's angle is a product modulo 2^64."""
    t = [int(round(float(f) / (2 * math.pi) * 2.0 ** 64)) for f in _frequencies(c)]
    return torch.tensor([x - (x >> 63 << 64) for x in t], dtype=torch.int64, device="cuda")


def _exponent(amax):
    """E8M0 byte of the smallest power of two that brings `amax` to at most 448 = 0.875 * 2^9."""
    m, e = torch.frexp(amax)
    e = e.to(torch.int32) - 9 + (m > 0.875).to(torch.int32) + 127
    return torch.where(amax > 0, e, E_MIN).clamp(E_MIN, E_MAX)


def _pow2(k):
    """2^k for whole k, by its bits: a power function may be off by a bit, which moves ties."""
    return ((k.to(torch.int32).clamp(-126, 127) + 127) << 23).view(torch.float32)


def _codes_of(g, n_pages, page, n_kv, dim):
    """(codes, scales) of pages filled with keys or values: [n_pages, n_kv, page, dim] E4M3, [n_pages, n_kv]."""
    amp = torch.exp2(torch.rand(1, n_kv, 1, 1, generator=g, device="cuda") * 4 - 2)
    x = torch.randn(n_pages, n_kv, page, dim, generator=g, device="cuda").mul_(amp)
    e = _exponent(x.abs().amax((2, 3)))
    return x.mul_(_pow2(127 - e)[:, :, None, None]).to(torch.float8_e4m3fn), e.to(torch.uint8)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(host, total, page, cols):
    """Block tables of requests of `total` tokens in pages of any order, and the number of pages."""
    held = [_pages(n, page) for n in total]
    n_pages = sum(held) + 3
    order = host.permutation(n_pages).astype(np.int32)
    table = np.full((len(total), cols), -1, dtype=np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    return table, n_pages


def prepare(c, seed):
    g, host = torch.Generator(device="cuda"), np.random.default_rng(seed)
    g.manual_seed(seed)
    lens = [int(v) for v in host.permutation(_lens(c))]
    n_seq, dt, rot = c["n_seq"], DTYPES[c["dtype"]], c["rot"]

    def normal(*shape, amp=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(amp).to(dt)

    def amps(heads):
        return torch.exp2(torch.rand(1, heads, 1, generator=g, device="cuda") * 4 - 2)

    st = {"case": c}
    if c["op"] == "latent_attn":
        table, n_pages = _table(host, lens, c["page"], _pages(c["hi"], c["page"]) + 1)
        rows = normal(n_pages, c["page"], c["dim"] + rot)
        st["latent"], st["rope"] = rows.split([c["dim"], rot], 2)
        st["table"], st["kv_lens"] = torch.from_numpy(table).cuda(), _i32(lens)
        st["starts"] = torch.arange(0, (n_seq + 1) * c["q_len"], c["q_len"], dtype=torch.int32, device="cuda")
        st["q"] = normal(n_seq * c["q_len"], c["heads"], c["dim"] + rot)
        st["scale"] = 1.5 * (c["dim"] + rot) ** -0.5  # scores of about N(0, 1.5^2)
        return st
    add = c["add"]
    pos = np.concatenate([np.arange(n, n + add) for n in lens])
    st["positions"], st["turns"] = torch.from_numpy(pos.astype(np.int32)).cuda(), _turns(c)
    if c["op"] == "rotate":
        st["x"] = normal(n_seq * add, c["heads"], c["dim"], amp=amps(c["heads"]))
        return st
    page = c["page"]
    table, n_pages = _table(host, [n + add for n in lens], page, _pages(c["hi"] + add, page) + 1)
    st["slots"] = torch.from_numpy(table[np.repeat(np.arange(n_seq), add), pos // page].astype(np.int64) * page
                                   + pos % page).cuda()
    if c["op"] == "latent_write":
        st["latent"], st["rope"] = normal(n_pages, page, c["dim"] + rot).split([c["dim"], rot], 2)
        st["new_latent"], st["new_rope"] = normal(n_seq * add, c["dim"]), normal(n_seq * add, rot, amp=4.0)
        return st
    n_kv, dim = c["n_kv"], c["dim"]
    k, st["ks"] = _codes_of(g, n_pages, page, n_kv, dim)
    v, st["vs"] = _codes_of(g, n_pages, page, n_kv, dim)
    st["k"], st["v"] = k.transpose(1, 2), v.transpose(1, 2)  # [page, token, head, dim]
    st["first"] = torch.arange(0, n_seq * add, add, device="cuda")  # each request's first new token
    # one projection's rows: queries, keys and values of a token next to each other
    qkv = torch.randn(n_seq * add, c["n_q"] + 2 * n_kv, dim, generator=g, device="cuda").mul_(amps(c["n_q"] + 2 * n_kv))
    qkv[:, c["n_q"]:c["n_q"] + n_kv, 3::dim // 4] *= 4
    st["q"], st["new_k"], st["new_v"] = qkv.to(dt).split([c["n_q"], n_kv, n_kv], 1)
    return st


# ------------------------------------------------------------------------------------------------------ plain forms --
def _turned(x, positions, turns, amplitude, inter, back=False):
    """x [tokens, heads, dim] with the first 2 * len(turns) elements of each head turned, float32."""
    half = turns.numel()
    angle = (positions.long()[:, None] * turns).double() * (2 * math.pi * 2.0 ** -64 * (-1 if back else 1))
    cos, sin = ((t * amplitude).float()[:, None] for t in (angle.cos(), angle.sin()))
    x = x.float()
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = part.unflatten(2, (half, 2)).unbind(3) if inter else part.unflatten(2, (2, half)).unbind(2)
    turned = torch.stack([a * cos - b * sin, a * sin + b * cos], 3 if inter else 2).flatten(2)
    return torch.cat([turned, rest], 2)


def _plain_rotate(st):
    c = st["case"]
    return _turned(st["x"], st["positions"], st["turns"], _amplitude(c), c["inter"], c["back"]).to(st["x"].dtype)


def _store_one(x, bad, codes, scales, page_of, off, first_page, first_off, nan_rows):
    """One of keys and values [tokens, heads, dim]: amax of each page and head, its exponent, the codes; the tokens that
    a request's first page holds already are scaled again where its exponent grew."""
    n_pages, page, n_kv, dim = codes.shape
    amax = torch.where(bad, 0.0, x.abs().amax(2))
    top = torch.full((n_pages, n_kv), -1.0, device=x.device)
    top = top.scatter_reduce(0, page_of[:, None].expand(-1, n_kv), amax, "amax")
    before = scales.int()
    kept = torch.full((n_pages,), page, device=x.device).scatter_reduce(0, page_of, off, "amin")  # first offset written
    run = _exponent(top)
    e = torch.where(top < 0, before, torch.where((kept > 0)[:, None], torch.maximum(before, run), run))
    scales.copy_(e.to(torch.uint8))
    shift = _pow2(before - e)[first_page][:, None, :, None]
    there = (torch.arange(page, device=x.device)[None] < first_off[:, None])[:, :, None, None] & (shift != 1)
    raw = codes.view(torch.uint8)
    held = raw[first_page]
    again = (held.view(torch.float8_e4m3fn).float() * shift).to(torch.float8_e4m3fn).view(torch.uint8)
    raw[first_page] = torch.where(there, again, held)
    y = (x * _pow2(127 - e[page_of])[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    y = torch.where(bad[:, :, None], torch.tensor(0x7f if nan_rows else 0, dtype=torch.uint8, device=x.device), y)
    raw[page_of, off] = y


def _plain_append(st):
    c = st["case"]
    dt, args = st["new_k"].dtype, (st["positions"], st["turns"], _amplitude(c), c["inter"])
    k = _turned(st["new_k"], *args).to(dt).float()  # what is stored is the turned key in its own type
    v = st["new_v"].float()
    page_of, off = st["slots"] // c["page"], st["slots"] % c["page"]
    first_page, first_off = page_of[st["first"]], off[st["first"]]
    bad = ~(k.isfinite().all(2) & v.isfinite().all(2))
    _store_one(k, bad, st["k"], st["ks"], page_of, off, first_page, first_off, True)
    _store_one(v, bad, st["v"], st["vs"], page_of, off, first_page, first_off, False)
    got = {"k": st["k"], "v": st["v"], "k_scale": st["ks"], "v_scale": st["vs"]}
    return dict(got, q=_turned(st["q"], *args).to(dt)) if c["n_q"] else got


def _plain_latent_write(st):
    c, rope = st["case"], st["new_rope"]
    turned = _turned(rope[:, None], st["positions"], st["turns"], _amplitude(c), c["inter"])[:, 0].to(rope.dtype)
    page_of, off = st["slots"] // c["page"], st["slots"] % c["page"]
    st["latent"][page_of, off], st["rope"][page_of, off] = st["new_latent"], turned
    return {"latent": st["latent"], "rope": st["rope"]}


def _plain_latent_attn(st):
    c = st["case"]
    n_seq, q_len, heads, dim, page = c["n_seq"], c["q_len"], c["heads"], c["dim"], c["page"]
    cols = _pages(c["hi"], page)
    table, T = st["table"][:, :cols].clamp(min=0).long(), cols * page
    t = torch.arange(T, device="cuda")
    held = (t[None] < st["kv_lens"][:, None])[:, :, None]
    latent = torch.where(held, st["latent"][table].reshape(n_seq, T, dim).float(), 0)
    rope = torch.where(held, st["rope"][table].reshape(n_seq, T, -1).float(), 0)
    q = st["q"].float().reshape(n_seq, q_len * heads, -1)
    s = torch.matmul(q[..., :dim], latent.transpose(1, 2)) + torch.matmul(q[..., dim:], rope.transpose(1, 2))
    s = s.mul_(st["scale"]).reshape(n_seq, q_len, heads, T)
    i = torch.arange(q_len, device="cuda")
    see = ((i // c["block"] + 1) * c["block"]).clamp(max=q_len) if c["block"] else q_len
    see = (st["kv_lens"][:, None] - q_len + see).expand(n_seq, q_len)
    s.masked_fill_(t >= see[:, :, None, None], -math.inf)
    m = s.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, 0, m)
    p = s.sub_(m).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p.reshape(n_seq, q_len * heads, T), latent).reshape(n_seq, q_len, heads, dim)
    o = torch.where(total > 0, o / total, torch.where(total == 0, 0, total))
    out = o.reshape(n_seq * q_len, heads, dim).to(st["q"].dtype)
    return (out, (m + total.log()).reshape(n_seq * q_len, heads)) if c["lse"] else out


def run(st):
    c = st["case"]
    if not own:
        return {"rotate": _plain_rotate, "append": _plain_append, "latent_write": _plain_latent_write,
                "latent_attn": _plain_latent_attn}[c["op"]](st)
    import paper_2609_33887_gb300 as bdc

    if c["op"] == "latent_attn":
        return bdc.kv_latent_attention(st["q"], bdc.KvLatent(st["latent"], st["rope"]), st["table"], st["kv_lens"],
                                       st["starts"], scale=st["scale"], max_q_len=c["q_len"], max_kv_len=c["hi"],
                                       mask_block=c["block"], return_lse=c["lse"])
    rotary = bdc.KvRotary(st["turns"], _amplitude(c), c["inter"])
    if c["op"] == "rotate":
        return bdc.kv_rotate(st["x"], st["positions"], rotary, inverse=c["back"])
    if c["op"] == "latent_write":
        bdc.kv_latent_write(st["new_latent"], st["new_rope"], st["slots"], bdc.KvLatent(st["latent"], st["rope"]),
                            positions=st["positions"], rotary=rotary)
        return {"latent": st["latent"], "rope": st["rope"]}
    q = bdc.kv_write_rotated(st["new_k"], st["new_v"], st["slots"], bdc.KvCache(st["k"], st["v"], st["ks"], st["vs"]),
                             st["positions"], rotary, q=st["q"] if c["n_q"] else None)
    got = {"k": st["k"], "v": st["v"], "k_scale": st["ks"], "v_scale": st["vs"]}
    return dict(got, q=q) if c["n_q"] else got


# ------------------------------------------------------------------------------------------------------------- work --
def _see(c, n, i):
    return n - c["q_len"] + (min(c["q_len"], (i // c["block"] + 1) * c["block"]) if c["block"] else c["q_len"])


def work(c):
    lens = _lens(c)
    if c["op"] == "latent_attn":
        rows = c["n_seq"] * c["q_len"] * c["heads"]
        seen = sum(_see(c, n, i) for n in lens for i in range(c["q_len"]))
        wide = c["dim"] + c["rot"]
        return {"bytes": 2 * sum(lens) * wide + rows * (2 * wide + 2 * c["dim"] + (4 if c["lse"] else 0)),
                "flops": 2 * seen * c["heads"] * (wide + c["dim"])}
    tokens = c["n_seq"] * c["add"]
    if c["op"] == "rotate":
        return {"bytes": tokens * (4 * c["heads"] * c["dim"] + 4), "flops": 3 * tokens * c["heads"] * c["rot"]}
    if c["op"] == "latent_write":
        return {"bytes": tokens * (4 * (c["dim"] + c["rot"]) + 12), "flops": 3 * tokens * c["rot"]}
    touched = sum(_pages(n + c["add"], c["page"]) - n // c["page"] for n in lens)
    return {"bytes": tokens * (c["n_kv"] * c["dim"] * 6 + c["n_q"] * c["dim"] * 4 + 12) + touched * c["n_kv"] * 2,
            "flops": 3 * tokens * (c["n_kv"] + c["n_q"]) * c["rot"]}


# ------------------------------------------------------------------------------------ from the definition, 64 bits --
def _pow2_64(k):
    return ((k + 1023) << 52).view(torch.float64)


def _rotation_64(x, st, back=False):
    """Each pair as a complex number times amplitude * exp(i position frequency)."""
    c = st["case"]
    x, n = x.double(), c["rot"]
    angle = st["positions"].double()[:, None] * torch.from_numpy(_frequencies(c)).cuda()
    by = torch.polar(torch.full_like(angle, _amplitude(c)), -angle if back else angle)[:, None]
    y = x.clone()
    first, second = (slice(0, n, 2), slice(1, n, 2)) if c["inter"] else (slice(0, n // 2), slice(n // 2, n))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * by
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_append(st):
    page, dt = st["case"]["page"], st["new_k"].dtype
    slots = st["slots"].cpu().numpy()
    # one entry for each run of slots in a page: [page, first offset, first token, tokens]
    cut = np.flatnonzero(np.concatenate([[True], (np.diff(slots) != 1) | (slots[1:] % page == 0)]))
    size = np.diff(np.concatenate([cut, [len(slots)]]))
    got = {}
    new = {"k": _rotation_64(st["new_k"], st).to(dt).double(), "v": st["new_v"].double()}
    for name, scales in (("k", "ks"), ("v", "vs")):
        x, held = new[name], st[name].double()
        e = st[scales].long()
        for r0, n in zip(cut.tolist(), size.tolist()):
            p, a = int(slots[r0]) // page, int(slots[r0]) % page
            y = x[r0:r0 + n]
            most = y.abs().amax((0, 2))
            up = (torch.log2(most / 448) - 0.5).floor().clamp(E_MIN - 127, E_MAX - 127).long()  # 2^up or less, then
            for _ in range(2):  # as many as it takes for 448 * 2^up to reach the largest
                up = up + (448 * _pow2_64(up) < most)
            up = up.clamp(E_MIN - 127, E_MAX - 127) + 127
            if a:
                up = torch.maximum(up, e[p])
                held[p, :a] = (held[p, :a] * _pow2_64(e[p] - up)[:, None]).to(torch.float8_e4m3fn).double()
            e[p] = up
            held[p, a:a + n] = (y * _pow2_64(127 - up)[:, None]).to(torch.float8_e4m3fn).double()
        got[name], got[name + "_scale"] = held, e.to(torch.uint8)
    return dict(got, q=_rotation_64(st["q"], st)) if st["case"]["n_q"] else got


def _exact_latent_write(st):
    got = {}
    for name, new in (("latent", st["new_latent"].double()), ("rope", _rotation_64(st["new_rope"][:, None], st)[:, 0])):
        held = st[name].double().contiguous()
        held.view(-1, held.shape[2])[st["slots"]] = new
        got[name] = held
    return got


def _exact_latent_attn(st):
    c = st["case"]
    n_seq, q_len, heads, dim, page = c["n_seq"], c["q_len"], c["heads"], c["dim"], c["page"]
    out = torch.zeros(n_seq * q_len, heads, dim, dtype=torch.float64, device="cuda")
    lse = torch.zeros(n_seq * q_len, heads, dtype=torch.float64, device="cuda")
    lens, table = st["kv_lens"].tolist(), st["table"].cpu()
    for s in range(n_seq):
        pages = table[s, :_pages(lens[s], page)].long().cuda()
        value = st["latent"][pages].double().reshape(-1, dim)[:lens[s]]
        key = torch.cat([value, st["rope"][pages].double().reshape(-1, c["rot"])[:lens[s]]], 1)
        see = torch.tensor([_see(c, lens[s], i) for i in range(q_len)], device="cuda")
        hide = torch.arange(lens[s], device="cuda")[None] >= see[:, None]
        rows = slice(s * q_len, (s + 1) * q_len)
        for h in range(heads):
            x = (st["q"][rows, h].double() @ key.T) * st["scale"]
            x[hide] = -math.inf
            out[rows, h] = torch.softmax(x, 1) @ value
            lse[rows, h] = torch.logsumexp(x, 1)
    return (out, lse) if c["lse"] else out


def exact(c, seed):
    st = prepare(c, seed)
    if c["op"] == "rotate":
        return _rotation_64(st["x"], st, c["back"])
    return {"append": _exact_append, "latent_write": _exact_latent_write, "latent_attn": _exact_latent_attn}[c["op"]](st)
