"""The paged 8-bit key/value cache on the GPU (kv_tables, kv_write, kv_attention) against the float64 oracle.

Tables and writes are compared exactly: whole numbers, and codes whose rounding is defined to the bit. Attention is
compared within bounds that follow from the number formats (see attention_bounds); what no call may read (a page's
tail, unused pages, table entries behind a request) holds NaN codes or page numbers far out of range.
"""

import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from workloads.cache_inputs import random_cache, random_tables

pytestmark = pytest.mark.gpu

bdc = pytest.importorskip("paper_2609_33887_gb300")

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)
    yield
    assert bdc.kvcache.kv_device_status() == 0


# ------------------------------------------------------------------ tables --
def run_tables(t, page, max_tokens=None):
    g = {k: torch.from_numpy(np.ascontiguousarray(t[k])).cuda() for k in ("lens", "new", "table", "ring", "pool")}
    r = bdc.kv_tables(g["lens"], g["new"], g["table"], g["ring"], g["pool"], page_size=page,
                      max_tokens=t["max_tokens"] if max_tokens is None else max_tokens)
    torch.cuda.synchronize()
    return dict({k: getattr(r, k).cpu().numpy() for k in r._fields}, block_table=g["table"].cpu().numpy(),
                free_pages=g["ring"].cpu().numpy()), g


def assert_tables(t, page, max_tokens=None):
    got, g = run_tables(t, page, max_tokens)
    ref = CO.tables(t["lens"], t["new"], t["table"], t["ring"], t["pool"], page,
                    t["max_tokens"] if max_tokens is None else max_tokens)
    for k, v in ref.items():
        assert got[k].dtype == v.dtype and np.array_equal(got[k], v), k
    return g


@pytest.mark.parametrize("n_seq", [1, 2, 31, 33, 513, 2000])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("spare", [4, 0, -3])
def test_tables_match_the_oracle(n_seq, page, spare):
    for seed in range(3):
        assert_tables(random_tables(n_seq, page, seed=seed, spare=spare), page)


def test_tables_of_the_most_requests_and_of_none():
    assert_tables(random_tables(8192, 32, seed=5, max_len=200, max_new=9), 32)
    t = random_tables(1, 16, seed=0)
    t.update(lens=t["lens"][:0], new=t["new"][:0], table=t["table"][:0], max_tokens=4)
    assert_tables(t, 16)


@pytest.mark.parametrize("max_tokens", [0, 1, 40])
def test_tables_with_fewer_token_entries_than_tokens(max_tokens):
    t = random_tables(9, 16, seed=2, give=0.0)
    assert_tables(t, 16, max_tokens)


def test_tables_refuse_requests_that_outgrow_their_row():
    for seed in range(4):
        t = random_tables(40, 16, seed=seed, cols=12)
        assert_tables(t, 16)
        assert (run_tables(t, 16)[0]["status"] == 2).any()


def test_tables_take_long_prompts_negative_lengths_and_everything_back():
    t = random_tables(5, 16, seed=3, max_len=3000, max_new=5000, give=0.0)
    assert_tables(t, 16)
    t = random_tables(6, 32, seed=4)
    t["lens"][1], t["new"][2], t["new"][3] = -7, -(2 ** 31), -1
    assert_tables(t, 32)


def test_tables_called_twice_on_the_same_inputs_give_the_same():
    t = random_tables(50, 16, seed=6)
    g = assert_tables(t, 16)
    again = bdc.kv_tables(g["lens"], g["new"], g["table"], g["ring"], g["pool"], page_size=16,
                          max_tokens=t["max_tokens"])
    ref = CO.tables(t["lens"], t["new"], t["table"], t["ring"], t["pool"], 16, t["max_tokens"])
    assert np.array_equal(again.slot_map.cpu().numpy(), ref["slot_map"])
    assert np.array_equal(g["ring"].cpu().numpy(), ref["free_pages"])
    assert np.array_equal(again.pool.cpu().numpy(), ref["pool"])


def test_tables_over_many_steps_lose_no_page():
    rng = np.random.default_rng(0)
    n_seq, page, n_pages = 12, 16, 120
    lens = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    table = torch.full((n_seq, 40), -1, dtype=torch.int32, device="cuda")
    ring = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    pool = torch.tensor([0, n_pages], dtype=torch.int64, device="cuda")
    for _ in range(60):
        new = torch.from_numpy(rng.integers(-60, 90, n_seq).astype(np.int32)).cuda()
        r = bdc.kv_tables(lens, new, table, ring, pool, page_size=page, max_tokens=1100)
        lens, pool = r.kv_lens, r.pool
        held = [int(p) for s, n in enumerate(lens.tolist()) for p in table[s, :-(-n // page)].tolist()]
        head, tail = pool.tolist()
        free = [int(ring[i % n_pages]) for i in range(head, tail)]
        assert sorted(held + free) == list(range(n_pages))


# ------------------------------------------------------------------ writes --
def laid_out(a: np.ndarray, layout: str) -> torch.Tensor:
    """Codes [pages, page, heads, dim] on the GPU in one of the layouts a cache may have."""
    t = torch.from_numpy(a).cuda()
    if layout == "head":  # a page's tokens of one head next to each other
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "token":
        return t
    more = (a.shape[0], a.shape[1] + 1, a.shape[2] + 1, a.shape[3] + 16)  # rows further apart than they are long
    wide = torch.full(more, 0x55, dtype=torch.uint8, device="cuda")
    wide[:, :-1, :-1, :-16] = t
    return wide[:, :-1, :-1, :-16]


def gpu_cache(c, layout="head"):
    return bdc.KvCache(laid_out(c.k, layout), laid_out(c.v, layout), torch.from_numpy(c.k_scale).cuda(),
                       torch.from_numpy(c.v_scale).cuda())


def slots_of(c, new, page):
    """(slots of `new[s]` tokens behind each request's length minus them, request of each)."""
    slots = []
    for s, n in enumerate(new):
        for p in range(int(c.kv_lens[s]) - int(n), int(c.kv_lens[s])):
            slots.append(int(c.table[s, p // page]) * page + p % page)
    return np.array(slots, dtype=np.int64)


def new_rows(n, n_kv, dim, dtype, seed, mag=1.0):
    rng = np.random.default_rng(seed + 77)
    x = rng.normal(0, 1, (2, n, n_kv, dim)) * mag * 2.0 ** rng.integers(-3, 4, (2, 1, n_kv, 1))
    t = torch.from_numpy(x).to(DTYPES[dtype])
    return t[0], t[1]


def assert_write(c, k, v, slots, layout="head", rows=lambda t: t.cuda()):
    cache = gpu_cache(c, layout)
    bdc.kv_write(rows(k), rows(v), torch.from_numpy(slots).cuda(), cache)
    torch.cuda.synchronize()
    ref = CO.write(k.double().numpy(), v.double().numpy(), slots, c.k, c.v, c.k_scale, c.v_scale)
    for name, got, want in zip(("k_scale", "v_scale"), cache[2:], ref[2:]):
        assert np.array_equal(got.cpu().numpy(), want), name
    for name, got, want in zip(("k", "v"), cache[:2], ref[:2]):
        got = CO.E4M3[got.cpu().numpy()]
        assert np.array_equal(got, CO.E4M3[want], equal_nan=True), name
    return cache


LENS = {"fresh": ([1, 16, 17, 40, 64, 300], [1, 16, 17, 40, 64, 300]),
        "append": ([20, 33, 64, 65, 130, 301], [1, 1, 1, 1, 1, 1]),
        "ragged": ([100, 7, 64, 129, 400, 257], [60, 7, 0, 64, 131, 1])}


@pytest.mark.parametrize("lens", sorted(LENS))
@pytest.mark.parametrize("page,n_kv,dim", [(16, 2, 128), (32, 5, 80), (64, 1, 64), (128, 8, 16), (256, 3, 112)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_writes_match_the_oracle(lens, page, n_kv, dim, dtype):
    total, new = LENS[lens]
    for seed, exp in enumerate([(-9, -5), (-30, 9)]):  # scales that the new tokens outgrow, and that they do not
        c = random_cache(total, page, n_kv, dim, seed=seed, k_exp=exp, v_exp=exp)
        k, v = new_rows(sum(new), n_kv, dim, dtype, seed, [1.0, 30.0][seed])
        assert_write(c, k, v, slots_of(c, new, page))


@pytest.mark.parametrize("layout", ["head", "token", "wide"])
def test_writes_take_any_strides(layout):
    c = random_cache([50, 90], 32, 3, 48, seed=3)
    k, v = new_rows(70, 3, 48, "bf16", 3)

    def rows(t):  # the middle of a wider projection
        w = torch.full((t.shape[0], 9, t.shape[2]), 7.0, dtype=t.dtype, device="cuda")
        w[:, 3:6] = t.cuda()
        return w[:, 3:6]

    cache = assert_write(c, k, v, slots_of(c, [30, 40], 32), layout, rows)
    if layout == "wide":  # the gaps are untouched
        base = cache.k._base if cache.k._base is not None else cache.k
        assert bool((base[:, -1] == 0x55).all()) and bool((base[:, :, -1] == 0x55).all())


def test_writes_skip_slots_outside_the_cache():
    c = random_cache([40], 16, 2, 32, seed=4)
    slots = slots_of(c, [20], 16)
    slots[3], slots[9], slots[15] = -1, c.k.shape[0] * 16, 2 ** 40
    k, v = new_rows(20, 2, 32, "bf16", 4)
    assert_write(c, k, v, slots)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_writes_mark_tokens_that_are_not_finite(bad):
    c = random_cache([30, 50], 16, 2, 48, seed=5)
    k, v = new_rows(45, 2, 48, "bf16", 5)
    k[3, 0, 47], v[7, 1, 0], k[8, :, 5], v[44, 0, 13] = bad, bad, bad, bad
    k[20:36], v[21] = bad, bad  # a whole page of them
    assert_write(c, k, v, slots_of(c, [10, 35], 16))


def test_writes_of_zeros_and_of_the_smallest_and_largest():
    c = random_cache([64], 16, 1, 16, seed=6)
    k, v = new_rows(64, 1, 16, "bf16", 6)
    k[:16], v[16:32] = 0, 0
    k[32:48] *= 2.0 ** -120
    v[48:] = torch.sign(v[48:]) * torch.finfo(torch.bfloat16).max
    assert_write(c, k, v, slots_of(c, [64], 16))


def test_writes_round_ties_to_even():
    c = random_cache([16], 16, 1, 128, seed=7)
    fin = np.sort(CO.E4M3[np.isfinite(CO.E4M3)])
    mids = np.unique((fin[1:] + fin[:-1]) / 2)  # 253 of them, each a bf16
    x = torch.from_numpy(np.resize(mids, (16, 1, 128))).to(torch.bfloat16)
    assert np.array_equal(np.unique(x.double().numpy()), mids)
    x[:, 0, 0] = 448.0  # the scale is 1
    assert_write(c, x, x.flip(2).contiguous(), slots_of(c, [16], 16))


def test_a_page_written_token_by_token_equals_its_scales_history():
    c = random_cache([0], 16, 2, 32, seed=8)
    c.table[0, 0] = 1
    k, v = new_rows(16, 2, 32, "bf16", 8)
    k *= (2.0 ** torch.arange(16) / 64)[:, None, None]  # the scale grows again and again
    cache = gpu_cache(c)
    kc, vc, ks, vs = c.k, c.v, c.k_scale, c.v_scale
    for i in range(16):
        slot = np.array([16 + i], dtype=np.int64)
        bdc.kv_write(k[i:i + 1].cuda(), v[i:i + 1].cuda(), torch.from_numpy(slot).cuda(), cache)
        kc, vc, ks, vs = CO.write(k[i:i + 1].double().numpy(), v[i:i + 1].double().numpy(), slot, kc, vc, ks, vs)
    assert np.array_equal(CO.E4M3[cache.k.cpu().numpy()], CO.E4M3[kc], equal_nan=True)
    assert np.array_equal(cache.k_scale.cpu().numpy(), ks) and np.array_equal(cache.v_scale.cpu().numpy(), vs)


# --------------------------------------------------------------- attention --
def attention_bounds(out, lse, spread, work, dtype, v_max):
    """How far a result may be off. The output is rounded once: 2^-8 of it in bf16 (8 significant bits, half a unit in
    the last), 2^-11 in f16. Weights are rounded to f16: 2^-11 of each, or 2^-37 of the largest one for weights that
    small (and 2^15 such tokens at most). A score is a sum of up to 128 exact products kept in fp32 by a tree whose nodes may
    drop 2^-22 of the largest partial sum each: 2^-15 of the sum of their magnitudes, which moves a weight, and the
    log-sum-exp, by as much (twice, for numerator and normaliser); exp2 and the sums of weights add 2^-19."""
    u = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    eps = 2.0 ** -11 + 2 * work[..., None] * 2.0 ** -15 + 2.0 ** -19
    tiny = 2.0 ** -24 if dtype == "f16" else 0.0  # f16 subnormals
    return (u * np.abs(out) + (1 + u) * (eps * spread + 2.0 ** -22 * v_max) + tiny,
            work * 2.0 ** -15 + 2.0 ** -19 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0))))


def assert_attention(c, q_lens, n_q, dtype="bf16", mask_block=1, layout="head", scale=None, seed=0, q_mag=1.0,
                     rows=None, max_q=None, max_kv=None, **kw):
    n_kv, dim, page = c.k.shape[2], c.k.shape[3], c.k.shape[1]
    rng = np.random.default_rng(seed + 9)
    starts = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    q = torch.from_numpy(rng.normal(0, q_mag, (int(starts[-1]), n_q, dim))).to(DTYPES[dtype])
    scale = dim ** -0.5 if scale is None else scale
    ref, ref_lse, spread, work = CO.attention(q.double().numpy(), c.k, c.v, c.k_scale, c.v_scale, c.table, c.kv_lens,
                                              starts, scale, mask_block)
    q_d = q.cuda() if rows is None else rows(q)
    out, lse = bdc.kv_attention(q_d, gpu_cache(c, layout), torch.from_numpy(c.table).cuda(),
                                torch.from_numpy(c.kv_lens).cuda(), torch.from_numpy(starts).cuda(),
                                max_q_len=int(max(q_lens)) if max_q is None else max_q,
                                max_kv_len=max(0, int(c.kv_lens.max())) if max_kv is None else max_kv, scale=scale,
                                mask_block=mask_block, return_lse=True, **kw)
    torch.cuda.synchronize()
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isnan(got_lse), np.isnan(ref_lse))
    fine = ~np.isnan(ref)
    codes, top = np.abs(CO.E4M3[c.v]), int(c.v_scale[c.v_scale != 255].max(initial=0))
    v_max = float(codes[np.isfinite(codes)].max(initial=0)) * 2.0 ** (top - 127)
    b, b_lse = attention_bounds(ref, ref_lse, spread, work, dtype, v_max)
    assert np.all((np.abs(got - ref) <= b)[fine])
    seen = np.isfinite(ref_lse)
    assert np.array_equal(got_lse == -np.inf, ref_lse == -np.inf)
    assert not got[ref_lse == -np.inf].any()
    assert np.all(np.abs(got_lse - ref_lse)[seen] <= b_lse[seen])
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,n_kv,g,dim", [(16, 2, 4, 128), (32, 1, 1, 64), (64, 3, 8, 80), (128, 1, 16, 16),
                                             (256, 2, 7, 112), (16, 1, 33, 96)])
def test_single_tokens(page, n_kv, g, dim, dtype):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 128, 129, 300, 511, 1025]
    assert_attention(random_cache(lens, page, n_kv, dim, seed=g), [1] * len(lens), n_kv * g, dtype, mask_block=0)


@pytest.mark.parametrize("mask_block", [0, 1, 2, 5, 32])
@pytest.mark.parametrize("n_kv,g,dim", [(2, 2, 128), (1, 5, 64), (1, 12, 48)])
def test_drafts_and_small_windows(mask_block, n_kv, g, dim):
    q_lens = [1, 5, 9, 0, 3, 20, 2]
    c = random_cache([1, 9, 9, 40, 67, 150, 300], 32, n_kv, dim, seed=2)
    assert_attention(c, q_lens, n_kv * g, "bf16", mask_block)


@pytest.mark.parametrize("mask_block", [0, 1, 20, 32, 64])
@pytest.mark.parametrize("page,n_kv,g,dim", [(16, 1, 1, 128), (64, 2, 4, 128), (32, 1, 3, 64), (128, 1, 4, 80)])
def test_windows(mask_block, page, n_kv, g, dim):
    q_lens = [64, 130, 1, 33, 257]
    lens = [64, 300, 200, 500, 260]
    assert_attention(random_cache(lens, page, n_kv, dim, seed=3), q_lens, n_kv * g, "bf16", mask_block)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("q_len", [1, 4, 40, 200])
def test_requests_that_see_nothing(q_len, dtype):
    c = random_cache([0, 7, -3, 30, 0], 16, 2, 64, seed=4)  # lengths below q_len: a failed kv_tables request
    assert_attention(c, [q_len] * 5, 4, dtype, mask_block=1)
    assert_attention(c, [q_len] * 5, 4, dtype, mask_block=0)
    assert_attention(random_cache([0, 0], 16, 2, 64, seed=4), [q_len] * 2, 4, dtype, mask_block=8)


@pytest.mark.parametrize("q_len", [1, 3, 70])
@pytest.mark.parametrize("layout", ["head", "token", "wide"])
def test_any_strides(layout, q_len):
    def rows(t):
        w = torch.full((t.shape[0], t.shape[1] + 5, t.shape[2] + 8), float("nan"), dtype=t.dtype, device="cuda")
        w[:, 2:-3, :-8] = t.cuda()
        return w[:, 2:-3, :-8]

    c = random_cache([100, 333, 250], 64, 2, 96, seed=5)
    assert_attention(c, [q_len] * 3, 6, "bf16", 1, layout, rows=rows)


@pytest.mark.parametrize("q_len", [1, 100])
def test_pages_of_very_different_scales(q_len):
    c = random_cache([400, 170], 16, 2, 64, seed=6, k_exp=(-16, -6), v_exp=(-60, 40))
    assert_attention(c, [q_len] * 2, 4, "bf16", 1)
    c = random_cache([400, 170], 16, 2, 64, seed=6, v_exp=(-60, 40))
    for p in c.table[0, 2:5]:  # pages of zero values under the smallest scale
        c.v[p], c.v_scale[p] = 0, CO.E_MIN
    assert_attention(c, [q_len] * 2, 4, "bf16", 1)
    c.v[:], c.v_scale[:] = 0, CO.E_MIN
    assert not assert_attention(c, [q_len] * 2, 4, "bf16", 1).any()


@pytest.mark.parametrize("q_len", [1, 150])
@pytest.mark.parametrize("q_mag", [0.0, 1e-30, 1e4])
def test_flat_and_peaked_scores(q_len, q_mag):
    c = random_cache([300, 170], 32, 2, 128, seed=7, k_exp=(-9, -9))
    if q_mag == 1e4:  # scores of +-1e4: one token takes all the weight; their rounding is bounded by `work`
        c.k[:, :, :, 1:] &= 0x80
    assert_attention(c, [q_len] * 2, 4, "bf16", 1, q_mag=q_mag)


@pytest.mark.parametrize("q_len,mask_block", [(1, 1), (6, 1), (130, 1), (130, 64)])
def test_tokens_that_are_not_finite_reach_only_the_queries_that_see_them(q_len, mask_block):
    c = random_cache([200, 300], 16, 2, 64, seed=8)
    for s, t in ((0, 199), (1, 250), (1, 299)):  # as kv_write stores them: a NaN key, a zero value
        p = c.table[s, t // 16]
        c.k[p, t % 16, 1], c.v[p, t % 16, 1] = 0x7F, 0
    out = assert_attention(c, [q_len] * 2, 4, "bf16", mask_block)
    assert bool(out.isnan().any()) and not bool(out.isnan().all())


@pytest.mark.parametrize("q_len", [1, 66])
def test_bounds_above_the_lengths_change_nothing(q_len):
    c = random_cache([100, 257, 70], 16, 2, 64, seed=9, extra_cols=30)
    a = assert_attention(c, [q_len] * 3, 4)
    b = assert_attention(c, [q_len] * 3, 4, max_q=q_len + 40, max_kv=257 + 400)
    assert torch.allclose(a.float(), b.float(), atol=2 ** -6)


@pytest.mark.parametrize("q_len,g,total", [(1, 4, 700), (20, 4, 300), (20, 4, 900), (31, 1, 513), (70, 4, 1300)])
def test_repeated_calls_give_the_same_bits(q_len, g, total):
    """Also the first one, whose warps run apart (code and data come from memory), in filled and in used scratch."""
    n_seq, n_kv, dim = 30, 2, 128
    c = random_cache([total] * n_seq, 16, n_kv, dim, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(q_len)
    args = (torch.randn(n_seq * q_len, n_kv * g, dim, generator=gen, device="cuda").to(torch.bfloat16), gpu_cache(c),
            torch.from_numpy(c.table).cuda(), torch.from_numpy(c.kv_lens).cuda(),
            torch.arange(0, (n_seq + 1) * q_len, q_len, dtype=torch.int32, device="cuda"))
    bounds = dict(max_q_len=q_len, max_kv_len=total)
    need = bdc.kv_attention_workspace(*args, **bounds)
    raw = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN
    ws = raw[-raw.data_ptr() % 256:][:need] if need else None
    torch.cuda.synchronize()
    first = bdc.kv_attention(*args, **bounds, workspace=ws)
    for i in range(100):
        assert torch.equal(bdc.kv_attention(*args, **bounds, workspace=ws if i % 2 else None), first), i


# More than 128 rows to a key/value head: two tiles to a CTA, unless all CTAs of one tile run at once and no length may
# pass 4096.
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("mask_block", [0, 1, 32])
@pytest.mark.parametrize("page,n_kv,g,dim", [(16, 1, 3, 128), (64, 2, 4, 64), (32, 1, 5, 80), (128, 1, 2, 16)])
def test_windows_under_a_long_bound(page, n_kv, g, dim, mask_block, dtype):
    c = random_cache([77, 900, 129, 0, 70], page, n_kv, dim, seed=12, extra_cols=5000 // page)
    assert_attention(c, [77, 110, 65, 0, 70], n_kv * g, dtype, mask_block, max_q=130, max_kv=5000)
    c = random_cache([400, 170], page, n_kv, dim, seed=13, k_exp=(-16, -6), v_exp=(-60, 40), extra_cols=5000 // page)
    assert_attention(c, [130, 66], n_kv * g, "bf16", mask_block, max_kv=4097)  # results up to 2^48: none in f16


@pytest.mark.parametrize("page,n_kv,g,dim,n_seq", [(16, 2, 2, 64, 80), (64, 1, 3, 96, 160)])
@pytest.mark.parametrize("mask_block", [0, 1, 20])
def test_many_windows(page, n_kv, g, dim, n_seq, mask_block):
    rng = np.random.default_rng(n_seq + mask_block)
    lens = rng.integers(-2, 330, n_seq)
    q_lens = np.minimum(rng.integers(0, 100, n_seq), np.maximum(lens, 0))
    assert_attention(random_cache(lens, page, n_kv, dim, seed=14), q_lens.tolist(), n_kv * g, "bf16", mask_block)


@pytest.mark.parametrize("q_len", [1, 4, 12])
@pytest.mark.parametrize("n_seq", [103, 256, 257])
def test_many_requests_of_any_lengths(n_seq, q_len):
    rng = np.random.default_rng(n_seq + q_len)
    lens = rng.integers(0, 180, n_seq)
    lens[rng.random(n_seq) < 0.3] = 64  # ranked by length, these are equals
    lens[rng.random(n_seq) < 0.05] = 700
    q_lens = np.minimum(rng.integers(0, q_len + 1, n_seq), lens)
    assert_attention(random_cache(lens, 16, 3, 64, seed=8), q_lens.tolist(), 12, "bf16", 1)


def test_page_numbers_out_of_range_are_not_read():
    c = random_cache([64, 64], 16, 1, 32, seed=10)
    c.table[1, 1], c.table[1, 2] = -1, 2 ** 31 - 1
    for q_len in (1, 64):
        starts = torch.tensor([0, q_len, 2 * q_len], dtype=torch.int32, device="cuda")
        q = torch.randn(2 * q_len, 2, 32, device="cuda", dtype=torch.bfloat16)
        out = bdc.kv_attention(q, gpu_cache(c), torch.from_numpy(c.table).cuda(), torch.from_numpy(c.kv_lens).cuda(),
                               starts, max_q_len=q_len, max_kv_len=64)
        torch.cuda.synchronize()
        assert bool(out.isfinite().all())
        ref = CO.attention(q.double().cpu().numpy(), c.k, c.v, c.k_scale, c.v_scale, c.table[:1], c.kv_lens[:1],
                           [0, q_len], 32 ** -0.5, 1)[0]
        assert np.allclose(out[:q_len].double().cpu().numpy(), ref[:q_len], atol=0.02)


def test_long_caches_with_offsets_past_32_bits():
    """A cache whose codes lie more than 2^32 bytes apart: the same few pages near its end as near its start."""
    page, n_kv, dim, far = 64, 2, 128, 300000
    n_pages = far + 8
    k = torch.zeros(n_pages, n_kv, page, dim, dtype=torch.uint8, device="cuda").transpose(1, 2)
    assert k.numel() > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(0)
    k[:8] = torch.randint(0, 100, (8, page, n_kv, dim), generator=g, device="cuda").to(torch.uint8)
    k[far:] = k[:8]
    s = torch.full((n_pages, n_kv), 118, dtype=torch.uint8, device="cuda")
    cache = bdc.KvCache(k, k, s, s)
    near = torch.tensor([[3, 1, 7, 0, 2, 5, 6, 4]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([500], dtype=torch.int32, device="cuda")
    for q_len in (1, 200):
        q = torch.randn(q_len, 8, dim, generator=g, device="cuda").to(torch.bfloat16)
        starts = torch.tensor([0, q_len], dtype=torch.int32, device="cuda")
        a, b = (bdc.kv_attention(q, cache, t, lens, starts, max_q_len=q_len, max_kv_len=500)
                for t in (near, near + far))
        assert torch.equal(a, b)
    x = torch.randn(3, n_kv, dim, generator=g, device="cuda").to(torch.bfloat16)
    bdc.kv_write(x, x, torch.arange((far + 7) * page, (far + 7) * page + 3, device="cuda"), cache)
    bdc.kv_write(x, x, torch.arange(7 * page, 7 * page + 3, device="cuda"), cache)
    assert torch.equal(k[far + 7, :3], k[7, :3]) and torch.equal(s[far + 7], s[7])


# ------------------------------------------------- streams, graphs, workspaces --
def attention_case(q_len, n_seq=6, total=900):
    c = random_cache([total] * n_seq, 64, 2, 128, seed=11)
    gen = torch.Generator(device="cuda").manual_seed(q_len)
    q = torch.randn(n_seq * q_len, 8, 128, generator=gen, device="cuda").to(torch.bfloat16)
    args = (q, gpu_cache(c), torch.from_numpy(c.table).cuda(), torch.from_numpy(c.kv_lens).cuda(),
            torch.arange(0, (n_seq + 1) * q_len, q_len, dtype=torch.int32, device="cuda"))
    return args, dict(max_q_len=q_len, max_kv_len=total)


@pytest.mark.parametrize("q_len", [1, 20, 64])
def test_streams_share_the_librarys_workspace(q_len):
    args, bounds = attention_case(q_len)
    assert bdc.kv_attention_workspace(*args, **bounds) > 0
    ref = bdc.kv_attention(*args, **bounds)
    outs = [torch.empty_like(ref) for _ in range(24)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):  # calls in flight at once, each in the one workspace
        bdc.kv_attention(*args, **bounds, out=out, stream=streams[i % 3])
    torch.cuda.synchronize()
    assert all(torch.equal(out, ref) for out in outs)


@pytest.mark.parametrize("q_len", [1, 64])
def test_a_forward_replays_from_a_graph(q_len):
    args, bounds = attention_case(q_len)
    q, cache, table, lens, starts = args
    need = bdc.kv_attention_workspace(*args, **bounds)
    raw = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    ws = raw[-raw.data_ptr() % 256:][:need]
    before = lens - q_len
    new = torch.full_like(lens, q_len)
    # free: the pages that the requests do not hold without the new tokens (their tables' last ones are taken again)
    held = -(-(900 - q_len) // 64)
    ring = torch.full((cache.k.shape[0],), -1, dtype=torch.int32, device="cuda")
    spare = table[:, held:15].reshape(-1)
    ring[:spare.numel()] = spare
    pool = torch.tensor([0, spare.numel()], dtype=torch.int64, device="cuda")
    k = torch.randn(6 * q_len, 2, 128, device="cuda").to(torch.bfloat16)

    def forward():
        t = bdc.kv_tables(before, new, table, ring, pool, page_size=64, max_tokens=6 * q_len)
        bdc.kv_write(k, k, t.slot_map, cache)
        return bdc.kv_attention(q, cache, table, t.kv_lens, t.query_start, workspace=ws, **bounds)

    ref = forward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = forward()
    k.mul_(2)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(out, ref)  # the new keys and values
    assert torch.equal(out, forward())


def test_a_capture_without_a_workspace_is_refused():
    args, bounds = attention_case(1)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(bdc.BdError) as e, torch.cuda.graph(graph):
        bdc.kv_attention(*args, **bounds)
    assert e.value.status == bdc.bdcommit.BD_ERR_WORKSPACE


def test_a_small_workspace_is_refused_and_shutdown_frees():
    args, bounds = attention_case(1)
    need = bdc.kv_attention_workspace(*args, **bounds)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    ws = ws[-ws.data_ptr() % 256:]
    with pytest.raises(bdc.BdError) as e:
        bdc.kv_attention(*args, **bounds, workspace=ws[:need - 1])
    assert e.value.status == bdc.bdcommit.BD_ERR_WORKSPACE
    ref = bdc.kv_attention(*args, **bounds, workspace=ws[:need])
    torch.cuda.synchronize()
    assert bdc.kvcache.kv_shutdown() == 0
    assert torch.equal(bdc.kv_attention(*args, **bounds), ref)


def test_negative_and_zero_scales():
    c = random_cache([200, 77], 32, 2, 64, seed=12)
    for q_len in (1, 60):
        for scale in (-0.125, 0.0):
            assert_attention(c, [q_len] * 2, 4, scale=scale)
