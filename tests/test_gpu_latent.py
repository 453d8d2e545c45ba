"""The paged latent cache on the GPU (kv_latent_write, kv_latent_attention) against the float64 oracle.

Writes are compared exactly where nothing is turned. Attention is compared within bounds that follow from the number
formats (see bounds); what no call may read is NaN (a page's tail, unused pages) or a page number far out of range.
"""

import math

import numpy as np
import pytest
import torch

from oracle import rotary_oracle as RO

pytestmark = pytest.mark.gpu

bdc = pytest.importorskip("paper_2609_33887_gb300")

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step, relative
BAD_PAGE = 0x7FFFFFF0


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)
    yield
    assert bdc.rotary.kv_latent_device_status() == 0


class Cache:
    """Requests of the given lengths in pages of any order; everything else is NaN or far out of range."""

    def __init__(self, lens, page, dim, rope, dtype, seed=0, extra_cols=2, mag=1.0):
        rng = np.random.default_rng(seed)
        lens = np.asarray(lens, dtype=np.int64)
        held = -(-np.maximum(lens, 0) // page)
        n_pages = int(held.sum()) + 3
        order = rng.permutation(n_pages)
        self.table = np.full((len(lens), int(held.max(initial=0)) + extra_cols), BAD_PAGE, dtype=np.int32)
        rows = torch.full((n_pages, page, dim + rope), math.nan, dtype=DTYPES[dtype])
        at = 0
        for s, h in enumerate(held):
            self.table[s, :h] = order[at:at + h]
            at += int(h)
            for j in range(int(h)):
                n = min(page, int(lens[s]) - j * page)
                rows[self.table[s, j], :n] = torch.from_numpy(rng.normal(0, mag, (n, dim + rope))).to(DTYPES[dtype])
        self.lens, self.page, self.dim, self.rope, self.dtype, self.rows = lens.astype(np.int32), page, dim, rope, dtype, rows

    def numpy(self):
        r = self.rows.double().numpy()
        return r[..., :self.dim], r[..., self.dim:]

    def gpu(self, layout="rows"):
        """rows: parts of the same rows. apart: tensors of their own. wide: rows and pages with gaps. tokens: pages next to
        each other, the tokens of a page far apart."""
        r = self.rows.cuda()
        if layout == "rows":
            return bdc.KvLatent(*r.split([self.dim, self.rope], 2))
        latent, rope = r[..., :self.dim].contiguous(), r[..., self.dim:].contiguous()
        if layout == "apart":
            return bdc.KvLatent(latent, rope)
        if layout == "wide":
            def wide(t):
                w = torch.full((t.shape[0], t.shape[1] + 3, t.shape[2] + 24), math.nan, dtype=t.dtype, device="cuda")
                w[:, 1:-2, 8:-16] = t
                return w[:, 1:-2, 8:-16]
            return bdc.KvLatent(wide(latent), wide(rope))
        return bdc.KvLatent(*(t.transpose(0, 1).contiguous().transpose(0, 1) for t in (latent, rope)))


def ints(v):
    return torch.from_numpy(np.asarray(v, dtype=np.int32)).cuda()


def bounds(out, lse, spread, work, dtype, width, n, v_max):
    """How far a result may be off. The output is rounded once and the weights once, each by U; f16 weights as small as
    2^-14 / 2^8 of the largest by 2^-33 of that, for each of n tokens. A score is a sum of `width` exact products kept in
    fp32, each addition of which may drop 2^-22 of the magnitudes: width 2^-22 of the sum of them, which moves a weight, and
    the log-sum-exp, by as much (twice, for numerator and normaliser); exp2 and the sums of weights add 2^-19."""
    score = work * width * 2.0 ** -22
    eps = U[dtype] + 2 * score[..., None] + 2.0 ** -19
    tiny = 2.0 ** -24 if dtype == "f16" else 0.0
    small = n * 2.0 ** -33 * v_max if dtype == "f16" else 0.0
    return (U[dtype] * np.abs(out) + (1 + U[dtype]) * (eps * spread + small) + tiny,
            score + 2.0 ** -19 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0))))


def attend(c, q, q_lens, heads, *, mask_block=1, layout="rows", scale=0.05, max_q=None, max_kv=None, **kw):
    starts = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    return bdc.kv_latent_attention(q, c.gpu(layout), ints(c.table), ints(c.lens), ints(starts), scale=scale,
                                   max_q_len=int(max(q_lens)) if max_q is None else max_q,
                                   max_kv_len=max(0, int(c.lens.max())) if max_kv is None else max_kv,
                                   mask_block=mask_block, return_lse=True, **kw)


def check(c, q_lens, heads, *, mask_block=1, scale=0.05, seed=0, q_mag=1.0, rows=None, edit=None, **kw):
    rng = np.random.default_rng(seed + 9)
    starts = np.concatenate([[0], np.cumsum(q_lens)])
    q = torch.from_numpy(rng.normal(0, q_mag, (int(starts[-1]), heads, c.dim + c.rope))).to(DTYPES[c.dtype])
    if edit is not None:
        edit(q)
    latent, rope = c.numpy()
    ref, ref_lse, spread, work = RO.latent_attention(q.double().numpy(), latent, rope, c.table, c.lens, starts, scale, mask_block)
    out, lse = attend(c, q.cuda() if rows is None else rows(q), q_lens, heads, mask_block=mask_block, scale=scale, **kw)
    torch.cuda.synchronize()
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isnan(got_lse), np.isnan(ref_lse))
    fine = ~np.isnan(ref)
    v_max = float(np.abs(latent[np.isfinite(latent)]).max(initial=0))
    b, b_lse = bounds(ref, ref_lse, spread, work, c.dtype, c.dim + c.rope, int(max(c.lens.max(), 1)), v_max)
    assert np.all((np.abs(got - ref) <= b)[fine]), float(np.max((np.abs(got - ref) / b)[fine]))
    seen = np.isfinite(ref_lse)
    assert np.array_equal(got_lse == -np.inf, ref_lse == -np.inf)
    assert np.all(np.abs(got_lse - ref_lse)[seen] <= b_lse[seen])
    return out, lse


# --------------------------------------------------------------- attention --
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page,heads,dim,rope", [(32, 16, 512, 64), (16, 1, 16, 16), (64, 64, 128, 32), (128, 20, 256, 48),
                                                 (256, 128, 512, 64), (16, 7, 144, 64), (64, 33, 448, 16), (32, 65, 64, 64),
                                                 (64, 3, 64, 48), (128, 12, 192, 32)])
def test_single_tokens(page, heads, dim, rope, dtype):
    lens = [1, 2, 15, 16, 17, 63, 64, 127, 128, 129, 255, 256, 300, 1025]
    check(Cache(lens, page, dim, rope, dtype, seed=heads), [1] * len(lens), heads, mask_block=0)


@pytest.mark.parametrize("mask_block", [0, 1, 2, 5, 32])
@pytest.mark.parametrize("heads,dim,rope", [(16, 512, 64), (5, 96, 16), (128, 256, 64)])
def test_drafts_and_windows(mask_block, heads, dim, rope):
    q_lens = [1, 5, 9, 0, 3, 20, 2, 70]
    check(Cache([1, 9, 9, 40, 67, 150, 300, 200], 32, dim, rope, "bf16", seed=2), q_lens, heads, mask_block=mask_block)


@pytest.mark.parametrize("mask_block", [0, 1, 20, 64])
@pytest.mark.parametrize("page,heads,dim,rope", [(16, 3, 512, 64), (128, 8, 128, 48), (256, 1, 384, 64)])
def test_prompts(mask_block, page, heads, dim, rope):
    check(Cache([64, 300, 200, 500, 260], page, dim, rope, "f16", seed=3), [64, 130, 1, 33, 257], heads, mask_block=mask_block)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("q_len", [1, 4, 90])
def test_requests_that_see_nothing(q_len, dtype):
    c = Cache([0, 7, -3, 30, 0], 16, 64, 16, dtype, seed=4)  # lengths below q_len: a failed kv_tables request
    for mask_block in (0, 1, 8):
        out, lse = check(c, [q_len] * 5, 4, mask_block=mask_block)
        assert not out[:q_len].any() and bool((lse[:q_len] == -math.inf).all())
    check(Cache([0, 0], 16, 512, 64, dtype, seed=4), [q_len] * 2, 4, mask_block=8)


@pytest.mark.parametrize("q_len", [1, 3, 40])
@pytest.mark.parametrize("layout", ["rows", "apart", "wide", "tokens"])
def test_any_strides(layout, q_len):
    def rows(t):
        w = torch.full((t.shape[0], t.shape[1] + 5, t.shape[2] + 8), math.nan, dtype=t.dtype, device="cuda")
        w[:, 2:-3, :-8] = t.cuda()
        return w[:, 2:-3, :-8]

    c = Cache([100, 333, 250], 64, 320, 32, "bf16", seed=5)
    out = torch.zeros(3 * q_len, 9, 320 + 16, dtype=torch.bfloat16, device="cuda")
    got, _ = check(c, [q_len] * 3, 6, layout=layout, rows=rows, out=out[:, 1:7, :320])
    assert got.data_ptr() == out[:, 1:].data_ptr() and not out[:, 0].any() and not out[:, 7:].any() and not out[..., 320:].any()


@pytest.mark.parametrize("q_len,total,heads", [(1, 20000, 16), (1, 5000, 128), (7, 9000, 4), (130, 3000, 2)])
def test_caches_in_parts(q_len, total, heads):
    c = Cache([total, total // 3, 130], 64, 128, 64, "bf16", seed=6)
    check(c, [q_len] * 3, heads)
    check(Cache([total], 64, 512, 64, "f16", seed=7), [q_len], heads, mask_block=0)


@pytest.mark.parametrize("mask_block", [0, 1, 32])
@pytest.mark.parametrize("n_seq,q_len,heads", [(1, 90, 64), (2, 150, 16), (7, 33, 40), (19, 64, 8), (150, 1, 3), (153, 1, 3),
                                               (31, 5, 64)])
def test_units_in_shares(n_seq, q_len, heads, mask_block):
    """Up to one unit of rows to an SM, whose tiles are shared out: whole units, parts that begin and end in a CTA, units over
    many CTAs, requests without rows or without tokens between them."""
    rng = np.random.default_rng(n_seq + q_len)
    lens, q_lens = rng.integers(0, 1500 if n_seq < 20 else 300, n_seq), rng.integers(0, q_len + 1, n_seq)
    lens[n_seq // 2], q_lens[n_seq // 3] = 1400, q_len
    check(Cache(lens, 32, 64, 16, "bf16", seed=23), q_lens.tolist(), heads, mask_block=mask_block, max_q=q_len)


@pytest.mark.parametrize("n_seq,q_len,heads,lo,hi", [(1, 140, 64, 3000, 3000), (1, 100, 64, 4000, 4000), (15, 5, 128, 2000, 2000),
                                                     (15, 5, 128, 100, 4000), (140, 1, 16, 1000, 1500), (60, 1, 16, 1000, 1500),
                                                     (3, 40, 16, 500, 5000)])
def test_whole_units_where_lengths_are_alike_and_parts_where_not(n_seq, q_len, heads, lo, hi):
    rng = np.random.default_rng(hi)
    lens, q_lens = rng.integers(lo, hi + 1, n_seq), np.full(n_seq, q_len)
    if n_seq > 1:
        lens[n_seq // 3], q_lens[n_seq // 2] = 0, 0
    check(Cache(lens, 64, 64, 16, "bf16", seed=25), q_lens.tolist(), heads, max_q=q_len)


def test_replayed_with_other_lengths():
    c = Cache([900, 40, 1300, 0], 32, 128, 16, "bf16", seed=24)
    q = torch.randn(4, 8, 144, device="cuda").to(torch.bfloat16)
    cache, table, lens, starts = c.gpu(), ints(c.table), ints(c.lens), ints([0, 1, 2, 3, 4])
    limits = dict(max_q_len=1, max_kv_len=1300)
    ws = torch.empty(bdc.kv_latent_attention_workspace(q, cache, table, lens, starts, **limits), dtype=torch.uint8, device="cuda")
    out = torch.empty(4, 8, 128, dtype=torch.bfloat16, device="cuda")
    args = dict(scale=0.1, workspace=ws, out=out, **limits)
    bdc.kv_latent_attention(q, cache, table, lens, starts, **args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bdc.kv_latent_attention(q, cache, table, lens, starts, **args)
    for other in ([900, 40, 1300, 0], [1, 0, 64, 0], [0, 0, 0, 0], [899, 33, 65, 0]):
        lens.copy_(ints(other))
        graph.replay()
        got = out.clone()
        assert torch.equal(got, bdc.kv_latent_attention(q, cache, table, lens, starts, scale=0.1, **limits)), other


@pytest.mark.parametrize("q_len", [1, 100])
@pytest.mark.parametrize("q_mag,scale", [(0.0, 0.05), (1e-6, 0.05), (30.0, 0.05), (300.0, 1.0), (1.0, -0.05), (1.0, 0.0)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_flat_and_peaked_scores(q_len, q_mag, scale, dtype):
    def edit(q):
        if q_mag == 300.0:  # one element a query: its products are exact sums, so scores of any size keep their order
            q[..., 1:] = 0

    check(Cache([300, 170], 32, 256, 64, dtype, seed=8), [q_len] * 2, 5, q_mag=q_mag, scale=scale, edit=edit)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [2.0 ** 21, 2.0 ** 27, 1.5 * 2.0 ** 28, 2.0 ** 60])
def test_scores_far_beyond_the_weights_range(size, dtype):
    """One key element decides: equal scores share the weight, a larger one takes it, at any size of the scores."""
    c = Cache([700], 64, 128, 16, dtype, seed=9)
    c.rows[..., 128:][~c.rows[..., 128:].isnan()] = 0.0
    best = torch.zeros(700)
    best[[3, 130, 131, 600]] = torch.tensor([1.0, 2.0, 2.0, 2.0])
    for t in range(700):
        c.rows[c.table[0, t // 64], t % 64, 128] = best[t]

    def edit(q):
        q[:] = 0
        q[..., 128] = 1.0

    out, lse = check(c, [1], 3, mask_block=0, scale=size, edit=edit)
    latent = torch.stack([c.rows[c.table[0, t // 64], t % 64, :128].double() for t in (130, 131, 600)])
    assert torch.allclose(out[0, 0].double().cpu(), latent.mean(0), rtol=2 * U[dtype], atol=2 * U[dtype])


@pytest.mark.parametrize("n", [1, 70, 9000])
@pytest.mark.parametrize("key", [-1.0, -0.9375, 1.0])
def test_scores_at_the_end_of_the_range(n, key):
    """Scores of up to 1.0625 * 3.2e38 as powers of two, either sign, that fp32 still holds: the largest, which are equal, share
    the weight. Their weights are 1, so a result is off by its rounding and the n - 1 additions of either sum alone."""
    c = Cache([n], 64, 128, 16, "bf16", seed=27)
    at = [c.rows[c.table[0, t // 64], t % 64] for t in range(n)]
    for t, r in enumerate(at):
        r[128:] = 0
        r[128] = -1.0625 if t % 7 == 3 else key
    q = torch.zeros(1, 3, 144, dtype=torch.bfloat16, device="cuda")
    q[..., 128] = 1.0
    scale = 3.2e38 * math.log(2)
    out, lse = attend(c, q, [1], 3, mask_block=0, scale=scale)
    latent = torch.stack([r[:128].double() for t, r in enumerate(at) if t % 7 != 3])
    want, spread = latent.mean(0), latent.abs().mean(0)
    off = (out[0].double().cpu() - want).abs()
    assert bool((off <= U["bf16"] * want.abs() + 2 * n * 2.0 ** -23 * spread).all()), float(off.max())
    assert torch.allclose(lse.double().cpu(), torch.full((1, 3), key * scale, dtype=torch.float64), rtol=2.0 ** -20)


@pytest.mark.parametrize("q_len,mask_block", [(1, 1), (6, 1), (130, 1), (130, 64)])
def test_tokens_that_are_not_finite_reach_only_the_queries_that_see_them(q_len, mask_block):
    c = Cache([200, 300], 16, 128, 32, "bf16", seed=10)
    for s, t in ((0, 199), (1, 250), (1, 299)):  # as kv_latent_write stores them
        r = c.rows[c.table[s, t // 16], t % 16]
        r[:128], r[128:] = 0, math.nan
    out, _ = check(c, [q_len] * 2, 3, mask_block=mask_block)
    assert bool(out.isnan().any()) and (q_len == 1 or not bool(out.isnan().all()))


def test_queries_that_are_not_finite_stay_in_their_row():
    def edit(q):
        q[0, 1, 5], q[2, 0, 130] = math.nan, math.nan
    c = Cache([200, 300], 16, 128, 32, "bf16", seed=11)
    out, _ = check(c, [2, 2], 3, edit=edit)
    assert {tuple(i) for i in out.isnan().any(2).nonzero().tolist()} == {(0, 1), (2, 0)}


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinite_scores(sign):
    """All scores +inf or -inf: NaN, as the formula's; -inf leaves a log-sum-exp of -inf."""
    c = Cache([40], 16, 64, 16, "bf16", seed=12)
    c.rows[..., 64] = torch.where(c.rows[..., 64].isnan(), c.rows[..., 64], torch.ones(()).to(torch.bfloat16))
    q = torch.zeros(1, 2, 80, dtype=torch.bfloat16, device="cuda")
    q[..., 64] = sign * math.inf
    out, lse = attend(c, q, [1], 2, mask_block=0)
    assert bool(out.isnan().all())
    assert bool((lse == -math.inf).all()) if sign < 0 else not bool(lse.isfinite().any())


def test_pages_outside_the_cache_are_zeros():
    c = Cache([300, 100], 32, 128, 16, "bf16", seed=13)
    c.table[0, 2], c.table[0, 9], c.table[1, 0] = -5, BAD_PAGE, c.rows.shape[0]
    check(c, [1, 1], 4, mask_block=0)
    check(c, [60, 60], 4, mask_block=1)
    # lengths beyond the table's columns are cut by the bound; no pages at all
    empty = bdc.kv_latent_cache(0, 32, 128, 16)
    q = torch.ones(1, 4, 144, dtype=torch.bfloat16, device="cuda")
    out = bdc.kv_latent_attention(q, empty, ints([[0, 1]]), ints([50]), ints([0, 1]), scale=1.0, max_q_len=1, max_kv_len=64)
    assert not out.any()


@pytest.mark.parametrize("q_len", [1, 66])
def test_bounds_above_and_below_the_lengths(q_len):
    c = Cache([100, 257, 70], 16, 128, 64, "bf16", seed=14, extra_cols=300)
    a, _ = check(c, [q_len] * 3, 4)
    b, _ = check(c, [q_len] * 3, 4, max_q=q_len + 40, max_kv=257 + 4000)
    assert torch.allclose(a.float(), b.float(), atol=2 ** -6)
    q = torch.randn(3 * q_len, 4, 192, device="cuda").to(torch.bfloat16)
    cut, _ = attend(c, q, [q_len] * 3, 4, mask_block=0, max_kv=64)
    c.lens[:] = 64
    assert torch.equal(cut, attend(c, q, [q_len] * 3, 4, mask_block=0, max_kv=64)[0])


@pytest.mark.parametrize("heads,pad", [(1, 0), (3, 24)])
def test_results_next_to_their_queries(heads, pad):
    c = Cache([300, 70, 129], 64, 64, 32, "bf16", seed=28)
    rows = torch.randn(3, heads * 160 + pad, device="cuda").to(torch.bfloat16)
    q, out = rows[:, :heads * 160].unflatten(1, (heads, 160)).split([96, 64], 2)
    if heads == 1:
        q, out = rows[:, :96].unsqueeze(1), rows[:, 96:].unsqueeze(1)  # a single head's stride is its width
    kept = q.clone()
    want, _ = attend(c, kept, [1] * 3, heads)
    got, _ = attend(c, q, [1] * 3, heads, out=out)
    assert got is out and torch.equal(out, want) and torch.equal(q, kept)


def test_rows_behind_the_last_sequence_stay_as_they_are():
    c = Cache([50, 60], 16, 64, 16, "bf16", seed=15)
    q = torch.randn(10, 3, 80, device="cuda").to(torch.bfloat16)
    out = torch.full((10, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    attend(c, q, [2, 3], 3, out=out)
    assert bool((out[5:] == 7).all()) and not bool((out[:5] == 7).all())


@pytest.mark.parametrize("n_seq", [3, 103, 256, 257])
@pytest.mark.parametrize("q_len", [1, 5])
def test_many_requests_of_any_lengths(n_seq, q_len):
    lens = np.random.default_rng(n_seq).integers(-2, 700, n_seq)
    check(Cache(lens, 32, 64, 16, "bf16", seed=16), [q_len] * n_seq, 6)


@pytest.mark.parametrize("q_len,heads,total", [(1, 16, 700), (5, 64, 900), (40, 8, 1300)])
def test_repeated_calls_give_the_same_bits(q_len, heads, total):
    n_seq = 20
    c = Cache([total] * n_seq, 16, 512, 64, "bf16", seed=17)
    gen = torch.Generator(device="cuda").manual_seed(q_len)
    q = torch.randn(n_seq * q_len, heads, 576, generator=gen, device="cuda").to(torch.bfloat16)
    args = (q, c.gpu(), ints(c.table), ints(c.lens), torch.arange(0, (n_seq + 1) * q_len, q_len, dtype=torch.int32, device="cuda"))
    limits = dict(max_q_len=q_len, max_kv_len=total)
    need = bdc.kv_latent_attention_workspace(*args, **limits)
    raw = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN
    ws = raw[-raw.data_ptr() % 256:][:need] if need else None
    first = bdc.kv_latent_attention(*args, **limits, scale=0.05, workspace=ws)
    for i in range(50):
        assert torch.equal(bdc.kv_latent_attention(*args, **limits, scale=0.05, workspace=ws if i % 2 else None), first), i


@pytest.mark.parametrize("dim,rope", [(64, 16), (128, 64), (256, 64), (512, 64)])
@pytest.mark.parametrize("n_seq,heads,total", [(3, 16, 9000), (40, 64, 1500), (160, 16, 1100)])
def test_rings_of_two_and_of_three_tiles(n_seq, heads, total, dim, rope):
    """Many tiles to a CTA, with sums that are rescaled at every tile: its scores are 16 above those of the tile before."""
    c = Cache(np.random.default_rng(n_seq).integers(total // 2, total + 1, n_seq), 64, dim, rope, "bf16", seed=26)
    for s in range(n_seq):
        for j in range(int(-(-c.lens[s] // 64))):
            c.rows[c.table[s, j], :, dim:] *= 0
            c.rows[c.table[s, j], :, dim] += j

    def edit(q):
        q[..., dim:] = 0
        q[..., dim] = 1.0

    out, lse = check(c, [1] * n_seq, heads, mask_block=0, scale=16.0, edit=edit, q_mag=0.001)
    args = (torch.randn(n_seq, heads, dim + rope, device="cuda").to(torch.bfloat16), c.gpu(), ints(c.table), ints(c.lens),
            torch.arange(n_seq + 1, dtype=torch.int32, device="cuda"))
    limits = dict(scale=0.05, max_q_len=1, max_kv_len=int(c.lens.max()))
    first = bdc.kv_latent_attention(*args, **limits)
    for i in range(30):
        assert torch.equal(bdc.kv_latent_attention(*args, **limits), first), i
    assert bdc.rotary.kv_latent_device_status() == 0


def test_workspaces():
    c = Cache([9000], 64, 128, 16, "bf16", seed=18)
    q = torch.randn(1, 4, 144, device="cuda").to(torch.bfloat16)
    args = (q, c.gpu(), ints(c.table), ints(c.lens), ints([0, 1]))
    limits = dict(max_q_len=1, max_kv_len=9000)
    need = bdc.kv_latent_attention_workspace(*args, **limits)
    assert need > 0
    with pytest.raises(bdc.BdError):
        bdc.kv_latent_attention(*args, **limits, scale=0.1, workspace=torch.empty(need - 256, dtype=torch.uint8, device="cuda"))
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    with pytest.raises(bdc.BdError):  # a capture brings its own
        with torch.cuda.graph(graph, stream=stream):
            bdc.kv_latent_attention(*args, **limits, scale=0.1)


def test_two_streams_and_two_threads_share_the_library_workspace():
    import threading

    caches = [Cache([9000 + 500 * i], 64, 128, 16, "bf16", seed=19 + i, extra_cols=12) for i in range(2)]
    q = torch.randn(1, 40, 144, device="cuda").to(torch.bfloat16)
    args = [(q, c.gpu(), ints(c.table), ints(c.lens), ints([0, 1])) for c in caches]
    ref = [bdc.kv_latent_attention(*a, scale=0.1, max_q_len=1, max_kv_len=9500) for a in args]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(60):
                if not torch.equal(bdc.kv_latent_attention(*args[i], scale=0.1, max_q_len=1, max_kv_len=9500), ref[i]):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_outputs_of_a_call_on_another_stream():
    c = Cache([3000], 64, 128, 16, "bf16", seed=20)
    q = torch.randn(1, 4, 144, device="cuda").to(torch.bfloat16)
    args = (q, c.gpu(), ints(c.table), ints(c.lens), ints([0, 1]))
    limits = dict(scale=0.1, max_q_len=1, max_kv_len=3000)
    ref = bdc.kv_latent_attention(*args, **limits)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got, _ = bdc.kv_latent_attention(*args, **limits, stream=stream, return_lse=True)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, ref)


# ------------------------------------------------------------------ writes --
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["rows", "apart", "wide", "tokens"])
@pytest.mark.parametrize("page,dim,rope,interleaved", [(16, 512, 64, True), (64, 16, 16, False), (256, 144, 48, True),
                                                       (32, 256, 32, None)])
def test_writes(page, dim, rope, interleaved, layout, dtype):
    c = Cache([300, 77, 0, 500], page, dim, rope, dtype, seed=21)
    rng = np.random.default_rng(22)
    slots = rng.permutation(c.rows.shape[0] * page)[:333].astype(np.int64)
    slots[[5, 9, 100]] = -1, 1 << 45, c.rows.shape[0] * page
    positions = rng.integers(0, 100000, 333).astype(np.int32)
    wide = torch.from_numpy(rng.normal(0, 2, (340, dim + 8 + rope))).to(DTYPES[dtype])
    wide[11, 3], wide[12, dim - 1], wide[13, dim + 8], wide[14, 0] = math.nan, math.inf, -math.inf, -math.inf
    wide_d = wide.cuda()
    new_l, new_r = wide_d[:, :dim], wide_d[:, dim + 8:]
    rotary = None if interleaved is None else bdc.kv_rotary(rope, interleaved=interleaved, scale=1.1)
    turned = new_r if rotary is None else bdc.kv_rotate(new_r[:333, None], ints(positions), rotary)[:, 0]
    cache = c.gpu(layout)
    bdc.kv_latent_write(new_l, new_r, torch.from_numpy(slots).cuda(), cache, rotary=rotary,
                        positions=None if rotary is None else ints(positions))
    ref = RO.latent_write(wide[:333, :dim].double().numpy(), turned[:333].double().cpu().numpy(), slots, *c.numpy())
    for got, want in zip(cache, ref):
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


def test_writes_of_nothing_and_of_one():
    cache = bdc.kv_latent_cache(4, 16, 64, 16)
    none = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    bdc.kv_latent_write(none, none[:, :16], torch.empty(0, dtype=torch.int64, device="cuda"), cache)
    assert not cache.latent.any()
    x = torch.randn(1, 80, device="cuda").to(torch.bfloat16)
    bdc.kv_latent_write(x[:, :64], x[:, 64:], torch.tensor([37], device="cuda"), cache)
    assert torch.equal(cache.latent[2, 5], x[0, :64]) and torch.equal(cache.rope[2, 5], x[0, 64:])
    assert int(cache.latent.any(2).sum()) == 1


def test_far_into_a_large_cache():
    """Slots and pages whose offsets pass 32 bits."""
    n_pages, page = 18000, 256
    rows = torch.empty(n_pages, page, 576, dtype=torch.bfloat16, device="cuda")  # 5.3 GB, 2.65e9 elements
    cache = bdc.KvLatent(*rows.split([512, 64], 2))
    pages = [n_pages - 1, 3, n_pages - 2]
    x = torch.randn(700, 576, device="cuda").to(torch.bfloat16)
    t = torch.arange(700, device="cuda")
    slots = torch.tensor(pages, device="cuda")[t // page] * page + t % page
    bdc.kv_latent_write(x[:, :512], x[:, 512:], slots, cache)
    q = torch.randn(1, 16, 576, device="cuda").to(torch.bfloat16)
    limits = dict(scale=0.05, max_q_len=1, max_kv_len=700)
    got = bdc.kv_latent_attention(q, cache, ints([pages]), ints([700]), ints([0, 1]), **limits)
    small = bdc.KvLatent(*rows[pages].split([512, 64], 2))
    assert torch.equal(got, bdc.kv_latent_attention(q, small, ints([[0, 1, 2]]), ints([700]), ints([0, 1]), **limits))


# ---------------------------------------------------------------- together --
def test_a_serving_run_over_the_latent_cache():
    """Tables, queries turned, latents written, attention, for prompts, windows that are taken back and single tokens;
    every forward against plain attention over all tokens kept by the request."""
    rng = np.random.default_rng(5)
    n_seq, page, heads, dim, rope, cols, scale = 5, 32, 4, 128, 32, 20, 0.1
    n_pages = n_seq * cols
    cache = bdc.kv_latent_cache(n_pages, page, dim, rope)
    rotary = bdc.kv_rotary(rope, interleaved=True, factor=4.0, original_len=128, scale=1.1)
    table = torch.full((n_seq, cols), -1, dtype=torch.int32, device="cuda")
    free, pool = torch.randperm(n_pages, device="cuda").to(torch.int32), torch.tensor([0, n_pages], device="cuda")
    lens = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    kept = [torch.empty(0, dim + rope, dtype=torch.bfloat16, device="cuda") for _ in range(n_seq)]
    for step in range(12):
        add = [int(rng.integers(20, 90)) if step == 0 else 24 if step % 3 else 1] * n_seq
        add[step % n_seq] = 0 if step else 1
        total = sum(add)
        r = bdc.kv_tables(lens, ints(add), table, free, pool, page_size=page, max_tokens=total + 3)
        pool = r.pool
        x = torch.randn(total + 3, dim + rope, device="cuda").to(torch.bfloat16)
        q = torch.randn(total + 3, heads, dim + rope, device="cuda").to(torch.bfloat16)
        bdc.kv_rotate(q[..., dim:], r.positions, rotary, out=q[..., dim:])
        bdc.kv_latent_write(x[:, :dim], x[:, dim:], r.slot_map, cache, positions=r.positions, rotary=rotary)
        out = bdc.kv_latent_attention(q, cache, table, r.kv_lens, r.query_start, scale=scale, max_q_len=max(add),
                                      max_kv_len=cols * page, mask_block=8)
        x[:, dim:] = bdc.kv_rotate(x[:, None, dim:].contiguous(), r.positions, rotary)[:, 0]
        at = 0
        for s in range(n_seq):
            keys = torch.cat([kept[s], x[at:at + add[s]]]).double()
            for i in range(add[s]):
                see = len(keys) - add[s] + min(add[s], (i // 8 + 1) * 8)
                p = torch.softmax(q[at + i].double() @ keys[:see].T * scale, 1)
                want, spread = p @ keys[:see, :dim], p @ keys[:see, :dim].abs()
                assert bool(((out[at + i].double() - want).abs() <= 2.0 ** -8 * (want.abs() + 1.1 * spread)).all())
            if step % 3 != 1:  # else the window is taken back
                kept[s] = torch.cat([kept[s], x[at:at + add[s]]])
            at += add[s]
        lens = r.kv_lens
        if step % 3 == 1:
            back = bdc.kv_tables(lens, ints([-a for a in add]), table, free, pool, page_size=page, max_tokens=0)
            lens, pool = back.kv_lens, back.pool
    assert lens.tolist() == [len(k) for k in kept] and min(lens.tolist()) > 40
