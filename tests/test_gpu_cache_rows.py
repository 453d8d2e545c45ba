"""Every row of kv_attention by its own measure: scores of any size, rows of very different magnitude in one call,
pages of very different scales, queries that are not finite. Bounds are those of test_gpu_cache.attention_bounds, but
for weights that are too small for f16: they are held times 2^8 or more against a reference that is at most the largest
weight of a token that the row itself sees, so each is off by at most 2^-33 of that (half a subnormal step, 2^-25, over
2^8)."""

import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from tests.test_gpu_cache import attention_bounds, gpu_cache
from workloads.cache_inputs import random_cache

pytestmark = pytest.mark.gpu

bdc = pytest.importorskip("paper_2609_33887_gb300")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)
    yield
    assert bdc.kvcache.kv_device_status() == 0


def queries(q_lens, n_q, dim, seed, dtype=torch.bfloat16):
    starts = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    q = np.random.default_rng(seed).normal(0, 1, (int(starts[-1]), n_q, dim))
    return torch.from_numpy(q).to(dtype), starts


def attention(c, q, starts, mask_block=1, max_kv=None):
    out, lse = bdc.kv_attention(
        q.cuda(), gpu_cache(c), torch.from_numpy(c.table).cuda(), torch.from_numpy(c.kv_lens).cuda(),
        torch.from_numpy(starts).cuda(), max_q_len=int(np.diff(starts).max()),
        max_kv_len=int(c.kv_lens.max()) if max_kv is None else max_kv, mask_block=mask_block, return_lse=True)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def assert_rows(c, q, starts, mask_block=1, max_kv=None):
    got, got_lse = attention(c, q, starts, mask_block, max_kv)
    args = (q.double().numpy(), c.k, c.v, c.k_scale, c.v_scale, c.table, c.kv_lens, starts, q.shape[2] ** -0.5, mask_block)
    ref, ref_lse, spread, work = CO.attention(*args)
    tiny = 2.0 ** -33 * CO.attention_largest_term(*args)
    b, b_lse = attention_bounds(ref, ref_lse, spread, work, {torch.bfloat16: "bf16", torch.float16: "f16"}[q.dtype],
                                2.0 ** 22 * tiny)
    off = np.abs(got - ref) > b
    assert not off.any(), (int(off.sum()), np.argwhere(off)[:4].tolist())
    assert np.all(np.abs(got_lse - ref_lse) <= b_lse)


@pytest.mark.parametrize("q_len", [1, 8, 9, 70])
@pytest.mark.parametrize("k", [0, 5, 10, 15, 20, 25, 30, 60, 90])
@pytest.mark.parametrize("page,dim,v_exp", [(16, 64, (-9, -5)), (64, 128, (-9, -5)), (64, 64, (-60, 40)), (32, 80, (-60, 40))])
def test_scores_of_any_size(k, q_len, page, dim, v_exp):
    """A row whose best score is above all others by more than any rounding takes that token's value, rounded twice: the
    weight to f16 (2^-11, and 2^-17 for references and exp2), the result to bf16. Scores are off by 2^-15 of `work`, and
    the others' values are at most 2^(40 + 60) times as large (70 in powers of e)."""
    c = random_cache([q_len + 150, q_len + 33], page, 2, dim, seed=24, v_exp=v_exp, extra_cols=5000 // page)
    q, starts = queries([q_len] * 2, 8, dim, 9)
    q *= 2.0 ** k
    got, _ = attention(c, q, starts, 1, 5000 if q_len == 70 else None)
    args = (q.double().numpy(), c.k, c.v, c.k_scale, c.v_scale, c.table, c.kv_lens, starts, dim ** -0.5, 1)
    work = CO.attention(*args)[3]
    value, gap, most = CO.attention_best_token(*args)
    assert np.all(np.abs(got) <= most * (1 + 2.0 ** -7))  # a weighted mean of the values it sees
    sure = gap - 2 * work * 2.0 ** -15 > 70 + 40
    b = (2.0 ** -8 + (1 + 2.0 ** -8) * (2.0 ** -11 + 2.0 ** -17)) * np.abs(value)
    off = (np.abs(got - value) > b) & sure[..., None]
    assert not off.any(), (int(off.sum()), np.argwhere(off)[:4].tolist())
    if k >= 20:
        assert sure.mean() > 0.9
    if k <= 10:
        assert_rows(c, q, starts, 1, 5000 if q_len == 70 else None)


# rows of a key/value head: 4 and 32 (16-row tiles), 36 (one tile of 128), 280 (two to a CTA, under a long bound)
@pytest.mark.parametrize("q_len", [1, 8, 9, 70])
@pytest.mark.parametrize("k", [31, 36, 40, 90, -40, -90])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_row_far_above_or_below_its_neighbours(q_len, k, dim):
    c = random_cache([q_len + 150, q_len + 33], 16, 2, dim, seed=21, extra_cols=330)
    q, starts = queries([q_len] * 2, 8, dim, 5)
    q[q_len // 2, 1] *= 2.0 ** k  # exact: whole powers of two
    q[-1, 6] *= 2.0 ** k
    assert_rows(c, q, starts, max_kv=5000 if q_len == 70 else None)


@pytest.mark.parametrize("q_len", [8, 9, 70])
def test_rows_of_all_magnitudes_in_one_call(q_len):
    c = random_cache([q_len + 90], 32, 1, 80, seed=22, extra_cols=160)
    q, starts = queries([q_len], 4, 80, 6)
    q *= torch.exp2(torch.arange(q.shape[0] * 4) % 41 * 5.0 - 100).view(-1, 4, 1).to(q.dtype)
    assert_rows(c, q, starts, max_kv=5000 if q_len == 70 else None)


@pytest.mark.parametrize("q_len", [1, 8, 100, 150])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("mask_block", [0, 1, 32])
def test_pages_of_very_different_scales_by_each_rows_own(q_len, page, mask_block):
    c = random_cache([400, 170], page, 2, 64, seed=6, k_exp=(-16, -6), v_exp=(-60, 40), extra_cols=5000 // page)
    q, starts = queries([q_len] * 2, 4, 64, 7)
    assert_rows(c, q, starts, mask_block)
    if q_len == 150:
        assert_rows(c, q, starts, mask_block, max_kv=5000)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("q_len", [1, 8, 9, 70])
@pytest.mark.parametrize("total", [90, 2000])  # in one part, in several
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_queries_that_are_not_finite(bad, total, q_len, dtype):
    """A softmax of scores that are all -inf, or hold +inf or NaN, is NaN, for that row alone."""
    c = random_cache([total, total - 7], 16, 2, 64, seed=23)
    c.k[c.k != 0x7F] &= 0x7F  # keys of one sign, none of them zero: scores of an infinity are infinities of one sign
    c.k[c.k == 0] = 1
    q, starts = queries([q_len] * 2, 8, 64, 8, dtype)
    q[q_len // 2, 1, 5] = bad
    got, lse = attention(c, q, starts, 0)
    want = np.zeros(got.shape[:2], dtype=bool)
    want[q_len // 2, 1] = True
    assert np.array_equal(np.isnan(got), np.repeat(want[..., None], 64, 2))
    assert np.all(np.isfinite(lse[~want]))
    if bad == -math.inf:
        assert lse[q_len // 2, 1] == -math.inf
