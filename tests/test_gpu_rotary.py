"""Rotary positions on the GPU (kv_rotate, kv_write_rotated) against the float64 oracle, whose angles are exact."""

import math

import numpy as np
import pytest
import torch

from oracle import rotary_oracle as RO
from tests.test_gpu_cache import gpu_cache
from workloads.cache_inputs import random_cache

pytestmark = pytest.mark.gpu

bdc = pytest.importorskip("paper_2609_33887_gb300")

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step, relative
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}  # half a subnormal step


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__

    __graft_entry__.build()
    torch.cuda.set_device(0)


def freqs(dim, base=10000.0):
    return [base ** (-2 * p / dim) for p in range(dim // 2)]


def rows(n, heads, dim, dtype, seed=0, mag=1.0):
    rng = np.random.default_rng(seed)
    return torch.from_numpy(rng.normal(0, mag, (n, heads, dim))).to(DTYPES[dtype]).cuda()


def ints(v):
    return torch.from_numpy(np.asarray(v, dtype=np.int32)).cuda()


def bound(x, ref, rot, scale, interleaved, dtype):
    """A result is rounded once (U). In fp32 before it, each 2^-24 of the pair's magnitudes or less: the angle within an
    eighth of a turn (and 2^-32 turns that it is cut to), the sine's and cosine's last two steps, and two products: 2^-21 in
    all, with room."""
    a = np.abs(x[..., :rot])
    both = a.reshape(*a.shape[:2], -1, 2).sum(3) if interleaved else a.reshape(*a.shape[:2], 2, -1).sum(2)
    both = np.repeat(both, 2, axis=2) if interleaved else np.concatenate([both, both], 2)
    b = np.zeros_like(x)
    b[..., :rot] = 2.0 ** -21 * abs(scale) * both * (1 + U[dtype]) + U[dtype] * np.abs(ref[..., :rot]) + TINY[dtype]
    return b


def check(x, positions, rot, dtype, *, interleaved=False, inverse=False, scale=1.0, base=10000.0, out=None, **kw):
    f = freqs(rot, base)
    rotary = bdc.kv_rotary(rot, base=base, scale=scale, interleaved=interleaved)
    before = x.double().cpu().numpy()
    got = bdc.kv_rotate(x, ints(positions), rotary, inverse=inverse, out=out, **kw)
    ref = RO.rotate(before, positions, f, scale, interleaved, inverse)
    off = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(off <= bound(before, ref, rot, scale, interleaved, dtype)), float(np.max(off))
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("n,heads,dim,rot", [(1, 1, 16, 16), (1, 32, 128, 128), (3, 5, 80, 48), (65, 2, 64, 64),
                                             (33, 28, 112, 32), (7, 3, 256, 256), (700, 12, 96, 96), (5, 1, 1024, 64),
                                             (260, 7, 208, 16)])
def test_rotations(n, heads, dim, rot, inverse, interleaved, dtype):
    positions = np.random.default_rng(n).integers(0, 5000, n)
    check(rows(n, heads, dim, dtype), positions, rot, dtype, interleaved=interleaved, inverse=inverse)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("scale,base", [(1.0, 10000.0), (1.3466, 5e6), (-0.25, 1.0), (0.0, 500.0)])
def test_far_and_negative_positions(scale, base, interleaved):
    positions = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131071, 900001, -12345678, 2 ** 30, 77, 4095, 2 ** 24 + 1]
    check(rows(len(positions), 4, 64, "f16"), positions, 64, "f16", scale=scale, base=base, interleaved=interleaved)


@pytest.mark.parametrize("scale", [2.0 ** -96, -1.37 * 2.0 ** -95, 1e30])
def test_smallest_and_large_scales(scale):
    check(rows(40, 3, 64, "bf16"), list(range(40)), 64, "bf16", scale=scale)


def test_position_zero_leaves_rows_as_they_are():
    x = rows(9, 3, 64, "bf16")
    for inter in (False, True):
        assert torch.equal(bdc.kv_rotate(x, ints([0] * 9), bdc.kv_rotary(64, interleaved=inter)), x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_in_parts_of_rows_and_out_of_wider_ones(interleaved):
    rng = np.random.default_rng(3)
    positions = rng.integers(0, 9000, 50)
    wide = rows(50, 9, 208, "bf16", 1)
    kept = wide.clone()
    part = wide[:, 2:7, 128:192]  # the last elements of some heads, in place
    fresh = check(part.clone(), positions, 64, "bf16", interleaved=interleaved)
    got = check(part, positions, 64, "bf16", interleaved=interleaved, out=part)
    assert got is part and torch.equal(part, fresh)
    kept[:, 2:7, 128:192] = fresh
    assert torch.equal(wide, kept)
    # into other heads of the same rows; from one row for all tokens; from one head for all heads
    out = wide[:, 7:9, :64]
    check(wide[:, :2, :64], positions, 64, "bf16", interleaved=interleaved, out=out)
    check(rows(1, 3, 80, "bf16").expand(50, 3, 80), positions, 48, "bf16", interleaved=interleaved)
    check(rows(50, 1, 80, "bf16").expand(50, 6, 80), positions, 80, "bf16", interleaved=interleaved)


def test_rows_that_meet_are_refused_and_nothing_is_written():
    x, rotary = rows(8, 4, 64, "bf16"), bdc.kv_rotary(64)
    wide = rows(9, 6, 64, "bf16")
    kept = wide.clone()
    for a, b in ((wide[:8, :4], wide[:8, 1:5]), (wide[:8, :4], wide[1:9, :4]), (wide[:8, ::2], wide[:8, :3])):
        with pytest.raises(bdc.BdError):
            bdc.kv_rotate(a, ints([1] * 8), rotary, out=b)
    with pytest.raises(bdc.BdError):
        bdc.kv_rotate(x, ints([1] * 8), rotary, out=torch.empty(1, 4, 64, dtype=x.dtype, device="cuda").expand(8, 4, 64))
    torch.cuda.synchronize()
    assert torch.equal(wide, kept)


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_inverse_is_the_adjoint(interleaved):
    """Against the formula and against differences: for y = R x and any g, the gradient of <g, y> is R' g, so <g, R d> =
    <R' g, d> for each direction d (R is linear: a difference of any size says so)."""
    n, heads, dim, rot, scale = 20, 3, 96, 64, 1.25
    rotary = bdc.kv_rotary(rot, scale=scale, interleaved=interleaved)
    positions = ints(np.random.default_rng(0).integers(0, 100000, n))
    x, g = rows(n, heads, dim, "f16", 1), rows(n, heads, dim, "f16", 2)
    d = rows(n, heads, dim, "f16", 3)
    host = [t.double().cpu().numpy() for t in (g, x, x + d)]
    back, before, after = (bdc.kv_rotate(t, positions, rotary, inverse=t is g).double().cpu().numpy()
                           for t in (g, x, x + d))
    step = host[2] - host[1]  # as f16 holds it
    slack = [bound(t, np.abs(r), rot, scale, interleaved, "f16") for t, r in zip(host, (back, before, after))]
    off = abs((host[0] * (after - before)).sum() - (back * step).sum())
    assert off <= 1.01 * ((np.abs(host[0]) * (slack[1] + slack[2])).sum() + (slack[0] * np.abs(step)).sum())
    assert off <= 1e-3 * np.abs(host[0] * (after - before)).sum()  # (what the bound leaves room for is far more)
    # twice, there and back: scale^2 x
    there = bdc.kv_rotate(x, positions, rotary)
    again = bdc.kv_rotate(there, positions, rotary, inverse=True).double().cpu().numpy()[..., :rot]
    there = there.double().cpu().numpy()
    # the first rounding moves both elements of a pair, by U of at most scale times their magnitudes' sum each
    one = bound(host[1], there, rot, scale, interleaved, "f16")
    both = bound(one, one, rot, 1.0, interleaved, "f16") * 2.0 ** 21  # a pair's errors added up
    ref = scale ** 2 * host[1][..., :rot]
    assert np.all(np.abs(again - ref) <= (1.01 * scale * both + bound(there, there, rot, scale, interleaved, "f16")
                                          + U["f16"] * np.abs(host[1]) * scale ** 2)[..., :rot])


def test_elements_that_are_not_finite_stay_in_their_pair():
    x = rows(4, 2, 64, "bf16")
    x[1, 0, 3], x[2, 1, 40] = math.nan, math.inf
    y = bdc.kv_rotate(x, ints([5, 6, 7, 8]), bdc.kv_rotary(64))
    bad = ~y.isfinite()
    assert {tuple(i) for i in bad.nonzero().tolist()} == {(1, 0, 3), (1, 0, 35), (2, 1, 8), (2, 1, 40)}


@pytest.mark.parametrize("n,heads", [(0, 3), (1, 1)])
def test_none_and_one(n, heads):
    x = rows(n, heads, 32, "bf16")
    assert bdc.kv_rotate(x, ints([9] * n), bdc.kv_rotary(32)).shape == x.shape


# ------------------------------------------------------------------------------------------------- stretched contexts --
def test_rotary_frequencies():
    def radians(r):
        return (r.turns.cpu().numpy().astype(object) % 2 ** 64 / 2.0 ** 64 * 2 * math.pi).astype(float)

    f = np.array(freqs(64))
    assert np.allclose(radians(bdc.kv_rotary(64)), f, rtol=1e-14)
    assert np.allclose(radians(bdc.kv_rotary(64, factor=4.0)), f / 4, rtol=1e-14)
    r = radians(bdc.kv_rotary(64, factor=8.0, original_len=4096))
    turns = 4096 * f / (2 * math.pi)
    assert np.allclose(r[turns >= 32], f[turns >= 32], rtol=1e-14)
    assert np.allclose(r[turns <= 1], f[turns <= 1] / 8, rtol=1e-14)
    between = (turns > 1) & (turns < 32)
    assert between.any() and np.all((r < f)[between]) and np.all((r > f / 8)[between])
    mine = [0.5, 0.25, 1e-3, 7.0, 0.0, -0.125, 3e-9, 1.0]
    assert np.allclose(radians(bdc.kv_rotary(16, frequencies=mine)), np.array(mine) % (2 * math.pi), rtol=1e-14, atol=1e-18)


# ------------------------------------------------------------------------------------------------------------ writes --
def slots_of(c, new, page):
    """Slots and positions of the last `new[s]` tokens of each request."""
    out, pos = [], []
    for s, n in enumerate(new):
        for p in range(int(c.kv_lens[s]) - n, int(c.kv_lens[s])):
            out.append(int(c.table[s, p // page]) * page + p % page)
            pos.append(p)
    return np.array(out, np.int64), np.array(pos, np.int32)


def check_write(page, lens, new, n_kv, dim, rot, n_q, dtype, interleaved, edit=None, scale=1.0):
    c = random_cache(lens, page, n_kv, dim, seed=page + dim)
    slots, pos = slots_of(c, new, page)
    n = len(slots)
    qkv = rows(n, n_q + 2 * n_kv, dim, dtype, seed=n + dim)
    if edit is not None:
        edit(qkv, slots)
    q, k, v = qkv.split([n_q, n_kv, n_kv], 1)
    rotary = bdc.kv_rotary(rot, interleaved=interleaved, scale=scale)
    slots, pos = torch.from_numpy(slots).cuda(), ints(pos)
    one, two = gpu_cache(c), gpu_cache(c)
    turned = bdc.kv_write_rotated(k, v, slots, one, pos, rotary, q=q if n_q else None)
    bdc.kv_write(bdc.kv_rotate(k, pos, rotary), v, slots, two)
    for a, b in zip(one, two):
        assert torch.equal(a, b)
    if n_q:
        assert torch.equal(turned.view(torch.int16), bdc.kv_rotate(q, pos, rotary).view(torch.int16))
    else:
        assert turned is None
    return qkv, q, k, v, slots, pos, rotary


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("page,n_kv,dim,rot,n_q", [(16, 2, 64, 64, 4), (32, 5, 80, 48, 10), (64, 8, 128, 128, 32),
                                                   (128, 1, 96, 16, 0), (256, 3, 128, 64, 3), (16, 1, 16, 16, 1)])
def test_writes_are_those_of_rows_turned_before(page, n_kv, dim, rot, n_q, interleaved, dtype):
    for lens, new in (([300, 77, 1, 500], [300, 40, 1, 257]), ([90, 33, 64, 200], [1, 1, 1, 1]), ([5, 0, 9], [0, 0, 3])):
        check_write(page, lens, new, n_kv, dim, rot, n_q, dtype, interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
def test_writes_of_what_is_not_finite_and_of_what_overflows(interleaved):
    def edit(qkv, slots):
        qkv[3, 3, 5], qkv[7, 4, 0], qkv[20, 2, 60], qkv[30, 5, 63] = math.nan, math.inf, -math.inf, math.nan
        qkv[40, 2:4] = 60000.0  # finite before, beyond f16 once turned and scaled
        slots[10:13] = -1
        slots[50] = 1 << 40
    check_write(16, [100, 50], [60, 20], 2, 64, 64, 2, "f16", interleaved, edit, scale=1.5)
    check_write(64, [100, 50], [60, 20], 2, 64, 32, 2, "bf16", interleaved, edit)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("page,n_kv,dim,n", [(16, 8, 64, 20000), (16, 3, 80, 2000), (16, 8, 128, 2000), (32, 8, 48, 20000),
                                             (32, 2, 16, 1000), (64, 8, 128, 20000), (128, 8, 64, 20000), (256, 8, 128, 20000),
                                             (256, 3, 48, 2000)])
def test_many_rows_with_some_that_are_not_finite(page, n_kv, dim, n, interleaved):
    """Calls in which a block takes several heads one after another, and others; requests begin inside pages."""
    def edit(qkv, slots):
        rng = np.random.default_rng(page)
        for value in (math.nan, math.inf, -math.inf):
            where = torch.from_numpy(rng.integers(0, len(slots), 40))
            qkv[where, torch.from_numpy(rng.integers(1, 1 + 2 * n_kv, 40)), torch.from_numpy(rng.integers(0, dim, 40))] = value
        slots[rng.integers(0, len(slots), 40)] = -1
        qkv[torch.from_numpy(rng.integers(0, len(slots), 9))] *= 1000.0
    lens = [n // 3 + 77, n // 3 + 130, n // 3 - 1, 300]
    check_write(page, lens, [n // 3, n // 3, n // 3 - 1, 1], n_kv, dim, dim, 1, "bf16", interleaved, edit)


@pytest.mark.parametrize("page,dim", [(16, 128), (16, 48), (32, 80), (64, 128)])
def test_single_tokens_of_many_requests(page, dim):
    """Blocks with far more runs than they do at once, each behind tokens that may need a larger scale."""
    rng = np.random.default_rng(page)
    lens = rng.integers(1, page + 4, 700)

    def edit(qkv, slots):
        qkv[torch.from_numpy(rng.integers(0, 700, 70))] *= 64.0
        qkv[torch.from_numpy(rng.integers(0, 700, 20)), 3] = math.inf
        slots[rng.integers(0, len(slots), 9)] = -1
    check_write(page, lens.tolist(), [1] * 700, 8, dim, 16, 2, "bf16", False, edit)
    check_write(page, lens.tolist(), rng.integers(0, np.minimum(lens, 9)).tolist(), 8, dim, 16, 2, "f16", True)


def test_queries_in_place_next_to_their_keys():
    qkv, q, k, v, slots, pos, rotary = check_write(32, [40, 70], [40, 33], 2, 64, 64, 4, "bf16", False)
    ref, keys = bdc.kv_rotate(q, pos, rotary), k.clone()
    cache = bdc.kv_cache(64, 32, 2, 64)
    got = bdc.kv_write_rotated(k, v, slots, cache, pos, rotary, q=q, q_out=q)
    assert got is q and torch.equal(q, ref) and torch.equal(k, keys)
    for out in (qkv[:, 1:5], qkv[:, 4:8]):  # on the queries otherwise, on the keys
        with pytest.raises(bdc.BdError):
            bdc.kv_write_rotated(k, v, slots, cache, pos, rotary, q=q, q_out=out)


@pytest.mark.parametrize("n_q,n_kv", [(1, 2), (4, 1), (1, 1)])
def test_single_heads_in_place_next_to_others(n_q, n_kv):
    n, dim, rotary = 50, 64, bdc.kv_rotary(64)
    x, pos, slots = rows(n, n_q + 2 * n_kv, dim, "bf16"), ints(np.arange(n) + 7), torch.arange(n, device="cuda")
    q, k, v = x.split([n_q, n_kv, n_kv], 1)
    if n_kv == 1:  # a head's stride as that of a [1, tokens, dim] tensor turned round
        k, v = (t.squeeze(1)[None].transpose(0, 1) for t in (k, v))
    keys, ref = k.clone(), bdc.kv_rotate(q, pos, rotary)
    one, two = bdc.kv_cache(5, 16, n_kv, dim), bdc.kv_cache(5, 16, n_kv, dim)
    bdc.kv_write(bdc.kv_rotate(k, pos, rotary), v, slots, two)
    assert bdc.kv_write_rotated(k, v, slots, one, pos, rotary, q=q, q_out=q) is q
    assert torch.equal(q, ref) and torch.equal(k, keys) and all(torch.equal(a, b) for a, b in zip(one, two))


def test_captured_and_replayed_on_a_stream_of_its_own():
    x, positions, rotary = rows(64, 8, 128, "bf16"), ints(np.arange(64)), bdc.kv_rotary(128)
    cache, slots = bdc.kv_cache(8, 16, 4, 128), torch.arange(64, device="cuda")
    q_out, out = torch.empty_like(x[:, :4]), torch.empty_like(x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        bdc.kv_rotate(x, positions, rotary, out=out)
        bdc.kv_write_rotated(x[:, 4:], x[:, 4:], slots, cache, positions, rotary, q=x[:, :4], q_out=q_out)
    x.copy_(rows(64, 8, 128, "bf16", 5))
    positions += 1000
    graph.replay()
    torch.cuda.synchronize()
    want = bdc.kv_rotate(x, positions, rotary)
    other = bdc.kv_cache(8, 16, 4, 128)
    bdc.kv_write(want[:, 4:], x[:, 4:], slots, other)
    assert torch.equal(out, want) and torch.equal(q_out, want[:, :4])
    assert all(torch.equal(a, b) for a, b in zip(cache, other))
    with torch.cuda.stream(stream):
        assert torch.equal(bdc.kv_rotate(x, positions, rotary, stream=stream), want)


@pytest.mark.parametrize("page", [64, 256])
def test_writes_replayed_with_other_rows_and_slots(page):
    n, rotary = 700, bdc.kv_rotary(96, interleaved=True)
    x, positions, slots = rows(n, 7, 96, "f16"), ints(np.arange(n)), torch.arange(n, device="cuda")
    cache, q_out = bdc.kv_cache(2048 // page, page, 3, 96), torch.empty_like(x[:, :1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bdc.kv_write_rotated(x[:, 1:4], x[:, 4:], slots, cache, positions, rotary, q=x[:, :1], q_out=q_out)
    rng = np.random.default_rng(page)
    for first in (0, 700, 1348):
        x.copy_(rows(n, 7, 96, "f16", first))
        positions += 311
        slots.copy_(torch.arange(first, first + n))
        slots[torch.from_numpy(rng.integers(0, n, 5)).cuda()] = -1
        before = [t.clone() for t in cache]
        graph.replay()
        torch.cuda.synchronize()
        other = bdc.KvCache(*before)
        turned = bdc.kv_rotate(x, positions, rotary)
        bdc.kv_write(turned[:, 1:4], x[:, 4:], slots, other)
        assert torch.equal(q_out, turned[:, :1])
        assert all(torch.equal(a, b) for a, b in zip(cache, other))
