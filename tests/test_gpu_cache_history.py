"""What tokens that were taken back leave behind in a page: its scale. A page's scale is the largest that its tokens have
needed since it was begun, also of tokens that are gone, and coarsens what it holds and what comes after them."""

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from tests.test_gpu_cache import gpu_cache
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


@pytest.mark.parametrize("grow", [1.0, 2.0 ** 4, 2.0 ** 9, 2.0 ** 14])
def test_tokens_taken_back_leave_their_scale(grow):
    """Eight tokens stay, a window of eight (up to `grow` times as large) is written and taken back three times, then eight
    more tokens stay. An element that stays is off by at most 2^-4 of it (E4M3 has four significant bits) and, for each
    scale that the page has had, half a subnormal step of that scale, 2^-10: together 2^-9 of the last, as each is at
    least twice the one before."""
    page, n_kv, dim, p = 32, 2, 64, 1
    c = random_cache([0], page, n_kv, dim, seed=31)
    cache = gpu_cache(c)
    kc, vc, ks, vs = c.k, c.v, c.k_scale, c.v_scale
    rng = np.random.default_rng(int(np.log2(grow)))
    kept = {}

    def write(first, n, mag):
        nonlocal kc, vc, ks, vs
        x = torch.from_numpy(rng.normal(0, 1, (2, n, n_kv, dim)) * mag).to(torch.bfloat16)
        slots = np.arange(p * page + first, p * page + first + n, dtype=np.int64)
        bdc.kv_write(x[0].cuda(), x[1].cuda(), torch.from_numpy(slots).cuda(), cache)
        kc, vc, ks, vs = CO.write(x[0].double().numpy(), x[1].double().numpy(), slots, kc, vc, ks, vs)
        for t in range(n):
            kept[first + t] = x[:, t].double().numpy()

    write(0, 8, 1.0)
    for i in range(3):
        write(8, 8, grow ** ((i + 1) / 3))
    write(8, 8, 1.0)
    assert np.array_equal(cache.k_scale.cpu().numpy(), ks) and np.array_equal(cache.v_scale.cpu().numpy(), vs)
    for i, (codes, scale, want) in enumerate(((cache.k, ks, kc), (cache.v, vs, vc))):
        got = CO.E4M3[codes[p].cpu().numpy()]
        assert np.array_equal(got[:16], CO.E4M3[want[p, :16]])
        step = CO.pow2(scale[p])[None, :, None]
        exact = np.stack([kept[t][i] for t in range(16)])
        assert np.all(np.abs(got[:16] * step - exact) <= 2.0 ** -4 * np.abs(exact) + 2.0 ** -9 * step)
        # the discarded window's largest element still sets the scale
        assert np.all(scale[p] >= CO.scale_byte(np.abs(exact).max((0, 2))) + max(0, int(np.log2(grow)) - 1))
    write(0, 16, 1.0)  # begun afresh: the scale is the tokens' own again
    assert np.array_equal(cache.k_scale.cpu().numpy(), ks)
    own = CO.scale_byte(np.abs(np.stack([kept[t][0] for t in range(16)])).max((0, 2)))
    assert np.array_equal(cache.k_scale[p].cpu().numpy(), own)
