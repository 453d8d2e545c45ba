"""The paged cache, the commit step and the sweep together, as examples/serve_loop.py runs them: no page is lost over
many forwards, the cache holds the committed blocks, and a forward's attention is the oracle's."""

import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO

pytestmark = pytest.mark.gpu

bdc = pytest.importorskip("paper_2609_33887_gb300")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def loop():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__

    __graft_entry__.build()
    spec = importlib.util.spec_from_file_location("serve_loop", os.path.join(ROOT, "examples", "serve_loop.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_serving_loop(loop):
    server = loop.Server(loop.Model(), n_seq=5, n_slots=3, block_len=16, page=32)
    n_pages = server.cache.k.shape[0]
    committed = torch.zeros(5, dtype=torch.int64, device="cuda")
    for i in range(25):
        done, _ = server.step()
        committed += done
        # held pages and free pages are all pages, once each
        held = [int(p) for s, n in enumerate(server.lens.tolist()) for p in server.table[s, :-(-n // 32)].tolist()]
        head, tail = server.pool.tolist()
        free = [int(server.free[j % n_pages]) for j in range(head, tail)]
        assert sorted(held + free) == list(range(n_pages))
        assert not bool(server.t.status.any())
        # committed blocks are in the cache, but for those of the last forward
        assert torch.equal(server.lens, ((committed - server.pending) * 16).int())
    assert int(committed.min()) > 0

    server.forward()  # its attention against the oracle, on the cache as it stands
    t = server.t
    start, lens = t.query_start.cpu().numpy(), t.kv_lens.cpu().numpy()
    n = int(start[-1])
    codes = [c.cpu().numpy() for c in server.cache]
    q, table = server.q[:n].double().cpu().numpy(), server.table.cpu().numpy()
    ref, _, spread, _ = CO.attention(q, *codes, table, lens, start, 64 ** -0.5, 16)
    got = server.a[:n].double().cpu().numpy()
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -9 * spread + 1e-6)
    assert bdc.kvcache.kv_device_status() == 0 and bdc.bd_get_device_status() == 0


def test_serving_loop_twice_is_the_same(loop):
    def run():
        torch.manual_seed(1)
        torch.cuda.manual_seed(1)
        server = loop.Server(loop.Model(seed=3), n_seq=4, n_slots=2, block_len=20, page=16)
        for _ in range(12):
            server.step()
        return server.tokens.clone(), server.lens.clone(), server.a[:4 * 40].clone()

    for a, b in zip(run(), run()):
        assert torch.equal(a, b)
