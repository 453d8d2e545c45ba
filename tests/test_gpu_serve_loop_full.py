"""examples/serve_loop.py past the end of its requests' tables: what a request has committed stays, in the cache and out
of it, and a forward that a request had no pages for changes nothing of it."""

import importlib.util
import os

import pytest
import torch

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


def held_tokens(server):
    """The codes of every cached token of each request, in its order, and its pages."""
    page, out = server.page, []
    for s, n in enumerate(server.lens.tolist()):
        pages = server.table[s, :-(-n // page)].long()
        out.append([c[pages].reshape(-1, *c.shape[2:])[:n].clone() for c in server.cache[:2]] + [pages])
    return out


@pytest.mark.parametrize("max_len,page", [(112, 16), (100, 32), (160, 64)])
def test_requests_that_fill_their_tables_lose_nothing(loop, max_len, page):
    n_seq, L = 4, 16
    server = loop.Server(loop.Model(), n_seq=n_seq, n_slots=2, block_len=L, page=page, max_len=max_len)
    n_pages = server.cache.k.shape[0]
    committed = torch.zeros(n_seq, dtype=torch.int64, device="cuda")
    stopped = 0
    for _ in range(200):
        before = {k: getattr(server, k).clone() for k in ("lens", "pending", "blocks", "tokens", "masked", "flags")}
        tokens = held_tokens(server)
        done, resolved = server.step()
        committed += done
        served = server.t.status == 0
        # nothing that was committed is gone: in the cache, or still to be computed once more
        assert bool((server.lens >= before["lens"]).all())
        assert torch.equal(server.lens, ((committed - server.pending) * L).int())
        held = [int(p) for s, n in enumerate(server.lens.tolist()) for p in server.table[s, :-(-n // page)].tolist()]
        head, tail = server.pool.tolist()
        assert sorted(held + [int(server.free[j % n_pages]) for j in range(head, tail)]) == list(range(n_pages))
        for s in range(n_seq):
            if served[s]:
                continue
            assert int(done[s]) == 0 and int(resolved[s]) == 0
            for k, was in before.items():
                assert torch.equal(getattr(server, k).view(n_seq, -1)[s], was.view(n_seq, -1)[s]), k
            for a, b in zip(held_tokens(server)[s], tokens[s]):
                assert torch.equal(a, b)
        stopped = stopped + 1 if not bool(served.any()) else 0
        if stopped == 3:
            break
    assert stopped == 3  # all of them came to their tables' end, and stayed there
    assert int(server.lens.max()) <= server.table.shape[1] * page
    assert bdc.kvcache.kv_device_status() == 0 and bdc.bd_get_device_status() == 0


def test_forwards_of_full_tables_see_all_of_their_tokens(loop):
    """max_len need not be a whole number of pages: a table's last page may be filled all the same."""
    server = loop.Server(loop.Model(), n_seq=1, n_slots=1, block_len=16, page=64, max_len=70)
    most = 0
    for _ in range(120):
        server.step()
        most = max(most, int(server.t.kv_lens.max()))
    assert most > 70
    assert server.max_len >= most
