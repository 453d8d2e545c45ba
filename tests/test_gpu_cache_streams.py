"""kv_attention's workspace shared by streams and threads: every stream has inputs, sizes and a reference of its own, so
that a call that reads another one's partial results shows."""

import threading

import pytest
import torch

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
    yield
    assert bdc.kvcache.kv_device_status() == 0


def case(seed, q_len, n_seq, total):
    """(arguments, bounds, result of the call alone) of requests whose caches are split."""
    c = random_cache([total - 3 * s for s in range(n_seq)], 64, 2, 128, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(n_seq * q_len, 8, 128, generator=g, device="cuda").to(torch.bfloat16)
    args = (q, gpu_cache(c), torch.from_numpy(c.table).cuda(), torch.from_numpy(c.kv_lens).cuda(),
            torch.arange(0, (n_seq + 1) * q_len, q_len, dtype=torch.int32, device="cuda"))
    bounds = dict(max_q_len=q_len, max_kv_len=total)
    need = bdc.kv_attention_workspace(*args, **bounds)
    assert need > 0
    raw = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    ref = bdc.kv_attention(*args, **bounds, workspace=raw[-raw.data_ptr() % 256:][:need])  # not the library's own
    torch.cuda.synchronize()
    return args, bounds, ref, need


SIZES = [(1, 6, 900), (5, 3, 1400), (20, 4, 700), (64, 2, 2000)]


def test_streams_with_their_own_inputs_share_the_workspace():
    cases = [case(s, *SIZES[s % 4]) for s in range(8)]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.zeros_like(ref) for _ in range(12)] for _, _, ref, _ in cases]
    torch.cuda.synchronize()
    for i in range(12):
        for (args, bounds, _, _), st, out in zip(cases, streams, outs):
            bdc.kv_attention(*args, **bounds, out=out[i], stream=st)
    torch.cuda.synchronize()
    for (_, _, ref, _), out in zip(cases, outs):
        assert all(torch.equal(o, ref) for o in out)


def test_a_call_that_needs_more_takes_a_larger_workspace():
    cases = sorted((case(20 + s, *SIZES[s]) for s in range(4)), key=lambda c: c[3])
    assert bdc.kvcache.kv_shutdown() == 0
    streams = [torch.cuda.Stream() for _ in cases]
    outs = []
    for _, _, ref, _ in cases:  # each needs more than the ones before, which are queued still
        outs += [(torch.zeros_like(ref), ref) for _ in range(6)]
    torch.cuda.synchronize()
    for i, (out, _) in enumerate(outs):
        args, bounds, _, _ = cases[i // 6]
        bdc.kv_attention(*args, **bounds, out=out, stream=streams[i // 6])
    torch.cuda.synchronize()
    assert all(torch.equal(out, ref) for out, ref in outs)


def test_threads_on_their_own_default_streams_share_the_workspace():
    """The per-thread default stream is one handle (2) for a stream of each thread."""
    cases = [case(40 + s, *SIZES[s % 4]) for s in range(4)]
    outs = [[torch.zeros_like(ref) for _ in range(25)] for _, _, ref, _ in cases]
    torch.cuda.synchronize()
    failed, start = [], threading.Barrier(len(cases))

    def work(i):
        args, bounds, _, _ = cases[i]
        try:
            start.wait()
            for out in outs[i]:
                bdc.kv_attention(*args, **bounds, out=out, stream=2)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for (_, _, ref, _), out in zip(cases, outs):
        assert all(torch.equal(o, ref) for o in out)


# ------------------------------------------------------------------ outputs of a call on another stream --
@pytest.mark.parametrize("handle", [False, True], ids=["stream", "handle"])
def test_outputs_of_a_call_on_another_stream_are_that_streams_memory(handle):
    """Memory that the current stream has freed may still be in use there: a call on another stream must not get it."""
    args, bounds, ref, _ = case(80, 20, 4, 700)
    _, ref_lse = bdc.kv_attention(*args, **bounds, return_lse=True)
    other = torch.cuda.Stream()
    stream = other.cuda_stream if handle else other
    torch.cuda.synchronize()
    freed = [torch.zeros_like(ref) for _ in range(8)] + [torch.zeros_like(ref_lse) for _ in range(8)]
    blocks = {t.data_ptr() for t in freed}
    del freed
    kept = []
    for _ in range(4):
        out, lse = bdc.kv_attention(*args, **bounds, return_lse=True, stream=stream)
        assert not {out.data_ptr(), lse.data_ptr()} & blocks
        kept.append((out, lse))
    other.synchronize()
    for out, lse in kept:
        assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    # and what such a call returned goes back to its own stream's memory
    ptrs = {out.data_ptr() for out, _ in kept}
    del kept, out, lse
    assert not {torch.empty_like(ref).data_ptr() for _ in range(8)} & ptrs


def test_tables_of_a_call_on_another_stream_are_that_streams_memory():
    lens = torch.tensor([5, 40, 0], dtype=torch.int32, device="cuda")
    new = torch.tensor([3, 20, 9], dtype=torch.int32, device="cuda")
    ring = torch.arange(40, dtype=torch.int32, device="cuda")
    pool = torch.tensor([10, 40], dtype=torch.int64, device="cuda")
    table = torch.arange(30, dtype=torch.int32, device="cuda").view(3, 10) % 10
    n = 1000
    kw = dict(page_size=16, max_tokens=n)
    ref = bdc.kv_tables(lens, new, table.clone(), ring.clone(), pool, **kw)
    other, mine, his = torch.cuda.Stream(), table.clone(), ring.clone()
    torch.cuda.synchronize()
    freed = [torch.zeros(n, dtype=d, device="cuda") for d in (torch.int64, torch.int32) for _ in range(8)]
    blocks = {t.data_ptr() for t in freed}
    del freed
    got = bdc.kv_tables(lens, new, mine, his, pool, **kw, stream=other)
    assert not {t.data_ptr() for t in got} & blocks
    other.synchronize()
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


@pytest.mark.parametrize("current", ["default", "other"])
def test_outputs_of_a_call_on_handle_0_are_the_default_streams_memory(current):
    args, bounds, ref, _ = case(81, 20, 4, 700)
    with torch.cuda.stream(torch.cuda.default_stream() if current == "default" else torch.cuda.Stream()):
        torch.cuda.synchronize()
        out = bdc.kv_attention(*args, **bounds, stream=0)
    torch.cuda.synchronize()
    home = [seg["stream"] for seg in torch.cuda.memory_snapshot()
            if seg["address"] <= out.data_ptr() < seg["address"] + seg["total_size"]]
    assert home == [0] and torch.equal(out, ref)
