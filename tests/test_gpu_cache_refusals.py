"""What the cache's calls refuse of tensors that are otherwise on the GPU: each argument in turn is one that the kernels
must not be given. Nothing is queued (the library is replaced by a record)."""

import pytest
import torch

pytestmark = pytest.mark.gpu

bdc = pytest.importorskip("paper_2609_33887_gb300")
K = bdc.kvcache


@pytest.fixture
def calls(monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    kept = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: kept.append(name) or 0

    monkeypatch.setattr(K, "load_library", lambda: Library())
    return kept


def ints(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def arguments():
    rows = torch.zeros(4, 2, 32, dtype=torch.bfloat16, device="cuda")
    return {"k": rows, "v": rows.clone(), "slot_map": ints(4, dtype=torch.int64), "cache": K.kv_cache(5, 16, 2, 32),
            "q": torch.zeros(4, 4, 32, dtype=torch.bfloat16, device="cuda"), "block_table": ints(4, 3),
            "kv_lens": ints(4), "query_start": ints(5), "lens": ints(4), "new_tokens": ints(4), "free_pages": ints(20),
            "pool": ints(2, dtype=torch.int64), "out": torch.zeros(4, 4, 32, dtype=torch.bfloat16, device="cuda"),
            "workspace": torch.zeros(4096, dtype=torch.uint8, device="cuda")}


CALLS = {
    "kv_write": lambda a: K.kv_write(a["k"], a["v"], a["slot_map"], a["cache"]),
    "kv_tables": lambda a: K.kv_tables(a["lens"], a["new_tokens"], a["block_table"], a["free_pages"], a["pool"],
                                       page_size=16, max_tokens=9),
    "kv_attention": lambda a: K.kv_attention(a["q"], a["cache"], a["block_table"], a["kv_lens"], a["query_start"],
                                             max_q_len=1, max_kv_len=48, out=a["out"], workspace=a["workspace"]),
}
READS = {"kv_write": ["k", "v", "slot_map"], "kv_tables": ["lens", "new_tokens", "block_table", "free_pages", "pool"],
         "kv_attention": ["q", "block_table", "kv_lens", "query_start", "out", "workspace"]}


@pytest.mark.parametrize("name,arg", [(n, a) for n, args in READS.items() for a in args])
def test_one_tensor_on_the_host_is_refused(calls, name, arg):
    a = arguments()
    CALLS[name](a)
    assert len(calls) == 1
    with pytest.raises(ValueError, match="GPU"):
        CALLS[name](dict(a, **{arg: a[arg].cpu()}))
    assert len(calls) == 1


@pytest.mark.parametrize("name", ["kv_write", "kv_attention"])
@pytest.mark.parametrize("part", K.KvCache._fields)
def test_a_part_of_the_cache_on_the_host_is_refused(calls, name, part):
    a = arguments()
    with pytest.raises(ValueError, match="GPU"):
        CALLS[name](dict(a, cache=a["cache"]._replace(**{part: getattr(a["cache"], part).cpu()})))
    assert not calls
