"""The checks of kvcache.py on the tensors that it turns into pointers, without a GPU: the library is replaced by a
record of the calls that reach it, so a call that should be refused and is not is seen and nothing runs."""

import pytest
import torch

from paper_2609_33887_gb300 import kvcache as K


class Library:
    """Takes every call and keeps its arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(K, "load_library", lambda: lib)
    monkeypatch.setattr(K, "_stream_handle", lambda stream: stream or 0)
    monkeypatch.setattr(K, "_same_gpu", lambda *tensors: None, raising=False)
    return lib


def ints(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype)


def attention(**kw):
    a = dict(q=torch.zeros(4, 4, 32, dtype=torch.bfloat16), cache=K.kv_cache(5, 16, 2, 32, device="cpu"),
             block_table=ints(4, 3), kv_lens=ints(4), query_start=ints(5), max_q_len=1, max_kv_len=48)
    a.update(kw)
    return K.kv_attention(a.pop("q"), a.pop("cache"), a.pop("block_table"), a.pop("kv_lens"), a.pop("query_start"), **a)


def tables(**kw):
    a = dict(lens=ints(4), new_tokens=ints(4), block_table=ints(4, 3), free_pages=ints(20),
             pool=ints(2, dtype=torch.int64))
    a.update(kw)
    return K.kv_tables(a["lens"], a["new_tokens"], a["block_table"], a["free_pages"], a["pool"], page_size=16,
                       max_tokens=9)


def test_tables_whose_rows_overlap_are_refused(library):
    """One row expanded over requests, and rows closer than they are long: their stride is what the kernels step by."""
    for table in (ints(1, 3).expand(4, 3), ints(20).as_strided((4, 3), (2, 1)), ints(20).as_strided((4, 3), (0, 1))):
        for call in (attention, tables):
            with pytest.raises(ValueError, match="block_table"):
                call(block_table=table)
    assert not library.calls


@pytest.mark.parametrize("call", [attention, tables])
def test_tables_of_one_row_and_wide_ones_keep_their_stride(library, call):
    one = dict(lens=ints(1), new_tokens=ints(1)) if call is tables else dict(kv_lens=ints(1), query_start=ints(2))
    # a single row's stride says nothing (it may be 0): the columns' number takes its place
    for kw, stride in ((dict(block_table=ints(4, 3)), 3), (dict(block_table=ints(4, 9)[:, :3]), 9),
                       (dict(one, block_table=ints(20).as_strided((1, 3), (0, 1))), 3)):
        call(**kw)
        name, args = library.calls[-1]
        fields = K.TABLES_FIELDS.unpack(args[0]) if call is tables else K.ATTN_FIELDS.unpack(args[1])
        assert (fields[4] if call is tables else fields[10]) == stride


def test_tensors_of_the_host_are_refused(monkeypatch):
    lib = Library()
    monkeypatch.setattr(K, "load_library", lambda: lib)
    monkeypatch.setattr(K, "_stream_handle", lambda stream: stream or 0)
    x = torch.zeros(4, 2, 32, dtype=torch.bfloat16)
    for call in (attention, tables, lambda: K.kv_write(x, x, ints(4, dtype=torch.int64), K.kv_cache(5, 16, 2, 32, device="cpu"))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    assert not lib.calls
