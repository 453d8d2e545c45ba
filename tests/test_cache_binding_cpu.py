"""The checks of kvcache.py on the tensors that it turns into pointers, without a GPU: the library is replaced by a
record of the calls that reach it, so a call that should be refused and is not is seen and nothing runs."""

import os
import shutil

import pytest
import torch

from paper_2609_33887_gb300 import kvcache as K
from paper_2609_33887_gb300.bdcommit import BD_ERR_ARG, BD_ERR_SHAPE, BD_OK, BdError


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


# ------------------------------------------------------- rows on top of each other --
@pytest.fixture(scope="module")
def checks():
    """The library itself: its argument checks come before any CUDA call."""
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("no CUDA toolkit")
    import __graft_entry__

    __graft_entry__.build()
    return K.load_library()


FAKE = 1 << 20  # a non-null, aligned address that is never dereferenced


def cache_fields(**kw):
    f = dict(n_pages=4, page=16, heads=2, dim=32, k=(1024, 64, 32), v=(1024, 64, 32), ks=2, vs=2)
    f.update(kw)
    return K.CACHE_FIELDS.pack(FAKE, FAKE, FAKE, FAKE, f["n_pages"], f["page"], f["heads"], f["dim"], *f["k"], *f["v"],
                               f["ks"], f["vs"])


def attn_fields(token, head, n_q=4, n_seq=2, max_q=3):
    return K.ATTN_FIELDS.pack(FAKE, K.BDKV_BF16, 0, 0, FAKE, K.BDKV_BF16, token, head, 0, FAKE, 8, 8, FAKE, FAKE, n_seq, n_q,
                              max_q, 100, 1, 0.5, 0, 0, 0)


OVERLAP = [dict(token=0, head=32), dict(token=128, head=0), dict(token=128, head=16), dict(token=120, head=32),
           dict(token=32, head=32), dict(token=16, head=400), dict(token=0, head=0, n_seq=1, max_q=1)]
APART = [dict(token=128, head=32), dict(token=32, head=96), dict(token=200, head=48), dict(token=0, head=32, n_seq=1, max_q=1)]


@pytest.mark.parametrize("kw", OVERLAP, ids=str)
def test_outputs_on_top_of_each_other_are_refused(checks, kw):
    assert checks.bdkv_attention(cache_fields(), attn_fields(**kw)) == BD_ERR_ARG


@pytest.mark.parametrize("kw", APART, ids=str)
def test_outputs_apart_in_any_order_are_not(checks, kw):
    if torch.cuda.is_available():
        pytest.skip("the call would run")
    assert checks.bdkv_attention(cache_fields(), attn_fields(**kw)) not in (BD_ERR_ARG, BD_OK)  # no device


def test_the_binding_refuses_an_out_whose_rows_overlap(library, checks, monkeypatch):
    x = torch.zeros(4, 4, 32, dtype=torch.bfloat16)
    base = torch.zeros(4000, dtype=torch.bfloat16)
    good = [x, x.transpose(0, 1).contiguous().transpose(0, 1), base.as_strided((4, 4, 32), (48, 192, 1))]
    for out in good:
        attention(out=out)
    assert len(library.calls) == len(good)
    attention(q=x[:1], out=base.as_strided((1, 4, 32), (0, 32, 1)))  # one token: its stride says nothing
    assert K.ATTN_FIELDS.unpack(library.calls[-1][1][1])[6] >= 4 * 32
    with pytest.raises(ValueError, match="overlap"):
        attention(out=base.as_strided((4, 4, 32), (32, 96, 1)))
    monkeypatch.setattr(K, "load_library", lambda: checks)
    for out in (x[:1].expand(4, 4, 32), x[:, :1].expand(4, 4, 32)):
        with pytest.raises(BdError) as e:
            attention(out=out)
        assert e.value.status == BD_ERR_ARG


def test_queries_may_share_memory(library):
    """Queries are only read: also where the workspace's size is asked for, which takes no outputs."""
    q = torch.zeros(1, 4, 32, dtype=torch.bfloat16).expand(4, 4, 32)
    args = (q, K.kv_cache(5, 16, 2, 32, device="cpu"), ints(4, 3), ints(4), ints(5))
    K.kv_attention_workspace(*args, max_q_len=1, max_kv_len=48)
    fields = K.ATTN_FIELDS.unpack(library.calls[-1][1][1])
    assert fields[2] == 0 and fields[6:8] == (128, 32)


@pytest.mark.parametrize("kw", [dict(k=(0, 64, 32)), dict(v=(1024, 0, 32)), dict(k=(1024, 64, 0)), dict(k=(1024, 64, 16)),
                                dict(v=(1024, 32, 32)), dict(k=(1008, 64, 32)), dict(v=(1024, 32, 496)), dict(ks=1),
                                dict(vs=0), dict(n_pages=2 ** 31 - 1, v=(2 ** 40, 2 ** 40, 2 ** 40))], ids=str)
def test_writes_into_shared_memory_are_refused(checks, kw):
    rows = K.ROWS_FIELDS.pack(FAKE, K.BDKV_BF16, 64, 32)
    assert checks.bdkv_write(cache_fields(**kw), rows, rows, FAKE, 3, None) == BD_ERR_ARG


@pytest.mark.parametrize("kw", [dict(), dict(k=(1024, 32, 512)), dict(v=(2048, 128, 64)), dict(k=(64, 256, 32)),
                                dict(n_pages=1, k=(0, 64, 32), ks=0), dict(heads=1, v=(1024, 64, 0)),
                                dict(n_pages=2 ** 31 - 1, v=(2 ** 40, 64, 32))], ids=str)
def test_writes_into_any_layout_are_not(checks, kw):
    if torch.cuda.is_available():
        pytest.skip("the call would run")
    rows = K.ROWS_FIELDS.pack(FAKE, K.BDKV_BF16, 64, 32)
    assert checks.bdkv_write(cache_fields(**kw), rows, rows, FAKE, 3, None) not in (BD_ERR_ARG, BD_OK)  # no device


def test_attention_reads_a_cache_that_shares_memory(checks):
    if torch.cuda.is_available():
        pytest.skip("the call would run")
    for kw in (dict(k=(1024, 64, 0)), dict(v=(0, 64, 32)), dict(ks=0)):
        assert checks.bdkv_attention(cache_fields(**kw), attn_fields(128, 32)) not in (BD_ERR_ARG, BD_OK)


# --------------------------------------------------------------- very long caches --
def test_lengths_that_32_bits_do_not_count_are_refused(checks):
    """A part's last token is begin + chunk, and its kernels look a few tiles further: past 2^31 those sums turn negative,
    which passes for a token inside the cache."""
    def call(max_kv):
        fields = list(K.ATTN_FIELDS.unpack(attn_fields(128, 32)))
        fields[10:12] = 2 ** 27, 2 ** 27  # the table's stride and columns: 2^31 tokens
        fields[17] = max_kv
        return checks.bdkv_attention(cache_fields(), K.ATTN_FIELDS.pack(*fields))

    for max_kv in (2 ** 30 + 1, 2 ** 31 - 200, 2 ** 31 - 1):
        assert call(max_kv) == BD_ERR_SHAPE
    if not torch.cuda.is_available():
        assert call(2 ** 30) not in (BD_ERR_SHAPE, BD_OK)  # no device


def test_a_workspace_has_to_be_one_piece(library):
    """Its bytes are counted from its elements: an expanded tensor has more of them than memory."""
    whole = torch.zeros(4096, dtype=torch.uint8)
    attention(workspace=whole)
    fields = K.ATTN_FIELDS.unpack(library.calls[-1][1][1])
    assert fields[20:22] == (whole.data_ptr(), 4096)
    for ws in (whole[:1].expand(4096), whole[::2], whole.view(64, 64)[:, :32]):
        with pytest.raises(ValueError, match="workspace"):
            attention(workspace=ws)
    assert len(library.calls) == 1
