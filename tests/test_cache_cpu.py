"""The paged cache without a GPU: the oracle against torch's E4M3 conversions and closed forms, the C ABI of
libbdcache.so (symbols, layout of its structures) and its argument checks, which come before any CUDA call."""

import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from paper_2609_33887_gb300 import kvcache as K
from paper_2609_33887_gb300.bdcommit import (BD_ERR_ALIGN, BD_ERR_ARG, BD_ERR_DTYPE, BD_ERR_NULL, BD_ERR_SHAPE, BD_OK,
                                             bd_status_string)
from workloads.cache_inputs import random_cache, random_tables

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "bdcache.h")


@pytest.fixture(scope="module")
def lib():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("no CUDA toolkit")
    import __graft_entry__

    __graft_entry__.build()
    return K.load_library()


# ------------------------------------------------------------------ oracle --
def test_e4m3_of_the_oracle_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    ref = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(CO.E4M3, ref, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).normal(0, s, 20000) for s in (1e-3, 0.02, 1.0, 100.0)])
    fin = ref[np.isfinite(ref)]
    mids = (np.sort(fin)[1:] + np.sort(fin)[:-1]) / 2  # every tie
    x = np.clip(np.concatenate([x, mids, fin]), -448, 448).astype(np.float32)
    got = CO.E4M3[CO.e4m3_encode(x)]
    assert np.array_equal(got, torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    assert CO.e4m3_encode(np.array([np.nan]))[0] == 0x7F


@pytest.mark.parametrize("amax", [0.0, 1e-45, 2.0 ** -120, 1e-3, 0.4375, 447.0, 448.0, 449.0, 1.0, 3e38])
def test_scale_byte_is_the_smallest_that_fits(amax):
    e = int(CO.scale_byte(np.float32(amax)))
    a = float(np.float32(amax))
    assert CO.E_MIN <= e <= CO.E_MAX
    assert a * 2.0 ** (127 - e) <= 448
    assert e == CO.E_MIN or a * 2.0 ** (128 - e) > 448


def test_tables_of_the_oracle_hand_out_every_page_once():
    for seed in range(20):
        t = random_tables(17, 16, seed=seed, spare=[5, -4][seed % 2])
        r = CO.tables(t["lens"], t["new"], t["table"], t["ring"], t["pool"], 16, t["max_tokens"])
        held = [int(p) for s in range(17) for p in r["block_table"][s, :-(-int(r["kv_lens"][s]) // 16)]]
        free = [int(r["free_pages"][i % len(r["free_pages"])]) for i in range(r["pool"][0], r["pool"][1])]
        assert sorted(held + free) == list(range(len(t["ring"])))
        live = r["slot_map"][r["slot_map"] >= 0]
        assert len(set(live.tolist())) == len(live)
        assert (seed % 2 == 1) == bool((r["status"] == 1).any())


def test_attention_of_the_oracle_on_one_token_and_none():
    c = random_cache([1, 0], 16, 2, 16, seed=1)
    q = np.random.default_rng(0).normal(size=(3, 4, 16))
    out, lse, _, _ = CO.attention(q, c.k, c.v, c.k_scale, c.v_scale, c.table, c.kv_lens, [0, 1, 3], 0.5, 1)
    p = c.table[0, 0]
    for h in range(4):
        v = CO.E4M3[c.v[p, 0, h // 2]] * 2.0 ** (int(c.v_scale[p, h // 2]) - 127)
        k = CO.E4M3[c.k[p, 0, h // 2]] * 2.0 ** (int(c.k_scale[p, h // 2]) - 127)
        assert np.allclose(out[0, h], v) and math.isclose(lse[0, h], 0.5 * float(k @ q[0, h]), rel_tol=1e-12)
    assert not out[1:].any() and np.all(lse[1:] == -np.inf)


# --------------------------------------------------------------------- ABI --
def test_library_exports_what_the_header_declares(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(re.findall(r"^(?:int|size_t)\s+(bdkv_\w+)\s*\(", text, flags=re.M))
    assert names == ["bdkv_attention", "bdkv_attention_workspace", "bdkv_get_device_status", "bdkv_shutdown",
                     "bdkv_tables", "bdkv_write"]
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm")
    out = subprocess.run([nm, "-D", "--defined-only", K.LIB_PATH], capture_output=True, text=True).stdout
    assert sorted(l.split()[-1] for l in out.splitlines() if " T " in l) == names


def test_binding_packs_the_structures_of_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "sizes.c"
    src.write_text("""#include "bdcache.h"
#include <stdio.h>
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu %zu\\n", sizeof(bdkv_cache), sizeof(bdkv_rows), sizeof(bdkv_tables_args),
         sizeof(bdkv_attention_args), offsetof(bdkv_cache, k_stride), offsetof(bdkv_attention_args, kv_lens),
         offsetof(bdkv_attention_args, scale));
  return 0;
}
""")
    exe = tmp_path / "sizes"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    packed = K.ATTN_FIELDS.pack(*[0, 0, 0, 0] * 2, 0, 0, 0, 0, 0x1122334455667788, 0, 0, 0, 0, 0, 0, 0.5, 0, 0, 0)
    assert got[:4] == [K.CACHE_FIELDS.size, K.ROWS_FIELDS.size, K.TABLES_FIELDS.size, K.ATTN_FIELDS.size]
    assert got[5] == packed.index((0x1122334455667788).to_bytes(8, "little"))
    assert got[6] == packed.index(np.float32(0.5).tobytes())
    cache = K.CACHE_FIELDS.pack(0, 0, 0, 0, 0, 0, 0, 0, 0x1122334455667788, 0, 0, 0, 0, 0, 0, 0)
    assert got[4] == cache.index((0x1122334455667788).to_bytes(8, "little"))


# ----------------------------------------------------- argument checks --
FAKE = 1 << 20  # a non-null, aligned address that is never dereferenced


def _cache(**kw):
    f = dict(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, n_pages=4, page=16, heads=2, dim=32, kst=(1024, 64, 32),
             vst=(1024, 64, 32), kss=2, vss=2)
    f.update(kw)
    return K.CACHE_FIELDS.pack(f["k"], f["v"], f["ks"], f["vs"], f["n_pages"], f["page"], f["heads"], f["dim"],
                               *f["kst"], *f["vst"], f["kss"], f["vss"])


def _rows(data=FAKE, dtype=K.BDKV_BF16, tok=128, head=32):
    return K.ROWS_FIELDS.pack(data, dtype, tok, head)


BAD_CACHE = [(dict(page=24), BD_ERR_SHAPE), (dict(page=8), BD_ERR_SHAPE), (dict(page=512), BD_ERR_SHAPE),
             (dict(dim=0), BD_ERR_SHAPE), (dict(dim=24), BD_ERR_SHAPE), (dict(dim=144), BD_ERR_SHAPE),
             (dict(heads=0), BD_ERR_SHAPE), (dict(n_pages=-1), BD_ERR_SHAPE), (dict(kst=(1024, -64, 32)), BD_ERR_SHAPE),
             (dict(kst=(1024, 65, 32)), BD_ERR_ALIGN), (dict(vst=(1024, 64, 8)), BD_ERR_ALIGN),
             (dict(k=FAKE + 8), BD_ERR_ALIGN), (dict(v=FAKE + 1), BD_ERR_ALIGN), (dict(k=0), BD_ERR_NULL),
             (dict(vs=0), BD_ERR_NULL), (dict(kss=-2), BD_ERR_SHAPE)]


@pytest.mark.parametrize("kw,want", BAD_CACHE, ids=lambda x: str(x))
def test_bad_caches_are_refused(lib, kw, want):
    rows = _rows()
    assert lib.bdkv_write(_cache(**kw), rows, rows, FAKE, 3, None) == want
    assert lib.bdkv_attention(_cache(**kw), _attn()) == want
    assert lib.bdkv_attention_workspace(_cache(**kw), _attn()) == 0


def test_write_refusals(lib):
    ok = _rows()
    for k, v, slots, n, want in [
            (None, ok, FAKE, 3, BD_ERR_NULL), (ok, ok, None, 3, BD_ERR_NULL), (_rows(data=0), ok, FAKE, 3, BD_ERR_NULL),
            (_rows(dtype=0), ok, FAKE, 3, BD_ERR_DTYPE), (ok, _rows(dtype=K.BDKV_F16), FAKE, 3, BD_ERR_DTYPE),
            (_rows(tok=129), ok, FAKE, 3, BD_ERR_ALIGN), (ok, _rows(head=4), FAKE, 3, BD_ERR_ALIGN),
            (_rows(data=FAKE + 2), ok, FAKE, 3, BD_ERR_ALIGN), (_rows(tok=-8), ok, FAKE, 3, BD_ERR_SHAPE),
            (ok, ok, FAKE + 4, 3, BD_ERR_ALIGN), (ok, ok, FAKE, -1, BD_ERR_SHAPE),
            (ok, ok, FAKE, 1 << 31, BD_ERR_SHAPE)]:
        assert lib.bdkv_write(_cache(), k, v, slots, n, None) == want
    assert lib.bdkv_write(None, ok, ok, FAKE, 3, None) == BD_ERR_NULL
    assert lib.bdkv_write(_cache(), ok, ok, None, 0, None) == BD_OK  # nothing to store: no CUDA call


def _attn(**kw):
    f = dict(q=(FAKE, K.BDKV_BF16, 128, 32), out=(FAKE, K.BDKV_BF16, 128, 32), lse=0, table=FAKE, stride=8, blocks=8,
             lens=FAKE, starts=FAKE, n_seq=2, n_q=4, max_q=3, max_kv=100, block=1, scale=0.5, ws=0, ws_bytes=0)
    f.update(kw)
    return K.ATTN_FIELDS.pack(*f["q"], *f["out"], f["lse"], f["table"], f["stride"], f["blocks"], f["lens"],
                              f["starts"], f["n_seq"], f["n_q"], f["max_q"], f["max_kv"], f["block"], f["scale"],
                              f["ws"], f["ws_bytes"], 0)


BAD_ATTN = [(dict(n_q=5), BD_ERR_SHAPE), (dict(n_q=0), BD_ERR_SHAPE), (dict(n_q=130), BD_ERR_SHAPE),
            (dict(n_seq=-1), BD_ERR_SHAPE), (dict(n_seq=65536), BD_ERR_SHAPE), (dict(max_q=-1), BD_ERR_SHAPE),
            (dict(max_kv=-1), BD_ERR_SHAPE), (dict(max_kv=129), BD_ERR_SHAPE), (dict(stride=7), BD_ERR_SHAPE),
            (dict(block=-1), BD_ERR_ARG), (dict(scale=math.nan), BD_ERR_ARG), (dict(scale=math.inf), BD_ERR_ARG),
            (dict(q=(0, 1, 128, 32)), BD_ERR_NULL), (dict(lens=0), BD_ERR_NULL), (dict(starts=0), BD_ERR_NULL),
            (dict(table=0), BD_ERR_NULL), (dict(q=(FAKE, 2, 128, 32)), BD_ERR_DTYPE),
            (dict(out=(FAKE, K.BDKV_F16, 128, 32)), BD_ERR_DTYPE), (dict(q=(FAKE, 1, 130, 32)), BD_ERR_ALIGN),
            (dict(out=(FAKE + 8, 1, 128, 32)), BD_ERR_ALIGN), (dict(lens=FAKE + 2), BD_ERR_ALIGN),
            (dict(lse=FAKE + 1), BD_ERR_ALIGN), (dict(ws=FAKE + 64, ws_bytes=1 << 20), BD_ERR_ALIGN)]


@pytest.mark.parametrize("kw,want", BAD_ATTN, ids=lambda x: str(x))
def test_attention_refusals(lib, kw, want):
    assert lib.bdkv_attention(_cache(), _attn(**kw)) == want


def test_attention_with_nothing_to_do_queues_nothing(lib):
    assert lib.bdkv_attention(_cache(), _attn(n_seq=0, lens=0, starts=0, table=0)) == BD_OK
    assert lib.bdkv_attention(_cache(), _attn(max_q=0)) == BD_OK
    assert lib.bdkv_attention(None, _attn()) == BD_ERR_NULL
    assert lib.bdkv_attention(_cache(), None) == BD_ERR_NULL


def _tables(**kw):
    f = dict(n_seq=2, page=16, blocks=4, max_tokens=9, stride=4, ring=8, ptrs=[FAKE + 4096 * i for i in range(11)])
    f.update(kw)
    return K.TABLES_FIELDS.pack(f["n_seq"], f["page"], f["blocks"], f["max_tokens"], f["stride"], f["ring"], *f["ptrs"])


def test_tables_refusals(lib):
    ptrs = [FAKE + 4096 * i for i in range(11)]
    for kw, want in [(dict(n_seq=-1), BD_ERR_SHAPE), (dict(n_seq=8193), BD_ERR_SHAPE), (dict(page=20), BD_ERR_SHAPE),
                     (dict(blocks=-1), BD_ERR_SHAPE), (dict(stride=3), BD_ERR_SHAPE), (dict(ring=0), BD_ERR_SHAPE),
                     (dict(max_tokens=-1), BD_ERR_SHAPE)]:
        assert lib.bdkv_tables(_tables(**kw), None) == want
    for i in range(11):
        assert lib.bdkv_tables(_tables(ptrs=ptrs[:i] + [0] + ptrs[i + 1:]), None) == BD_ERR_NULL, i
        assert lib.bdkv_tables(_tables(ptrs=ptrs[:i] + [ptrs[i] + 2] + ptrs[i + 1:]), None) == BD_ERR_ALIGN, i
    assert lib.bdkv_tables(_tables(ptrs=ptrs[:5] + [ptrs[4]] + ptrs[6:]), None) == BD_ERR_ARG  # pool_out = pool_in
    assert lib.bdkv_tables(_tables(ptrs=ptrs[:6] + [ptrs[0]] + ptrs[7:]), None) == BD_ERR_ARG  # kv_lens = lens
    assert lib.bdkv_tables(None, None) == BD_ERR_NULL


def test_binding_checks_tensors_before_the_library():
    c = K.kv_cache(3, 16, 2, 32, device="cpu")
    x = torch.zeros(4, 2, 32, dtype=torch.bfloat16)
    slots = torch.zeros(4, dtype=torch.int64)
    for bad in (lambda: K.kv_write(x[:, :1], x[:, :1], slots, c), lambda: K.kv_write(x.float(), x.float(), slots, c),
                lambda: K.kv_write(x, x, slots.int(), c), lambda: K.kv_write(x[:3], x[:3], slots, c),
                lambda: K.kv_write(x.transpose(1, 2).contiguous().transpose(1, 2), x, slots, c),
                lambda: K.kv_write(x, x, slots, c._replace(k=c.k[:2])),
                lambda: K.kv_write(x, x, slots, c._replace(k_scale=c.k_scale.int()))):
        with pytest.raises(ValueError):
            bad()
    table, lens, starts = (torch.zeros(n, dtype=torch.int32) for n in ((1, 3), 1, 2))
    for bad in (dict(block_table=table.long()), dict(kv_lens=lens.long()), dict(query_start=starts[:1]),
                dict(q=x.float()), dict(q=x[:, :, :16])):
        kw = dict(dict(q=x, cache=c, block_table=table, kv_lens=lens, query_start=starts), **bad)
        with pytest.raises(ValueError):
            K.kv_attention(kw["q"], kw["cache"], kw["block_table"], kw["kv_lens"], kw["query_start"], max_q_len=1,
                           max_kv_len=16)
    assert bd_status_string(BD_ERR_SHAPE)
