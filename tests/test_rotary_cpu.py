"""Rotary positions and the latent cache without a GPU: the oracle against closed forms, the C ABI of libbdrotary.so
(symbols, layout of its structures), its argument checks, which come before any CUDA call, and the binding's."""

import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import rotary_oracle as RO
from paper_2609_33887_gb300 import kvcache as K
from paper_2609_33887_gb300 import rotary as R
from paper_2609_33887_gb300.bdcommit import (BD_ERR_ALIGN, BD_ERR_ARG, BD_ERR_DTYPE, BD_ERR_NULL, BD_ERR_SHAPE, BD_OK,
                                             BdError)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "bdrotary.h")
BF16, F16 = K.BDKV_BF16, K.BDKV_F16


@pytest.fixture(scope="module")
def lib():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("no CUDA toolkit")
    import __graft_entry__

    __graft_entry__.build()
    return R.load_library()


# ------------------------------------------------------------------ oracle --
def test_rotations_of_the_oracle_are_rotations():
    rng = np.random.default_rng(0)
    x, f = rng.normal(size=(3, 2, 40)), [1.0, 0.5, 0.01, 3.0]
    for inter in (False, True):
        y = RO.rotate(x, [0, 1, 5], f, 1.0, inter)
        assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 8:], x[..., 8:])
        a, b = ((slice(0, 8, 2), slice(1, 8, 2)) if inter else (slice(0, 4), slice(4, 8)))
        assert np.allclose(y[..., a] ** 2 + y[..., b] ** 2, x[..., a] ** 2 + x[..., b] ** 2, rtol=1e-14)
        # by 1 five times is by 5; back by 5 is where it began; the scale is a factor
        five = x[2:]
        for _ in range(5):
            five = RO.rotate(five, [1], f, 1.0, inter)
        assert np.allclose(five[0], y[2], rtol=1e-13, atol=1e-13)
        assert np.allclose(RO.rotate(y, [0, 1, 5], f, 1.0, inter, inverse=True), x, rtol=1e-14, atol=1e-14)
        assert np.allclose(RO.rotate(x, [0, 1, 5], f, 2.5, inter)[..., :8], 2.5 * y[..., :8], rtol=1e-14)
    # scores depend on distances alone
    q, k = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
    s = [float((RO.rotate(q, [p + 9], f) * RO.rotate(k, [p], f)).sum()) for p in (0, 100, 2 ** 31 - 10)]
    assert np.allclose(s, s[0], rtol=1e-11, atol=1e-11)


def test_angles_of_the_oracle_keep_far_positions():
    assert np.allclose(RO.angles([7, -3], [0.25])[:, 0], [1.75, 2 * math.pi - 0.75], rtol=1e-15)
    # 355 / 113 is pi but for 2.667641890624e-7 (355 - 113 pi = 3.0144353364053721e-5)
    assert math.isclose(RO.angles([2 * 355], [1.0])[0, 0], 2 * 3.0144353364053721e-5, rel_tol=1e-12)


def test_latent_attention_of_the_oracle_on_one_token_none_and_masks():
    rng = np.random.default_rng(1)
    latent, rope = rng.normal(size=(3, 16, 32)), rng.normal(size=(3, 16, 16))
    q = rng.normal(size=(4, 2, 48))
    out, lse, _, _ = RO.latent_attention(q, latent, rope, np.array([[1], [2], [0]]), [1, 0, 2], [0, 1, 2, 4], 0.5, 1)
    key = np.concatenate([latent[1, 0], rope[1, 0]])
    assert np.allclose(out[0], latent[1, 0][None]) and np.allclose(lse[0], 0.5 * q[0] @ key)
    assert not out[1].any() and np.all(lse[1] == -np.inf)
    assert np.allclose(out[2], latent[0, 0][None])  # the first of two causal queries
    w = np.exp(0.5 * q[3] @ np.concatenate([latent[0, :2], rope[0, :2]], 1).T)
    assert np.allclose(out[3], w @ latent[0, :2] / w.sum(1, keepdims=True))


# --------------------------------------------------------------------- ABI --
def test_library_exports_what_the_header_declares(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(re.findall(r"^(?:int|size_t)\s+(bdrot_\w+)\s*\(", text, flags=re.M))
    assert len(names) == 7
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm")
    out = subprocess.run([nm, "-D", "--defined-only", R.LIB_PATH], capture_output=True, text=True).stdout
    assert sorted(l.split()[-1] for l in out.splitlines() if " T " in l) == names


def test_binding_packs_the_structures_of_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "sizes.c"
    src.write_text("""#include "bdrotary.h"
#include <stdio.h>
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu %zu %zu\\n", sizeof(bdrot_rotary), sizeof(bdrot_latent),
         sizeof(bdrot_latent_attention_args), offsetof(bdrot_rotary, scale), offsetof(bdrot_latent, n_pages),
         offsetof(bdrot_latent, latent_stride), offsetof(bdrot_latent_attention_args, kv_lens),
         offsetof(bdrot_latent_attention_args, scale));
  return 0;
}
""")
    exe = tmp_path / "sizes"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    mark = 0x1122334455667788
    word = mark.to_bytes(8, "little")
    attn = R.LATENT_ATTN_FIELDS.pack(*[0, 0, 0, 0] * 2, 0, 0, 0, 0, mark, 0, 0, 0, 0, 0, 0, 0.5, 0, 0, 0)
    half = np.float32(0.5).tobytes()
    assert got == [R.ROTARY_FIELDS.size, R.LATENT_FIELDS.size, R.LATENT_ATTN_FIELDS.size,
                   R.ROTARY_FIELDS.pack(0, 0, 0, 0.7).index(np.float64(0.7).tobytes()), R.LATENT_FIELDS.pack(0, 0, 0, 0, mark, 0, 0, 0, 0, 0, 0).index(word),
                   R.LATENT_FIELDS.pack(0, 0, 0, 0, 0, 0, 0, mark, 0, 0, 0).index(word), attn.index(word), attn.index(half)]


# ----------------------------------------------------- argument checks --
FAKE = 1 << 20  # a non-null, aligned address that is never dereferenced


def rotary(turns=FAKE, dim=32, inter=0, scale=1.0):
    return R.ROTARY_FIELDS.pack(turns, dim, inter, scale)


def rows(data=FAKE, dtype=BF16, tok=128, head=32):
    return K.ROWS_FIELDS.pack(data, dtype, tok, head)


OUT = FAKE + (1 << 24)


def rotate(lib, rot=None, x=None, out=None, heads=4, dim=32, pos=FAKE, n=3, inverse=0):
    return lib.bdrot_rotate(rotary() if rot is None else rot, rows() if x is None else x,
                            rows(OUT) if out is None else out, heads, dim, pos, n, inverse, None)


BAD_ROTARY = [(dict(dim=0), BD_ERR_SHAPE), (dict(dim=24), BD_ERR_SHAPE), (dict(dim=272), BD_ERR_SHAPE),
              (dict(dim=48), BD_ERR_SHAPE), (dict(inter=2), BD_ERR_ARG), (dict(scale=math.nan), BD_ERR_ARG),
              (dict(scale=math.inf), BD_ERR_ARG), (dict(scale=1e39), BD_ERR_ARG),
              (dict(turns=0), BD_ERR_NULL), (dict(turns=FAKE + 8), BD_ERR_ALIGN)]


@pytest.mark.parametrize("kw,want", BAD_ROTARY, ids=str)
def test_bad_rotations_are_refused(lib, kw, want):
    assert rotate(lib, rot=rotary(**kw)) == want
    assert write(lib, rot=rotary(**kw)) == want
    assert latent_write(lib, rot=rotary(**kw)) == want


@pytest.mark.parametrize("scale", [2.0 ** -97, -2.0 ** -97, 1e-37, -5e-324])
def test_scales_whose_sines_fp32_does_not_hold_are_refused(lib, scale):
    """A sine is its angle in 2^-32 turns times scale * 2 pi / 2^32, in two fp32 terms, which lose their bits below 2^-126."""
    assert rotate(lib, rot=rotary(scale=scale)) == BD_ERR_ARG
    assert write(lib, rot=rotary(scale=scale)) == BD_ERR_ARG
    assert latent_write(lib, rot=rotary(scale=scale)) == BD_ERR_ARG
    if not torch.cuda.is_available():
        for fine in (0.0, 2.0 ** -96, -2.0 ** -96, 3e38):
            assert rotate(lib, rot=rotary(scale=fine)) not in (BD_ERR_ARG, BD_OK)


@pytest.mark.parametrize("kw,want", [
    (dict(heads=0), BD_ERR_SHAPE), (dict(heads=1025), BD_ERR_SHAPE), (dict(dim=40), BD_ERR_SHAPE), (dict(dim=1040), BD_ERR_SHAPE),
    (dict(dim=16), BD_ERR_SHAPE), (dict(n=-1), BD_ERR_SHAPE), (dict(n=1 << 31), BD_ERR_SHAPE), (dict(inverse=2), BD_ERR_ARG),
    (dict(x=rows(dtype=2)), BD_ERR_DTYPE), (dict(x=rows(dtype=F16)), BD_ERR_DTYPE), (dict(x=rows(0)), BD_ERR_NULL),
    (dict(out=rows(0)), BD_ERR_NULL), (dict(pos=0), BD_ERR_NULL), (dict(pos=FAKE + 2), BD_ERR_ALIGN),
    (dict(x=rows(FAKE + 8)), BD_ERR_ALIGN), (dict(x=rows(tok=132)), BD_ERR_ALIGN), (dict(out=rows(OUT, tok=-128)), BD_ERR_SHAPE),
    (dict(out=rows(OUT, tok=32, head=64)), BD_ERR_ARG), (dict(out=rows(OUT, tok=0)), BD_ERR_ARG), (dict(out=rows(OUT, head=16)), BD_ERR_ARG), (dict(out=rows(OUT, tok=120)), BD_ERR_ARG),
    # on x otherwise than in place
    (dict(out=rows(FAKE + 16)), BD_ERR_ARG), (dict(out=rows(FAKE + 256)), BD_ERR_ARG), (dict(out=rows(FAKE + 512)), BD_ERR_ARG),
    (dict(out=rows(FAKE - 512)), BD_ERR_ARG), (dict(out=rows(FAKE, tok=256)), BD_ERR_ARG), (dict(x=rows(tok=0), out=rows(FAKE)), BD_ERR_ARG)],
    ids=str)
def test_rotate_refusals(lib, kw, want):
    assert rotate(lib, **kw) == want


def test_rotations_that_are_apart_or_in_place_reach_the_device(lib):
    refused = (BD_ERR_ARG, BD_ERR_SHAPE, BD_ERR_ALIGN, BD_ERR_NULL, BD_ERR_DTYPE, BD_OK)
    for kw in (dict(), dict(out=rows(OUT, tok=32, head=96)), dict(out=rows(FAKE)), dict(x=rows(tok=0)), dict(x=rows(head=0)), dict(out=rows(FAKE + 768)),
               dict(x=rows(tok=256), out=rows(FAKE + 256, tok=256)),  # other heads of the same rows
               dict(x=rows(tok=512, head=64), out=rows(FAKE + 64, tok=512, head=64)),  # other elements of the same heads
               dict(x=rows(tok=0, head=0), out=rows(FAKE, tok=0, head=0), heads=1, n=1)):
        assert rotate(lib, **kw) not in refused, kw  # no device here
    assert rotate(lib, n=0, pos=0, x=rows(0), out=rows(0)) == BD_OK
    assert lib.bdrot_rotate(None, rows(), rows(OUT), 4, 32, FAKE, 3, 0, None) == BD_ERR_NULL


def test_rows_that_meet_are_found_as_a_set_of_elements_finds_them(lib):
    """Every offset, on 8-element steps, of rows over others with the same strides."""
    for tok, head, heads, n in ((64, 16, 3, 4), (16, 80, 2, 4), (120, 40, 2, 3), (24, 24, 1, 5)):
        own = {t * tok + h * head + e for t in range(n) for h in range(heads) for e in range(16)}
        for off in range(-40, 41):
            meets = any(x + 8 * off in own for x in own)
            got = rotate(lib, rot=rotary(dim=16), x=rows(tok=tok, head=head), out=rows(FAKE + 16 * off, tok=tok, head=head),
                         heads=heads, dim=16, n=n)
            assert (got == BD_ERR_ARG) == (meets and off != 0), (tok, head, off)


def cache(**kw):
    f = dict(n_pages=4, page=16, heads=2, dim=32, k=(1024, 64, 32))
    f.update(kw)
    return K.CACHE_FIELDS.pack(FAKE, FAKE, FAKE, FAKE, f["n_pages"], f["page"], f["heads"], f["dim"], *f["k"], *f["k"], 2, 2)


def write(lib, rot=None, c=None, k=None, v=None, slots=FAKE, pos=FAKE, n=3, q=None, q_out=None, n_q=0):
    return lib.bdrot_write(rotary() if rot is None else rot, cache() if c is None else c, rows() if k is None else k,
                           rows() if v is None else v, slots, pos, n, q, q_out, n_q, None)


@pytest.mark.parametrize("kw,want", [
    (dict(c=cache(page=24)), BD_ERR_SHAPE), (dict(c=cache(k=(1024, 64, 16))), BD_ERR_ARG), (dict(k=rows(dtype=F16)), BD_ERR_DTYPE),
    (dict(slots=0), BD_ERR_NULL), (dict(pos=0), BD_ERR_NULL), (dict(slots=FAKE + 4), BD_ERR_ALIGN), (dict(pos=FAKE + 1), BD_ERR_ALIGN),
    (dict(n=-1), BD_ERR_SHAPE), (dict(q=rows(OUT)), BD_ERR_NULL), (dict(q_out=rows(OUT)), BD_ERR_NULL),
    (dict(q=rows(OUT), q_out=rows(OUT), n_q=0), BD_ERR_SHAPE), (dict(q=rows(OUT, F16), q_out=rows(OUT, F16), n_q=4), BD_ERR_DTYPE),
    (dict(q=rows(OUT), q_out=rows(FAKE), n_q=4), BD_ERR_ARG), (dict(q=rows(OUT), q_out=rows(OUT + 16), n_q=4), BD_ERR_ARG)], ids=str)
def test_write_refusals(lib, kw, want):
    assert write(lib, **kw) == want


@pytest.mark.parametrize("n_k,n_q", [(2, 1), (1, 4), (1, 1), (2, 3)])
@pytest.mark.parametrize("single", [0, 8, 48, 4096])
def test_the_head_stride_of_a_single_head_says_nothing(lib, n_k, n_q, single):
    """Queries in place at every offset from keys of the same rows, on 8-element steps: refused where an element is of both."""
    if torch.cuda.is_available():
        pytest.skip("the calls would run")
    tok, dim, n = 256, 32, 3
    k = {t * tok + h * dim + e for t in range(n) for h in range(n_k) for e in range(dim)}
    q = {t * tok + h * dim + e for t in range(n) for h in range(n_q) for e in range(dim)}
    k_head, q_head = (single if heads == 1 else dim for heads in (n_k, n_q))
    for off in range(-40, 41):
        meets = any(x + 8 * off in k for x in q)
        at = rows(FAKE + 16 * off, tok=tok, head=q_head)
        got = write(lib, c=cache(heads=n_k), k=rows(tok=tok, head=k_head), v=rows(OUT, tok=tok, head=k_head), q=at, q_out=at, n_q=n_q, n=n)
        assert (got == BD_ERR_ARG) == meets and got != BD_OK, off


def test_the_binding_takes_single_heads_next_to_others(lib, monkeypatch):
    if torch.cuda.is_available():
        pytest.skip("the calls would run")
    monkeypatch.setattr(R, "_same_gpu", lambda *tensors: None)
    monkeypatch.setattr(R, "_stream_handle", lambda stream: 0)
    turn, pos, slots = R.kv_rotary(32, device="cpu"), zeros(6, dtype=torch.int32), zeros(6, dtype=torch.int64)

    def status(q, k, v):
        with pytest.raises(BdError) as e:  # no device here
            R.kv_write_rotated(k, v, slots, K.kv_cache(3, 16, k.shape[1], 32, device="cpu"), pos, turn, q=q, q_out=q)
        return e.value.status

    row = zeros(6, 5, 32)
    assert status(row[:, :1], row[:, 1:3], row[:, 3:]) != BD_ERR_ARG  # one query head, two of keys
    flat = zeros(6, 6 * 32)  # four query heads, and one of keys as [1, tokens, dim] turned round
    q, k, v = flat[:, :128].unflatten(1, (4, 32)), flat[None, :, 128:160].transpose(0, 1), flat[None, :, 160:].transpose(0, 1)
    assert k.stride(1) == 6 * 192 and status(q, k, v) != BD_ERR_ARG
    assert status(q, flat[None, :, 96:128].transpose(0, 1), v) == BD_ERR_ARG


def test_a_write_of_nothing_queues_nothing(lib):
    assert write(lib, n=0, slots=0, pos=0) == BD_OK
    assert lib.bdrot_write(None, cache(), rows(), rows(), FAKE, FAKE, 3, None, None, 0, None) == BD_ERR_NULL


def latent(**kw):
    f = dict(latent=FAKE, rope=FAKE + 128, dtype=BF16, page=16, n_pages=4, dim=64, rdim=32, ls=(1536, 96), rs=(1536, 96))
    f.update(kw)
    return R.LATENT_FIELDS.pack(f["latent"], f["rope"], f["dtype"], f["page"], f["n_pages"], f["dim"], f["rdim"], *f["ls"], *f["rs"])


def latent_write(lib, rot=None, c=None, x=None, r=None, slots=FAKE, pos=FAKE, n=3):
    return lib.bdrot_latent_write(rotary() if rot is None else rot, latent() if c is None else c, rows() if x is None else x,
                                  rows() if r is None else r, slots, pos, n, None)


BAD_LATENT = [(dict(page=24), BD_ERR_SHAPE), (dict(page=512), BD_ERR_SHAPE), (dict(dim=0), BD_ERR_SHAPE), (dict(dim=528), BD_ERR_SHAPE),
              (dict(dim=72), BD_ERR_SHAPE), (dict(rdim=8), BD_ERR_SHAPE), (dict(rdim=80), BD_ERR_SHAPE), (dict(n_pages=-1), BD_ERR_SHAPE),
              (dict(n_pages=1 << 31), BD_ERR_SHAPE), (dict(ls=(-1536, 96)), BD_ERR_SHAPE), (dict(ls=(1 << 38, 96)), BD_ERR_SHAPE),
              (dict(dtype=3), BD_ERR_DTYPE), (dict(ls=(1536, 100)), BD_ERR_ALIGN), (dict(latent=FAKE + 8), BD_ERR_ALIGN),
              (dict(rope=FAKE + 2), BD_ERR_ALIGN), (dict(latent=0), BD_ERR_NULL), (dict(rope=0), BD_ERR_NULL),
              (dict(ls=(1536, 56)), BD_ERR_ARG), (dict(ls=(0, 96)), BD_ERR_ARG), (dict(rs=(1400, 96)), BD_ERR_ARG),
              (dict(rs=(32, 96)), BD_ERR_ARG)]


@pytest.mark.parametrize("kw,want", BAD_LATENT, ids=str)
def test_bad_latent_caches_are_refused(lib, kw, want):
    assert latent_write(lib, c=latent(**kw)) == want
    assert lib.bdrot_latent_attention(latent(**kw), attn()) == want
    assert lib.bdrot_latent_attention_workspace(latent(**kw), attn()) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(rot=rotary(dim=16)), BD_ERR_SHAPE), (dict(x=rows(dtype=F16)), BD_ERR_DTYPE), (dict(r=rows(dtype=F16)), BD_ERR_DTYPE),
    (dict(x=rows(0)), BD_ERR_NULL), (dict(r=rows(0)), BD_ERR_NULL), (dict(slots=0), BD_ERR_NULL), (dict(pos=0), BD_ERR_NULL),
    (dict(slots=FAKE + 4), BD_ERR_ALIGN), (dict(pos=FAKE + 2), BD_ERR_ALIGN), (dict(x=rows(tok=100)), BD_ERR_ALIGN),
    (dict(n=-1), BD_ERR_SHAPE), (dict(c=latent(rope=FAKE + 64)), BD_ERR_ARG), (dict(c=latent(rope=FAKE)), BD_ERR_ARG),
    (dict(c=latent(rope=FAKE - 16)), BD_ERR_ARG), (dict(c=latent(rope=FAKE + 1536, rs=(1536, 32))), BD_ERR_ARG)], ids=str)
def test_latent_write_refusals(lib, kw, want):
    assert latent_write(lib, **kw) == want


def test_latent_writes_that_may_run_reach_the_device(lib):
    refused = (BD_ERR_ARG, BD_ERR_SHAPE, BD_ERR_ALIGN, BD_ERR_NULL, BD_ERR_DTYPE, BD_OK)
    for c in (latent(), latent(rope=OUT, rs=(512, 32)), latent(ls=(64, 256), rope=OUT, rs=(512, 32)),
              latent(rope=FAKE + 12288 * 4), latent(n_pages=1, ls=(0, 96), rs=(0, 96))):
        assert latent_write(lib, c=c) not in refused
    assert lib.bdrot_latent_write(None, latent(), rows(), rows(), FAKE, None, 3, None) not in refused  # nothing turned
    assert latent_write(lib, n=0, slots=0, pos=0) == BD_OK


def attn(**kw):
    f = dict(q=(FAKE, BF16, 384, 96), out=(OUT, BF16, 256, 64), lse=0, table=FAKE, stride=8, blocks=8, lens=FAKE, starts=FAKE,
             n_seq=2, heads=4, max_q=3, max_kv=100, block=1, scale=0.5, ws=0, ws_bytes=0)
    f.update(kw)
    return R.LATENT_ATTN_FIELDS.pack(*f["q"], *f["out"], f["lse"], f["table"], f["stride"], f["blocks"], f["lens"], f["starts"],
                                     f["n_seq"], f["heads"], f["max_q"], f["max_kv"], f["block"], f["scale"], f["ws"],
                                     f["ws_bytes"], 0)


@pytest.mark.parametrize("kw,want", [
    (dict(heads=0), BD_ERR_SHAPE), (dict(heads=1025), BD_ERR_SHAPE), (dict(n_seq=-1), BD_ERR_SHAPE), (dict(n_seq=65536), BD_ERR_SHAPE),
    (dict(max_q=-1), BD_ERR_SHAPE), (dict(max_q=1 << 25), BD_ERR_SHAPE), (dict(max_kv=129), BD_ERR_SHAPE), (dict(max_kv=-1), BD_ERR_SHAPE),
    (dict(blocks=1 << 30, stride=1 << 30, max_kv=(1 << 30) + 1), BD_ERR_SHAPE), (dict(stride=7), BD_ERR_SHAPE),
    (dict(block=-1), BD_ERR_ARG), (dict(scale=math.nan), BD_ERR_ARG), (dict(scale=-math.inf), BD_ERR_ARG),
    (dict(q=(0, BF16, 384, 96)), BD_ERR_NULL), (dict(out=(0, BF16, 256, 64)), BD_ERR_NULL), (dict(lens=0), BD_ERR_NULL),
    (dict(starts=0), BD_ERR_NULL), (dict(table=0), BD_ERR_NULL), (dict(q=(FAKE, 2, 384, 96)), BD_ERR_DTYPE),
    (dict(q=(FAKE, F16, 384, 96), out=(OUT, F16, 256, 64)), BD_ERR_DTYPE), (dict(out=(OUT, F16, 256, 64)), BD_ERR_DTYPE),
    (dict(q=(FAKE, BF16, 386, 96)), BD_ERR_ALIGN), (dict(out=(OUT + 8, BF16, 256, 64)), BD_ERR_ALIGN), (dict(lens=FAKE + 2), BD_ERR_ALIGN),
    (dict(lse=FAKE + 1), BD_ERR_ALIGN), (dict(ws=FAKE + 64, ws_bytes=1 << 20), BD_ERR_ALIGN),
    (dict(out=(OUT, BF16, 0, 64)), BD_ERR_ARG), (dict(out=(OUT, BF16, 256, 48)), BD_ERR_ARG), (dict(out=(OUT, BF16, 240, 64)), BD_ERR_ARG)],
    ids=str)
def test_attention_refusals(lib, kw, want):
    assert lib.bdrot_latent_attention(latent(), attn(**kw)) == want


# (q: rows of 4 heads of 64 + 32 at FAKE)
@pytest.mark.parametrize("out,meets", [((FAKE, 256, 64), True), ((FAKE, 384, 96), True), ((FAKE + 16, 384, 96), True),
                                       ((FAKE - 16, 384, 96), True), ((FAKE + 2 * 96, 384, 96), True), ((FAKE + 2 * 320, 384, 96), True),
                                       ((FAKE + 2 * 384, 384, 96), False), ((FAKE - 2 * 352, 384, 96), False),
                                       ((FAKE - 2 * 344, 384, 96), True)], ids=str)
def test_attention_onto_its_queries_is_refused(lib, out, meets):
    args = attn(out=(out[0], BF16, *out[1:]))
    if meets:
        assert lib.bdrot_latent_attention(latent(), args) == BD_ERR_ARG
    elif not torch.cuda.is_available():
        assert lib.bdrot_latent_attention(latent(), args) not in (BD_ERR_ARG, BD_OK)


def test_attention_between_its_queries_is_not(lib):
    """Rows of a head's queries and its result next to each other, 96 and 64 elements."""
    for off in range(0, 160, 8):
        args = attn(q=(FAKE, BF16, 640, 160), out=(FAKE + 2 * off, BF16, 640, 160))
        if off != 96:
            assert lib.bdrot_latent_attention(latent(), args) == BD_ERR_ARG, off
        elif not torch.cuda.is_available():
            assert lib.bdrot_latent_attention(latent(), args) not in (BD_ERR_ARG, BD_OK)


@pytest.mark.parametrize("scale", [2.4e38, -3.4e38])
def test_attention_scales_that_are_infinite_as_powers_of_two_are_refused(lib, scale):
    assert lib.bdrot_latent_attention(latent(), attn(scale=scale)) == BD_ERR_ARG
    if not torch.cuda.is_available():
        assert lib.bdrot_latent_attention(latent(), attn(scale=math.copysign(2.3e38, scale))) not in (BD_ERR_ARG, BD_OK)


def test_attention_with_nothing_to_do_queues_nothing(lib):
    assert lib.bdrot_latent_attention(latent(), attn(n_seq=0, lens=0, starts=0, table=0)) == BD_OK
    assert lib.bdrot_latent_attention(latent(), attn(max_q=0)) == BD_OK
    assert lib.bdrot_latent_attention(None, attn()) == BD_ERR_NULL
    assert lib.bdrot_latent_attention(latent(), None) == BD_ERR_NULL


# -------------------------------------------------------------------- binding --
def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_checks_tensors_before_the_library(monkeypatch):
    monkeypatch.setattr(R, "_stream_handle", lambda stream: stream or 0)
    x, pos, turn = zeros(4, 2, 32), zeros(4, dtype=torch.int32), R.kv_rotary(32, device="cpu")
    slots, c, lat = zeros(4, dtype=torch.int64), K.kv_cache(3, 16, 2, 32, device="cpu"), R.kv_latent_cache(3, 16, 64, 32, device="cpu")
    l, r = zeros(4, 64), zeros(4, 32)
    table, lens, starts = (zeros(*n, dtype=torch.int32) for n in ((1, 3), (1,), (2,)))
    q = zeros(4, 5, 96)

    def attend(**kw):
        a = dict(q=q, cache=lat, table=table, lens=lens, starts=starts, scale=1.0, max_q_len=1, max_kv_len=48)
        a.update(kw)
        return R.kv_latent_attention(a.pop("q"), a.pop("cache"), a.pop("table"), a.pop("lens"), a.pop("starts"), **a)

    for bad in (lambda: R.kv_rotate(x.float(), pos, turn), lambda: R.kv_rotate(x[0], pos, turn), lambda: R.kv_rotate(x, pos[:3], turn),
                lambda: R.kv_rotate(x, pos.long(), turn), lambda: R.kv_rotate(x, pos, turn, out=x[:, :1]),
                lambda: R.kv_rotate(x, pos, turn, out=x.half()), lambda: R.kv_rotate(x, pos, turn._replace(turns=turn.turns.int())),
                lambda: R.kv_rotate(x.transpose(1, 2), pos, turn), lambda: R.kv_rotate(x, pos, turn),  # not on a GPU
                lambda: R.kv_write_rotated(x[:3], x[:3], slots, c, pos, turn), lambda: R.kv_write_rotated(x, x, slots, c, pos[:3], turn),
                lambda: R.kv_write_rotated(x, x, slots, c, pos, turn, q=x[:3]), lambda: R.kv_write_rotated(x, x, slots, c, pos, turn, q_out=x),
                lambda: R.kv_write_rotated(x, x, slots, c, pos, turn, q=zeros(4, 2, 48)), lambda: R.kv_write_rotated(x, x, slots, c, pos, turn),
                lambda: R.kv_latent_write(l[:3], r, slots, lat), lambda: R.kv_latent_write(l, r.half(), slots, lat),
                lambda: R.kv_latent_write(l, l, slots, lat), lambda: R.kv_latent_write(l, r, slots.int(), lat),
                lambda: R.kv_latent_write(l, r, slots, lat, rotary=turn), lambda: R.kv_latent_write(l, r, slots, lat, positions=pos),
                lambda: R.kv_latent_write(l, r, slots, lat._replace(rope=lat.rope[:2])), lambda: R.kv_latent_write(l, r, slots, lat),
                lambda: attend()):
        with pytest.raises(ValueError):
            bad()
    monkeypatch.setattr(R, "_same_gpu", lambda *tensors: None)
    for kw in (dict(q=zeros(4, 5, 64)), dict(q=q.half()), dict(out=zeros(4, 5, 96)), dict(starts=starts[:1]), dict(lens=lens.long()),
               dict(table=table.long()), dict(workspace=zeros(8, 8).t()[:, :4]), dict(cache=lat._replace(rope=lat.rope.half()))):
        with pytest.raises(ValueError):
            attend(**kw)
    wide = zeros(4, 5, 160)
    for out in (q[..., :64], wide[..., 32:96], zeros(8, 5, 96)[4:, :, :64]):
        attended = wide[..., :96] if out.data_ptr() == wide[..., 32:].data_ptr() else q
        if out.data_ptr() in (q.data_ptr(), wide[..., 32:].data_ptr()):
            with pytest.raises(ValueError, match="lie on"):
                attend(q=attended, out=out)
    monkeypatch.setattr(R, "load_library", lambda: type("Library", (), {"bdrot_latent_attention": lambda *a: 0}))
    assert attend(q=wide[..., :96], out=wide[..., 96:]).shape == (4, 5, 64)  # between the rows of the queries
    for bad in (dict(dim=24), dict(dim=0), dict(dim=32, frequencies=[1.0]), dict(dim=16, frequencies=[math.nan] * 8),
                dict(dim=32, factor=0.0), dict(dim=32, factor=2.0, original_len=128, slow=4.0, fast=4.0)):
        with pytest.raises(ValueError):
            R.kv_rotary(**bad, device="cpu")


@pytest.mark.parametrize("dim,base,factor,length,slow,fast", [(64, 10000.0, 8.0, 4096, 1.0, 32.0), (128, 5e5, 40.0, 8192, 1.0, 4.0),
                                                              (96, 10000.0, 0.5, 100, 0.0, 7.5)])
def test_the_kept_share_of_a_band_grows_linearly_with_its_turns(dim, base, factor, length, slow, fast):
    """Each frequency from the definition; in the middle bands far from those of a blend by the pair's index."""
    got = R.kv_rotary(dim, base=base, factor=factor, original_len=length, slow=slow, fast=fast, device="cpu").turns.tolist()
    middle = 0
    for p, turns in enumerate(got):
        f = base ** (-2 * p / dim)
        n = length * f / (2 * math.pi)
        kept = 0.0 if n <= slow else 1.0 if n >= fast else (n - slow) / (fast - slow)
        want = (kept * f + (1 - kept) * f / factor) / (2 * math.pi) * 2.0 ** 64
        assert abs(turns % 2 ** 64 - want) <= 1e-13 * want + 0.5  # (turns are whole numbers)
        if slow > 0 and 0.05 < kept < 0.95:
            middle += 1
            by_index = math.log(n / slow) / math.log(fast / slow)
            other = (by_index * f + (1 - by_index) * f / factor) / (2 * math.pi) * 2.0 ** 64
            assert other > 1.01 * want
            # the frequencies of such a model, given as they are
            own = R.kv_rotary(16, frequencies=[other / 2.0 ** 64 * 2 * math.pi] * 8, device="cpu").turns[0].item()
            assert abs(own % 2 ** 64 - other) <= 1e-13 * other + 0.5
    assert middle >= 3 or slow == 0


@pytest.mark.parametrize("n,heads,token,head", [(3, 2, 100, 40), (3, 2, 104, 52), (3, 1, 40, 24), (1, 3, 0, 44), (1, 1, 8, 8), (2, 3, 48, 200),
                                                (4, 2, 30, 120), (3, 2, 0, 60), (3, 3, 40, 0), (5, 1, 33, 7)])
@pytest.mark.parametrize("o_single", [None, 0, 72])
def test_results_are_apart_from_queries_where_no_element_is_of_both(n, heads, token, head, o_single):
    """Every offset of results of 16 elements from queries of 24. Strides that are of a single token or head are arbitrary."""
    base = zeros(2048)

    def view(at, wide, token, head):
        return base.as_strided((n, heads, wide), (token, head, 1), at)

    def elements(at, wide):
        return {at + t * token + h * head + e for t in range(n) for h in range(heads) for e in range(wide)}

    o_token, o_head = (x if o_single is None or size > 1 else o_single for x, size in ((token, n), (head, heads)))
    for at in range(1024 - 300, 1024 + 300):
        meets = bool(elements(1024, 24) & elements(at, 16))
        try:
            R._apart(view(1024, 24, token, head), view(at, 16, o_token, o_head))
            refused = False
        except ValueError:
            refused = True
        assert refused == meets, at


def test_results_next_to_the_queries_of_a_single_head():
    row = zeros(5, 160)
    R._apart(row[:, :96].unsqueeze(1), row[:, 96:].unsqueeze(1))
    with pytest.raises(ValueError, match="lie on"):
        R._apart(row[:, :96].unsqueeze(1), row[:, 32:96].unsqueeze(1))


def test_turns_are_the_frequencies_to_the_last_bit():
    f = [1.0, 0.5, 1e-4, 6.25, -0.25, 0.0, 1e-9, 2.0]
    turns = R.kv_rotary(16, frequencies=f, device="cpu").turns.tolist()
    for x, t in zip(f, turns):
        exact = RO.Fraction(x) / (2 * RO.PI) * 2 ** 64
        assert abs((t - exact + 2 ** 63) % 2 ** 64 - 2 ** 63) <= 0.5
    assert BdError
