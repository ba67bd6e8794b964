"""The quantised K/V cache without a GPU: its oracle against brute force, and what the C ABI refuses
before it launches anything."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import quant_cache as oq
from paper_2605_28115_b200 import build, civic


@pytest.fixture(scope="module")
def lib():
    build.build()
    return civic.load()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_oracle_values_are_within_half_a_step(bits, dtype):
    gen = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn((200, 64), generator=gen) * 10.0**e for e in (-3, 0, 2)]).to(dtype)
    x[0], x[1, :32], x[2, 32:] = 0.0, 3.5, -1.25
    codes, s, m = oq.quantise(x, bits)
    assert codes.min() >= 0 and codes.max() == (1 << bits) - 1
    got = oq.values(codes, s, m)
    half = (s.double() / 2).repeat_interleave(32, -1)
    assert bool(((got - x.double()).abs() <= half).all())
    # the scale is the least one of the type that spans the group
    span = (x.double().unflatten(-1, (-1, 32)).amax(-1) - m.double())
    top = (1 << bits) - 1
    assert bool((s.double() * top >= span).all())
    below = (s.view(torch.int16) - 1).view(dtype).double()
    assert bool((below * top < span)[s > 0].all())
    assert torch.equal(got[0], torch.zeros(64, dtype=torch.float64)) and bool((got[1, :32] == 3.5).all())


def test_oracle_groups_that_are_not_finite():
    x = torch.ones(5, 64, dtype=torch.bfloat16)
    x[0, 3], x[1, 40], x[2, 0], x[3, 0], x[3, 1] = float("nan"), float("inf"), float("-inf"), 3e38, -3e38
    v = oq.values(*oq.quantise(x, 4))
    for row, group in ((0, 0), (1, 1), (2, 0), (3, 0)):
        assert bool(torch.isnan(v[row, 32 * group : 32 * group + 32]).all())
        other = v[row, 32 - 32 * group : 64 - 32 * group]
        assert bool((other == 1.0).all())


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bits", [4, 8])
def test_layout_gives_every_code_a_place_of_its_own(dim, bits):
    """Codes and parameters tile the tile: every bit is used once."""
    used = np.zeros((oq.tile_bytes(dim, bits), 8), np.int64)
    for which in "kv":
        byte, shift, par = oq.places(dim, bits, which)
        for b, s in zip(byte.ravel(), shift.ravel()):
            used[b, s : s + bits] += 1
        for p in par.ravel():
            used[p : p + 4] += 1
    assert (used == 1).all()
    assert civic.quant_tile_bytes(dim, bits) == oq.tile_bytes(dim, bits)


def test_oracle_attention_matches_a_masked_softmax():
    gen = torch.Generator().manual_seed(2)
    q = torch.randn((3, 4, 8), generator=gen)
    k, v = torch.randn((2, 5, 2, 8), generator=gen, dtype=torch.float64)
    out, lse = oq.attention(q, k, v, 0.3, True)
    s = torch.einsum("ihd,jhd->hij", q.double(), k.repeat_interleave(2, 1)) * 0.3
    s = s + torch.triu(torch.full((3, 5), -np.inf, dtype=torch.float64), 3)
    want = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v.repeat_interleave(2, 1))
    assert torch.allclose(out, want, atol=1e-14) and torch.allclose(lse, torch.logsumexp(s, -1).T, atol=1e-14)
    out, lse = oq.attention(q, k[:2], v[:2], 0.3, True)
    assert bool((out[0] == 0).all()) and bool((lse[0] == -np.inf).all()) and bool(torch.isfinite(lse[1:]).all())


# ---- refusals ---------------------------------------------------------------------------------

OK, ARG, ALIGN, UNSUP, WORK = 0, 1, 4, 5, 7
GOOD = dict(n_pages=10, page_size=16, n_heads=2, head_dim=128, bits=4, dtype=0)


def desc(**kw):
    return ctypes.byref(civic.QuantDesc(*{**GOOD, **kw}.values()))


def ptrs(*at):
    return (ctypes.c_void_p * len(at))(*at)


def strides(seq=1 << 20, token=256, head=128):
    return ctypes.byref(civic.RowStrides(seq, token, head))


K, V, C, IDX, TAB = 0x10_0000_0000, 0x20_0000_0000, 0x30_0000_0000, 0x1000, 0x8000


def compact(lib, k=(K,), v=(V,), st=None, n_layers=1, n_seq=1, seq_len=40, s_out=20, idx=IDX, cache=(C,), d=None, tab=TAB,
            pages=2):
    return lib.civic_compact_kv_quant(ptrs(*k), ptrs(*v), st or strides(), n_layers, n_seq, seq_len, s_out, idx, ptrs(*cache),
                                      d or desc(), tab, pages, None)


def append(lib, k=(K,), v=(V,), st=None, n_layers=1, n_seq=1, n_new=2, start=IDX, counts=None, cache=(C,), d=None, tab=TAB,
           pages=2):
    return lib.civic_append_kv_quant(ptrs(*k), ptrs(*v), st or strides(), n_layers, n_seq, n_new, start, counts, ptrs(*cache),
                                     d or desc(), tab, pages, None)


def read(lib, k=(K,), v=(V,), st=None, n_layers=1, n_seq=1, rows=20, start=None, counts=IDX, cache=(C,), d=None, tab=TAB, pages=2):
    return lib.civic_read_kv_quant(ptrs(*cache), d or desc(), tab, pages, n_layers, n_seq, rows, start, counts, ptrs(*k), ptrs(*v),
                                   st or strides(), None)


def attend(lib, q=K, st=None, cache=C, d=None, tab=TAB, pages=2, lens=IDX, q_lens=None, n_seq=1, q_len=1, q_heads=4, scale=0.1,
           causal=1, out=V, lse=None, ws=0x40_0000_0000, ws_bytes=1 << 30):
    return lib.civic_quant_attention(q, st or strides(), cache, d or desc(), tab, pages, lens, q_lens, n_seq, q_len, q_heads,
                                     ctypes.c_float(scale), causal, out, lse, ws, ws_bytes, None)


BAD_DESC = [(dict(n_pages=0), ARG), (dict(n_heads=0), ARG), (dict(page_size=0), ARG), (dict(head_dim=-64), ARG),
            (dict(page_size=24), UNSUP), (dict(page_size=8), UNSUP), (dict(page_size=2048), UNSUP), (dict(head_dim=96), UNSUP),
            (dict(bits=5), UNSUP), (dict(dtype=2), UNSUP), (dict(n_heads=2000), UNSUP)]


@pytest.mark.parametrize("kw,status", BAD_DESC)
def test_descriptions_that_are_refused(lib, kw, status):
    before = lib.civic_launch_count()
    d = desc(**kw)
    assert lib.civic_quant_page_bytes(d) == 0
    assert lib.civic_quant_attention_workspace_bytes(d, 100, 1, 1, 4) == 0
    for call in (compact, append, read):
        assert call(lib, d=d) == status
    assert attend(lib, d=d) == status
    assert lib.civic_launch_count() == before


def test_page_bytes(lib):
    for dim in (64, 128, 256):
        for bits in (4, 8):
            assert lib.civic_quant_page_bytes(desc(head_dim=dim, bits=bits, page_size=48)) == 2 * 3 * oq.tile_bytes(dim, bits)


def test_row_calls_refuse_on_the_host(lib):
    before = lib.civic_launch_count()
    for call in (compact, append, read):
        assert call(lib, n_layers=0) == ARG
        assert call(lib, n_seq=-1) == ARG
        assert call(lib, pages=-1) == ARG
        assert call(lib, k=(None,)) == ARG
        assert call(lib, cache=(None,)) == ARG
        assert call(lib, tab=None) == ARG
        assert call(lib, tab=TAB + 2) == ALIGN
        assert call(lib, v=(V + 8,)) == ALIGN
        assert call(lib, cache=(C + 4,)) == ALIGN
        assert call(lib, st=strides(token=-256)) == ARG
        assert call(lib, st=strides(token=260)) == ALIGN
        assert call(lib, st=strides(token=1 << 50)) == UNSUP
        assert call(lib, k=(C + 16,)) == ARG  # rows inside the cache
        assert call(lib, n_seq=1 << 30, st=strides(seq=0)) in (UNSUP, ARG)
        assert call(lib, n_seq=0, k=(None,), tab=None) == OK
    assert compact(lib, idx=None) == ARG
    assert compact(lib, idx=IDX + 1) == ALIGN
    assert compact(lib, idx=C) == ARG  # the index array inside the cache
    assert compact(lib, s_out=33) == ARG  # 2 pages of 16
    assert compact(lib, seq_len=-1) == ARG
    assert compact(lib, s_out=0, idx=None) == OK
    assert compact(lib, n_layers=2, k=(K, K), v=(V, V), cache=(C, C)) == ARG  # two layers, one cache
    assert compact(lib, n_layers=2, k=(K, K), v=(V, V), cache=(C + 4096, C)) == ARG
    assert append(lib, start=None) == ARG
    assert append(lib, counts=IDX + 2) == ALIGN
    assert append(lib, n_new=0, start=None) == OK
    assert append(lib, n_new=-1) == ARG
    assert read(lib, counts=None) == ARG
    assert read(lib, v=(K,)) == ARG  # K and V into one place
    assert read(lib, st=strides(token=128, head=128)) == ARG  # rows that share places
    assert read(lib, st=strides(token=0)) == ARG
    assert read(lib, n_seq=2, st=strides(seq=256 * 10)) == ARG
    assert read(lib, counts=K + 64) == ARG  # counts inside the output
    assert read(lib, rows=0, counts=None) == OK
    assert lib.civic_launch_count() == before


def test_attention_refuses_on_the_host(lib):
    before = lib.civic_launch_count()
    assert attend(lib, q_heads=3) == ARG  # no multiple of the K/V heads
    assert attend(lib, q_heads=0) == ARG
    assert attend(lib, n_seq=-1) == ARG
    assert attend(lib, q_len=-1) == ARG
    assert attend(lib, pages=-1) == ARG
    assert attend(lib, scale=float("nan")) == ARG
    assert attend(lib, scale=float("inf")) == ARG
    assert attend(lib, q=None) == ARG
    assert attend(lib, cache=None) == ARG
    assert attend(lib, lens=None) == ARG
    assert attend(lib, out=None) == ARG
    assert attend(lib, tab=None) == ARG
    assert attend(lib, q=K + 8) == ALIGN
    assert attend(lib, lse=IDX + 2) == ALIGN
    assert attend(lib, st=strides(head=132)) == ALIGN
    assert attend(lib, ws=None, pages=100) == WORK
    assert attend(lib, ws_bytes=100, pages=100) == WORK
    assert attend(lib, ws=0x40_0000_0010, pages=100) == ALIGN
    assert attend(lib, out=K) == ARG  # over q
    assert attend(lib, out=C + 16) == ARG  # inside the cache
    assert attend(lib, lse=V) == ARG  # over out
    assert attend(lib, ws=V - 4096, pages=100) == ARG
    assert attend(lib, n_seq=70000) == UNSUP
    assert attend(lib, q_len=1 << 24) == UNSUP
    assert attend(lib, pages=1 << 28) == UNSUP
    assert attend(lib, n_seq=0, q=None, lens=None) == OK
    assert attend(lib, q_len=0, q=None, out=None) == OK
    assert lib.civic_launch_count() == before


def test_binding_refuses_wrong_tensors(lib):
    with pytest.raises(ValueError):
        civic.QuantCache(torch.zeros((1, 2, 2, 2560), dtype=torch.uint8), 16, 128, 4)  # not on a GPU
    with pytest.raises(ValueError):
        civic.QuantCache(torch.zeros((1, 2, 2, 2560), dtype=torch.uint8), 16, 128, 4, torch.float32)
    with pytest.raises(ValueError):
        civic.quant_cache(1, 2, 2, 128, page_size=20, device="cpu")
