"""Writing rows into the quantised cache and reading them back, on the GPU, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import quant_cache as oq
from paper_2605_28115_b200 import build, civic

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    civic.load()


def filled(n_layers, n_pages, heads, dim, page, bits, dtype, byte=0xFF):
    """A cache whose every byte is `byte`: 0xFF makes every parameter a NaN."""
    cache = civic.quant_cache(n_layers, n_pages, heads, dim, page, bits, dtype, DEV)
    cache.buffer.fill_(byte)
    return cache


def tables(rng, n_seq, pages, n_pages):
    order = rng.permutation(n_pages)[: n_seq * pages].reshape(n_seq, pages)
    return torch.from_numpy(order.astype(np.int32)).to(DEV)


def read_oracle(cache):
    return oq.Cache(cache.buffer.cpu().numpy(), cache.page_size, cache.head_dim, cache.bits, cache.dtype)


def check_rows(got_raw, x, bits):
    """Codes and parameters read from a cache against rows x [n, heads, dim] (CPU, 16 bit).

    Parameters are equal.  A code may differ by one from the oracle's where the quotient is so near a
    border that fp32 cannot tell: the kernel's 1 / s is at most 2 units in the last place above the
    exact one (2^-22 relative), and x - (m - s / 2) is rounded twice (2^-24 of |x| + 2 |m| + s)."""
    codes, s, m = got_raw
    want, ws, wm = oq.quantise(x, bits)
    same = lambda a, b: torch.equal(torch.nan_to_num(a.double(), nan=-7.0), torch.nan_to_num(b.double(), nan=-7.0))
    assert same(s, ws) and same(m, wm)
    fine = torch.isfinite(ws.double()).repeat_interleave(32, -1)
    differ = (codes != want) & fine
    if bool(differ.any()):
        q = oq.quotients(x, ws, wm)
        wide = lambda p: p.double().repeat_interleave(32, -1)
        slack = 2.0**-22 * (q + 1) + 2.0**-24 * (x.double().abs() + 2 * wide(wm).abs() + wide(ws)) / wide(ws)
        border = (q + 0.5 - torch.round(q + 0.5)).abs()
        assert bool((border <= slack)[differ].all()) and bool(((codes - want).abs() == 1)[differ].all())


def touched_bytes(cache, table, positions):
    """Mask over the buffer (one layer) of the bytes that tokens `positions[s]` occupy."""
    tb, ps = oq.tile_bytes(cache.head_dim, cache.bits), cache.page_size
    mask = np.zeros((cache.n_pages, cache.n_heads, ps // 16, tb), bool)
    for which in "kv":
        byte, _, par = oq.places(cache.head_dim, cache.bits, which)
        for s, tokens in enumerate(positions):
            for t in tokens:
                page, sub, r = int(table[s, t // ps]), t % ps // 16, t % 16
                mask[page, :, sub, byte[r]] = True
                for i in range(4):
                    mask[page, :, sub, par[r] + i] = True
    return mask.reshape(cache.n_pages, cache.n_heads, -1)


def rows(gen, dtype, *shape, spread=True):
    x = torch.randn(shape, generator=gen)
    if spread:
        x = x * torch.exp2(torch.randint(-6, 7, shape[:-1] + (1,), generator=gen).float())
        x[..., 3] *= 20
    return x.to(dtype)


CASES = [  # layers, n_seq, seq_len, s_out, heads, dim, bits, page, layout, dtype
    (1, 1, 1, 1, 1, 64, 4, 16, "token", torch.bfloat16),
    (2, 3, 70, 37, 2, 128, 4, 16, "token", torch.bfloat16),
    (2, 3, 70, 37, 2, 128, 8, 32, "head", torch.bfloat16),
    (1, 2, 129, 129, 3, 64, 8, 48, "head", torch.float16),
    (3, 2, 50, 16, 1, 64, 4, 64, "list", torch.float16),
    (1, 2, 90, 33, 5, 256, 4, 128, "fused", torch.bfloat16),
    (2, 1, 40, 31, 2, 256, 8, 16, "list", torch.float16),
    (1, 4, 200, 100, 8, 128, 4, 1024, "token", torch.float16),
    (2, 2, 60, 45, 2, 128, 4, 16, "odd", torch.bfloat16),
    (1, 2, 60, 45, 2, 64, 8, 16, "odd", torch.float16),
]


@pytest.mark.parametrize("case", CASES)
def test_compaction_writes_what_the_oracle_quantises_and_nothing_else(case):
    layers, n_seq, seq_len, s_out, heads, dim, bits, page, layout, dtype = case
    gen = torch.Generator().manual_seed(hash(case[:8]) % 1000)
    rng = np.random.default_rng(5)
    k, v = (rows(gen, dtype, layers, n_seq, seq_len, heads, dim) for _ in "kv")
    idx = torch.stack([torch.randperm(seq_len, generator=gen)[:s_out].sort().values for _ in range(n_seq)]).int()
    pages = -(-s_out // page)
    cache = filled(layers, n_seq * pages + 2, heads, dim, page, bits, dtype, 0xA5)
    table = tables(rng, n_seq, pages, cache.n_pages)
    if layout == "token":
        kd, vd = k.to(DEV), v.to(DEV)
    elif layout == "head":
        kd, vd = (x.transpose(2, 3).contiguous().to(DEV).transpose(2, 3) for x in (k, v))
    elif layout == "list":
        kd, vd = [x.to(DEV) for x in k], [x.to(DEV) for x in v]
    elif layout == "odd":  # rows aligned to 16 bytes only
        kd, vd = (torch.cat([torch.zeros_like(x[..., :8]), x], 4).to(DEV)[..., 8:] for x in (k, v))
        assert kd.data_ptr() % 32 == 16 and kd.stride(3) % 16 == 8
    else:  # slices of one projection [.., 3 * heads, dim]
        both = torch.cat([torch.zeros_like(k), k, v], 3).to(DEV)
        kd, vd = both[..., heads : 2 * heads, :], both[..., 2 * heads :, :]
    civic.civic_compact_kv_quant(kd, vd, idx.to(DEV), cache, table)
    torch.cuda.synchronize()
    got, mask = read_oracle(cache), touched_bytes(cache, table.cpu(), [range(s_out)] * n_seq)
    for layer in range(layers):
        for s in range(n_seq):
            for which, x in (("k", k), ("v", v)):
                check_rows(got.raw(layer, which, table[s].cpu(), s_out), x[layer, s][idx[s].long()], bits)
        assert bool((cache.buffer[layer].cpu().numpy()[~mask] == 0xA5).all())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_groups_of_special_values(bits, dtype):
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    x = torch.zeros(24, 1, 64, dtype=dtype)
    x[1], x[2], x[3] = 1.5, -0.0, big
    x[4, 0, 5], x[5, 0, 33], x[6, 0, 0], x[7, 0, 63] = float("nan"), float("inf"), float("-inf"), float("nan")
    x[8, 0, 0], x[8, 0, 1] = big, -big
    x[9, 0, 0], x[9, 0, 1] = big / 4, -big / 4
    x[10, 0, ::2] = small
    x[11, 0, ::2] = small / 2
    x[12, 0, ::3] = small * 32
    x[13] = torch.arange(64).to(dtype)  # exact multiples of scales, quotients on borders
    x[14] = (torch.arange(64) * 0.5).to(dtype)
    x[15] = (1000 + torch.arange(64)).to(dtype)
    x[16, 0, 1::2] = -0.0
    x[17, 0, 7] = float("nan")
    x[17, 0, 8] = float("inf")
    x[18] = torch.linspace(-1, 1, 64).to(dtype)
    x[19, 0, ::2], x[20, 0, ::2] = big, -big
    x[21], x[22] = -big, big
    x[21, 0, ::2], x[22, 0, ::2] = -0.8 * big, 0.8 * big
    cache = filled(1, 2, 1, 64, 32, bits, dtype)
    table = torch.tensor([[1]], dtype=torch.int32, device=DEV)
    idx = torch.arange(24, dtype=torch.int32, device=DEV)[None]
    xd = x[None, None].to(DEV)
    civic.civic_compact_kv_quant(xd, xd, idx, cache, table)
    got = read_oracle(cache)
    for which in "kv":
        check_rows(got.raw(0, which, [1], 24), x, bits)
    # and back: the same numbers, rounded once; NaN groups stay NaN
    k, v = (torch.zeros((1, 1, 24, 1, 64), dtype=dtype, device=DEV) for _ in "kv")
    civic.civic_read_kv_quant(cache, table, torch.tensor([24], dtype=torch.int32, device=DEV), k, v)
    # (a rounded-up scale may put the largest value a little beyond the type's range)
    want = got.rows(0, "k", [1], 24).clamp(-big, big).float().to(dtype)
    for y in (k, v):
        assert torch.equal(torch.nan_to_num(y[0, 0].cpu(), nan=9.0), torch.nan_to_num(want, nan=9.0))
        assert not bool(torch.isinf(y).any())


@pytest.mark.parametrize("dim,bits,page,dtype", [(64, 4, 16, torch.float16), (128, 4, 32, torch.bfloat16),
                                                (128, 8, 16, torch.bfloat16), (256, 8, 64, torch.float16)])
def test_appending_in_pieces_equals_one_compaction(dim, bits, page, dtype):
    gen = torch.Generator().manual_seed(7)
    rng = np.random.default_rng(8)
    layers, n_seq, total, heads = 2, 3, 53, 2
    k, v = (rows(gen, dtype, layers, n_seq, total, heads, dim).to(DEV) for _ in "kv")
    pages = -(-total // page)
    a, b = (filled(layers, n_seq * pages + 1, heads, dim, page, bits, dtype, 0x3C) for _ in "ab")
    table = tables(rng, n_seq, pages, a.n_pages)
    idx = torch.arange(total, dtype=torch.int32, device=DEV).repeat(n_seq, 1)
    civic.civic_compact_kv_quant(k, v, idx, a, table)
    # pieces of different lengths for different sequences, single tokens among them
    at = torch.zeros(n_seq, dtype=torch.int32)
    steps = [[1, 7, 16], [1, 1, 0], [15, 3, 1], [2, 20, 17], [17, 0, 2], [16, 21, 16], [1, 1, 1]]
    for step in steps:
        count = torch.minimum(torch.tensor(step, dtype=torch.int32), total - at)
        n_new = max(1, int(count.max()))
        kn, vn = (torch.zeros((layers, n_seq, n_new, heads, dim), dtype=dtype, device=DEV) for _ in "kv")
        for s in range(n_seq):
            n, p = int(count[s]), int(at[s])
            kn[:, s, :n], vn[:, s, :n] = k[:, s, p : p + n], v[:, s, p : p + n]
        civic.civic_append_kv_quant(kn, vn, at.to(DEV), b, table, counts=count.to(DEV))
        at = at + count
    assert at.tolist() == [53, 53, 53]
    assert torch.equal(a.buffer, b.buffer)


def test_append_without_counts_and_what_it_leaves_alone():
    gen = torch.Generator().manual_seed(9)
    cache = filled(1, 6, 2, 128, 16, 4, torch.bfloat16, 0x77)
    table = torch.tensor([[4, 2], [0, 5], [1, -1]], dtype=torch.int32, device=DEV)
    start = torch.tensor([15, 3, 16], dtype=torch.int32, device=DEV)  # the third would need the page that is not there
    k, v = (rows(gen, torch.bfloat16, 1, 3, 2, 2, 128) for _ in "kv")
    record = torch.zeros(4, dtype=torch.int32, device=DEV)
    with civic.index_check(record):
        civic.civic_append_kv_quant(k.to(DEV), v.to(DEV), start, cache, table)
    got = read_oracle(cache)
    for s, tokens in ((0, (15, 16)), (1, (3, 4))):
        for which, x in (("k", k), ("v", v)):
            raw = [t[list(tokens)] for t in got.raw(0, which, table[s].cpu(), tokens[-1] + 1)]
            check_rows(raw, x[0, s], 4)
    mask = touched_bytes(cache, table.cpu(), [(15, 16), (3, 4)])
    assert bool((cache.buffer[0].cpu().numpy()[~mask] == 0x77).all())
    assert record.tolist() == [3, 2, 1, -1]  # CIVIC_INDEX_BAD_PAGE, sequence 2, page slot 1


@pytest.mark.parametrize("bad", [-1, 40, 2**31 - 1])
def test_source_rows_out_of_range_are_neither_read_nor_written(bad):
    gen = torch.Generator().manual_seed(10)
    cache = filled(1, 3, 1, 64, 16, 8, torch.bfloat16, 0x11)
    table = torch.tensor([[2, 0]], dtype=torch.int32, device=DEV)
    k, v = (rows(gen, torch.bfloat16, 1, 1, 40, 1, 64) for _ in "kv")
    idx = torch.arange(20, dtype=torch.int32)[None]
    idx[0, 7] = bad
    record = torch.zeros(4, dtype=torch.int32, device=DEV)
    with civic.index_check(record):
        civic.civic_compact_kv_quant(k.to(DEV), v.to(DEV), idx.to(DEV), cache, table)
    tokens = [t for t in range(20) if t != 7]
    mask = touched_bytes(cache, table.cpu(), [tokens])
    assert bool((cache.buffer[0].cpu().numpy()[~mask] == 0x11).all())
    got = read_oracle(cache)
    for which, x in (("k", k), ("v", v)):
        check_rows([t[tokens] for t in got.raw(0, which, table[0].cpu(), 20)], x[0, 0][tokens], 8)
    assert record.tolist() == [1, 0, 7, bad]


@pytest.mark.parametrize("dim,bits,page,dtype,layout", [(64, 4, 16, torch.bfloat16, "token"), (64, 8, 32, torch.float16, "head"),
                                                        (128, 4, 48, torch.float16, "fused"), (128, 8, 16, torch.bfloat16, "list"),
                                                        (256, 4, 16, torch.bfloat16, "head"), (256, 8, 16, torch.float16, "token")])
def test_reading_rows_back(dim, bits, page, dtype, layout):
    gen = torch.Generator().manual_seed(11)
    rng = np.random.default_rng(12)
    layers, n_seq, total, heads, most = 2, 4, 61, 2, 50
    k, v = (rows(gen, dtype, layers, n_seq, total, heads, dim).to(DEV) for _ in "kv")
    pages = -(-total // page)
    cache = filled(layers, n_seq * pages + 1, heads, dim, page, bits, dtype)
    table = tables(rng, n_seq, pages, cache.n_pages)
    civic.civic_compact_kv_quant(k, v, torch.arange(total, dtype=torch.int32, device=DEV).repeat(n_seq, 1), cache, table)
    oracle = read_oracle(cache)
    canary = torch.tensor(-77.0, dtype=dtype)
    for start, counts in ((None, [0, 1, 50, 17]), ([0, 16, 11, 60], [50, 7, 33, 1]), ([3, 60, 0, 5], [-5, 1, 99, 50])):
        if layout == "token":
            kd, vd = (torch.full((layers, n_seq, most, heads, dim), canary, dtype=dtype, device=DEV) for _ in "kv")
        elif layout == "head":
            kd, vd = (torch.full((layers, n_seq, heads, most, dim), canary, dtype=dtype, device=DEV).transpose(2, 3) for _ in "kv")
        elif layout == "list":
            kd, vd = ([torch.full((n_seq, most, heads, dim), canary, dtype=dtype, device=DEV) for _ in range(layers)] for _ in "kv")
        else:
            both = torch.full((layers, n_seq, most, 2 * heads, dim), canary, dtype=dtype, device=DEV)
            kd, vd = both[..., :heads, :], both[..., heads:, :]
        at = None if start is None else torch.tensor(start, dtype=torch.int32, device=DEV)
        out = civic.civic_read_kv_quant(cache, table, torch.tensor(counts, dtype=torch.int32, device=DEV), kd, vd, start=at)
        assert out[0] is kd and out[1] is vd
        for layer in range(layers):
            for s in range(n_seq):
                n, p = min(max(counts[s], 0), most), 0 if start is None else start[s]
                for which, y in (("k", kd), ("v", vd)):
                    want = torch.full((most, heads, dim), canary, dtype=dtype)
                    if n:  # s * code + m is rounded once, from the exact sum to fp32 and then to 16 bits
                        want[:n] = oracle.rows(layer, which, table[s].cpu(), p + n)[p:].float().to(dtype)
                    assert torch.equal(y[layer][s].cpu(), want)


def test_no_rows_no_launch_and_more_layers_than_one_launch_takes():
    before = civic.launch_count()
    cache = filled(83, 1, 1, 64, 16, 4, torch.bfloat16)
    table = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    empty = torch.zeros((83, 1, 0, 1, 64), dtype=torch.bfloat16, device=DEV)
    civic.civic_append_kv_quant(empty, empty, torch.zeros(1, dtype=torch.int32, device=DEV), cache, table)
    assert civic.launch_count() == before
    x = rows(torch.Generator().manual_seed(13), torch.bfloat16, 83, 1, 3, 1, 64)
    civic.civic_append_kv_quant(x.to(DEV), (x * 2).to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV), cache, table)
    assert civic.launch_count() == before + 2
    got = read_oracle(cache)
    for layer in (0, 79, 80, 82):
        check_rows(got.raw(layer, "k", [0], 3), x[layer, 0], 4)
        check_rows(got.raw(layer, "v", [0], 3), x[layer, 0] * 2, 4)
