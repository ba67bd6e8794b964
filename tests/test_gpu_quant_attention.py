"""Attention over the quantised cache, on the GPU, against softmax in 64 bits over the same cache."""
import math

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


class Setup:
    """A cache with `lens` tokens per sequence; what no token wrote is NaN parameters, and table
    entries behind a sequence's last page are garbage."""

    def __init__(self, lens, heads, dim, bits, page, dtype, seed=0, n_pages=None, k_scale=1.0, edit=None, spare=0):
        """`spare`: entries of the block table that no length needs."""
        gen = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens_host, self.dtype, self.dim = lens, dtype, dim
        n_seq, most = len(lens), max(max(lens), 1)
        per = -(-most // page) + spare
        self.cache = civic.quant_cache(1, n_pages or n_seq * per + 3, heads, dim, page, bits, dtype, DEV)
        if n_pages is None:
            self.cache.buffer.fill_(0xFF)
        total = self.cache.n_pages
        pick = total - 1 - rng.permutation(min(total, n_seq * per + 3))[: n_seq * per]
        self.table_host = pick.reshape(n_seq, per).astype(np.int32)
        if n_pages is not None:
            self.cache.buffer[0, torch.from_numpy(pick).long().to(DEV)] = 0xFF
        self.k, self.v = (torch.randn((n_seq, most, heads, dim), generator=gen) for _ in "kv")
        self.k[..., 5] *= 6
        self.k *= k_scale
        if edit:
            edit(self.k, self.v)
        self.k, self.v = self.k.to(dtype), self.v.to(dtype)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        table = torch.from_numpy(self.table_host.copy()).to(DEV)
        civic.civic_append_kv_quant(self.k[None].to(DEV), self.v[None].to(DEV), torch.zeros_like(self.lens), self.cache, table,
                                    counts=self.lens)
        for s, n in enumerate(lens):
            self.table_host[s, -(-n // page):] = rng.choice([-1, -(2**31), 2**31 - 1, total])
        self.table = torch.from_numpy(self.table_host).to(DEV)
        self.gen = gen

    def queries(self, q_len, q_heads, scale=1.0):
        return (torch.randn((len(self.lens_host), q_len, q_heads, self.dim), generator=self.gen) * scale).to(self.dtype)

    def reader(self):
        pages = sorted({int(p) for s, n in enumerate(self.lens_host) for p in self.table_host[s, : -(-n // self.cache.page_size)]})
        small = self.cache.buffer[:, pages].cpu().numpy() if pages else np.zeros((1, 0, 1, 1), np.uint8)
        remap = {p: i for i, p in enumerate(pages)}
        read = oq.Cache(small, self.cache.page_size, self.dim, self.cache.bits, self.dtype) if pages else None
        rows = [[remap[int(p)] for p in self.table_host[s, : -(-n // self.cache.page_size)]] for s, n in enumerate(self.lens_host)]
        return read, rows


def takes_tcgen05(setup, q):
    return setup.dtype == torch.bfloat16 and setup.dim <= 128 and q.shape[1] * (q.shape[2] // setup.cache.n_heads) > 40 and \
        q.shape[:3].numel() > 2048


def many_rows(lens, q_len, q_heads):
    """`lens` with empty slots behind, so that the batch has enough query rows for the tcgen05 kernels."""
    return lens + [0] * max(0, 2049 // (q_len * q_heads) + 1 - len(lens))


def check(setup, q, out, lse, scale, causal, q_lens=None, canary=None, sample=None, wide=None):
    """Tolerance of an output element: the rounding to T (eps / 2 of it); P' rounded to fp16 (2^-11 of the
    weighted sum of s * code, which is the output without the minima), elements of P' below 2^-14 of the
    largest to 2^-25 (2^-24 of the largest s * code a token); and the scores' error d, which moves each
    weight by a factor of at most exp(2 d).  A score goes through at most 64 roundings of 2^-23 (32-bit sums
    that the matrix unit may cut instead of rounding) of partial sums below B = scale * sum |q| (s code + |m|).

    The kernels for many rows (bf16, heads up to 128) round v to fp16, by half a step of 2^-11, or by 2^-25
    against 2^-7 of the tile's largest (2^-18 of it), and weights the same way (below 2^-14 of the largest by
    2^-25).  Their scores are exact products but for K groups whose scale is below 2^-5 of the tile's largest S:
    such a scale is off by at most 2^-25 against 2^-9 (2^-16 S), a value of up to 16 of them by 2^-12 S."""
    wide = takes_tcgen05(setup, q) if wide is None else wide
    read, rows = setup.reader()
    eps = torch.finfo(setup.dtype).eps / 2
    for s, n in enumerate(setup.lens_host):
        ql = q.shape[1] if q_lens is None else q_lens[s]
        if canary is not None:
            assert bool((out[s, ql:] == canary).all()) and bool((lse[s, ql:] == canary).all())
        if n == 0:
            assert bool((out[s, :ql] == 0).all()) and bool((lse[s, :ql] == -math.inf).all())
            continue
        parts = {w: read.raw(0, w, rows[s], n) for w in "kv"}
        k, v = (oq.values(*parts[w]) for w in "kv")
        zero = lambda p: oq.values(p[0] * 0, p[1], p[2])
        vm, km = zero(parts["v"]), zero(parts["k"])
        group = q.shape[2] // k.shape[1]
        pairs = [(i, h) for i in range(ql) for h in range(q.shape[2])]
        if sample and len(pairs) > sample:
            pairs = [pairs[i] for i in np.random.default_rng(1).permutation(len(pairs))[:sample]]
        for i, h in pairs:
            seen = max(0, min(n, n - ql + i + 1)) if causal else n
            o, e = out[s, i, h].double(), float(lse[s, i, h])
            if seen == 0:
                assert bool((o == 0).all()) and e == -math.inf
                continue
            kk, vv, mm, x = k[:seen, h // group], v[:seen, h // group], vm[:seen, h // group], q[s, i, h].double()
            sc = kk @ x * scale
            w = torch.softmax(sc, 0)
            want = w @ vv
            b = float(((kk - km[:seen, h // group] + km[:seen, h // group].abs()) @ x.abs()).max() * abs(scale))
            d = 64 * 2.0**-23 * b + 2.0**-20
            codes = vv - mm
            if wide:
                tiles = -(-seen // 16) * 16  # with the tokens that share a tile with seen ones
                steps = parts["k"][1][:tiles, h // group].double().nan_to_num(0.0)
                if bool((steps < steps.max() * 2.0**-5).any()):
                    d += 2.0**-12 * float(steps.max() * x.abs().sum()) * abs(scale)
                codes = vv.abs() + 2.0**-7 * v[:tiles, h // group].abs().nan_to_num(0.0).max()
            tol = eps * want.abs() * 1.01 + 2.0**-11 * (w @ codes) + seen * 2.0**-24 * float(w.max()) * codes.amax(0) \
                + (math.exp(2 * d) - 1) * vv.abs().amax(0) + torch.finfo(setup.dtype).tiny
            off = (o - want).abs()
            assert bool((off <= tol).all()), (s, i, h, float((off / tol).max()))
            want_lse = float(torch.logsumexp(sc, 0))
            assert abs(e - want_lse) <= d + 2.0**-22 * (abs(want_lse) + float(sc.abs().max())), (s, i, h, e, want_lse, d)


def attend(setup, q, **kw):
    out, lse = civic.civic_quant_attention(q.to(DEV), setup.cache, 0, setup.table, setup.lens, want_lse=True, **kw)
    return out.cpu(), lse.cpu()


SHAPES = [  # lens, heads, q_heads, dim, bits, page, q_len, dtype
    ([1], 1, 1, 64, 4, 16, 1, torch.bfloat16),
    ([0], 2, 4, 128, 4, 16, 1, torch.bfloat16),
    ([15, 16, 17, 0, 1, 33], 2, 8, 128, 4, 16, 1, torch.bfloat16),
    ([15, 16, 17, 0, 1, 33], 2, 8, 128, 8, 32, 1, torch.bfloat16),
    ([129], 8, 32, 128, 4, 16, 1, torch.bfloat16),
    ([405, 1, 77], 8, 32, 128, 4, 64, 1, torch.float16),
    ([700, 2, 1999], 2, 14, 64, 8, 48, 5, torch.float16),
    ([300, 40], 1, 8, 64, 4, 16, 3, torch.bfloat16),
    ([300, 40], 4, 4, 64, 8, 16, 17, torch.bfloat16),
    ([513, 0, 250], 1, 5, 256, 4, 32, 1, torch.bfloat16),
    ([100, 61], 2, 6, 256, 8, 16, 7, torch.float16),
    ([260, 3], 2, 16, 128, 8, 128, 2, torch.float16),
    ([200, 90], 2, 10, 128, 4, 16, 40, torch.bfloat16),
    ([5000], 1, 7, 128, 4, 1024, 1, torch.bfloat16),
]


@pytest.mark.parametrize("case", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("spare", [0, 65])  # tables beyond 1024 tokens take the kernels that share items between blocks
def test_against_64_bits(case, causal, spare):
    lens, heads, q_heads, dim, bits, page, q_len, dtype = case
    setup = Setup(lens, heads, dim, bits, page, dtype, seed=3, spare=spare)
    q = setup.queries(q_len, q_heads)
    out, lse = attend(setup, q, causal=causal)
    check(setup, q, out, lse, dim**-0.5, causal, sample=150)
    again, lse2 = attend(setup, q, causal=causal)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


WIDE = [  # lens, heads, q_heads, dim, bits, page, q_len
    ([1], 1, 48, 128, 4, 16, 1),
    ([40], 1, 20, 64, 8, 16, 40),
    ([127, 128, 129, 0, 300], 2, 8, 128, 4, 16, 33),
    ([500, 20, 61], 2, 14, 64, 4, 48, 61),
    ([700, 257], 3, 3, 128, 8, 64, 129),
    ([1000], 2, 8, 128, 4, 32, 300),
    ([300, 299, 5], 1, 4, 64, 8, 128, 300),
    ([2500], 1, 5, 128, 8, 16, 52),
    ([513], 1, 8, 64, 4, 256, 32),
]


@pytest.mark.parametrize("case", WIDE)
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows_against_64_bits(case, causal):
    lens, heads, q_heads, dim, bits, page, q_len = case
    setup = Setup(many_rows(lens, q_len, q_heads), heads, dim, bits, page, torch.bfloat16, seed=23)
    q = setup.queries(q_len, q_heads)
    assert takes_tcgen05(setup, q)
    out, lse = attend(setup, q, causal=causal)
    check(setup, q, out, lse, dim**-0.5, causal, sample=200)
    again, lse2 = attend(setup, q, causal=causal)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    # as a whole no further off than a rounding to bf16 may be, whatever the operands' roundings add up to
    read, rows = setup.reader()
    n = lens[0]
    want, want_lse = oq.attention(q[0, -40:], *(read.rows(0, w, rows[0], n) for w in "kv"), dim**-0.5, causal)
    assert float((out[0, -40:].double() - want).norm() / want.norm()) < 2.0**-8
    seen = torch.isfinite(want_lse)
    assert float((lse[0, -40:].double() - want_lse)[seen].abs().max()) < 2.0**-14


def test_many_rows_padded_batch():
    setup = Setup([400, 130, 100, 0, 31], 2, 128, 4, 16, torch.bfloat16, seed=24)
    q = setup.queries(70, 8)
    assert takes_tcgen05(setup, q)
    for q_lens in ([70, 1, 0, 2, 64], [33, 64, 70, 0, 70], [1, 65, 64, 70, -4]):
        some = torch.tensor(q_lens, dtype=torch.int32, device=DEV)
        out = torch.full((5, 70, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((5, 70, 8), 7.0, dtype=torch.float32, device=DEV)
        civic.civic_quant_attention(q.to(DEV), setup.cache, 0, setup.table, setup.lens, q_lens=some, out=out, lse=lse)
        check(setup, q, out.cpu(), lse.cpu(), 128**-0.5, True, q_lens=[min(max(x, 0), 70) for x in q_lens], canary=7.0, sample=120)


def test_many_rows_many_items():
    rng = np.random.default_rng(25)
    lens = [int(x) for x in rng.integers(0, 200, 70)]
    lens[33] = 3000
    setup = Setup(lens, 2, 64, 4, 16, torch.bfloat16, seed=25)
    q = setup.queries(9, 12)
    assert takes_tcgen05(setup, q)
    out, lse = attend(setup, q)
    check(setup, q, out, lse, 0.125, True, sample=12)


def test_many_rows_masked_tokens_may_hold_anything():
    """NaN rows of later query tokens stay out of the earlier ones' results."""
    def edit(k, v):
        k[0, 150:], v[0, 150:] = float("nan"), float("inf")
        v[0, 145] = float("nan")

    setup = Setup(many_rows([160], 20, 8), 2, 64, 4, 16, torch.bfloat16, seed=26, edit=edit)
    q = setup.queries(20, 8)  # tokens 140 .. 159
    assert takes_tcgen05(setup, q)

    def same_rows(k, v):
        k[0], v[0] = setup.k[0, :145].float(), setup.v[0, :145].float()

    out, lse = attend(setup, q)
    clean = Setup([145], 2, 64, 4, 16, torch.bfloat16, seed=26, edit=same_rows)
    check(clean, q[:1, :5], out[:1, :5], lse[:1, :5], 0.125, True, wide=True)
    assert bool(torch.isnan(out[:1, 5:]).all()) and bool(torch.isnan(lse[:1, 10:]).all())
    assert bool((out[1:] == 0).all()) and bool((lse[1:] == -math.inf).all())


def test_many_rows_nan_in_v_stays_in_its_group_where_all_see_it():
    def edit(k, v):
        v[0, 20, 1, 40] = float("nan")

    setup = Setup(many_rows([400], 11, 8), 2, 128, 8, 16, torch.bfloat16, seed=27, edit=edit)
    q = setup.queries(11, 8)
    assert takes_tcgen05(setup, q)
    out, lse = attend(setup, q)
    assert bool(torch.isnan(out[0, :, 4:, 32:64]).all()) and bool(torch.isfinite(lse[0]).all())
    assert int(torch.isnan(out).sum()) == 11 * 4 * 32


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("kind", ["large_scores", "sink", "tiny_v", "huge_v", "tiny_q", "zero_q", "equal_rows", "uneven", "negative"])
def test_many_rows_extreme_ranges(bits, kind):
    def edit(k, v):
        if kind == "sink":
            k[:, 3] = -4.0
            v[:, 3] *= 2.0**30
        elif kind == "tiny_v":
            v *= 2.0**-70
        elif kind == "huge_v":
            v *= 2.0**70
        elif kind == "equal_rows":
            k[:], v[:] = 1.25, -3.5
        elif kind == "uneven":  # tokens of one tile that differ by far more than fp16's range allows
            size = torch.exp2(torch.randint(-30, 4, k.shape[:2] + (1, 1), generator=torch.Generator().manual_seed(1)).float())
            k *= size
            v *= size.flip(1)

    setup = Setup(many_rows([277, 20], 14, 3), 1, 64, bits, 16, torch.bfloat16, seed=28, edit=edit,
                  k_scale=8.0 if kind == "large_scores" else 1.0)
    q = setup.queries(14, 3, {"large_scores": 60.0, "tiny_q": 2.0**-110, "zero_q": 0.0}.get(kind, 1.0))
    if kind == "sink":
        q = q.abs() * 2
    scale = {"tiny_q": 2.0**105, "negative": -0.2}.get(kind, 0.125)
    assert takes_tcgen05(setup, q)
    out, lse = attend(setup, q, scale=scale)
    check(setup, q, out, lse, scale, True)


def test_many_rows_bad_pages_are_left_out():
    setup = Setup(many_rows([300], 12, 8), 2, 128, 4, 16, torch.bfloat16, seed=29)
    q = setup.queries(12, 8)
    assert takes_tcgen05(setup, q)
    for bad in (-1, setup.cache.n_pages, 2**31 - 1):
        setup.table[0, 2] = bad
        record = torch.zeros(4, dtype=torch.int32, device=DEV)
        with civic.index_check(record):
            out, lse = attend(setup, q, causal=False)
        assert record.tolist() == [3, 0, 2, bad]
        read, rows = setup.reader()
        keep = [t for t in range(300) if not 32 <= t < 48]
        k, v = (read.rows(0, w, rows[0], 300)[keep] for w in "kv")
        want, want_lse = oq.attention(q[0], k, v, 128**-0.5, False)
        assert float((out[0].double() - want).norm() / want.norm()) < 2.0**-8
        assert float((lse[0].double() - want_lse).abs().max()) < 2.0**-14


def test_many_rows_captured_and_replayed_and_on_two_streams():
    setup = Setup(many_rows([600, 290], 30, 8), 2, 128, 4, 16, torch.bfloat16, seed=30)
    n_seq = len(setup.lens_host)
    q = setup.queries(30, 8).to(DEV)
    assert takes_tcgen05(setup, q)
    out = torch.empty_like(q)
    need = civic.quant_attention_workspace_bytes(setup.cache, setup.table.shape[1], n_seq, 30, 8)
    ws = [torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(3)]
    lens = setup.lens.clone()
    run = lambda: civic.civic_quant_attention(q, setup.cache, 0, setup.table, lens, out=out, workspace=ws[0])
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for now in ([600, 290], [30, 64], [0, 289], [7, 0]):
        lens.copy_(torch.tensor(now + [0] * (n_seq - 2), dtype=torch.int32))
        out.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = civic.civic_quant_attention(q, setup.cache, 0, setup.table, lens, workspace=ws[1])
        assert torch.equal(out, want)
    lens.copy_(setup.lens)
    want, _ = civic.civic_quant_attention(q, setup.cache, 0, setup.table, lens)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [civic.civic_quant_attention(q, setup.cache, 0, setup.table, lens, workspace=ws[1 + i % 2], stream=streams[i % 2])[0]
           for i in range(12)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


@pytest.mark.parametrize("spare", [0, 65])
def test_padded_queries_and_rows_that_see_nothing(spare):
    setup = Setup([40, 3, 100, 0], 2, 128, 4, 16, torch.bfloat16, seed=4, spare=spare)
    q = setup.queries(6, 8)
    for q_lens in ([6, 5, 0, 2], [1, 6, 3, 6], [9, -2, 1, 1]):
        some = torch.tensor(q_lens, dtype=torch.int32, device=DEV)
        out = torch.full((4, 6, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((4, 6, 8), 7.0, dtype=torch.float32, device=DEV)
        civic.civic_quant_attention(q.to(DEV), setup.cache, 0, setup.table, setup.lens, q_lens=some, out=out, lse=lse)
        # sequence 1 has 3 tokens: with 5 or 6 query tokens the first ones see nothing
        check(setup, q, out.cpu(), lse.cpu(), 128**-0.5, True, q_lens=[min(max(x, 0), 6) for x in q_lens], canary=7.0)


def test_tokens_that_are_masked_may_hold_anything():
    def edit(k, v):
        k[0, 30:], v[0, 30:] = float("nan"), float("inf")

    setup = Setup([33], 2, 64, 8, 16, torch.bfloat16, seed=5, edit=edit)
    q = setup.queries(5, 4)
    out, lse = attend(setup, q)  # query tokens at 28 .. 32

    def same_rows(k, v):
        k[0], v[0] = setup.k[0, :30].float(), setup.v[0, :30].float()

    clean = Setup([30], 2, 64, 8, 16, torch.bfloat16, seed=5, edit=same_rows)
    want, want_lse = attend(clean, q[:, :2])
    assert torch.equal(out[:, :2], want) and torch.equal(lse[:, :2], want_lse)
    assert bool(torch.isnan(out[:, 2:]).all()) and bool(torch.isnan(lse[:, 2:]).all())


def test_nan_in_v_stays_in_its_group():
    def edit(k, v):
        v[0, 20, 1, 40] = float("nan")

    setup = Setup([50], 2, 128, 4, 16, torch.bfloat16, seed=6, edit=edit)
    out, lse = attend(setup, setup.queries(1, 4))
    assert bool(torch.isnan(out[0, 0, 2:, 32:64]).all()) and bool(torch.isfinite(lse).all())
    assert int(torch.isnan(out).sum()) == 64


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("kind", ["large_scores", "sink", "tiny_v", "huge_v", "tiny_q", "zero_q", "equal_rows"])
def test_extreme_ranges(bits, kind):
    def edit(k, v):
        if kind == "sink":  # a token without weight whose values are a million times the others'
            k[:, 3] = -4.0
            v[:, 3] *= 2.0**30
        elif kind == "tiny_v":
            v *= 2.0**-70
        elif kind == "huge_v":
            v *= 2.0**70
        elif kind == "equal_rows":
            k[:], v[:] = 1.25, -3.5

    setup = Setup([77, 20], 1, 64, bits, 16, torch.bfloat16, seed=7, edit=edit, k_scale=8.0 if kind == "large_scores" else 1.0)
    scale = {"large_scores": 60.0, "tiny_q": 2.0**-110, "zero_q": 0.0}.get(kind, 1.0)
    q = setup.queries(2, 3, scale)
    if kind == "sink":
        q = q.abs() * 2
    out, lse = attend(setup, q, scale=2.0**105 if kind == "tiny_q" else None)
    check(setup, q, out, lse, 2.0**105 if kind == "tiny_q" else 0.125, True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", ["large_scores", "sink", "tiny_v", "equal_rows", "flat"])
def test_extreme_ranges_in_fp16(bits, dim, kind):
    def edit(k, v):
        if kind == "sink":
            k[:, 3] = -4.0
            v[:, 3] *= 2.0**10
        elif kind == "tiny_v":  # scales among fp16's subnormals
            v *= 2.0**-12
        elif kind == "equal_rows":
            k[:], v[:] = 1.25, -3.5
        elif kind == "flat":  # scores alike: sums of many weights
            k *= 0.01

    setup = Setup([1900, 20] if kind == "flat" else [177, 20], 1, dim, bits, 16, torch.float16, seed=31, edit=edit,
                  k_scale=8.0 if kind == "large_scores" else 1.0)
    q = setup.queries(5, 5, 60.0 if kind == "large_scores" else 1.0)
    if kind == "sink":
        q = q.abs() * 2
    out, lse = attend(setup, q)
    check(setup, q, out, lse, dim**-0.5, True)


def test_strides_of_dimensions_of_size_one_do_not_matter():
    setup = Setup([50], 1, 128, 4, 16, torch.bfloat16, seed=32)
    q = setup.queries(1, 1).to(DEV)
    want, _ = civic.civic_quant_attention(q, setup.cache, 0, setup.table, setup.lens)
    odd = q.as_strided((1, 1, 1, 128), (3, 5, 7, 1))
    got, _ = civic.civic_quant_attention(odd, setup.cache, 0, setup.table, setup.lens)
    assert torch.equal(got, want)
    before = setup.cache.buffer.clone()
    x = setup.k[None, :, 40:41].to(DEV)
    start = torch.tensor([40], dtype=torch.int32, device=DEV)
    y = setup.v[None, :, 40:41].to(DEV)
    civic.civic_append_kv_quant(x.as_strided((1, 1, 1, 1, 128), (9, 3, 5, 7, 1)), y.as_strided((1, 1, 1, 1, 128), (9, 3, 5, 7, 1)),
                                start, setup.cache, setup.table)
    assert torch.equal(setup.cache.buffer, before)


def test_empty_batches():
    setup = Setup([20], 2, 128, 4, 16, torch.bfloat16, seed=33)
    before = civic.launch_count()
    none = torch.empty((0,), dtype=torch.int32, device=DEV)
    table = torch.empty((0, 4), dtype=torch.int32, device=DEV)
    out, lse = civic.civic_quant_attention(torch.empty((0, 3, 4, 128), dtype=torch.bfloat16, device=DEV), setup.cache, 0, table, none,
                                           want_lse=True)
    assert out.shape == (0, 3, 4, 128) and lse.shape == (0, 3, 4)
    out, _ = civic.civic_quant_attention(torch.empty((1, 0, 4, 128), dtype=torch.bfloat16, device=DEV), setup.cache, 0, setup.table,
                                         setup.lens)
    assert out.shape == (1, 0, 4, 128) and civic.launch_count() == before
    # a block table without entries: every sequence is empty
    out, lse = civic.civic_quant_attention(setup.queries(2, 4).to(DEV), setup.cache, 0,
                                           torch.empty((1, 0), dtype=torch.int32, device=DEV), setup.lens, want_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_q_slices_scale_and_given_buffers():
    setup = Setup([1030, 64], 2, 128, 4, 32, torch.bfloat16, seed=8)
    fused = torch.randn((2, 3, 4 + 2 + 2, 128), generator=setup.gen).to(torch.bfloat16)
    q = fused[:, :, :4]
    out = torch.empty((2, 3, 4, 128), dtype=torch.bfloat16, device=DEV)
    ws = torch.full((civic.quant_attention_workspace_bytes(setup.cache, 33, 2, 3, 4),), 0xFF, dtype=torch.uint8, device=DEV)
    got, lse = civic.civic_quant_attention(fused.to(DEV)[:, :, :4], setup.cache, 0, setup.table, setup.lens, scale=-0.2, out=out,
                                           workspace=ws)
    assert got is out and lse is None
    _, lse = attend(setup, q, scale=-0.2)
    check(setup, q, out.cpu(), lse, -0.2, True)
    head_major = q.transpose(1, 2).contiguous().to(DEV).transpose(1, 2)
    again, _ = civic.civic_quant_attention(head_major, setup.cache, 0, setup.table, setup.lens, scale=-0.2)
    assert torch.equal(again, out)


def test_bad_pages_are_left_out_and_recorded():
    setup = Setup([100], 2, 128, 4, 16, torch.bfloat16, seed=9)
    q = setup.queries(1, 8)
    good = int(setup.table_host[0, 2])
    for bad in (-1, setup.cache.n_pages, 2**31 - 1):
        setup.table[0, 2] = bad
        record = torch.zeros(4, dtype=torch.int32, device=DEV)
        with civic.index_check(record):
            out, lse = attend(setup, q, causal=False)
        assert record.tolist() == [3, 0, 2, bad]
        read, rows = setup.reader()
        keep = [t for t in range(100) if not 32 <= t < 48]
        k, v = (read.rows(0, w, rows[0], 100)[keep] for w in "kv")
        want, want_lse = oq.attention(q[0], k, v, 128**-0.5, False)
        # the tolerances of `check` at these sizes come to less
        assert float((out[0].double() - want).abs().max()) < 0.02 and float((lse[0] - want_lse).abs().max()) < 1e-3
    setup.table[0, 2] = good
    out, lse = attend(setup, q)
    check(setup, q, out, lse, 128**-0.5, True)


def test_lengths_beyond_the_table_and_below_zero():
    setup = Setup([48, 20, 31], 1, 64, 4, 16, torch.bfloat16, seed=10)
    q = setup.queries(1, 4)
    want, want_lse = attend(setup, q)
    setup.lens = torch.tensor([10**9, -3, 31], dtype=torch.int32, device=DEV)
    out, lse = attend(setup, q)
    assert torch.equal(out[0], want[0]) and torch.equal(lse[0], want_lse[0]) and torch.equal(out[2], want[2])
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())


def test_pages_beyond_four_gigabytes():
    per_page = 8 * civic.quant_tile_bytes(128, 4)
    n_pages = (1 << 32) // per_page + 5000
    setup = Setup([400, 77], 8, 128, 4, 16, torch.bfloat16, seed=11, n_pages=n_pages)
    assert int(setup.table_host[0, :25].min()) * per_page > 1 << 32
    q = setup.queries(1, 32)
    out, lse = attend(setup, q)
    check(setup, q, out, lse, 128**-0.5, True, sample=40)


def test_many_sequences_share_blocks_evenly():
    rng = np.random.default_rng(12)
    lens = [int(x) for x in rng.integers(0, 90, 150)]
    lens[60] = 2500
    setup = Setup(lens, 2, 64, 4, 16, torch.bfloat16, seed=12)
    q = setup.queries(1, 4)
    out, lse = attend(setup, q)
    check(setup, q, out, lse, 0.125, True)


@pytest.mark.parametrize("spare", [0, 60])  # short tables: a block per item; longer ones: shared items
def test_captured_and_replayed_with_new_lengths(spare):
    setup = Setup([200, 90], 2, 128, 4, 16, torch.bfloat16, seed=13, spare=spare)
    q = setup.queries(1, 8).to(DEV)
    out = torch.empty_like(q)
    ws = torch.empty(max(256, civic.quant_attention_workspace_bytes(setup.cache, 13 + spare, 2, 1, 8)), dtype=torch.uint8, device=DEV)
    lens = setup.lens.clone()
    run = lambda: civic.civic_quant_attention(q, setup.cache, 0, setup.table, lens, out=out, workspace=ws)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for now in ([200, 90], [1, 64], [0, 89], [77, 0], [200, 1]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = civic.civic_quant_attention(q, setup.cache, 0, setup.table, lens)
        assert torch.equal(out, want)


def test_two_streams_with_workspaces_of_their_own():
    setups = [Setup([900, 333], 2, 128, 4, 16, torch.bfloat16, seed=s) for s in (14, 15)]
    qs = [s.queries(1, 8).to(DEV) for s in setups]
    want = [civic.civic_quant_attention(q, s.cache, 0, s.table, s.lens)[0] for s, q in zip(setups, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in setups]
    got = []
    for _ in range(20):
        for s, q, st in zip(setups, qs, streams):
            got.append(civic.civic_quant_attention(q, s.cache, 0, s.table, s.lens, stream=st)[0])
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, want[i % 2])


def test_select_compact_append_attend_and_read_together():
    """The path as a user runs it: choose visual tokens, compact every layer's K/V into the cache, then
    decode: append a token and attend, layer by layer."""
    gen = torch.Generator().manual_seed(16)
    layers, n_seq, heads, q_heads, dim, steps = 2, 3, 2, 8, 128, 20
    desc = civic.SelectDesc(1, 8, 8, 2, 2, 1, 24)
    seq_len, text_before = 64 + 13, 5
    scores = torch.rand((n_seq, 64), generator=gen).to(DEV)
    keep, idx = civic.civic_select_seq(scores, desc, seq_len, text_before)
    k, v = (torch.randn((layers, n_seq, seq_len, heads, dim), generator=gen).to(torch.bfloat16).to(DEV) for _ in "kv")
    cache = civic.quant_cache(layers, 20, heads, dim, 16, 4, device=DEV)
    table = torch.from_numpy(np.random.default_rng(17).permutation(20)[:12].reshape(3, 4).astype(np.int32)).to(DEV)
    civic.civic_compact_kv_quant(k, v, idx, cache, table)
    kept = idx.shape[1]
    lens = torch.full((n_seq,), kept, dtype=torch.int32, device=DEV)
    news = []
    for _ in range(steps):
        kn, vn = (torch.randn((layers, n_seq, 1, heads, dim), generator=gen).to(torch.bfloat16) for _ in "kv")
        news.append((kn, vn))
        civic.civic_append_kv_quant(kn.to(DEV), vn.to(DEV), lens, cache, table)
        lens += 1
    rows = []
    for i, x in enumerate((k, v)):
        old = torch.stack([x[:, s].cpu()[:, idx[s].cpu().long()] for s in range(n_seq)], 1)
        rows.append(torch.cat([old] + [new[i] for new in news], 2))
    dense = [oq.values(*oq.quantise(x, 4)) for x in rows]
    back = [torch.zeros((layers, n_seq, kept + steps, heads, dim), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    civic.civic_read_kv_quant(cache, table, lens, *back)
    for y, x in zip(back, dense):
        # a code next to a border may differ by one step, at most a handful of them
        assert float((y.cpu().double() != x.float().bfloat16().double()).double().mean()) < 1e-4
    for layer in range(layers):
        q = torch.randn((n_seq, 1, q_heads, dim), generator=gen).to(torch.bfloat16)
        out, _ = civic.civic_quant_attention(q.to(DEV), cache, layer, table, lens)
        for s in range(n_seq):
            want, _ = oq.attention(q[s], dense[0][layer, s], dense[1][layer, s], dim**-0.5, True)
            # bf16 rounding and fp16 weights: outputs are averages of about 57 values below 5
            assert float((out[s].cpu().double() - want).abs().max()) < 2.0**-8 * 2 + 2.0**-11 * 5


def test_wrong_shapes_devices_and_types_raise():
    setup = Setup([20], 2, 128, 4, 16, torch.bfloat16, seed=18)
    q = setup.queries(1, 4).to(DEV)
    call = lambda q=q, layer=0, table=setup.table, lens=setup.lens, **kw: civic.civic_quant_attention(
        q, setup.cache, layer, table, lens, **kw)
    for kw in (dict(q=q.float()), dict(q=q.cpu()), dict(q=q[..., :64]), dict(q=q.transpose(2, 3)), dict(q=q[0]), dict(layer=1),
               dict(layer=-1), dict(table=setup.table.long()), dict(table=setup.table[0]), dict(lens=setup.lens.cpu()),
               dict(lens=setup.lens[:0]), dict(q_lens=setup.lens.float()), dict(out=torch.empty_like(q[:, :0])),
               dict(out=torch.empty_like(q).float()), dict(lse=torch.empty((1, 1, 3), device=DEV)),
               dict(lse=torch.empty((1, 1, 4), device=DEV, dtype=torch.float64))):
        with pytest.raises(ValueError):
            call(**kw)
    long_table = torch.zeros((1, 65), dtype=torch.int32, device=DEV)
    with pytest.raises(civic.CivicError):
        call(table=long_table, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(civic.CivicError):
        call(q=setup.queries(1, 5).to(DEV))
    with pytest.raises(civic.CivicError):
        call(scale=float("nan"))
    x = torch.zeros((1, 1, 4, 2, 128), dtype=torch.bfloat16, device=DEV)
    start = torch.zeros(1, dtype=torch.int32, device=DEV)
    for k, v in ((x.float(), x), (x, x.cpu()), (x[:, :, :2], x), (x[0], x), ([x[0], x[0]], [x[0], x[0]]), (x[..., :64], x[..., :64]),
                 (x.transpose(3, 4).contiguous().transpose(3, 4), x)):
        with pytest.raises(ValueError):
            civic.civic_append_kv_quant(k, v, start, setup.cache, setup.table)
    with pytest.raises(civic.CivicError):
        civic.civic_read_kv_quant(setup.cache, setup.table, start, x, x)


def test_pinned_queries_and_rows():
    """Pinned tensors may stand for device ones; what the call allocates is on the cache's device all the same."""
    setup = Setup([20, 33], 2, 128, 4, 16, torch.bfloat16, seed=19)
    q = setup.queries(2, 4)
    want, want_lse = civic.civic_quant_attention(q.to(DEV), setup.cache, 0, setup.table, setup.lens, want_lse=True)
    out, lse = civic.civic_quant_attention(q.pin_memory(), setup.cache, 0, setup.table, setup.lens, want_lse=True)
    assert out.device == lse.device == torch.device(DEV)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    own = torch.empty_like(q).pin_memory()
    out, lse = civic.civic_quant_attention(q.pin_memory(), setup.cache, 0, setup.table, setup.lens, want_lse=True, out=own)
    torch.cuda.synchronize()
    assert out is own and lse.device == torch.device(DEV)
    assert torch.equal(own, want.cpu()) and torch.equal(lse, want_lse)
    for kw in (dict(out=torch.empty_like(q)), dict(lse=torch.empty((2, 2, 4)))):
        with pytest.raises(ValueError):
            civic.civic_quant_attention(q.to(DEV), setup.cache, 0, setup.table, setup.lens, **kw)
    # one pinned layer does not vouch for the next
    cache = civic.quant_cache(2, 4, 2, 128, 16, 4, torch.bfloat16, DEV)
    start, table = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    x = torch.randn(1, 4, 2, 128).bfloat16()
    for rows in ([x.pin_memory(), x], [x.pin_memory(), x.to(DEV)], [x, x.pin_memory()]):
        with pytest.raises(ValueError):
            civic.civic_append_kv_quant(rows, [x.to(DEV)] * 2, start, cache, table)
        with pytest.raises(ValueError):
            civic.civic_append_kv_quant([x.to(DEV)] * 2, rows, start, cache, table)
    pinned = x.pin_memory()
    got = []
    for rows in ([pinned, pinned], [x.to(DEV)] * 2):
        cache.buffer.fill_(0)
        civic.civic_append_kv_quant(rows, rows, start, cache, table)
        got.append(cache.buffer.clone())
    assert torch.equal(*got)


def test_k_and_v_may_have_layer_strides_of_their_own():
    cache = civic.quant_cache(2, 4, 2, 128, 16, 4, torch.bfloat16, DEV)
    start, table = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    k = torch.randn(2, 1, 4, 2, 128, device=DEV).bfloat16()
    v = torch.randn(4, 1, 4, 2, 128, device=DEV).bfloat16()
    got = []
    for other in (v[::2], v[::2].contiguous()):
        cache.buffer.fill_(0)
        civic.civic_append_kv_quant(k, other, start, cache, table)
        got.append(cache.buffer.clone())
    assert torch.equal(*got)
    with pytest.raises(ValueError):
        civic.civic_append_kv_quant(k, v[:2, :, ::2].repeat(1, 1, 2, 1, 1)[:, :, ::2], start, cache, table)


@pytest.mark.parametrize("pages", [4, 80])
def test_results_on_another_stream_do_not_take_memory_that_the_current_one_still_writes(pages):
    setup = Setup([20, 33], 2, 128, 4, 16, torch.bfloat16, seed=33, spare=pages)
    q = setup.queries(40, 4).to(DEV)  # results of 80 KB
    want, want_lse = civic.civic_quant_attention(q, setup.cache, 0, setup.table, setup.lens, want_lse=True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    olds = [torch.empty_like(q) for _ in range(8)] + [torch.empty_like(want_lse) for _ in range(8)]
    torch.cuda._sleep(20_000_000)
    for old in olds:
        old.fill_(7.0)
    del olds, old
    out, lse = civic.civic_quant_attention(q, setup.cache, 0, setup.table, setup.lens, want_lse=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("bits", [4, 8])
def test_values_at_the_end_of_fp16_stay_finite(bits):
    """A rounded-up scale may put a group's largest value a little beyond 65504."""
    big = torch.finfo(torch.float16).max

    def edit(k, v):
        v[..., ::2], v[..., 1::2] = big, -big

    setup = Setup([20, 700], 1, 128, bits, 16, torch.float16, seed=34, edit=edit)
    q = setup.queries(3, 2)
    out, lse = attend(setup, q)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    # off by at most half a step, the weights' and sums' roundings (2^-11 and less of 65504) and the last rounding
    step = 2 * big / (15 if bits == 4 else 255) * (1 + 2.0**-10)
    want = torch.tensor([big, -big], dtype=torch.float64).repeat(64)
    assert float((out.double() - want).abs().max()) <= step / 2 + big * 2.0**-10


@pytest.mark.parametrize("q_len", [3, 300])
def test_a_query_that_is_not_finite_spoils_its_row_only(q_len):
    setup = Setup([900, 400], 2, 128, 4, 16, torch.bfloat16, seed=35)
    q = setup.queries(q_len, 8).to(DEV)
    assert takes_tcgen05(setup, q) == (q_len == 300)
    want, want_lse = attend(setup, q, causal=False)
    bad = q.clone()
    bad[0, 1, 3, 7], bad[1, 2, 0, 0], bad[1, 0, 5, 127] = float("nan"), float("inf"), float("-inf")
    got, lse = attend(setup, bad, causal=False)
    spoilt = torch.zeros(2, q_len, 8, dtype=torch.bool)
    spoilt[0, 1, 3] = spoilt[1, 2, 0] = spoilt[1, 0, 5] = True
    assert bool(torch.isnan(got[spoilt]).all()) and bool(torch.isnan(lse[spoilt]).all())
    assert bool(torch.isfinite(got).all(-1)[~spoilt].all())
    # weights of the other rows may be taken relative to another reference: a rounding of each weight (fp16) and of the result
    assert float((got[~spoilt].double() - want[~spoilt].double()).abs().max()) <= (2.0**-10 + 2.0**-8) * 8
    assert float((lse[~spoilt] - want_lse[~spoilt]).abs().max()) <= 1e-5


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128])
def test_many_rows_repeated_calls_agree(dim, bits):
    """Short items cut between blocks, thousands of them: the kernel's warps meet in many orders."""
    setup = Setup([640, 1, 14, 1024, 0], 2, dim, bits, 16, torch.bfloat16, seed=36)
    q = setup.queries(138, 66).to(DEV)
    assert takes_tcgen05(setup, q)
    want, want_lse = civic.civic_quant_attention(q, setup.cache, 0, setup.table, setup.lens, want_lse=True)
    assert bool(torch.isfinite(want).all())
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(1500):
        out, lse = civic.civic_quant_attention(q, setup.cache, 0, setup.table, setup.lens, want_lse=True)
        bad += (out != want).sum() + (lse != want_lse).sum()
    assert int(bad) == 0


def test_many_rows_of_tokens_much_smaller_than_their_tile():
    """Rows that see a tile's small tokens only: their values keep 2^-18 of the tile's largest."""
    def edit(k, v):
        v[:, ::3] *= 2.0**-7
        v[:, 1::5] *= 2.0**6

    lens, q_len, q_heads = [40, 5, 260], 40, 24
    setup = Setup(many_rows(lens, q_len, q_heads), 2, 128, 4, 16, torch.bfloat16, seed=37, edit=edit)
    q = setup.queries(q_len, q_heads)
    out, lse = attend(setup, q)
    check(setup, q, out, lse, 128**-0.5, True, sample=300)
