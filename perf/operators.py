"""Work and plain forms of the quantised K/V cache: writing kept rows and new tokens into it in 4 or 8
bits, reading rows back, and attention over it.

The cache holds, for every layer, pages [n_pages, kv_heads, page_size / 16] of tiles.  A tile is 16
tokens of one K/V head: K codes, V codes, K parameters, V parameters (see `pack`).  A group is 32
consecutive channels of one row: minimum m, scale s = (max - m) / (2^bits - 1) rounded up to the
payload type, code = floor((x - m) / s + 1/2), value = s * code + m.
"""

import math

import torch

own = False

GROUP = 32
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- the cases -------------------------------------------------------------------------------


def listed():
    return [
        # one 448x448 image (196 visual tokens, 65 kept, 64 of text) compacted for every layer: the smallest prefill
        dict(name="compact_1x448_int4", op="compact", layers=36, n_seq=1, seq_len=260, s_out=129, heads=8, dim=128,
             bits=4, page=16, layout="token", dtype="bf16"),
        # sixteen 896x896 images with text, the K/V configuration of the benchmark
        dict(name="compact_16x896_int4", op="compact", layers=36, n_seq=16, seq_len=1088, s_out=405, heads=8, dim=128,
             bits=4, page=16, layout="token", dtype="bf16"),
        # four 1792x1792 images, half of the tokens kept, head-major cache tensors, 8 bits
        dict(name="compact_4x1792_int8", op="compact", layers=36, n_seq=4, seq_len=3136, s_out=1568, heads=8, dim=128,
             bits=8, page=64, layout="head", dtype="bf16"),
        # one layer of one short sequence read back, as a debugger or a cache migration does
        dict(name="read_layer_int8", op="read", layers=1, n_seq=1, max_len=1045, ragged=False, heads=8, dim=128,
             bits=8, page=32, dtype="bf16"),
        # the benchmark's whole cache read back for an engine that wants it dense
        dict(name="read_16x896_int4", op="read", layers=36, n_seq=16, max_len=405, ragged=False, heads=8, dim=128,
             bits=4, page=16, dtype="bf16"),
        # a decode step's new token of 64 sequences, one layer, read back where it went
        dict(name="append_64_tokens_int4", op="append", layers=1, n_seq=64, n_new=1, max_len=1088, heads=8, dim=128,
             bits=4, page=16, dtype="bf16"),
        # the second turn's prompt, 37 tokens at odd places for 33 sequences and all layers, heads of 64 in fp16
        dict(name="append_33x37_int8", op="append", layers=36, n_seq=33, n_new=37, max_len=777, heads=4, dim=64,
             bits=8, page=32, dtype="fp16"),
        # decoding from one compacted image: the smallest call, where latency counts
        dict(name="decode_1x129_int4", op="attend", n_seq=1, q_len=1, max_len=129, ragged=False, q_heads=32, heads=8,
             dim=128, bits=4, page=16, dtype="bf16"),
        # decoding the benchmark's sixteen compacted sequences
        dict(name="decode_16x405_int4", op="attend", n_seq=16, q_len=1, max_len=405, ragged=False, q_heads=32, heads=8,
             dim=128, bits=4, page=16, dtype="bf16"),
        # long videos: ragged lengths up to 32768 and an empty slot of a padded batch
        dict(name="decode_9x32768_int4", op="attend", n_seq=9, q_len=1, max_len=32768, ragged=True, q_heads=32, heads=8,
             dim=128, bits=4, page=64, dtype="bf16"),
        # five drafted tokens verified at once against 8-bit caches of odd lengths, heads of 64 in fp16
        dict(name="verify_48x4999_int8", op="attend", n_seq=48, q_len=5, max_len=4999, ragged=True, q_heads=28, heads=4,
             dim=64, bits=8, page=32, dtype="fp16"),
        # a second turn's prompt of 500 tokens against compacted high-resolution images
        dict(name="chunk_4x4001_int4", op="attend", n_seq=4, q_len=500, max_len=4001, ragged=False, q_heads=32, heads=8,
             dim=128, bits=4, page=16, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    common = dict(heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128, 128, 256]), bits=rng.choice([4, 4, 8]),
                  page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "bf16", "fp16"]))
    op = rng.choice(["compact", "read", "append", "attend", "attend", "attend"])
    row = common["heads"] * common["dim"]
    if op == "attend":
        kind = rng.choice(["decode", "decode", "verify", "chunk"])
        q_len = {"decode": 1, "verify": rng.randint(2, 16), "chunk": _log(rng, 17, 500)}[kind]
        n_seq = _log(rng, 1, 64)
        # visible (query row, token) pairs and cache elements stay below the largest listed cases'
        group = rng.choice([1, 2, 4, 5, 7, 8])
        pairs = 4 * 500 * 3751 * 32 * 128 // (n_seq * q_len * group * row)
        elems = 5 * 32768 * 8 * 128 // (n_seq * row)
        most = max(q_len, min(32768, pairs, elems))
        return dict(op=op, n_seq=n_seq, q_len=q_len, max_len=_log(rng, max(1, q_len), most), ragged=rng.random() < 0.5,
                    q_heads=group * common["heads"], **common)
    layers, n_seq = _log(rng, 1, 36), _log(rng, 1, 16 if op != "append" else 128)
    most = 36 * 16 * 405 * 8 * 128 // (layers * n_seq * row)
    if op == "compact":
        s_out = _log(rng, 1, min(1600, most))
        return dict(op=op, layers=layers, n_seq=n_seq, seq_len=s_out + rng.randint(0, 2 * s_out), s_out=s_out,
                    layout=rng.choice(["token", "head"]), **common)
    if op == "read":
        return dict(op=op, layers=layers, n_seq=n_seq, max_len=_log(rng, 1, min(4096, most)), ragged=rng.random() < 0.5,
                    **common)
    n_new = _log(rng, 1, min(64, most))
    return dict(op=op, layers=layers, n_seq=n_seq, n_new=n_new, max_len=_log(rng, n_new, 1600), **common)


def lens_of(case):
    """Tokens of every sequence: all alike, or from max_len down to a quarter of it with an empty slot behind."""
    n, most = case["n_seq"], case["max_len"]
    if not case.get("ragged") or n < 3:
        return [most] * n
    return [most - (3 * most // 4) * i // (n - 2) for i in range(n - 1)] + [0]


def row_bytes(case):
    """Bytes of one token's K (or V) row of all heads in the cache."""
    return case["heads"] * (case["dim"] * case["bits"] // 8 + case["dim"] // GROUP * 4)


def work(case):
    wide, narrow = case["heads"] * case["dim"] * 2, row_bytes(case)
    if case["op"] == "compact":
        rows = 2 * case["layers"] * case["n_seq"] * case["s_out"]
        return {"bytes": 2 * rows * (wide + narrow) + 4 * case["n_seq"] * case["s_out"], "flops": 0}
    if case["op"] == "read":
        rows = 2 * case["layers"] * sum(lens_of(case))
        return {"bytes": rows * (wide + narrow), "flops": 0}
    if case["op"] == "append":
        rows = 2 * case["layers"] * case["n_seq"] * case["n_new"]
        return {"bytes": 2 * rows * (wide + narrow), "flops": 0}
    lens, q_len = lens_of(case), case["q_len"]
    pairs = sum(max(0, n - q_len + i + 1) for n in lens for i in range(q_len))
    io = case["n_seq"] * q_len * case["q_heads"] * (case["dim"] * 4 + 4)
    return {"bytes": 2 * sum(lens) * narrow + io, "flops": 4 * pairs * case["q_heads"] * case["dim"]}


# ---- the plain forms -------------------------------------------------------------------------


def quantise(x, bits):
    """x [..., dim] -> codes uint8 [..., dim], scale and minimum [..., dim / 32] of x's type."""
    top = 2**bits - 1
    g = x.unflatten(-1, (-1, GROUP))
    low = g.amin(-1)
    # a divisor that is a tensor: by a plain number the GPU multiplies with its reciprocal
    step = (g.amax(-1).float() - low.float()) / torch.full_like(low, top, dtype=torch.float32)
    scale = step.to(x.dtype)
    up = (scale.view(torch.int16) + 1).view(x.dtype)
    scale = torch.where(scale.float() < step, up, scale)
    # the quotient in 64 bits: values at the border between two codes are common in 16-bit data
    at = (g.double() - low.double().unsqueeze(-1)) / scale.double().unsqueeze(-1)
    codes = torch.where(scale.unsqueeze(-1) > 0, torch.floor(at + 0.5), torch.zeros_like(at))
    return codes.to(torch.uint8).flatten(-2), scale, low


def values(codes, scale, low):
    """The numbers that codes stand for, in 32 bits."""
    g = codes.unflatten(-1, (-1, GROUP)).float()
    return (g * scale.float().unsqueeze(-1) + low.float().unsqueeze(-1)).flatten(-2)


def _bytes(x):
    return x.contiguous().view(torch.uint8)


def pack(k, v, bits):
    """(codes, scale, minimum) of K and of V, tokens padded to a multiple of 16: [..., tokens, dim] ->
    tiles uint8 [..., tokens / 16, tile bytes].

    K codes are in 32-bit words of consecutive channels of one token; word t of each of four (two in
    8 bits: twice two) groups lie together.  A V word holds consecutive channels of token a in its
    low half and the same channels of token a + 1 in its high half."""
    per = 32 // bits  # codes of a word
    lead = k[0].shape[:-2]
    n = len(lead)
    dim = k[0].shape[-1]
    words = dim // GROUP * bits // 4  # words of a lane and row
    plane = min(4, words)

    def nibbles(c):
        return c if bits == 8 else c[..., 0::2] | (c[..., 1::2] << 4)

    # K: token, group, lane of four, word of the lane, codes -> plane, token, lane, word, bytes
    c = nibbles(k[0].reshape(*lead, -1, 16, dim // GROUP, 4, 8 // per, per))
    c = c.transpose(n + 2, n + 3).reshape(*lead, -1, 16, 4, words // plane, plane, 4)
    kc = c.movedim(n + 3, n + 1).flatten(n + 1)
    # V: half, lane t, token of the pair, group, lane g, word, codes -> half, plane, g, t, word, token, bytes
    c = nibbles(v[0].reshape(*lead, -1, 2, 4, 2, dim // GROUP, 8, bits // 4, per // 2))
    i = n + 1
    c = c.permute(*range(n + 1), i, i + 3, i + 5, i + 4, i + 1, i + 2, i + 6)
    c = c.reshape(*lead, -1, 2, words // plane, plane, 8, 4, 2, 2)
    vc = c.permute(*range(n + 1), i, i + 1, i + 3, i + 4, i + 2, i + 5, i + 6).flatten(n + 1)
    par = [_bytes(torch.stack((x[1], x[2]), -1).reshape(*lead, -1, 16, dim // GROUP * 2)).flatten(n + 1) for x in (k, v)]
    return torch.cat([kc, vc] + par, -1)


def unpack(tiles, dim, bits, dtype):
    """The inverse of `pack`: ((codes, scale, minimum) of K, the same of V)."""
    per, groups = 32 // bits, dim // GROUP
    words = groups * bits // 4
    plane = min(4, words)
    lead, n = tiles.shape[:-2], tiles.dim() - 2
    cb, pb = 16 * dim * bits // 8, 16 * groups * 4
    kc, vc, kp, vp = tiles.split([cb, cb, pb, pb], -1)

    def codes(c):
        return c if bits == 8 else torch.stack((c & 15, c >> 4), -1).flatten(-2)

    i = n + 1
    c = kc.reshape(*lead, -1, words // plane, 16, 4, plane, 4).movedim(i, i + 2)
    c = codes(c.reshape(*lead, -1, 16, 4, groups, bits // 4, 4)).transpose(i + 1, i + 2)
    kc = c.reshape(*lead, -1, dim)
    c = vc.reshape(*lead, -1, 2, words // plane, 8, 4, plane, 2, 2)
    c = c.permute(*range(i), i, i + 1, i + 4, i + 2, i + 3, i + 5, i + 6).reshape(*lead, -1, 2, groups, bits // 4, 8, 4, 2, 2)
    c = codes(c.permute(*range(i), i, i + 4, i + 5, i + 1, i + 3, i + 2, i + 6))
    vc = c.reshape(*lead, -1, dim)
    out = []
    for c, p in ((kc, kp), (vc, vp)):
        p = p.contiguous().view(dtype).reshape(*lead, -1, groups, 2)
        out.append((c, p[..., 0], p[..., 1]))
    return out


def rows(buffer, table, dim, bits, dtype):
    """Cached rows in 32 bits through the block table: buffer [..., n_pages, heads, page bytes], table
    [n_seq, pages] -> K and V [..., n_seq, heads, tokens, dim]."""
    groups = dim // GROUP
    tile = 2 * (16 * dim * bits // 8 + 16 * groups * 4)
    got = buffer[..., table.clamp(min=0).long(), :, :]  # [..., n_seq, pages, heads, bytes]
    got = got.transpose(-3, -2).unflatten(-1, (-1, tile)).flatten(-3, -2)
    return [values(*x) for x in unpack(got, dim, bits, dtype)]


# ---- inputs ----------------------------------------------------------------------------------


def _pages(case):
    most = max(case.get("max_len", 0) + case.get("n_new", 0), case.get("s_out", 0))
    return -(-most // case["page"])


def _table(case, gen, n_pages):
    """Every sequence's pages in an arbitrary order of the pool; -1 behind a sequence's last page."""
    per = _pages(case)
    order = torch.randperm(n_pages, generator=gen, device="cuda")[: case["n_seq"] * per]
    return order.to(torch.int32).reshape(case["n_seq"], per).contiguous()


def _kv(gen, dtype, *shape):
    """K rows with a few channels that stand out, as keys have them, and V rows."""
    k = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
    stand = torch.where(torch.rand((shape[-1],), generator=gen, device="cuda") < 0.05, 6.0, 1.0).to(dtype)
    return k.mul_(stand), torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _cache(case, gen, layers, table, n_pages):
    """A cache [layers, n_pages, heads, page bytes] whose pages in the table hold quantised rows."""
    bits, dim, page, dtype = case["bits"], case["dim"], case["page"], TYPES[case["dtype"]]
    pages = table.flatten().long()
    groups = dim // GROUP
    tile = 2 * (16 * dim * bits // 8 + 16 * groups * 4)
    buffer = torch.zeros((layers, n_pages, case["heads"], page // 16 * tile), dtype=torch.uint8, device="cuda")
    for layer in range(layers):
        k, v = _kv(gen, dtype, pages.numel(), case["heads"], page, dim)
        buffer[layer, pages] = pack(quantise(k, bits), quantise(v, bits), bits).flatten(-2)
    return buffer


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, n_seq, heads, dim = TYPES[case["dtype"]], case["n_seq"], case["heads"], case["dim"]
    n_pages = n_seq * _pages(case) + 3
    table = _table(case, gen, n_pages)
    state = dict(case=case, table=table)
    if case["op"] == "compact":
        # sources as a prefill leaves them, token-major or head-major, and the kept rows' numbers
        seq_len, s_out = case["seq_len"], case["s_out"]
        shape = (seq_len, heads) if case["layout"] == "token" else (heads, seq_len)
        k, v = _kv(gen, dtype, case["layers"], n_seq, *shape, dim)
        if case["layout"] == "head":
            k, v = k.transpose(2, 3), v.transpose(2, 3)
        order = torch.rand((n_seq, seq_len), generator=gen, device="cuda").argsort(-1)[:, :s_out]
        state.update(k=k, v=v, idx=order.sort(-1).values.to(torch.int32))
        state["lens"] = torch.full((n_seq,), s_out, dtype=torch.int32, device="cuda")
        state["cache"] = _empty(case, case["layers"], n_pages)
    elif case["op"] == "append":
        k, v = _kv(gen, dtype, case["layers"], n_seq, case["n_new"], heads, dim)
        # the sequences have grown to different lengths
        start = torch.randint(0, case["max_len"] + 1, (n_seq,), generator=gen, device="cuda", dtype=torch.int32)
        state.update(k=k, v=v, start=start)
        state["lens"] = torch.full((n_seq,), case["n_new"], dtype=torch.int32, device="cuda")
        state["cache"] = _empty(case, case["layers"], n_pages)
    else:
        state["lens"] = torch.tensor(lens_of(case), dtype=torch.int32, device="cuda")
        state["cache"] = _cache(case, gen, case.get("layers", 1), table, n_pages)
    if case["op"] == "attend":
        state["q"] = torch.randn((n_seq, case["q_len"], case["q_heads"], dim), generator=gen, device="cuda", dtype=dtype)
    else:
        most = case["max_len"] if case["op"] == "read" else case["s_out"] if case["op"] == "compact" else case["n_new"]
        state["out"] = [torch.zeros((case["layers"], n_seq, most, heads, dim), dtype=dtype, device="cuda") for _ in "kv"]
    return state


def _empty(case, layers, n_pages):
    tile = 2 * (16 * case["dim"] * case["bits"] // 8 + 16 * case["dim"] // GROUP * 4)
    return torch.zeros((layers, n_pages, case["heads"], case["page"] // 16 * tile), dtype=torch.uint8, device="cuda")


# ---- one pass --------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    if own:
        return run_own(state, case)
    bits, dim, dtype = case["bits"], case["dim"], TYPES[case["dtype"]]
    if case["op"] == "compact":
        # what the cache holds of the kept rows, as the values the codes stand for
        at = state["idx"].long()[None, :, :, None, None].expand(case["layers"], -1, -1, case["heads"], dim)
        return [values(*quantise(state[x].gather(2, at), bits)).to(dtype) for x in ("k", "v")]
    if case["op"] == "append":
        return [values(*quantise(state[x], bits)).to(dtype) for x in ("k", "v")]
    if case["op"] == "read":
        most, lens = case["max_len"], state["lens"]
        seen = (torch.arange(most, device=lens.device)[None] < lens[:, None])[None, :, :, None, None]
        got = rows(state["cache"], state["table"], dim, bits, dtype)
        return [torch.where(seen, x.transpose(2, 3)[:, :, :most], torch.zeros_like(x[:1, :1, :1, :1])).to(dtype) for x in got]
    k, v = rows(state["cache"][0], state["table"], dim, bits, dtype)  # [n_seq, heads, tokens, dim]
    n_seq, q_len, q_heads, _ = state["q"].shape
    q = state["q"].float().reshape(n_seq, q_len, case["heads"], -1, dim).permute(0, 2, 3, 1, 4).flatten(2, 3)
    s = (q @ k.transpose(-1, -2)) / math.sqrt(dim)  # [n_seq, heads, group * q_len, tokens]
    last = state["lens"][:, None] - q_len + 1 + torch.arange(q_len, device=q.device)[None]  # tokens a query row sees
    seen = torch.arange(k.shape[2], device=q.device)[None, None] < last[:, :, None]
    seen = seen[:, None, None].expand(-1, -1, q_heads // case["heads"], -1, -1).flatten(2, 3)
    s = s.masked_fill(~seen, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).squeeze(-1)
    split = (n_seq, case["heads"], -1, q_len)
    out = out.reshape(*split, dim).permute(0, 3, 1, 2, 4).reshape(n_seq, q_len, q_heads, dim)
    return out.to(dtype), lse.reshape(*split).permute(0, 3, 1, 2).reshape(n_seq, q_len, q_heads)


def run_own(state, case):
    from paper_2605_28115_b200 import civic

    cache = civic.QuantCache(state["cache"], case["page"], case["dim"], case["bits"], TYPES[case["dtype"]])
    if case["op"] == "compact":
        civic.civic_compact_kv_quant(state["k"], state["v"], state["idx"], cache, state["table"])
        return civic.civic_read_kv_quant(cache, state["table"], state["lens"], *state["out"])
    if case["op"] == "append":
        civic.civic_append_kv_quant(state["k"], state["v"], state["start"], cache, state["table"])
        return civic.civic_read_kv_quant(cache, state["table"], state["lens"], *state["out"], start=state["start"])
    if case["op"] == "read":
        return civic.civic_read_kv_quant(cache, state["table"], state["lens"], *state["out"])
    return civic.civic_quant_attention(state["q"], cache, 0, state["table"], state["lens"], causal=True, want_lse=True)


# ---- the same in 64 bits, from the definition ------------------------------------------------


def _round_trip64(x, bits):
    """Values that 16-bit rows have after quantisation, one group a row, in 64 bits throughout."""
    flat = x.reshape(-1, GROUP)
    g = flat.to(torch.float64)
    low, high = g.min(1, keepdim=True).values, g.max(1, keepdim=True).values
    step = (high - low).div(torch.full_like(low, (1 << bits) - 1))
    # the least number of the payload type that is not below the step
    near = step.to(x.dtype)
    above = (near.view(torch.int16) + 1).view(x.dtype)  # the next larger one, for numbers >= 0
    near = torch.where(near.to(torch.float64) < step, above, near).to(torch.float64)
    code = torch.where(near > 0, ((g - low) / near + 0.5).floor(), torch.zeros_like(g))
    return (low + near * code).reshape(x.shape)


def _cached64(tiles, dim, bits, dtype, token, which):
    """One token's K (which = 0) or V (which = 1) rows in 64 bits, read element by element from tiles
    uint8 [..., tile bytes] by the layout's definition: where each channel's code and parameters lie."""
    groups = dim // GROUP
    cb, pb = 16 * dim * bits // 8, 64 * groups
    words = groups * bits // 4
    plane = min(4, words)
    ch = torch.arange(dim, device=tiles.device)
    j, r = ch // GROUP, ch % GROUP
    per = 32 // bits
    if which == 0:
        word, place = j * (bits // 4) + (r % 8) // per, r % per
        at = (((word // plane) * 16 + token) * 4 + r // 8) * plane + word % plane
        byte, low = at * 4 + place * bits // 8, (place * bits) % 8
    else:
        word, place = j * (bits // 4) + (r % 4) // (per // 2), r % (per // 2)
        lane = (r // 4) * 4 + (token % 8) // 2
        at = (((token // 8) * (words // plane) + word // plane) * 32 + lane) * plane + word % plane
        byte, low = cb + at * 4 + (token % 2) * 2 + place * bits // 8, (place * bits) % 8
    code = (tiles[..., byte].to(torch.int32) >> low.to(torch.int32)) & ((1 << bits) - 1)
    par = tiles[..., 2 * cb + which * pb + token * groups * 4 : 2 * cb + which * pb + (token + 1) * groups * 4]
    par = par.contiguous().view(dtype).to(torch.float64)
    return code.to(torch.float64) * par[..., 0::2][..., j] + par[..., 1::2][..., j]


def _rows64(buffer, pages, dim, bits, dtype):
    """K and V [heads, tokens, dim] in 64 bits of one sequence's pages of one layer."""
    tile = 2 * (16 * dim * bits // 8 + 64 * (dim // GROUP))
    tiles = buffer[pages.long()].reshape(pages.numel(), buffer.shape[1], -1, tile)  # page, head, tile, bytes
    both = []
    for which in (0, 1):
        x = torch.stack([_cached64(tiles, dim, bits, dtype, t, which) for t in range(16)], 3)  # page, head, tile, token, dim
        both.append(x.permute(1, 0, 2, 3, 4).reshape(buffer.shape[1], -1, dim))
    return both


def exact(case, seed):
    state = prepare(case, seed)
    bits, dim, dtype = case["bits"], case["dim"], TYPES[case["dtype"]]
    if case["op"] in ("compact", "append"):
        out = []
        for src in (state["k"], state["v"]):
            got = []
            for layer in src:
                if case["op"] == "compact":
                    layer = torch.stack([layer[s][state["idx"][s].long()] for s in range(case["n_seq"])])
                got.append(_round_trip64(layer, bits))
            out.append(torch.stack(got))
        return out
    lens = lens_of(case)
    if case["op"] == "read":
        out = [torch.zeros(state["out"][0].shape, dtype=torch.float64, device="cuda") for _ in "kv"]
        for layer in range(case["layers"]):
            for s, n in enumerate(lens):
                for o, x in zip(out, _rows64(state["cache"][layer], state["table"][s], dim, bits, dtype)):
                    o[layer, s, :n] = x[:, :n].transpose(0, 1)
        return out
    n_seq, q_len, q_heads, _ = state["q"].shape
    out = torch.zeros((n_seq, q_len, q_heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((n_seq, q_len, q_heads), float("-inf"), dtype=torch.float64, device="cuda")
    group = q_heads // case["heads"]
    for s, n in enumerate(lens):
        if n == 0:
            continue
        k, v = _rows64(state["cache"][0], state["table"][s], dim, bits, dtype)
        visible = n - q_len + 1 + torch.arange(q_len, device="cuda")
        hidden = torch.arange(n, device="cuda")[None] >= visible[:, None]
        for h in range(q_heads):
            x = state["q"][s, :, h].double() @ k[h // group, :n].T / math.sqrt(dim)
            x = x.masked_fill(hidden, float("-inf"))
            lse[s, :, h] = torch.logsumexp(x, -1)
            w = torch.softmax(x, -1)
            out[s, :, h] = torch.where(visible[:, None] > 0, w, torch.zeros_like(w)) @ v[h // group, :n]
    return out, lse
