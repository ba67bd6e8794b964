"""Quantised K/V cache and attention over it, in numpy and 64 bits, from the definitions.

Test infrastructure: shares no code with the CUDA library.  16-bit numbers arrive as torch tensors
and are taken to float64 exactly."""

from __future__ import annotations

import math

import numpy as np
import torch

GROUP = 32
TILE = 16


def _next_up(x: torch.Tensor) -> torch.Tensor:
    """The next larger number of a 16-bit type, for x >= 0."""
    return (x.contiguous().view(torch.int16) + 1).view(x.dtype)


def quantise(x: torch.Tensor, bits: int):
    """x [..., dim] (bfloat16 / float16, CPU) -> codes int64 [..., dim], scale and minimum of x's type
    [..., dim / 32].  Groups that are not finite: scale and minimum NaN, codes 0."""
    top = (1 << bits) - 1
    g = x.double().unflatten(-1, (-1, GROUP))
    low, high = g.amin(-1), g.amax(-1)
    span = (high - low).float().double()
    step = (high - low) / top
    s = step.to(x.dtype)
    s = torch.where(s.double() < step, _next_up(s), s)
    if x.dtype == torch.bfloat16:
        s = torch.where(s.double() < 2.0**-126, torch.zeros_like(s), s)
    bad = ~torch.isfinite(span)
    nan = torch.full_like(s, float("nan"))
    s, m = torch.where(bad, nan, s), torch.where(bad, nan, low.to(x.dtype))
    sd = s.double().unsqueeze(-1)
    q = torch.where(sd > 0, torch.floor((g - low.unsqueeze(-1)) / sd + 0.5), torch.zeros_like(g))
    return q.to(torch.int64).flatten(-2), s, m


def quotients(x: torch.Tensor, s: torch.Tensor, m: torch.Tensor) -> torch.Tensor:
    """(x - m) / s before rounding, for judging codes next to a border."""
    g = x.double().unflatten(-1, (-1, GROUP))
    return ((g - m.double().unsqueeze(-1)) / s.double().unsqueeze(-1)).flatten(-2)


def values(codes, s, m) -> torch.Tensor:
    """float64 [..., dim]"""
    g = codes.double().unflatten(-1, (-1, GROUP))
    return (g * s.double().unsqueeze(-1) + m.double().unsqueeze(-1)).flatten(-2)


def tile_bytes(dim: int, bits: int) -> int:
    return 2 * (TILE * dim * bits // 8 + TILE * dim // GROUP * 4)


def code_place(dim: int, bits: int, which: str, token: int, channel: int):
    """(byte offset in the tile, bit shift) of one code, from the layout's description in civic.h."""
    words = dim // GROUP * bits // 4
    plane = min(4, words)
    per_word = 32 // bits
    j, r = divmod(channel, GROUP)
    if which == "k":
        lane, inside = divmod(r, 8)
        w, place = divmod(inside, per_word)
        w += j * (bits // 4)
        word = ((w // plane * TILE + token) * 4 + lane) * plane + w % plane
        bit = place * bits
    else:
        g, inside = divmod(r, 4)
        w, place = divmod(inside, per_word // 2)
        w += j * (bits // 4)
        half, t, second = token // 8, token % 8 // 2, token % 2
        word = ((half * (words // plane) + w // plane) * 32 + 4 * g + t) * plane + w % plane
        bit = 16 * second + place * bits
    base = 0 if which == "k" else TILE * dim * bits // 8
    return base + 4 * word + bit // 8, bit % 8


def param_place(dim: int, bits: int, which: str, token: int, group: int) -> int:
    base = 2 * TILE * dim * bits // 8 + (0 if which == "k" else TILE * dim // GROUP * 4)
    return base + (token * (dim // GROUP) + group) * 4


def places(dim: int, bits: int, which: str):
    """Arrays [16, dim] of byte offsets and shifts, and [16, dim / 32] of parameter offsets."""
    at = np.array([[code_place(dim, bits, which, t, c) for c in range(dim)] for t in range(TILE)])
    par = np.array([[param_place(dim, bits, which, t, j) for j in range(dim // GROUP)] for t in range(TILE)])
    return at[..., 0], at[..., 1], par


class Cache:
    """Reads a cache buffer uint8 [n_layers, n_pages, heads, page bytes] (numpy) element by element."""

    def __init__(self, buffer: np.ndarray, page_size: int, dim: int, bits: int, dtype: torch.dtype):
        self.tiles = buffer.reshape(*buffer.shape[:3], page_size // TILE, tile_bytes(dim, bits))
        self.page_size, self.dim, self.bits, self.dtype = page_size, dim, bits, dtype
        self.where = {w: places(dim, bits, w) for w in "kv"}

    def raw(self, layer: int, which: str, table_row, n: int):
        """codes [n, heads, dim], scale and minimum [n, heads, groups] of a sequence's first n tokens."""
        byte, shift, par = self.where[which]
        heads = self.tiles.shape[2]
        codes = np.zeros((n, heads, self.dim), np.int64)
        pairs = np.zeros((n, heads, self.dim // GROUP, 2), np.int16)
        for first in range(0, n, TILE):
            page, sub = int(table_row[first // self.page_size]), first % self.page_size // TILE
            tile = self.tiles[layer, page, :, sub]  # [heads, bytes]
            got = (tile[:, byte] >> shift) & ((1 << self.bits) - 1)  # [heads, 16, dim]
            two = np.stack([tile[:, par + i] for i in range(4)], -1).astype(np.uint8)  # [heads, 16, groups, 4]
            m = min(TILE, n - first)
            codes[first : first + m] = got.transpose(1, 0, 2)[:m]
            pairs[first : first + m] = np.ascontiguousarray(two).view(np.int16).transpose(1, 0, 2, 3)[:m]
        p = torch.from_numpy(pairs).view(self.dtype)
        return torch.from_numpy(codes), p[..., 0], p[..., 1]

    def rows(self, layer: int, which: str, table_row, n: int) -> torch.Tensor:
        """float64 [n, heads, dim]"""
        return values(*self.raw(layer, which, table_row, n))


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float, causal: bool):
    """One sequence: q [q_len, q_heads, dim], k and v float64 [n, heads, dim] -> out float64 like q,
    lse float64 [q_len, q_heads].  Tokens a query does not see do not enter, whatever they hold."""
    q_len, q_heads, dim = q.shape
    n, heads = k.shape[:2]
    out = torch.zeros((q_len, q_heads, dim), dtype=torch.float64)
    lse = torch.full((q_len, q_heads), -math.inf, dtype=torch.float64)
    for i in range(q_len):
        seen = max(0, min(n, n - q_len + i + 1)) if causal else n
        if seen == 0:
            continue
        for h in range(q_heads):
            kv = h // (q_heads // heads)
            s = (k[:seen, kv] @ q[i, h].double()) * scale
            lse[i, h] = torch.logsumexp(s, 0)
            out[i, h] = torch.softmax(s, 0) @ v[:seen, kv]
    return out, lse
