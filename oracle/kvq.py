"""Plain form of the KV cache in 8 bits (numpy, 64-bit arithmetic), written from the definition in include/tc.h.

TEST INFRASTRUCTURE, like the rest of this package.  Rows are handled one page at a time: E4M3
numbers by a table of the 256 bytes and their steps, places in a page by the layout's formulas.
Attention over such a cache is oracle.attention over a cache in 16 bits that holds what the bytes stand for
(`widened_pools`), which is exact in both element types.
"""
from __future__ import annotations

import numpy as np

import oracle

BLOCK = 16
LIMITS = {"bf16": (-117, 120), "fp16": (-15, 8)}


def _table():
    t = np.zeros(256)
    for b in range(256):
        s, e, m = b >> 7, (b >> 3) & 15, b & 7
        x = np.nan if (e == 15 and m == 7) else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        t[b] = -x if s else x
    return t


NUMBER = _table()


def encode(x, top=448.0):
    """Bytes of the E4M3 numbers nearest to x (ties to the even byte), magnitudes limited to top; NaN and infinities: 0x7F."""
    x = np.asarray(x, np.float64)
    special = ~np.isfinite(x)
    a = np.minimum(np.abs(np.where(special, 0, x)), top)
    power = np.where(a > 0, np.maximum(np.frexp(a)[1] - 1, -6), -6)  # of two, at or below a; subnormal numbers have the steps of the lowest
    byte = ((power + 6) * 8 + np.rint(a / np.exp2(power - 3.0))).astype(np.uint8)
    byte |= np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(special, 0x7F, byte).astype(np.uint8)


def widen(bits, dtype):
    """uint16 patterns of bf16 or IEEE half as float64."""
    bits = np.asarray(bits, np.uint16)
    if dtype == "fp16":
        return bits.view(np.float16).astype(np.float64)
    return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


def narrow(x, dtype):
    """float64 numbers that are exact in the type (or NaN) as uint16 patterns."""
    if dtype == "fp16":
        with np.errstate(over="ignore", invalid="ignore"):
            h = x.astype(np.float16)
        assert np.array_equal(h.astype(np.float64), x, equal_nan=True)
        return h.view(np.uint16)
    f = x.astype(np.float32)
    assert np.array_equal(f.astype(np.float64), x, equal_nan=True)
    u = f.view(np.uint32)
    assert np.all((u & 0xFFFF) == 0) or np.isnan(x).any()
    return (u >> 16).astype(np.uint16)


def k_place(t, d):
    return (d // 16 * BLOCK + t) * 16 + d % 16


def v_place(t, d, dim):
    return (((d // 16 % 2 * 4 + t // 4) * 16 + d % 16) * (dim // 32) + d // 32) * 4 + t % 4


class Cache:
    """k, v uint8 [blocks][kv heads][16 * dim], scales uint8 [blocks][kv heads][2]."""

    def __init__(self, num_blocks, num_kv_heads, head_dim, dtype="bf16", fill=0x7F, scale_fill=0xFF):
        self.shape = (num_blocks, num_kv_heads, head_dim)
        self.dtype = dtype
        self.k = np.full((num_blocks, num_kv_heads, BLOCK * head_dim), fill, np.uint8)
        self.v = self.k.copy()
        self.scales = np.full((num_blocks, num_kv_heads, 2), scale_fill, np.uint8)
        t, d = np.meshgrid(np.arange(BLOCK), np.arange(head_dim), indexing="ij")
        self.places = (k_place(t, d), v_place(t, d, head_dim))

    def tensors(self):
        return (self.k, self.v)

    def append(self, q_start, ctx_len, block_table, k_new, v_new):
        """k_new, v_new: uint16 patterns [T][kv heads][dim]."""
        lo, hi = LIMITS[self.dtype]
        for s, c in enumerate(int(x) for x in ctx_len):
            a, b = int(q_start[s]), int(q_start[s + 1])
            i = a
            while i < b:
                pos = c + i - a
                t0 = pos % BLOCK
                n = min(BLOCK - t0, b - i)
                blk = int(block_table[s][pos // BLOCK])
                for x, new in enumerate((k_new, v_new)):
                    self._append_page(x, blk, t0, widen(new[i:i + n], self.dtype), lo, hi)
                i += n

    def _append_page(self, x, blk, t0, rows, lo, hi):  # rows [n][kv heads][dim]
        tile, place = self.tensors()[x][blk], self.places[x]
        amax = np.abs(np.where(np.isfinite(rows), rows, 0.0)).max((0, 2))  # of every KV head
        e = np.full(amax.shape, lo)
        some = amax > 0
        e[some] = np.ceil(np.log2(amax[some] / 448.0)).astype(int)
        e[some & (amax > 448.0 * 2.0 ** e)] += 1  # (a logarithm may be a rounding off)
        e[some & (amax <= 448.0 * 2.0 ** (e - 1))] -= 1
        e = np.clip(e, lo, hi)
        if t0 > 0:
            before = self.scales[blk, :, x].astype(int) - 127
            e = np.maximum(e, before)
            old = place[:t0].reshape(-1)
            for h in np.flatnonzero(e > before):
                tile[h, old] = encode(NUMBER[tile[h, old]] * 2.0 ** (before[h] - e[h]))
        scaled = (rows * 2.0 ** -e[None, :, None]).transpose(1, 0, 2)
        at_top = e == hi
        for top, some in ((240.0, at_top), (448.0, ~at_top)):
            if some.any():
                tile[np.ix_(np.flatnonzero(some), place[t0:t0 + len(rows)].reshape(-1))] = encode(scaled[some], top).reshape(int(some.sum()), -1)
        self.scales[blk, :, x] = e + 127

    def read(self, table_row, kv_len):
        """What tokens 0..kv_len-1 of a sequence stand for: two float64 [kv_len][kv heads][dim]."""
        ids = np.asarray(table_row[:-(-kv_len // BLOCK)], np.int64)
        out = []
        for x, t in enumerate(self.tensors()):
            scale = 2.0 ** (self.scales[ids][:, :, x].astype(np.float64) - 127)  # [page][kv heads]
            tile = NUMBER[t[ids][:, :, self.places[x]]] * scale[:, :, None, None]  # [page][kv heads][token][d]
            out.append(tile.transpose(0, 2, 1, 3).reshape(-1, self.shape[1], self.shape[2])[:kv_len])
        return out

    def widened_pools(self, block_table, kv_lens):
        """Pools in 16 bits (as oracle.attention reads them) that hold what the tokens of the sequences stand for."""
        nb, hkv, dim = self.shape
        kp, vp = oracle.new_pool(nb, hkv, dim)
        for row, n in zip(block_table, kv_lens):
            k, v = self.read(row, int(n))
            oracle.kv_append(kp, vp, hkv, dim, BLOCK, np.array([0, n], np.int32), np.zeros(1, np.int32), np.asarray(row)[None, :],
                             narrow(k, self.dtype), narrow(v, self.dtype))
        return kp, vp
