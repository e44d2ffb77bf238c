"""4-bit pages written down from their definition (NumPy, no code of the library): codes and
scales of rows, tiles of pages, and a pool of them."""
from __future__ import annotations

import numpy as np
import torch

import workloads as wl
from cache_util import Cache

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
FP4 = 4


def bf16_of(x):
    """fp32 to bf16 bits, nearest even."""
    with np.errstate(over="ignore", invalid="ignore"):
        x = np.ascontiguousarray(x, np.float32)
    return torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def bf16_value(bits):
    return (np.asarray(bits, np.uint32) << 16).view(np.float32)


def enc4(y):
    """Code of the nearest of GRID (the even code at a tie, 6 beyond) with y's sign; 0 for a NaN."""
    a = np.where(np.isnan(y), 0.0, np.minimum(np.abs(y), 6.0))
    far = np.abs(a[..., None] - GRID)
    best = far.min(-1, keepdims=True)
    near = far == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1)).astype(np.uint8)
    return np.where(np.isnan(y), 0, code | (np.signbit(y).astype(np.uint8) << 3)).astype(np.uint8)


def dec4(code):
    v = GRID[code & 7]
    return np.where(code & 8, -v, v)


def key_codes(bits):
    """bf16 bits [..., d] -> codes [..., d], exponents [..., d / 32]."""
    b = bits.reshape(bits.shape[:-1] + (-1, 32))
    top = (b & 0x7FFF).max(-1).astype(np.int64)
    e = np.clip(((top + 0x20) >> 7) - 2, 1, 252)
    with np.errstate(invalid="ignore"):
        x = bf16_value(b).astype(np.float64)
    codes = enc4(x / np.exp2(e[..., None] - 127.0))
    nan = top > 0x7F80
    return np.where(nan[..., None], 0, codes).astype(np.uint8).reshape(bits.shape), np.where(nan, 255, e).astype(np.uint8)


def value_codes(bits):
    """bf16 bits [..., d] -> codes [..., d], bf16 scales (bits) [..., d / 64]."""
    b = bits.reshape(bits.shape[:-1] + (-1, 64))
    top = (b & 0x7FFF).max(-1)
    nan = top > 0x7F80
    with np.errstate(all="ignore"):
        s = bf16_of(bf16_value(np.minimum(top, 0x7F7F)) / np.float32(6))
        s = np.maximum(s, 0x0080)  # 2^-126
        codes = enc4((bf16_value(b) / bf16_value(s)[..., None]).astype(np.float32).astype(np.float64))
    return (np.where(nan[..., None], 0, codes).astype(np.uint8).reshape(bits.shape),
            np.where(nan, 0x7FC0, s).astype(np.uint16))


def tile_bytes(d, P):
    return P * d * 17 // 32


def put_keys(tile, slot, codes, exps):
    """Slots [n] of a tile [bytes] from codes [n][d], exponents [n][d / 32]."""
    d = codes.shape[1]
    P = tile.shape[0] * 32 // (17 * d)
    c = tile[:P * d // 2].reshape(d // 32, P, 16)
    c[:, slot] = (codes[:, 0::2] | (codes[:, 1::2] << 4)).reshape(-1, d // 32, 16).transpose(1, 0, 2)
    s = tile[P * d // 2:].reshape(d // 32, P // 16, 4, 4)
    s[:, slot // 16, slot % 4, slot % 16 // 4] = exps.T


def put_values(tile, slot, codes, scales):
    d = codes.shape[1]
    P = tile.shape[0] * 32 // (17 * d)
    rows = tile[:P * d // 2].reshape(d, P // 2)
    for i, u in enumerate(slot):
        shift = 4 * (u % 2)
        rows[:, u // 2] = (rows[:, u // 2] & (0xF0 >> shift)) | (codes[i] << shift)
    s = tile[P * d // 2:].view(np.uint16).reshape(d // 64, P)
    s[:, slot] = scales.T


def get_keys(tile, slot, d):
    """Values [n][d] of slots [n], 64 bits."""
    P = tile.shape[0] * 32 // (17 * d)
    b = tile[:P * d // 2].reshape(d // 32, P, 16)[:, slot].transpose(1, 0, 2).reshape(len(slot), -1)
    codes = np.stack([b & 15, b >> 4], -1).reshape(len(slot), d)
    e = tile[P * d // 2:].reshape(d // 32, P // 16, 4, 4)[:, slot // 16, slot % 4, slot % 16 // 4].T.astype(np.float64)
    return dec4(codes) * np.repeat(np.where(e == 255, np.nan, np.exp2(e - 127)), 32, axis=1)


def get_values(tile, slot, d):
    P = tile.shape[0] * 32 // (17 * d)
    b = tile[:P * d // 2].reshape(d, P // 2)[:, slot // 2].T
    codes = np.where(slot[:, None] % 2, b >> 4, b & 15)
    s = bf16_value(np.ascontiguousarray(tile[P * d // 2:]).view(np.uint16).reshape(d // 64, P)[:, slot].T).astype(np.float64)
    return dec4(codes) * np.repeat(s, 64, axis=1)


class Cache4(Cache):
    """A pool of sequences in 4-bit pages.  Slots behind a sequence's end, and pages that no
    sequence holds, have NaN exponents and scales."""

    def __init__(self, lens, Hkv, d, P, seed=0, extra_pages=3, stride=None, extra_tokens=0):
        rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, np.int32)
        self.Hkv, self.d, self.P, self.dt, self.ks, self.vs = Hkv, d, P, FP4, None, None
        room = self.lens + extra_tokens
        self.num_pages = int(wl.pages_needed(room, P).sum()) + extra_pages
        self.bt, _ = wl.place_pages(room, P, self.num_pages, seed=seed + 1, stride=stride)
        size = tile_bytes(d, P)
        k, v = (np.full((self.num_pages, Hkv, size), 0xFF, np.uint8) for _ in range(2))
        for b, L in enumerate(self.lens):
            for j in range(-(-int(L) // P)):
                slot = np.arange(min(P, int(L) - j * P))
                for h in range(Hkv):
                    x = rng.standard_normal((2, len(slot), d)) * np.exp(rng.normal(0, 0.5, (2, len(slot), 1)))
                    x = bf16_of(x)
                    put_keys(k[self.bt[b, j], h], slot, *key_codes(x[0]))
                    put_values(v[self.bt[b, j], h], slot, *value_codes(x[1]))
        self.k, self.v = torch.from_numpy(k), torch.from_numpy(v)

    def tokens(self, b, t):
        t = np.asarray(t, np.int64)
        k, v = np.zeros((2, len(t), self.Hkv, self.d))
        for j in np.unique(t // self.P):
            at = t // self.P == j
            for h in range(self.Hkv):
                page = int(self.bt[b, j])
                k[at, h] = get_keys(self.k[page, h].numpy(), t[at] % self.P, self.d)
                v[at, h] = get_values(self.v[page, h].numpy(), t[at] % self.P, self.d)
        return k, v


def make_cache(lens, Hkv, d, P, dt, **kw):
    return Cache4(lens, Hkv, d, P, **kw) if dt == FP4 else Cache(lens, Hkv, d, P, dt, **kw)
