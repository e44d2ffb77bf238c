"""Shared helpers of the tests of tree and window attention, path append and page
copies: poisoned pools, and the operators written down in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import torch

import workloads as wl

BF16 = 2.0 ** -8       # half a step of bf16, relative to the value
# Weights: scores of N(0,1) rows are sums of 128 products at most, off by at most
# 128 * 2^-24 * sum |q k| * scale * log2(e), about 1e-4 for |q k| sums of 80; the exponent's
# own rounding and the fp32 sums are below that.  2^-12 covers both.
FP32 = 2.0 ** -12


def bound(out, spread, roundings=1):
    """How far a result may be from the 64-bit `out`: the weights are rounded to bf16 once
    (each by half a step, so the sum by half a step of sum w |v| / sum w, `spread`), or
    `roundings` times, and the result is once more."""
    return BF16 * (1 + BF16) * (roundings * spread + np.abs(out)) + FP32 * spread


def check(got, want, spread, what="", roundings=1):
    got = got.float().cpu().double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    assert np.array_equal(np.isinf(got), np.isinf(want)), f"{what}: infinities in other places"
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) - bound(want, spread, roundings)
    off = np.where(np.isnan(want) | (np.isinf(want) & (got == want)), -1.0, off)
    worst = np.unravel_index(np.argmax(off), off.shape) if off.size else None
    assert off.size == 0 or off[worst] <= 0, \
        f"{what}: {got[worst]} for {want[worst]} at {worst}, {off[worst]} beyond the bound"


class Cache:
    """A pool of sequences with random contents.  Slots behind a sequence's end, and pages
    that no sequence holds, are NaN."""

    def __init__(self, lens, Hkv, d, P, dt, seed=0, extra_pages=3, stride=None, extra_tokens=0):
        g = torch.Generator().manual_seed(seed)
        self.lens = np.asarray(lens, np.int32)
        self.Hkv, self.d, self.P, self.dt = Hkv, d, P, dt
        room = self.lens + extra_tokens
        self.num_pages = int(wl.pages_needed(room, P).sum()) + extra_pages
        self.bt, _ = wl.place_pages(room, P, self.num_pages, seed=seed + 1, stride=stride)
        X = wl.chunk_elems(dt)
        kshape, vshape = (self.num_pages, Hkv, d // X, P, X), (self.num_pages, Hkv, d, P)
        used = torch.zeros(self.num_pages, P, dtype=torch.bool)
        for b, L in enumerate(self.lens):
            for j in range(-(-int(L) // P)):
                used[self.bt[b, j], :max(0, min(P, int(L) - j * P))] = True
        k, v = torch.randn(kshape, generator=g), torch.randn(vshape, generator=g)
        if dt == 0:
            k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
            nan = float("nan")
            self.ks = self.vs = None
        else:
            k, v = ((x * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v))
            nan = 0x7F
            self.ks = (torch.rand(self.num_pages, generator=g) + 0.5) / 100
            self.vs = (torch.rand(self.num_pages, generator=g) + 0.5) / 100
        k = torch.where(used[:, None, None, :, None], k, torch.full_like(k, nan))
        v = torch.where(used[:, None, None, :], v, torch.full_like(v, nan))
        self.k, self.v = k, v

    def gpu(self):
        dev = {"k": self.k.cuda(), "v": self.v.cuda(), "bt": torch.from_numpy(self.bt).cuda(),
               "lens": torch.from_numpy(self.lens).cuda()}
        dev["kw"] = dict(num_kv_heads=self.Hkv, page_size=self.P, kv_dtype=self.dt,
                         k_scales=None if self.ks is None else self.ks.cuda(),
                         v_scales=None if self.vs is None else self.vs.cuda())
        return dev

    def tokens(self, b, t):
        """Keys and values [len(t)][Hkv][d] of tokens t of sequence b, in 64 bits."""
        t = np.asarray(t, np.int64)
        ids, slot = torch.from_numpy(self.bt[b, t // self.P].astype(np.int64)), torch.from_numpy(t % self.P)
        k, v = self.k[ids, :, :, slot], self.v[ids, :, :, slot]
        if self.dt == 1:
            k, v = (x.view(torch.float8_e4m3fn) for x in (k, v))
        k, v = k.float().double().reshape(len(t), self.Hkv, self.d).numpy(), v.float().double().numpy()
        if self.dt == 1:
            with np.errstate(invalid="ignore"):
                k = k * self.ks[ids].double().numpy()[:, None, None]
                v = v * self.vs[ids].double().numpy()[:, None, None]
        return k, v


def odd_scales(c):
    """fp8 pages whose scales are 0, negative, infinite, or far from 1, in turn over the sequences
    after the first, which keep their other pages as they are.  The V scale of most pages is a
    part of the weights; where it cannot be, a weight is rounded before and after the product with
    it: twice."""
    ks, vs = [1.0, 0.0, -0.01, 1.0, 1.0, 1.0], [0.0, -0.01, 0.02, 2.0 ** -45, 2.0 ** 45, float("inf")]
    for b in range(1, len(c.lens)):
        n = -(-int(c.lens[b]) // c.P)
        for j in range(b % 2, n, 2 if b < 7 else 3):
            at = int(c.bt[b, j])
            if ks[(b - 1) % 6] != 1.0:
                c.ks[at] = ks[(b - 1) % 6]
            c.vs[at] = vs[(b - 1) % 6]


def attend(q, k, v, seen, scale):
    """Softmax attention of rows q [n][Hq][d] over tokens k, v [m][Hkv][d], row i seeing token
    j where seen[i][j], in 64 bits: (out, sum w |v| / sum w); 0 where a row sees nothing."""
    n, Hq, d = q.shape
    g = Hq // k.shape[1]
    out, spread = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    with np.errstate(all="ignore"):
        for i in range(n):
            at = np.nonzero(seen[i])[0]
            if len(at) == 0:
                continue
            for h in range(Hq):
                s = scale * (k[at, h // g] @ q[i, h])
                w = np.exp(s - s.max())
                out[i, h] = w @ v[at, h // g] / w.sum()
                spread[i, h] = w @ np.abs(v[at, h // g]) / w.sum()
    return out, spread


def random_trees(rng, counts, T):
    """Masks [B][T] (int64 bits): a node sees itself and its ancestors; bits of nodes that a
    sequence does not have are set at random."""
    B = len(counts)
    mask = np.zeros((B, T), np.uint64)
    for b in range(B):
        for i in range(T):
            up = int(rng.integers(0, i + 1))
            above = int(mask[b, up - 1]) if up > 0 else 0
            mask[b, i] = np.uint64((above | 1 << i))
        for i in range(T):
            if counts[b] < 64:
                low = (1 << int(counts[b])) - 1
                noise = int(rng.integers(0, 1 << 63)) * 2 + int(rng.integers(0, 2))
                mask[b, i] = np.uint64((int(mask[b, i]) & low) | (noise & ~low & (2 ** 64 - 1)))
    return mask


def tree_reference(cache, q, kd, vd, mask, counts, out, sm_scale=0.0):
    """out with the rows of the nodes that exist replaced; and sum w |v| / sum w."""
    scale = sm_scale or 1 / math.sqrt(cache.d)
    q, kd, vd = (x.float().double().numpy() for x in (q, kd, vd))
    want, spread = out.float().double().numpy().copy(), np.zeros(out.shape)
    for b, L in enumerate(cache.lens):
        n, L = int(counts[b]), int(L)
        if n == 0:
            continue
        k, v = cache.tokens(b, np.arange(L))
        bits = np.array([[(int(mask[b, i]) >> j) & 1 for j in range(n)] for i in range(n)], bool)
        seen = np.concatenate([np.ones((n, L), bool), bits], 1)
        want[b, :n], spread[b, :n] = attend(q[b, :n], np.concatenate([k, kd[b, :n]]),
                                            np.concatenate([v, vd[b, :n]]), seen, scale)
    return want, spread


def window_reference(cache, q, window, sinks, sm_scale=0.0):
    scale = sm_scale or 1 / math.sqrt(cache.d)
    q = q.float().double().numpy()
    want, spread = np.zeros(q.shape), np.zeros(q.shape)
    for b, L in enumerate(cache.lens):
        t = np.arange(max(0, int(L)))
        t = t[(t < sinks) | (t >= int(L) - window)]
        k, v = cache.tokens(b, t)
        o, s = attend(q[b][None], k, v, np.ones((1, len(t)), bool), scale)
        want[b], spread[b] = o[0], s[0]
    return want, spread
