"""Inputs and 64-bit references of the 8-bit caches and of the rotation in front of them, on the CPU."""
import math

import numpy as np
import torch

from tests.shared_common import U

MOST = {"int8": 127.0, "e4m3": 448.0}


def table(fmt):
    """What every byte stands for."""
    if fmt == "int8":
        return np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        out[b] = math.copysign(m / 512 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7), -1 if b & 128 else 1) if b & 127 != 127 else np.nan
    return out


def spots(n, d):
    """Where the bytes of positions 0 .. n - 1 and channels lie in the codes of a unit and KV head: keys [n, d], values [n, d]."""
    p, c = np.arange(n)[:, None], np.arange(d)[None, :]
    tile, r, w = p // 32 * 64 * d, p % 32, min(32, d)
    keys = tile + c // 16 * 512 + r * 16 + c % 16
    # positions of half h: 0-3, 8-11, 16-19, 24-27 and the others
    order = [j for h in (0, 1) for j in range(32) if (j // 4) % 2 == h]
    slot = np.empty(32, dtype=np.int64)
    slot[order] = np.arange(32)
    at = slot[r]
    values = tile + 32 * d + c // w * 32 * w + at // 16 * 16 * w + c % w * 16 + at % 16
    return keys, values


def nearest(x, fmt):
    """The nearest code (as a number) to x, ties to even, x exact in 64 bits."""
    kinds = np.unique(table(fmt)[np.abs(np.nan_to_num(table(fmt), nan=1e9)) <= MOST[fmt]])
    middle = int(np.where(kinds == 0)[0][0])
    at = np.clip(np.searchsorted(kinds, x), 1, len(kinds) - 1)
    lo, hi = kinds[at - 1], kinds[at]
    below, above = x - lo, hi - x
    even_lo = (at - 1 - middle) % 2 == 0
    return np.where((below < above) | ((below == above) & even_lo), lo, hi)


class Cache:
    """codes [units, heads, tiles, 2, 32 d] and scales [units, heads, blocks, 2] on the CPU; lens: positions that a unit holds."""

    def __init__(self, units, Hkv, d, positions, block, fmt, seed=0, lens=None, size=1.5):
        rng = np.random.default_rng(seed)
        n = -(-positions // max(32, block)) * max(32, block)
        self.units, self.Hkv, self.d, self.n, self.block, self.fmt, self.positions, self.lens = units, Hkv, d, n, block, fmt, positions, lens
        self.held = [min(max(x, 0), positions) for x in lens] if lens is not None else [positions] * units
        codes = rng.integers(0, 256, (units, Hkv, 64 * n * d // 32), dtype=np.uint8)
        if fmt == "e4m3":
            codes[(codes & 127) == 127] = 0
            # (uniform bytes are mostly tiny numbers: bring them near the top)
            codes = np.where((codes & 0x78) < 0x60, codes | 0x60, codes).astype(np.uint8)
            codes[(codes & 127) == 127] = 0x70
        scales = (size / (73 if fmt == "int8" else 120) * 2.0 ** rng.uniform(-1, 1, (units, Hkv, n // block, 2))).astype(np.float32)
        # what lies behind a unit's positions must not matter
        keys, values = spots(n, d)
        for u, m in enumerate(self.held):
            codes[u][:, keys[m:]] = 0xff if fmt == "e4m3" else 0x80
            codes[u][:, values[m:]] = 0x7f if fmt == "e4m3" else 0x80
            scales[u, :, -(-m // block):] = np.nan
        self.codes, self.scales = codes.reshape(units, Hkv, n // 32, 2, 32 * d), scales

    def read(self, u):
        """keys, values [positions held, heads, d] in 64 bits."""
        m = self.held[u]
        t, at = table(self.fmt), spots(self.n, self.d)
        s = self.scales[u].astype(np.float64)[:, np.arange(m) // self.block]
        flat = self.codes[u].reshape(self.Hkv, -1)
        return tuple(np.swapaxes(t[flat[:, at[i][:m]]] * s[:, :, i, None], 0, 1) for i in (0, 1))

    def device(self, dev, length=None, per=1, pad=0):
        import paper_2605_15609_amd as psd
        codes, scales = torch.from_numpy(self.codes), torch.from_numpy(self.scales)
        if pad:      # units further apart than they are long
            wide = torch.zeros((self.units, self.codes[0].size + 16 * pad), dtype=torch.uint8, device=dev)
            wide[:, :self.codes[0].size] = codes.reshape(self.units, -1).to(dev)
            codes = wide.as_strided(codes.shape, (wide.stride(0),) + codes.stride()[1:])
        lens = None if self.lens is None else torch.tensor(self.lens, dtype=torch.int32, device=dev)
        return psd.Kv8Cache(codes.to(dev), scales.to(dev), self.d, format=self.fmt, length=self.positions if length is None else length, lens=lens, seqs_per_unit=per)


def stored(cache, k, v, starts, counts):
    """(codes as numbers, scales) of keys and values [units, n, heads, d] behind a store, in place of cache's: [units, heads, positions, d] and
    [units, heads, blocks], each a pair.  k, v: float arrays; the rules of include/psd.h, one block at a time."""
    t, (ka, va) = table(cache.fmt), spots(cache.n, cache.d)
    flat = cache.codes.reshape(cache.units, cache.Hkv, -1)
    number = [t[flat[:, :, a]] for a in (ka, va)]
    scale = [cache.scales[..., i].copy() for i in (0, 1)]
    for u in range(cache.units):
        start, end = starts[u], min(starts[u] + counts[u], cache.n)
        for b in range(max(start, 0) // cache.block, -(-max(end, 0) // cache.block)):
            lo, hi = max(b * cache.block, start), min((b + 1) * cache.block, end)
            if lo >= hi:
                continue
            for i, x in enumerate((k, v)):
                new = np.swapaxes(x[u, lo - start:hi - start].astype(np.float64), 0, 1)     # [heads, rows, d]
                for g in range(cache.Hkv):
                    had = scale[i][u, g, b] if lo > b * cache.block else np.float32(0)
                    need = np.float32(np.abs(new[g]).max() / MOST[cache.fmt])
                    s = max(had, need) if np.isfinite(had) and np.isfinite(need) else np.float32(np.nan)
                    old = number[i][u, g, b * cache.block:lo]
                    if np.isfinite(s):
                        if s > had > 0:
                            number[i][u, g, b * cache.block:lo] = nearest(old * float(had) / float(s), cache.fmt)
                        number[i][u, g, lo:hi] = nearest(new[g] / float(s), cache.fmt) if s > 0 else 0.0
                    else:
                        number[i][u, g, lo:hi] = 0.0
                    scale[i][u, g, b] = s
    return number, scale


def attention(q, cache, per, k=None, v=None):
    """out, lse and what bounds the error of each.  q [S, L, H, d], k, v [S, L, Hkv, d]: tensors of the type of the call.

    A score is a sum of d products of exact inputs in fp32, off by at most d 2^-24 sum|q||k| / sqrt(d) (a code's scale is taken out of the sum), and
    is scaled, shifted and exponentiated with at most 2^-21 |x| + 2^-22 more, E together; so is the lse, whose sum of n positive terms adds n 2^-24.  A
    probability is off by a factor within 2 E + n 2^-24, the sum of n products with values by n 2^-24 more, an output by that much of sum p|v|.  A
    probability times its value scale is rounded to fp32 (2^-24) and with bf16 to that (half a step u: factors 1 + e_j), and so is the result.  With bf16 the
    sum that divides has the same factors: sum p (1 + e) v / sum p (1 + e) is off by at most u sum p|v| + u |o| before it is rounded."""
    S, L, H, d = q.shape
    Hkv, u, x64 = cache.Hkv, U[q.dtype], q.double().numpy()
    out, lse = np.zeros((S, L, H, d)), np.full((S, L, H), -np.inf)
    out_tol, lse_tol = np.zeros_like(out), np.zeros_like(lse)
    for s in range(S):
        keys, values = cache.read(s // per)
        if k is not None:
            keys = np.concatenate([keys, k[s].double().numpy()])
            values = np.concatenate([values, v[s].double().numpy()])
        n = len(keys)
        if n == 0:
            continue
        for h in range(H):
            kk, vv = keys[:, h // (H // Hkv)], values[:, h // (H // Hkv)]
            x = x64[s, :, h] @ kk.T / math.sqrt(d)
            size = np.abs(x64[s, :, h]) @ np.abs(kk).T / math.sqrt(d)
            m = x.max(-1, keepdims=True)
            z = m + np.log(np.exp(x - m).sum(-1, keepdims=True))
            p = np.exp(x - z)
            E = (d * 2.0 ** -24 * size + 2.0 ** -21 * np.abs(x) + 2.0 ** -21 * np.abs(z) + 2.0 ** -22).max(-1, keepdims=True)
            rel = 2 * E + 2 * n * 2.0 ** -24
            o = p @ vv
            out[s, :, h], lse[s, :, h], lse_tol[s, :, h] = o, z[:, 0], rel[:, 0]
            given = u if q.dtype == torch.bfloat16 else 0
            out_tol[s, :, h] = (rel + 2.0 ** -23 + given) * (p @ np.abs(vv)) + (u + given) * np.abs(o) + 1e-30
    return {"out": out, "lse": lse, "out_tol": out_tol, "lse_tol": lse_tol}


def rotation(x, positions, frequencies, interleaved, factor, gain, eps):
    """(result, what bounds the error) of x [S, L, heads, d]: tensors; positions [S, L].

    A normed channel is off by a factor within (d / 2 + 6) 2^-24: a sum of d squares in fp32, halved by the root, the mean, eps, the root, the
    quotient and two products.  An angle of t turns is off by 2^-51 t (three products in 64 bits) and, in half turns up to 1, rounded to fp32 (2^-25);
    sine and cosine by 2^-23 more (two steps of a number up to 1), the factor's product by half a step.  Two products and a sum: three half steps."""
    y = x.double().numpy()
    d, u = y.shape[-1], U[x.dtype]
    rel = 0.0
    if gain is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * gain.double().numpy()
        rel = (d / 2 + 6) * 2.0 ** -24
    f = frequencies.numpy()
    n = 2 * len(f)
    t = positions.double().numpy()[..., None] * f
    c, s = factor * np.cos(t)[:, :, None], factor * np.sin(t)[:, :, None]
    at = np.arange(n).reshape(-1, 2) if interleaved else np.arange(n).reshape(2, -1).T
    a, b = y[..., at[:, 0]], y[..., at[:, 1]]
    out, tol = y.copy(), rel * np.abs(y)
    out[..., at[:, 0]], out[..., at[:, 1]] = a * c - b * s, b * c + a * s
    off = math.pi * 2.0 ** -25 + np.abs(t)[:, :, None] * 2.0 ** -51 + 2.0 ** -23 + 2.0 ** -24 + (0 if n == 0 else 2.0 ** -52 * np.abs(t)[:, :, None])
    slack = abs(factor) * (np.abs(a) + np.abs(b)) * (off + rel + 3 * 2.0 ** -24)
    tol[..., at[:, 0]], tol[..., at[:, 1]] = slack, slack
    return out, tol + u * np.abs(out) + 1e-30
