"""Inputs and 64-bit references of the shared-key operators (attention over segments, weights, eviction), on the CPU."""
import math

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}     # half a step, relative to the value
NAN16 = 0x7FFF


def slots(n):
    """Where position 0 .. n-1 stands in a transposed value row: groups of 16 in the order 0-3, 8-11, 4-7, 12-15."""
    order = [0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15]
    place = np.empty(16, dtype=np.int64)
    place[order] = np.arange(16)
    j = np.arange(n)
    return torch.from_numpy(j // 16 * 16 + place[j % 16])


class Case:
    """q and segments on the CPU.  segments: (seqs_per_unit, positions, lens or None).  Rows of q, keys and values are padded (pad
    elements) and what lies behind a unit's keys is NaN."""

    def __init__(self, dtype, H, Hkv, dh, S, L, segments, seed=0, pad=0, scale=1.5, weights=True):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.H, self.Hkv, self.dh, self.S, self.L = dtype, H, Hkv, dh, S, L

        def normal(*dims):
            return torch.randn(dims, generator=g).to(dtype)
        self.q = (scale * torch.randn((S, L, H, dh), generator=g)).to(dtype)
        self.pad, self.segments = pad, []
        for per, n, lens in segments:
            units = S // per
            cap = n + (pad and 3)
            k, v = normal(units, cap, Hkv * dh), normal(units, cap, Hkv * dh)
            held = [min(max(x, 0), n) for x in lens] if lens is not None else [n] * units
            ld = (cap + 15) // 16 * 16 + 16 * pad
            vt = torch.full((units, Hkv * dh, ld), float("nan"), dtype=dtype)
            for u, m in enumerate(held):
                k[u, m:] = float("nan")
                vt[u][:, slots(m)] = v[u, :m].t()
            self.segments.append({"per": per, "n": n, "lens": lens, "held": held, "k": k, "v": v, "vt": vt})

    def device(self, dev, weights=()):
        """(q, KvSegments, weight tensors): weights: indices of the segments that collect them; they start as -7."""
        import paper_2605_15609_amd as psd
        pad = self.pad

        def rows(t, chunk=8):     # the last dimension padded on the device
            if not pad:
                return t.to(dev)
            wide = torch.full(t.shape[:-1] + (t.shape[-1] + pad * chunk,), float("nan"), dtype=t.dtype, device=dev)
            wide[..., :t.shape[-1]] = t.to(dev)
            return wide[..., :t.shape[-1]]
        q = rows(self.q.view(self.S, self.L, -1))
        q = q.as_strided((self.S, self.L, self.H, self.dh), (q.stride(0), q.stride(1), self.dh, 1))
        segs, ws = [], []
        for i, s in enumerate(self.segments):
            w = None
            if i in weights:
                w = torch.full((s["k"].shape[0], self.Hkv, s["n"] + 5), -7.0, device=dev)
            ws.append(w)
            lens = None if s["lens"] is None else torch.tensor(s["lens"], dtype=torch.int32, device=dev)
            segs.append(psd.KvSegment(rows(s["k"]), s["vt"].to(dev), self.dh, length=s["n"], seqs_per_unit=s["per"], lens=lens, weights=w))
        return q, psd.KvSegments(segs), ws

    def reference(self):
        """out, lse, weights per segment, and what bounds the error of each: dicts of float64 arrays.

        A score is a sum of dh products of exact inputs in fp32, off by at most E = dh 2^-24 sum|q||k| / sqrt(dh), and is scaled, shifted by
        the maximum and exponentiated with at most 2^-21 |x| + 2^-22 more; so is the lse, whose sum of n positive terms adds n 2^-24.  A
        probability is then off by a factor within 2 E (its own score and those in the sum) + n 2^-24, an output by that much of sum p|v| and,
        with bf16, half a step for p and half a step for the result."""
        q = self.q.double()
        out = np.zeros((self.S, self.L, self.H, self.dh))
        lse = np.full((self.S, self.L, self.H), -np.inf)
        out_tol, lse_tol = np.zeros_like(out), np.zeros_like(lse)
        w = [np.zeros((s["k"].shape[0], self.Hkv, s["n"])) for s in self.segments]
        w_tol = [np.zeros_like(x) for x in w]
        group = self.H // self.Hkv
        u = U[self.dtype]
        for s in range(self.S):
            k = torch.cat([g["k"][s // g["per"], :g["held"][s // g["per"]]] for g in self.segments]).double()
            v = torch.cat([g["v"][s // g["per"], :g["held"][s // g["per"]]] for g in self.segments]).double()
            n = k.shape[0]
            if n == 0:
                continue
            for h in range(self.H):
                at = slice(h // group * self.dh, (h // group + 1) * self.dh)
                x = q[s, :, h] @ k[:, at].t() / math.sqrt(self.dh)
                size = q[s, :, h].abs() @ k[:, at].abs().t() / math.sqrt(self.dh)
                z = torch.logsumexp(x, -1, keepdim=True)
                p = torch.exp(x - z)
                E = (self.dh * 2.0 ** -24 * size + 2.0 ** -21 * x.abs() + 2.0 ** -21 * z.abs() + 2.0 ** -22).max(-1, keepdim=True).values
                rel = 2 * E + n * 2.0 ** -24
                o = p @ v[:, at]
                out[s, :, h] = o.numpy()
                out_tol[s, :, h] = ((rel + (u if self.dtype == torch.bfloat16 else 0)) * (p @ v[:, at].abs()) + u * o.abs() + 1e-30).numpy()
                lse[s, :, h] = z[:, 0].numpy()
                lse_tol[s, :, h] = rel[:, 0].numpy()
                begin = 0
                for i, g in enumerate(self.segments):
                    unit = s // g["per"]
                    m = g["held"][unit]
                    w[i][unit, h // group, :m] += p[:, begin:begin + m].sum(0).numpy()
                    w_tol[i][unit, h // group, :m] += ((2 * rel + self.S * self.L * group * 2.0 ** -24) * p[:, begin:begin + m]).sum(0).numpy()
                    begin += m
        return {"out": out, "lse": lse, "w": w, "out_tol": out_tol, "lse_tol": lse_tol, "w_tol": w_tol}


def near(got, want, tol, what):
    got = got.double().cpu().numpy() if torch.is_tensor(got) else got
    same = (got == want) | (np.isneginf(got) & np.isneginf(want))
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want))
        worst = np.max(np.where(same, 0.0, off / np.maximum(tol, 1e-300)), initial=0.0)
    assert np.isfinite(off).all(), f"{what}: not finite"
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound, off by {off.max():.3e}"
    return worst


def kept_positions(w, length, keep, first, last):
    """The positions that stay, by the definition: a Python sort of (stays, -weight, position)."""
    n = min(max(int(length), 0), len(w))

    def key(i):
        stays = i < first or i >= n - last
        x = float(w[i])
        return (not stays, math.inf if math.isnan(x) else -x if not stays else 0.0, math.isnan(x) and not stays, i)
    return sorted(sorted(range(n), key=key)[:keep])
