"""Pools, batches and error bounds of the paged cache's tests."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged_oracle as orc

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


class Pool:
    """A pool whose every byte is NaN until something is written to it, and a table of pages in random order.

    lengths: [(tokens before the call, new tokens)] of the sequences.  Table entries behind a sequence's last page hold numbers that are
    no pages."""

    def __init__(self, lengths, h_kv, d, page, dtype="bf16", held="e4m3", device="cuda", seed=0, token_major=False, spare=3):
        self.lengths, self.h_kv, self.d, self.page, self.dtype, self.held, self.device = lengths, h_kv, d, page, dtype, held, device
        self.rng = np.random.default_rng(seed)
        need = [-(-(t0 + n) // page) for t0, n in lengths]
        self.n_pages = sum(need) + spare
        order = self.rng.permutation(self.n_pages)
        width = max(need + [1]) + 1
        self.table = np.full((len(lengths), width), 2 ** 31 - 1, dtype=np.int32)
        for b, n in enumerate(need):
            self.table[b, :n] = order[sum(need[:b]):sum(need[:b + 1])]
        shape = (self.n_pages, page, h_kv, d) if token_major else (self.n_pages, h_kv, page, d)
        self.caches = []
        for _ in "kv":
            if held == "e4m3":
                t = torch.full(shape, 0x7F, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
            else:
                t = torch.full(shape, float("nan"), dtype=TYPES[dtype], device=device)
            self.caches.append(t.transpose(1, 2) if token_major else t)
        self.scales = [torch.full((self.n_pages, h_kv), 255, dtype=torch.uint8, device=device) for _ in "kv"] if held == "e4m3" else [None, None]
        self.cu = torch.tensor(np.concatenate(([0], np.cumsum([n for _, n in lengths]))), dtype=torch.int32, device=device)
        self.start = torch.tensor([t0 for t0, _ in lengths], dtype=torch.int32, device=device)
        self.pages = torch.tensor(self.table, device=device)
        self.n_tok = sum(n for _, n in lengths)

    def rows(self, n, heads, size=1.0):
        x = torch.from_numpy(self.rng.standard_normal((n, heads, self.d)) * size).to(TYPES[self.dtype])
        return x.to(self.device)

    def batch(self, first=None):
        """cu, start, pages, caches and scales, as the calls take them; first: lengths before the call instead of the pool's."""
        return (self.cu, self.start if first is None else torch.tensor(first, dtype=torch.int32, device=self.device), self.pages,
                self.caches[0], self.caches[1], self.scales[0], self.scales[1])

    def fill(self, sizes=(1.0, 1.0)):
        """Values at every position below a sequence's length, scales for them; the rest of the pool keeps its NaN."""
        for which, size in enumerate(sizes):
            cache, scale = self.caches[which], self.scales[which]
            host = cache.contiguous().cpu()
            host = host.view(torch.uint8) if self.held == "e4m3" else host
            for b, (t0, n) in enumerate(self.lengths):
                for p in range(-(-(t0 + n) // self.page)):
                    rows = min(t0 + n - p * self.page, self.page)
                    x = torch.from_numpy(self.rng.standard_normal((self.h_kv, rows, self.d)) * size).to(TYPES[self.dtype])
                    if self.held == "e4m3":
                        for g in range(self.h_kv):
                            byte = orc.scale_byte(float(x[g].abs().max()))
                            scale[self.table[b, p], g] = byte
                            x8 = torch.from_numpy(orc.to_e4m3(f64(x[g]) * 2.0 ** (127 - byte))).to(torch.float8_e4m3fn)
                            host[self.table[b, p], g, :rows] = x8.view(torch.uint8)
                    else:
                        host[self.table[b, p], :, :rows] = x
            (cache.view(torch.uint8) if self.held == "e4m3" else cache).copy_(host)
        return self

    def values(self):
        """The pool's e4m3 or stored numbers and scales, in float64: k, v, k_scale, v_scale."""
        return [f64(c.contiguous()) for c in self.caches] + [None if s is None else s.cpu().numpy().copy() for s in self.scales]

    def seen(self, b, positions):
        """Keys and values [n, h_kv, d] at positions of sequence b, in float64."""
        at = np.asarray(positions, dtype=np.int64)
        page, slot = self.table[b][at // self.page], at % self.page
        got = []
        for cache, scale in zip(self.caches, self.scales):
            raw = cache.view(torch.uint8) if self.held == "e4m3" else cache
            x = raw[torch.from_numpy(page.astype(np.int64)).to(self.device), :, torch.from_numpy(slot).to(self.device)].cpu()
            if self.held == "e4m3":
                x = orc.e4m3_table()[x.numpy()] * np.exp2(scale.cpu().numpy()[page].astype(np.float64) - 127)[:, :, None]
            got.append(f64(x) if isinstance(x, torch.Tensor) else x)
        return got


def check_attention(pool, q, out, lse, l_i=None, l_l=0, idx=None, scale=None, cap=0.0, p_half_step=0.0, skip=()):
    """out, lse against the oracle.  What an element may be off, with e = 2^-24 and A = sum_j p_j |v_j| of the row:
      rounding of the output to storage: half a step of |out|
      logits: a dot product of d terms and its scaling, (d + 8) e sum|q||k|; a cap's tanh 8 e cap; the exponent's own rounding and the
        exponential, 8 e (1 + |largest logit - smallest|), bounded by twice the largest sum|q||k|: together `delta` relative on p, twice
        (numerator and normaliser)
      probabilities rounded to fewer bits: p_half_step, twice
      sums of n terms: (n + 64) e, of the products and of the normaliser."""
    e = 2.0 ** -24
    d, dtype = pool.d, pool.dtype
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    qf, of = f64(q), f64(out)
    lf = None if lse is None else f64(lse)
    row0, worst = 0, 0.0
    for b, (t0, n) in enumerate(pool.lengths):
        if n and b not in skip:
            at = orc.visible(t0, n, l_i, l_l, None if idx is None else idx[b].cpu().numpy())
            k, v = pool.seen(b, at)
            want, want_lse, spread, most = orc.attend(qf[row0:row0 + n], t0, k, v, at, scale, cap)
            delta = (d + 8) * e * most + 8 * e * cap + 8 * e * (1 + 2 * most)
            share = 2 * delta + 2 * p_half_step + 2 * (len(at) + 64) * e
            tol = HALF_STEP[dtype] * np.abs(want) + share[..., None] * spread + 1e-30
            off = np.abs(of[row0:row0 + n] - want)
            assert np.all(off <= tol), (b, t0, n, float(np.max(off / tol)))
            worst = max(worst, float(np.max(off / tol)))
            if lf is not None:
                tol = delta + (len(at) + 64) * e + 2 * p_half_step + 4 * e * np.abs(want_lse)
                assert np.all(np.abs(lf[row0:row0 + n] - want_lse) <= tol), (b, t0, n, float(np.max(np.abs(lf[row0:row0 + n] - want_lse) / tol)))
        row0 += n
    return worst
