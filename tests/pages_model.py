"""A cache in pages worked through one sequence after another on the host, and attention over it in 64 bits."""
import math

import numpy as np
import torch


class PageModel:
    """The tables and the pool (fp64 on the host) of a cache in pages; every call changes them one entry after another."""

    def __init__(self, layers, kv_heads, head_dim, page, n_pages, max_seqs, max_pages):
        self.page, self.max_pages = page, max_pages
        self.pool = np.full((layers, 2, n_pages, kv_heads, page, head_dim), np.nan)
        self.table = [[] for _ in range(max_seqs)]
        self.lens, self.refs = [0] * max_seqs, [0] * n_pages

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def drop(self, p):
        if p >= 0:
            self.refs[p] -= 1

    def pages_needed(self, seqs, n_new):
        refs, need = list(self.refs), 0
        for s, n in zip(seqs, n_new):
            L = self.lens[s]
            if n and L % self.page and refs[self.table[s][-1]] > 1:
                refs[self.table[s][-1]] -= 1
                need += 1
            need += -(-(L + n) // self.page) - -(-L // self.page)
        return need

    def extend(self, seqs, n_new):
        if self.pages_needed(seqs, n_new) > self.refs.count(0):
            return False
        for s, n in zip(seqs, n_new):
            L = self.lens[s]
            if n and L % self.page and self.refs[self.table[s][-1]] > 1:
                old = self.table[s][-1]
                self.refs[old] -= 1
                self.table[s][-1] = self.take()
                self.pool[:, :, self.table[s][-1], :, :L % self.page] = self.pool[:, :, old, :, :L % self.page]
            while len(self.table[s]) * self.page < L + n:
                self.table[s].append(self.take())
            self.lens[s] = L + n
        return True

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.table[b], self.lens[b] = list(self.table[a]), self.lens[a]
            for p in self.table[b]:
                if p >= 0:
                    self.refs[p] += 1

    def compact(self, seqs, n_rows, n_keep, rows=None):
        for i, s in enumerate(seqs):
            base = self.lens[s] - n_rows[i]
            for j in range(n_keep[i] if rows is not None else 0):
                a, b = base + rows[i][j], base + j
                self.pool[:, :, self.table[s][b // self.page], :, b % self.page] = self.pool[:, :, self.table[s][a // self.page], :, a % self.page]
            self.lens[s] = base + n_keep[i]
            while len(self.table[s]) > -(-self.lens[s] // self.page):
                self.drop(self.table[s].pop())

    def trim(self, seqs, window, sinks):
        for s in seqs:
            for c in range(len(self.table[s])):
                if c * self.page >= sinks and (c + 1) * self.page <= self.lens[s] - window:
                    self.drop(self.table[s][c])
                    self.table[s][c] = -1

    def free(self, seqs):
        for s in seqs:
            for p in self.table[s]:
                self.drop(p)
            self.table[s], self.lens[s] = [], 0

    def write(self, layer, seq, rows_k, rows_v):
        m = len(rows_k)
        for r in range(m):
            pos = self.lens[seq] - m + r
            p = self.table[seq][pos // self.page]
            self.pool[layer, 0, p, :, pos % self.page] = rows_k[r]
            self.pool[layer, 1, p, :, pos % self.page] = rows_v[r]

    def check(self, cache, pool=True):
        """The library's tables (and, bit by bit, its pool) against these."""
        want = np.array([t + [-1] * (self.max_pages - len(t)) for t in self.table])
        assert np.array_equal(cache.page_table.cpu().numpy(), want)
        assert cache.lens.tolist() == self.lens and cache.refs.tolist() == self.refs
        bits = [sum((self.refs[p] == 0) << (p - w * 32) for p in range(w * 32, min(len(self.refs), w * 32 + 32)))
                for w in range(-(-len(self.refs) // 32))]
        assert cache.free_bits.cpu().numpy().view(np.uint32).tolist() == bits
        if pool:
            got = cache.pool.double().cpu().numpy()
            assert np.array_equal(got, self.pool, equal_nan=True)


def attend(q, k, v, pos, window=0, sinks=0, scale=None):
    """Rows q [m, heads, hd] at positions pos [m] over keys k, v [n, kv_heads, hd] in 64 bits.  Returns the output, the softmax's
    log denominator, sum_j p_j |v_j| and the largest sum_d |q_d k_d| of a visible key.  A row without keys: zeros, -inf."""
    q, k, v = q.double(), k.double(), v.double()
    m, heads, hd = q.shape
    n, kv = k.shape[0], k.shape[1]
    scale = 1 / math.sqrt(hd) if scale is None else scale
    j, p = torch.arange(n, device=q.device)[None], torch.as_tensor(pos, device=q.device)[:, None]
    seen = j <= p
    if window:
        seen &= (j > p - window) | (j < sinks)
    out, lse = torch.zeros_like(q), torch.full((m, heads), -math.inf, dtype=torch.float64, device=q.device)
    absv, absqk = torch.zeros_like(q), torch.zeros(m, heads, dtype=torch.float64, device=q.device)
    if n == 0:
        return out, lse, absv, absqk
    for h in range(heads):
        kh, vh = k[:, h * kv // heads], v[:, h * kv // heads]
        ok = seen[:, :, None]
        for r0 in range(0, m, 256):
            r = slice(r0, min(m, r0 + 256))
            # what a row does not see is selected away before any arithmetic: it may be anything
            mask = seen[r]
            if torch.isfinite(kh).all() and torch.isfinite(vh).all():
                s = q[r, h] @ kh.T * scale
                a = q[r, h].abs() @ kh.abs().T
                vv, va = None, None
            else:
                kk = torch.where(ok[r], kh[None], 0.)
                s, a = torch.einsum("md,mnd->mn", q[r, h], kk) * scale, torch.einsum("md,mnd->mn", q[r, h].abs(), kk.abs())
                vv = torch.where(ok[r], vh[None], 0.)
            s = torch.where(mask, s, -math.inf)
            top = s.amax(1, keepdim=True)
            e = torch.exp(s - torch.where(torch.isinf(top) & (top < 0), 0., top))
            den = e.sum(1, keepdim=True)
            w = torch.where(den > 0, e / den, torch.where(den.isnan(), den, 0.))
            if vv is None:
                out[r, h], absv[r, h] = w @ vh, w @ vh.abs()
            else:
                out[r, h], absv[r, h] = torch.einsum("mn,mnd->md", w, vv), torch.einsum("mn,mnd->md", w, vv.abs())
            lse[r, h] = torch.where(den[:, 0] > 0, torch.log(den[:, 0]) + torch.where(den[:, 0] > 0, top[:, 0], 0.), torch.where(den[:, 0].isnan(), den[:, 0], -math.inf))
            absqk[r, h] = torch.where(mask, a, 0.).amax(1)
    return out, lse, absv, absqk


def tolerance(dtype, out, absv, absqk, n_keys, scale):
    """How far an output may be off, element by element.  Half a step of the output's type; half a bf16 step of every weight
    that multiplies V (bf16: sum_j p_j |v_j| 2^-8); the scores' fp32 sums ((hd + 8) 2^-24 sum |q_d k_d| scale each, in numerator
    and denominator); exponentials (2^-20); fp32 sums over the keys (n 2^-24)."""
    hd = out.shape[-1]
    es = ((hd + 8) * 2.0 ** -24 * absqk * scale)[..., None]
    half, weight = (2.0 ** -8, 2.0 ** -8) if dtype == torch.bfloat16 else (2.0 ** -24, 0.0)
    return half * out.abs() + (weight + 2 * es + 2.0 ** -19 + 2 * (n_keys + 16) * 2.0 ** -24) * absv * (1 + half) + 1e-30
