"""A paged cache with random contents, and the operators' definitions in 64 bits to hold it against."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2510_14961_b200 as rd

FILL = 7.0                      # what outputs hold before a call


class Case:
    """Groups of rows over a paged cache.  groups: (positions of the rows in order, or (n, before)) per sequence."""

    def __init__(self, dtype, H, G, D, page, groups, pad=0, seed=0, uniform=False, ld_extra=0, spare_pages=3, max_context=None,
                 n_layers=1, layer=0, rope_base=10000.0, hint=True, kscale=1.0):
        dev = "cuda"
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.dtype, self.H, self.G, self.D, self.page, self.layer = dtype, H, G, D, page, layer
        self.td = torch.bfloat16 if dtype == rd.RD_BF16 else torch.float32
        self.pos = [list(g) if not isinstance(g, tuple) else list(range(g[1], g[1] + g[0])) for g in groups]
        self.len = [max([p for p in ps if p >= 0], default=-1) + 1 for ps in self.pos]
        self.n = sum(len(p) for p in self.pos)
        self.total = self.n + pad
        held = [(L + page - 1) // page for L in self.len]
        n_pages = sum(held) + spare_pages
        stride = max(max(held), 1)
        order = rng.permutation(n_pages).astype(np.int32)
        table = np.full((len(groups), stride), -1, dtype=np.int32)
        at = 0
        for i, h in enumerate(held):
            table[i, :h] = order[at:at + h]
            at += h
        self.n_pages, self.table_np, self.free = n_pages, table, order[at:]
        pos = np.concatenate([np.asarray(p, dtype=np.int32) for p in self.pos] + [np.full(pad, -1, dtype=np.int32)])
        start = np.concatenate([[0], np.cumsum([len(p) for p in self.pos])]).astype(np.int32)
        self.row_pos, self.table = torch.from_numpy(pos).to(dev), torch.from_numpy(table).to(dev)
        self.start = None if uniform else torch.from_numpy(start).to(dev)
        self.most = max(len(p) for p in self.pos)

        def rows(heads, scale=1.0):
            buf = torch.randn(self.total, heads * D + ld_extra, generator=gen, device=dev) * scale
            return buf.to(self.td)[:, :heads * D]

        self.q, self.k, self.v = rows(H), rows(G, kscale), rows(G)
        shape = (n_layers, n_pages, G, page, D)
        self.kp = (torch.randn(shape, generator=gen, device=dev) * kscale).to(self.td)
        self.vp = torch.randn(shape, generator=gen, device=dev).to(self.td)
        self.out = torch.full((self.total, H * D + ld_extra), FILL, device=dev, dtype=self.td)[:, :H * D]
        self.q_out = torch.full((self.total, H * D + ld_extra), FILL, device=dev, dtype=self.td)[:, :H * D]
        self.lse = torch.full((self.total, H), FILL, device=dev, dtype=torch.float32)
        self.rope_base = rope_base
        self.cache = rd.PagedCache(H, G, D, page, n_pages, n_layers=n_layers, max_context=max_context or max(max(self.len), 1),
                                   dtype=dtype, rope_base=rope_base, k_pages=self.kp, v_pages=self.vp)
        self.rows = rd.PagedRows(self.row_pos, self.table, group_start=self.start, max_group_rows=self.most if hint or uniform else 0)

    # ---- calls ----
    def attend(self, window=0, sinks=0, scale=0.0, lse=True, **kw):
        self.cache.attend(self.rows, self.q, self.out, self.lse if lse else None, layer=self.layer, window=window, sinks=sinks, scale=scale, **kw)
        self.cache.sync()

    def append(self, q_out=None):
        self.cache.append(self.rows, self.q, self.k, self.v, self.q_out if q_out is None else q_out, layer=self.layer)
        self.cache.sync()

    # ---- definitions in 64 bits ----
    def sequence(self, pages, g):
        """[positions, G, D] of group g, from the pages one by one."""
        L, out = self.len[g], []
        for i in range((L + self.page - 1) // self.page):
            out.append(pages[self.layer, int(self.table_np[g, i])].double().transpose(0, 1))
        return torch.cat(out)[:L] if out else torch.zeros(0, self.G, self.D, dtype=torch.float64, device="cuda")

    def want_attend(self, window=0, sinks=0, scale=0.0):
        """(out, lse, tolerance of out, tolerance of lse) of every row with a position; rows are [n_real, H, D].

        Tolerances.  u = 2^-24 (float32), h = half a step of the stored type (2^-8 bf16).
        Score: a float32 sum of D products errs by at most D u sum|q_i k_i| =: D u b, the multiplication by the
        scale and the subtraction of the maximum by 3 u (|s| + |m|) <= 6 u b' with b' the largest b of the row.
        Hence every p_j has relative error e = (D + 6) u b' scale (base e) + 2^-22 (exponential); l and the
        products over n keys add n u each (joins included: they only regroup the sum).  bf16: p is rounded for the
        product (h).  With A = sum p_j |v_j| / sum p_j, the output is off by at most (2 e + 2 n u + h) A, and by
        another h |out| when it is stored.  lse: e + n u + 2^-22 |lse|.  The factor 1 + 2^-6 covers products of errors."""
        D, G, rep = self.D, self.G, self.H // self.G
        scale = scale or 1.0 / math.sqrt(D)
        u = 2.0 ** -24
        h = 2.0 ** -8 if self.dtype == rd.RD_BF16 else 0.0
        outs, lses, tols, ltols = [], [], [], []
        r = 0
        for g, ps in enumerate(self.pos):
            if self.len[g] == 0:                       # rows without a position only: nothing is wanted of them
                for some, shape in ((outs, (len(ps), self.H, D)), (lses, (len(ps), self.H)), (tols, (len(ps), self.H, D)), (ltols, (len(ps), self.H))):
                    some.append(torch.zeros(shape, dtype=torch.float64, device="cuda"))
                r += len(ps)
                continue
            K, V = self.sequence(self.kp, g), self.sequence(self.vp, g)
            j = torch.arange(self.len[g], device="cuda")
            for i0 in range(0, len(ps), 256):
                chunk = ps[i0:i0 + 256]
                p = torch.tensor(chunk, device="cuda")[:, None]
                see = j[None] <= p
                if window:
                    see = see & ((p - j[None] < window) | (j[None] < sinks))
                see = see & (p >= 0)
                q = self.q[r + i0:r + i0 + len(chunk)].double().reshape(len(chunk), G, rep, D)
                s = torch.einsum("ngrd,jgd->ngrj", q, K) * scale
                s = torch.where(see[:, None, None], s, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
                m = s.amax(-1, keepdim=True)
                m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
                e = torch.exp(s - m)
                l = e.sum(-1, keepdim=True)
                # (a key nobody sees must not turn 0 into a NaN here either)
                Vc = torch.where(torch.isfinite(V), V, torch.zeros_like(V))
                o = torch.einsum("ngrj,jgd->ngrd", e / l, Vc)
                A = torch.einsum("ngrj,jgd->ngrd", e / l, Vc.abs())
                b = torch.einsum("ngrd,jgd->ngrj", q.abs(), torch.where(torch.isfinite(K), K, torch.zeros_like(K)).abs())
                b = torch.where(see[:, None, None], b, torch.zeros_like(b)).amax(-1, keepdim=True) * scale
                n = see.sum(-1)[:, None, None, None].double()
                err = (D + 6) * u * b + 2.0 ** -22
                outs.append(o.reshape(len(chunk), self.H, D))
                tols.append((((2 * err + 2 * n * u + h) * A + (h + 2 * u) * o.abs()) * (1 + 2.0 ** -6) + 1e-30).reshape(len(chunk), self.H, D))
                L = m + torch.log(l)
                lses.append(L.reshape(len(chunk), self.H))
                ltols.append((err + n * u + 2.0 ** -22 * (1 + L.abs())).reshape(len(chunk), self.H))
            r += len(ps)
        return torch.cat(outs), torch.cat(lses), torch.cat(tols), torch.cat(ltols)

    def check_attend(self, window=0, sinks=0, scale=0.0):
        want, lse, tol, ltol = self.want_attend(window, sinks, scale)
        real = self.row_pos >= 0
        live = real[:self.n]
        got = self.out[:self.n].double().reshape(self.n, self.H, self.D)
        off = (got - want).abs()[live] - tol[live]
        assert not torch.isnan(got[live]).any(), "NaN in rows that see finite keys"
        assert off.numel() == 0 or off.max() <= 0, f"output off by {(got - want).abs()[live].max():.3e}, {off.max():.3e} over the bound"
        loff = (self.lse[:self.n].double() - lse).abs()[live] - ltol[live]
        assert loff.numel() == 0 or loff.max() <= 0, f"lse off by {(self.lse[:self.n].double() - lse).abs()[live].max():.3e}"
        assert (self.out[~real] == FILL).all() and (self.lse[~real] == FILL).all(), "a row without a sequence was written"

    def want_rope(self, x, heads):
        """x [n, heads * D] turned to the rows' positions, 64 bits."""
        x = x[:self.n].double().reshape(self.n, heads, self.D)
        if self.rope_base == 0:
            return x
        pos = self.row_pos[:self.n].double()
        i = torch.arange(self.D // 2, device="cuda", dtype=torch.float64)
        ang = pos[:, None] * self.rope_base ** (-2.0 * i / self.D)
        z = torch.view_as_complex(x.reshape(self.n, heads, self.D // 2, 2).contiguous()) * torch.polar(torch.ones_like(ang), ang)[:, None]
        return torch.view_as_real(z).reshape(self.n, heads, self.D)
