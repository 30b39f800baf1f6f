"""Latent attention, its cache rows and its pages from their definitions: 64 bits, no code of the library."""
import math

import numpy as np
import torch

STEP = 2.0 ** -8                       # half a step of bf16, relative


def positions(cu, lens, t):
    for i in range(len(lens)):
        if cu[i] <= t < cu[i + 1]:
            return i, lens[i] - cu[i + 1] + t
    return None, None


def context(cache, table_row, n):
    """The first n rows of a sequence, [n][row] in 64 bits"""
    page = cache.shape[1]
    pages = table_row[:(n + page - 1) // page].long()
    return cache[pages].flatten(0, 1)[:n].double()


def attention(cache, table, cu, lens, q, q_rope, W_uk, W_uv, scale):
    """(y, sigma) [T][heads][d_v].  sigma: what the bf16 roundings inside either form leave on y, as a standard deviation.  A rounding is
    uniform within half a step, sigma_0 = 2^-8 / sqrt 3 relative, and they are independent; to first order
        weights      sum_j p_j^2 v_j^2,                       values    the same again,
        keys         sum_j p_j^2 scale^2 (sum_n q_n^2 k_jn^2) (v_j - y)^2,
        q_lat        sum_c (scale q_lat_c)^2 (sum_j p_j c_jc (v_j - y))^2,
    times sigma_0^2.  Rows that see nothing give zero; rows behind the last sequence NaN."""
    T, H, dn = q.shape[0], q.shape[1], W_uk.shape[1]
    dl, dv = W_uk.shape[2], W_uv.shape[1]
    y = torch.full((T, H, dv), math.nan, dtype=torch.float64, device=q.device)
    var = torch.zeros_like(y)
    for i in range(len(lens)):
        a, b, n = cu[i], cu[i + 1], lens[i]
        m = b - a
        if m == 0:
            continue
        if n == 0:
            y[a:b] = 0
            continue
        rows = context(cache, table[i], n)
        c, pos = rows[:, :dl], rows[:, dl:]
        seen = torch.arange(n, device=q.device)[None] <= (n - m + torch.arange(m, device=q.device))[:, None]
        for h in range(H):
            uk, uv = W_uk[h].double(), W_uv[h].double()
            qn, qr = q[a:b, h, :dn].double(), q_rope[a:b, h].double()
            key, val, ql = c @ uk.T, c @ uv.T, qn @ uk
            s = (scale * (qn @ key.T + qr @ pos.T)).masked_fill(~seen, -math.inf)
            top = s.amax(dim=1, keepdim=True)
            p = torch.where(seen, torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top)), torch.zeros_like(s))
            tot = p.sum(dim=1, keepdim=True)
            p = p / torch.where(tot > 0, tot, torch.ones_like(tot))
            o = p @ val
            y[a:b, h] = o
            p2 = p * p
            v = 2 * (p2 @ val ** 2)
            w = p2 * (scale ** 2) * (qn ** 2 @ (key ** 2).T)
            v = v + (w @ val ** 2) - 2 * o * (w @ val) + o ** 2 * w.sum(dim=1, keepdim=True)
            g = torch.einsum("mj,jl,jv->mlv", p, c, val) - (p @ c)[:, :, None] * o[:, None, :]
            v = v + ((scale * ql) ** 2)[:, :, None].mul(g ** 2).sum(dim=1)
            var[a:b, h] = v.clamp(min=0)
    return y, var.sqrt() * (STEP / math.sqrt(3.0))


def append_rows(cache, table, cu, lens, kv, gain, eps, inv_freq, q, dn, halves, dl):
    """(cache in 64 bits after the new rows, rotated parts of the queries [T][heads][d_rope])"""
    out = cache.double().clone()
    dr = kv.shape[1] - dl
    half = dr // 2
    first = torch.arange(half) if halves else 2 * torch.arange(half)
    second = first + (half if halves else 1)
    first, second = first.to(kv.device), second.to(kv.device)
    qr = q[..., dn:].double().clone()
    page = cache.shape[1]
    for t in range(cu[-1]):
        i, pos = positions(cu, lens, t)
        if pos < 0:
            qr[t] = math.nan
            continue
        angle = pos * inv_freq.double()
        co, si = angle.cos(), angle.sin()
        row = kv[t].double().clone()
        lat = row[:dl]
        row[:dl] = lat / torch.sqrt((lat * lat).mean() + eps) * (1.0 if gain is None else gain.double())
        x, z = kv[t, dl:].double()[first], kv[t, dl:].double()[second]
        row[dl + first], row[dl + second] = x * co - z * si, x * si + z * co
        x, z = q[t, :, dn:].double()[:, first], q[t, :, dn:].double()[:, second]
        qr[t][:, first], qr[t][:, second] = x * co - z * si, x * si + z * co
        out[int(table[i, pos // page]), pos % page] = row
    return out, qr


class Pages:
    """The pool as a plain state machine: one call at a time, one entry at a time."""

    def __init__(self, n_pages, page, n_seqs, max_pages, layers=1):
        self.page, self.max_pages = page, max_pages
        self.refs, self.lens = np.zeros(n_pages, np.int64), np.zeros(n_seqs, np.int64)
        self.pages = [[] for _ in range(n_seqs)]
        self.rows = [[[None] * page for _ in range(n_pages)] for _ in range(layers)]

    def _ok(self, s):
        return 0 <= s < len(self.pages)

    def fork(self, parents, children):
        bad = False
        for i, (a, c) in enumerate(zip(parents, children)):
            if not self._ok(a) or not self._ok(c) or a in children or c in children[:i] or self.lens[c] != 0:
                bad = True
                continue
            self.pages[c] = list(self.pages[a])
            self.lens[c] = self.lens[a]
            for p in self.pages[a]:
                self.refs[p] += 1
        return bad

    def reserve(self, seqs, counts):
        """(range error, too few pages)"""
        bad, plan, free = False, [], [p for p in range(len(self.refs)) if self.refs[p] == 0]
        refs = self.refs.copy()
        for i, (s, n) in enumerate(zip(seqs, counts)):
            if not self._ok(s) or n < 0 or s in seqs[:i] or self.lens[s] + n > self.max_pages * self.page:
                bad = True
                continue
            old = self.lens[s]
            need = -(-(old + n) // self.page) - len(self.pages[s])
            copy = n > 0 and old % self.page != 0 and refs[self.pages[s][-1]] > 1
            if copy:
                refs[self.pages[s][-1]] -= 1
            plan.append((s, n, need, copy))
        if sum(need + copy for _, _, need, copy in plan) > len(free):
            return bad, True
        for s, n, need, copy in plan:
            if copy:
                src, dst = self.pages[s][-1], free.pop(0)
                for layer in self.rows:
                    for r in range(self.lens[s] % self.page):
                        layer[dst][r] = layer[src][r]
                self.refs[src] -= 1
                self.refs[dst] = 1
                self.pages[s][-1] = dst
            for _ in range(need):
                p = free.pop(0)
                self.refs[p] = 1
                self.pages[s].append(p)
            self.lens[s] += n
        return bad, False

    def free(self, seqs):
        bad = False
        for s in seqs:
            if not self._ok(s):
                bad = True
                continue
            for p in self.pages[s]:
                self.refs[p] -= 1
            self.pages[s], self.lens[s] = [], 0
        return bad

    def compact(self):
        used = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        src = [p for p in used if p >= len(used)]
        dst = [p for p in range(len(used)) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            for layer in self.rows:
                layer[b] = list(layer[a])
        self.pages = [[to.get(p, p) for p in ps] for ps in self.pages]
