"""Plain 64-bit forms of the paged cache's operators, on the CPU, and the bounds that the tests compare with."""
import numpy as np
import torch

EPS = 1e-6
U32 = 2.0 ** -24      # a rounding to float32, relative
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}      # a rounding to the type


class Pool:
    """The bookkeeping, request by request, with Python lists."""

    def __init__(self, n_pages, page, n_req, max_pages):
        self.n_pages, self.page, self.max_pages = n_pages, page, max_pages
        self.table = [[-1] * max_pages for _ in range(n_req)]
        self.held = [0] * n_req
        self.free = list(range(n_pages - 1, -1, -1))

    def step(self, start, rows, max_rows):
        """(status, cu, pos, slots): as dmtd_page_tables is documented."""
        n = len(start)
        none = [0] * (n + 1)
        for i in range(n):
            if start[i] < 0 or rows[i] < 0 or start[i] + rows[i] > self.max_pages * self.page:
                return (-1, i), none, [], []
        if sum(rows) > max_rows:
            return (-1, -1), none, [], []
        need = [-(-(s + r) // self.page) for s, r in zip(start, rows)]
        give = [self.table[i][need[i]:self.held[i]] for i in range(n)]
        lack = sum(max(need[i] - self.held[i], 0) for i in range(n)) - sum(map(len, give)) - len(self.free)
        if lack > 0:
            return (-3, lack), none, [], []
        self.free += reversed([p for g in give for p in g])
        for i in range(n):
            for j in range(self.held[i], need[i]):
                self.table[i][j] = None
            for j in range(need[i], self.held[i]):
                self.table[i][j] = -1
        for i in range(n):
            for j in range(self.held[i], need[i]):
                self.table[i][j] = self.free.pop()
        self.held = need
        cu, pos, slots = [0], [], []
        for i in range(n):
            cu.append(cu[-1] + rows[i])
            for p in range(start[i], start[i] + rows[i]):
                pos.append(p)
                slots.append(self.table[i][p // self.page] * self.page + p % self.page)
        return (0, 0), cu, pos, slots


def rope_table(n, hd, theta=1e6):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def normed_rotated(x, gain, rope, pos):
    """x float64 [rows, heads, hd]; gain None: no norm; rope None: no rotation.  Also the sum of the magnitudes behind each value."""
    if gain is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
    if rope is None:
        return x, x.abs()
    cos, sin = rope.double()[pos][:, None].unbind(-1)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1), torch.cat([(a * cos).abs() + (b * sin).abs(), (b * cos).abs() + (a * sin).abs()], -1)


def attention(qkv, nq, k, v, table, page, start, rows, gain, rope, two_parts):
    """Outputs float64 [rows, nq, hd] and how far a kernel's may be off.

    A score is a sum of hd products.  float32 throughout: each product and each of the additions rounds, hd + 8 steps of U32 of the products'
    magnitudes with what norm, rotation and scale bring.  Queries as two bf16 parts: the second is off by half a step of 2^-8 of at most 2^-8 of
    the query, 2^-16 of the magnitudes on top.  A probability exp(s - m) is then off by both scores' errors and the exponential's own (below 2^-20
    for arguments above -20; smaller ones weigh less), as two bf16 parts by 2^-16 more; sums over the keys round once a key.  Numerator and
    denominator each carry that, so the output is off by at most twice it, in units of sum p |v|; then it is rounded once."""
    nkv, hd = k.shape[1], k.shape[3]
    total = sum(rows)
    out, tol = torch.zeros(total, nq, hd, dtype=torch.float64), torch.zeros(total, nq, hd, dtype=torch.float64)
    at = 0
    for i, (s, r) in enumerate(zip(start, rows)):
        if r == 0:
            continue
        pos = torch.arange(s, s + r)
        q, mag = normed_rotated(qkv[at:at + r, :nq * hd].double().view(r, nq, hd), gain, rope, pos)
        pages = torch.as_tensor(table[i][:-(-(s + r) // page)]).long()
        good = (pages >= 0) & (pages < k.shape[0])
        there = good.repeat_interleave(page)[:s + r]
        for g in range(nkv):
            kk = k[pages.clamp(0, k.shape[0] - 1), g].reshape(-1, hd)[:s + r].double()
            vv = v[pages.clamp(0, k.shape[0] - 1), g].reshape(-1, hd)[:s + r].double()
            for h in range(g * (nq // nkv), (g + 1) * (nq // nkv)):
                z = q[:, h] @ kk.T / hd ** 0.5
                err = (mag[:, h] @ kk.abs().T / hd ** 0.5) * ((hd + 8) * U32 + (2.0 ** -16 if two_parts else 0))
                hidden = (torch.arange(s + r) > pos[:, None]) | ~there
                z = z.masked_fill(hidden, -np.inf)
                p = torch.nan_to_num(torch.softmax(z, -1))            # a row without keys: 0
                vis = torch.where(hidden.all(0)[:, None], 0.0, vv)
                # values that only later rows see must not reach this one
                out[at:at + r, h] = torch.stack([p[j][~hidden[j]] @ vis[~hidden[j]] for j in range(r)]) if not torch.isfinite(vis).all() else p @ vis
                size = p @ torch.nan_to_num(vis, 0, 0, 0).abs()
                off = 2 * (2 * err.masked_fill(hidden, 0).amax(-1, keepdim=True) + 2.0 ** -20 + (2.0 ** -16 if two_parts else 0) + (s + r + 16) * U32)
                tol[at:at + r, h] = off * size
        at += r
    return out, tol + out.abs() * HALF[k.dtype] + 1e-30
