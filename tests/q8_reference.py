"""The paged 8-bit cache, its rotation and its attention as the header defines them, in plain loops on the CPU: 64 bits but where
the definition itself rounds (a turned value: 32 bits; a row: bf16; a full block: 8 bits).  Shares no code with the kernels."""
import math

import numpy as np
import torch

BLOCK = 64


def table(rows, D, base=10000.0):
    """fp32 [rows, D]: cosines, then sines"""
    a = np.arange(rows, dtype=np.float64)[:, None] * base ** (-np.arange(0, D, 2, dtype=np.float64) / D)[None]
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], axis=1).astype(np.float32))


def angles(tab, pos, section, b, t):
    """cosines and sines of token (b, t): pair by pair the row of its axis"""
    half, c, s, i = tab.shape[1] // 2, [], [], 0
    for axis, n in enumerate(section):
        row = tab[min(max(int(pos[axis, b, t]), 0), tab.shape[0] - 1)]
        c.append(row[i:i + n])
        s.append(row[half + i:half + i + n])
        i += n
    return torch.cat(c), torch.cat(s)


def turned(x, tab, pos, section):
    """x [B, H, L, D] fp32 -> fp32, every product and sum rounded to fp32 by itself"""
    half, y = x.shape[-1] // 2, torch.empty_like(x)
    for b in range(x.shape[0]):
        cs = [angles(tab, pos, section, b, t) for t in range(x.shape[2])]
        c, s = torch.stack([e[0] for e in cs]), torch.stack([e[1] for e in cs])      # [L, D/2]
        lo, hi = x[b, :, :, :half], x[b, :, :, half:]
        y[b, :, :, :half] = lo * c - hi * s
        y[b, :, :, half:] = hi * c + lo * s
    return y


def turned64(x, tab, pos, section):
    half, y = x.shape[-1] // 2, torch.empty(x.shape, dtype=torch.float64)
    for b in range(x.shape[0]):
        for t in range(x.shape[2]):
            c, s = (e.double() for e in angles(tab, pos, section, b, t))
            lo, hi = x[b, :, t, :half].double(), x[b, :, t, half:].double()
            y[b, :, t, :half], y[b, :, t, half:] = lo * c - hi * s, hi * c + lo * s
    return y


def place(D, values):
    """[64, D]: where value (t, d) of a block lies in its page"""
    p = torch.empty(BLOCK, D, dtype=torch.int64)
    for t in range(BLOCK):
        for d in range(D):
            if values:
                p[t, d] = (d // 16 * 4 + t // 4 % 4) * 256 + d % 16 * 16 + t // 16 * 4 + t % 4
            else:
                p[t, d] = ((t // 16 * (D // 64) + d // 64) * 4 + d // 16 % 4) * 256 + t % 16 * 16 + d % 16
    return p


_PLACES = {}


def places(D):
    if D not in _PLACES:
        _PLACES[D] = (place(D, False), place(D, True))
    return _PLACES[D]


def eight_bits(block):
    """A block's bf16 values (fp32 tensor) -> (values of the codes, scale): value = code * scale"""
    x = block.double()
    finite = x.abs()[torch.isfinite(x)]
    top = float(finite.max()) if finite.numel() else 0.0
    e = -100
    if top > 0.0:
        m, ex = math.frexp(top)                   # top = m 2^ex, 448 = 0.875 2^9
        e = max(-100, ex - 9 if m <= 0.875 else ex - 8)
    y = x * 2.0 ** -e
    _, yx = torch.frexp(torch.where(torch.isfinite(y), y, 0.0))
    step = torch.exp2((yx.double() - 4).clamp(min=-9))   # a number keeps 4 significant bits; the least spacing is 2^-9
    code = torch.round(y / step) * step
    return torch.where(torch.isfinite(y), code, torch.nan), 2.0 ** e


class Cache:
    """Host copy of a cache: codes [n_pages, 64 D] as values, scales, tails (values of bf16), page, len."""

    def __init__(self, B, Hkv, D, n_pages, max_blocks, g, lens, page=None, magnitude=1.0):
        U = B * Hkv
        self.B, self.Hkv, self.D, self.n_pages, self.max_blocks = B, Hkv, D, n_pages, max_blocks
        self.page = torch.randperm(n_pages, generator=g)[:U * max_blocks].int().view(U, max_blocks) if page is None else page
        self.len = torch.tensor(lens, dtype=torch.int32)
        self.codes = [torch.empty(n_pages, BLOCK * D), torch.empty(n_pages, BLOCK * D)]
        self.scales = [torch.empty(n_pages), torch.empty(n_pages)]
        for x in range(2):
            rows = (torch.randn(n_pages, BLOCK * D, generator=g) * magnitude).bfloat16().float()
            for p in range(n_pages):
                c, s = eight_bits(rows[p])
                self.codes[x][p], self.scales[x][p] = c.float(), s
        self.tails = [(torch.randn(U, BLOCK * D, generator=g) * magnitude).bfloat16().float() for _ in range(2)]

    def rows(self, u, x):
        """float64 [len, D]: the rows of unit u (x = 0: keys, 1: values); those of pages outside the pool are left out"""
        n, at = int(self.len[u]), places(self.D)[x].reshape(-1)
        out = []
        for j in range(n // BLOCK):
            p = int(self.page[u, j])
            if 0 <= p < self.n_pages:
                out.append((self.codes[x][p].double() * float(self.scales[x][p]))[at].view(BLOCK, self.D))
        out.append(self.tails[x][u].double()[at].view(BLOCK, self.D)[:n % BLOCK])
        return torch.cat(out)

    def room(self, u, want):
        """how many of `want` more rows unit u takes"""
        n = int(self.len[u])
        for r in range(want):
            j = (n + r) // BLOCK
            if (n + r) % BLOCK == BLOCK - 1 and not (j < self.max_blocks and 0 <= int(self.page[u, j]) < self.n_pages):
                return r
        return want

    def append(self, u, k, v):
        """k, v fp32 [n, D] join unit u, as far as there is room"""
        n = int(self.len[u])
        take = self.room(u, k.shape[0])
        for x, new in enumerate((k[:take], v[:take])):
            at = places(self.D)[x]
            rows = torch.cat([self.tails[x][u][at.reshape(-1)].view(BLOCK, self.D)[:n % BLOCK], new.bfloat16().float()])
            j = n // BLOCK
            while rows.shape[0] >= BLOCK:
                c, s = eight_bits(rows[:BLOCK])
                p = int(self.page[u, j])
                self.codes[x][p][at.reshape(-1)] = c.float().reshape(-1)
                self.scales[x][p] = s
                rows, j = rows[BLOCK:], j + 1
            first = 0 if j > n // BLOCK else n % BLOCK
            self.tails[x][u][at[first:rows.shape[0]].reshape(-1)] = rows[first:].reshape(-1)
        self.len[u] = n + take
        return take


def attend(cache, q, k, v, flags, scale):
    """q [B, Hq, L, D], k, v [B, Hkv, L, D] (turned), flags [B, Hkv, L] bool -> float64 [B, Hq, L, D]"""
    B, Hq, L, D = q.shape
    G = Hq // cache.Hkv
    out = torch.empty(B, Hq, L, D, dtype=torch.float64)
    for u in range(B * cache.Hkv):
        b, h = divmod(u, cache.Hkv)
        K, V = cache.rows(u, 0), cache.rows(u, 1)
        kept = torch.nonzero(flags[b, h]).view(-1)
        kept = kept[:cache.room(u, kept.numel())]
        own_k, own_v = k[b, h].double(), v[b, h].double()
        for j in range(L):
            mine = torch.cat([kept[kept < j], torch.tensor([j])])
            kk, vv = torch.cat([K, own_k[mine]]), torch.cat([V, own_v[mine]])
            s = q[b, h * G:(h + 1) * G, j].double() @ kk.T * scale
            out[b, h * G:(h + 1) * G, j] = torch.softmax(s, dim=1) @ vv if kk.shape[0] > 1 else vv.expand(G, D)
    return out
