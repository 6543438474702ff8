"""64-bit statements of the paged 8-bit cache on the CPU (numpy / torch float64), one row and one page at a time: the
values the GPU calls are compared with.  Nothing here is shared with the library."""
import math

import numpy as np
import torch

FP8 = torch.float8_e4m3fn
MIN_EXP = -100


def decode(codes):
    """e4m3 codes (uint8 tensor) -> float64, from the format: sign, 4 exponent bits (bias 7), 3 mantissa bits."""
    c = codes.cpu().numpy().astype(np.int64)
    s, e, m = np.where(c & 128, -1.0, 1.0), (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    return np.where((c & 127) == 127, np.nan, s * v)


def encode(x):
    """float64 array -> e4m3 codes: nearest, ties to the even code, +-448 beyond the range, NaN 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    grid = decode(torch.arange(0, 127, dtype=torch.uint8))           # 0 ... 448 ascending
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=1e300, neginf=-1e300)), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d_lo, d_hi = a - grid[lo], grid[hi] - a
    pick = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    out = pick + np.where(np.signbit(x), 128, 0)
    return np.where(np.isnan(x), 127, out).astype(np.uint8)


def block_scale(x):
    """Smallest power of two s with max|x| <= 448 s over the finite elements, at least 2^MIN_EXP."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a)]
    top, e = (a.max() if a.size else 0.0), MIN_EXP
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def present(n_rep, n_tok, g, x):
    return 0 <= x < n_rep or n_rep * g <= x < n_tok


def rows_of(n_rep, n_tok, g):
    return list(range(n_rep)) + list(range(n_rep * g, n_tok))


class Pages:
    """Reference of the page tables: Python lists, changed one page at a time."""

    def __init__(self, table, free, n_free, page, g, n_pages):
        self.table = [list(map(int, r)) for r in table]
        self.free, self.top, self.page, self.g, self.n_pages = list(map(int, free)), int(n_free), page, g, n_pages
        self.held = [(0, 0)] * len(self.table)

    def pages(self, r, t):
        P = self.page
        return set(range(-(-r // P))) | set(range(r * self.g // P, -(-t // P)))

    def update(self, target, limit=None):
        """Returns (slots per sequence, status)."""
        P, width = self.page, len(self.table[0])
        for (r0, t0), (r1, t1) in zip(self.held, target):
            if r1 < 0 or t1 < 0 or r1 * self.g > t1 or t1 > width * P or (r1 < r0 and t1 > 0):
                return [[] for _ in target], -1
        new_rows = [list(range(r0, r1)) + list(range(max(t0, r1 * self.g), t1)) for (r0, t0), (r1, t1) in zip(self.held, target)]
        if limit is not None and limit(new_rows):
            return [[] for _ in target], -2
        gone = [(b, e) for b, (h, n) in enumerate(zip(self.held, target)) for e in sorted(self.pages(*h) - self.pages(*n))]
        need = [(b, e) for b, (h, n) in enumerate(zip(self.held, target)) for e in sorted(self.pages(*n) - self.pages(*h))]
        if len(need) > self.top + len(gone):
            return [[] for _ in target], len(need) - self.top - len(gone)
        for b, e in reversed(gone):
            self.free[self.top] = self.table[b][e]
            self.table[b][e] = -1
            self.top += 1
        for b, e in need:
            self.top -= 1
            self.table[b][e] = self.free[self.top]
        self.held = list(target)
        return [[self.table[b][x // P] * P + x % P for x in xs] for b, xs in enumerate(new_rows)], 0


def write(codes_sem, codes_pos, scale_sem, scale_pos, rows_sem, rows_pos, slots, page):
    """Writes rows (float64 arrays [T, Hkv, d]) one run after the other into copies of the pools; scale_pos None: MLA."""
    cs, cp = codes_sem.copy(), codes_pos.copy()
    ss, sp = scale_sem.copy(), None if scale_pos is None else scale_pos.copy()
    n_slots = cs.shape[0] * page
    i, T = 0, len(slots)
    while i < T:
        if not 0 <= slots[i] < n_slots:
            i += 1
            continue
        n = 1
        while i + n < T and slots[i + n] == slots[i] + n and slots[i + n] % page != 0:
            n += 1
        pg, off = slots[i] // page, slots[i] % page
        for h in range(cs.shape[1]):
            blocks = [((cs, rows_sem), (cp, rows_pos))] if sp is None else [((cs, rows_sem),), ((cp, rows_pos),)]
            for parts, scale in zip(blocks, (ss, sp)):
                s = block_scale(np.concatenate([x[i:i + n, h] for _, x in parts], -1))
                if off > 0 and scale[pg, h] >= s:
                    s = float(scale[pg, h])
                for c, x in parts:
                    if off > 0 and s > scale[pg, h]:
                        c[pg, h, :off] = encode(decode(torch.from_numpy(c[pg, h, :off])) * (float(scale[pg, h]) / s))
                    c[pg, h, off:off + n] = encode(x[i:i + n, h] / s)
                scale[pg, h] = s
        i += n
    return cs, cp, ss, sp


def values(codes, scale, table_row, x, page, n_pages):
    """Values [len(x), Hkv, d] of logical rows x and a mask of those that are on a page."""
    ok = np.array([0 <= r // page < len(table_row) and 0 <= table_row[r // page] < n_pages for r in x], dtype=bool)
    v = np.stack([codes[table_row[r // page], :, r % page] * scale[table_row[r // page]][:, None] if o else np.zeros((codes.shape[1], codes.shape[3]))
                  for r, o in zip(x, ok)]) if len(x) else np.zeros((0, codes.shape[1], codes.shape[3]))
    return v, ok


def attend(q_sem, q_pos, codes_sem, codes_pos, scale_sem, scale_pos, table, n_rep, n_tok, g, page, softmax_scale, bias=0.0):
    """float64 (out [B, Q, H, d_sem], lse [B, Q, H], mean |v| under the weights, largest |logit| product sum) of every query."""
    B, Q, H, _ = q_pos.shape
    n_pages, Hkv, _, d_sem = codes_sem.shape
    vs, ks = decode(torch.from_numpy(codes_sem)), decode(torch.from_numpy(codes_pos))
    cap = table.shape[1] * page
    out, lse = np.zeros((B, Q, H, d_sem)), np.full((B, Q, H), -np.inf)
    absv, big = np.zeros((B, Q, H, d_sem)), np.zeros((B, Q, H))
    for b in range(B):
        r, t = min(max(int(n_rep[b]), 0), cap), min(max(int(n_tok[b]), 0), cap)
        x = [y for y in rows_of(r, t, g) if y < cap]
        v, ok = values(vs, scale_sem, table[b], x, page, n_pages)
        k, _ = values(ks, scale_sem if scale_pos is None else scale_pos, table[b], x, page, n_pages)
        x = np.array(x, dtype=np.int64)
        for i in range(Q):
            see = ok & (x < t - Q + 1 + i)
            if not see.any():
                continue
            for h in range(H):
                hk = h // (H // Hkv)
                kk = k[see, hk] if scale_pos is not None else np.concatenate([v[see, hk], k[see, hk]], -1)
                qq = q_pos[b, i, h] if scale_pos is not None else np.concatenate([q_sem[b, i, h], q_pos[b, i, h]])
                z = softmax_scale * (kk @ qq) + np.where(x[see] < r, bias, 0.0)
                m = z.max()
                p = np.exp(z - m)
                out[b, i, h] = p @ v[see, hk] / p.sum()
                absv[b, i, h] = p @ np.abs(v[see, hk]) / p.sum()
                lse[b, i, h] = m + math.log(p.sum())
                big[b, i, h] = softmax_scale * np.abs(qq).max() * np.abs(kk).sum(-1).max()
    return out, lse, absv, big


def update(codes_sem, codes_pos, scale_sem, scale_pos, table, n_rep, n_tok, qbar, g, w, page, softmax_scale):
    """(n_rep_new, rep_sem, rep_pos, anchor): float64 representatives (None rows: nothing condensed)."""
    n_pages, Hkv = codes_sem.shape[:2]
    vs, ks = decode(torch.from_numpy(codes_sem)), decode(torch.from_numpy(codes_pos))
    B = len(n_tok)
    new, anchor = np.array(n_rep), np.full((B, Hkv), -1)
    sem, pos = {}, {}
    for b in range(B):
        r, t = int(n_rep[b]), int(n_tok[b])
        if r < 0 or t - r * g < w + g or t > table.shape[1] * page:
            continue
        x = list(range(r * g, (r + 1) * g))
        v, ok = values(vs, scale_sem, table[b], x, page, n_pages)
        k, _ = values(ks, scale_sem if scale_pos is None else scale_pos, table[b], x, page, n_pages)
        if not ok.all():
            continue
        new[b] += 1
        for h in range(Hkv):
            key = k[:, h] if scale_pos is not None else np.concatenate([v[:, h], k[:, h]], -1)
            z = softmax_scale * (key @ qbar[b, h].astype(np.float64))
            a = np.exp(z - z.max())
            anchor[b, h] = int(np.argmax(z))
            sem[b, h], pos[b, h] = (a / a.sum()) @ v[:, h], k[anchor[b, h], h]
    return new, sem, pos, anchor
