"""64-bit statements of the paged 4-bit cache, of rotary positions and of draft verification on the CPU (numpy), from their
definitions: the values the GPU calls are compared with.  Nothing here is shared with the library."""
import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
SIGN_BIT = [7, 15, 23, 31, 3, 11, 19, 27]
MIN_EXP, MAX_SHIFT = -94, 14


def encode_row(parts):
    """Rows (list of float64 vectors that share an exponent) -> (list of (codes, shifts), exponent).  A code is the magnitude's
    index, 8 more where the value is negative."""
    scales = []
    for x in parts:
        e = []
        for block in x.reshape(-1, 32):
            a = np.abs(block[np.isfinite(block)])
            top = a.max() if a.size else 0.0
            k = -1000
            if top > 0:
                k = math.frexp(top)[1] - 4
                while top > 6.0 * 2.0 ** k:
                    k += 1
            e.append(k)
        scales.append(e)
    E = max([MIN_EXP] + [k for e in scales for k in e])
    out = []
    for x, e in zip(parts, scales):
        codes, shifts = [], []
        for block, k in zip(x.reshape(-1, 32), e):
            s = min(E - k, MAX_SHIFT)
            a = np.minimum(np.abs(np.nan_to_num(block, nan=0.0, posinf=1e300, neginf=-1e300)) / 2.0 ** (E - s), 6.0)
            hi = np.clip(np.searchsorted(LEVELS, a), 1, 7)
            lo = hi - 1
            up, down = LEVELS[hi] - a, a - LEVELS[lo]
            m = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
            codes += list(m + 8 * np.signbit(block))
            shifts.append(15 if np.isnan(block).any() else s)
        out.append((np.array(codes), np.array(shifts)))
    return out, E


def pack(codes):
    """Codes [..., d] -> bytes [..., d / 2]."""
    c = codes.reshape(codes.shape[:-1] + (-1, 8)).astype(np.uint64)
    w = np.zeros(c.shape[:-1], dtype=np.uint64)
    for i in range(8):
        w |= ((c[..., i] & np.uint64(7)) << np.uint64(4 * i)) | ((c[..., i] >> np.uint64(3)) << np.uint64(SIGN_BIT[i]))
    return w.astype("<u4").view(np.uint8).reshape(codes.shape[:-1] + (-1,))


def unpack(pages):
    """Bytes [..., d / 2] -> codes [..., d]."""
    w = np.ascontiguousarray(pages).view("<u4").astype(np.uint64)
    return np.stack([((w >> np.uint64(4 * i)) & np.uint64(7)) + np.uint64(8) * ((w >> np.uint64(SIGN_BIT[i])) & np.uint64(1)) for i in range(8)],
                    -1).reshape(pages.shape[:-1] + (-1,)).astype(np.int64)


def pack_shifts(s):
    return (s[..., 0::2] | (s[..., 1::2] << 4)).astype(np.uint8)


def unpack_shifts(b):
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (-1,)).astype(np.int64)


def values(pages, shifts, exps):
    """Bytes of a pool -> float64 values [..., d]."""
    c, s = unpack(pages), unpack_shifts(shifts)
    e = np.maximum(exps.astype(np.int64) - 127, MIN_EXP)[..., None] - s
    scale = np.where(s == 15, np.nan, 2.0 ** e)
    v = LEVELS[c & 7] * np.where(c > 7, -1.0, 1.0)
    return (v.reshape(v.shape[:-1] + (-1, 32)) * scale[..., None]).reshape(v.shape)


class Pool:
    """Pages of a 4-bit cache as numpy arrays; sem / pos: (pages, shifts), exps (exp_pos None: MLA)."""

    def __init__(self, n_pages, kv, page, d_sem, d_pos, mla, seed):
        r = np.random.RandomState(seed)
        self.mla, self.page, self.kv = mla, page, kv
        row = (n_pages, kv, page)
        codes = lambda d: pack(np.minimum(np.abs(np.rint(r.randn(*row, d) * 2.5)), 7).astype(np.int64) + 8 * r.randint(0, 2, row + (d,)))  # noqa: E731
        shifts = lambda d: pack_shifts(r.randint(0, 3, row + (d // 32,)))  # noqa: E731
        exps = lambda: r.randint(124, 128, row).astype(np.uint8)           # noqa: E731
        self.pages_sem, self.pages_pos, self.shift_sem, self.shift_pos = codes(d_sem), codes(d_pos), shifts(d_sem), shifts(d_pos)
        self.exp_sem, self.exp_pos = exps(), None if mla else exps()

    def arrays(self):
        return self.pages_sem, self.pages_pos, self.shift_sem, self.shift_pos, self.exp_sem, self.exp_pos

    def sem(self):
        return values(self.pages_sem, self.shift_sem, self.exp_sem)

    def pos(self):
        return values(self.pages_pos, self.shift_pos, self.exp_sem if self.mla else self.exp_pos)

    def write(self, rows_sem, rows_pos, slots):
        """Writes rows (float64 [T, kv, d]) one after the other."""
        for t, s in enumerate(slots):
            if not 0 <= s < self.pages_sem.shape[0] * self.page:
                continue
            for h in range(self.kv):
                at = s // self.page, h, s % self.page
                groups = [(rows_sem[t, h], rows_pos[t, h])] if self.mla else [(rows_sem[t, h],), (rows_pos[t, h],)]
                fields = [[(self.pages_sem, self.shift_sem), (self.pages_pos, self.shift_pos)]] if self.mla else \
                    [[(self.pages_sem, self.shift_sem)], [(self.pages_pos, self.shift_pos)]]
                for parts, field, exps in zip(groups, fields, (self.exp_sem, self.exp_pos)):
                    coded, E = encode_row(list(parts))
                    for (codes, shifts), (pages, sh) in zip(coded, field):
                        pages[at], sh[at] = pack(codes), pack_shifts(shifts)
                    exps[at] = E + 127


def rows_of(n_rep, n_tok, g):
    return list(range(n_rep)) + list(range(n_rep * g, n_tok))


def gather(v, table_row, x, page):
    """Values [len(x), kv, d] of logical rows x and a mask of those that are on a page."""
    n = v.shape[0]
    ok = np.array([y // page < len(table_row) and 0 <= table_row[y // page] < n for y in x], dtype=bool)
    out = np.zeros((len(x),) + (v.shape[1], v.shape[3]))
    for i, y in enumerate(x):
        if ok[i]:
            out[i] = v[table_row[y // page], :, y % page]
    return out, ok


def attend(q_sem, q_pos, pool, table, n_rep, n_tok, g, scale, bias=0.0):
    """float64 (out [B, Q, H, d_sem], lse [B, Q, H], mean |v| under the weights, largest |q| sum|k|) of every query."""
    B, Q, H, _ = q_pos.shape
    vs, ks = pool.sem(), pool.pos()
    cap = table.shape[1] * pool.page
    out, lse = np.zeros((B, Q, H, vs.shape[3])), np.full((B, Q, H), -np.inf)
    absv, big = np.zeros((B, Q, H, vs.shape[3])), np.zeros((B, Q, H))
    for b in range(B):
        r, t = min(max(int(n_rep[b]), 0), cap), min(max(int(n_tok[b]), 0), cap)
        x = [y for y in rows_of(r, t, g) if y < cap]
        v, ok = gather(vs, table[b], x, pool.page)
        k, _ = gather(ks, table[b], x, pool.page)
        x = np.array(x, dtype=np.int64)
        for i in range(Q):
            see = ok & (x < t - Q + 1 + i)
            if not see.any():
                continue
            for h in range(H):
                hk = h // (H // pool.kv)
                kk, qq = k[see, hk], q_pos[b, i, h]
                if pool.mla:
                    kk, qq = np.concatenate([v[see, hk], kk], -1), np.concatenate([q_sem[b, i, h], qq])
                z = scale * (kk @ qq) + np.where(x[see] < r, bias, 0.0)
                m = z.max()
                p = np.exp(z - m)
                out[b, i, h] = p @ v[see, hk] / p.sum()
                absv[b, i, h] = p @ np.abs(v[see, hk]) / p.sum()
                lse[b, i, h] = m + math.log(p.sum())
                big[b, i, h] = scale * np.abs(qq).max() * np.abs(kk).sum(-1).max()
    return out, lse, absv, big


def update(pool, table, n_rep, n_tok, qbar, g, w, scale):
    """(n_rep_new, {sequence: [kv, d] representatives}, the same of the anchors' keys, anchors [B, kv])."""
    vs, ks = pool.sem(), pool.pos()
    new, anchor, sem, pos = np.array(n_rep), np.full((len(n_tok), pool.kv), -1), {}, {}
    for b in range(len(n_tok)):
        r, t = int(n_rep[b]), int(n_tok[b])
        if r < 0 or t - r * g < w + g or t > table.shape[1] * pool.page:
            continue
        x = list(range(r * g, (r + 1) * g))
        v, ok = gather(vs, table[b], x, pool.page)
        k, _ = gather(ks, table[b], x, pool.page)
        if not ok.all():
            continue
        new[b] += 1
        key = np.concatenate([v, k], -1) if pool.mla else k
        z = scale * np.einsum("xhd,hd->hx", key, qbar[b].astype(np.float64))
        a = np.exp(z - z.max(-1, keepdims=True))
        anchor[b] = z.argmax(-1)
        sem[b] = np.einsum("hx,xhd->hd", a / a.sum(-1, keepdims=True), v)
        pos[b] = k[anchor[b], np.arange(pool.kv)]
    return new, sem, pos, anchor


def rope(x, positions, freqs, interleaved, inverse, factor):
    """x [T, heads, d] float64, every pair on its own."""
    y = np.array(x, dtype=np.float64)
    n = len(freqs)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        angle = (positions.astype(np.float64) * float(freqs[i]))[:, None] * (-1.0 if inverse else 1.0)
        c, s = np.cos(angle), np.sin(angle)
        y[..., a], y[..., b] = factor * (x[..., a] * c - x[..., b] * s), factor * (x[..., a] * s + x[..., b] * c)
    return y


def mass(p, q):
    with np.errstate(invalid="ignore"):
        r = np.asarray(p, dtype=np.float64) - q
    return np.where((r > 0) & (r < np.inf), r, 0.0)


def verify(target, draft, tokens, u_accept, u_sample, n_draft):
    """(accepted, tokens [n + 1]) of one request: target [n + 1, V], draft [n, V] or None, as float64."""
    n, V = len(tokens), target.shape[1]
    out, rest = [], None
    for i in range(min(max(int(n_draft), 0), n)):
        x = int(tokens[i])
        inside = 0 <= x < V
        if inside and float(u_accept[i]) * (1.0 if draft is None else float(draft[i, x])) < float(target[i, x]):
            out.append(x)
            continue
        q = np.zeros(V) if draft is None else draft[i]
        rest = mass(target[i], q)
        if draft is None and inside:
            rest[x] = 0.0
        if not rest.sum() > 0:
            rest = mass(target[i], 0.0)
        break
    if rest is None:
        rest = mass(target[len(out)], 0.0)
    k, new = len(out), -1
    if rest.sum() > 0:
        cum = np.cumsum(rest)
        hit = np.nonzero((cum > float(u_sample) * cum[-1]) & (rest > 0))[0]
        new = int(hit[0]) if hit.size else int(np.nonzero(rest)[0][-1])
    return k, np.array(out + [new] + [-1] * (n - k))
