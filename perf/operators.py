"""Measured cases of the paged 8-bit condensed cache: page tables and slot maps, the quantising write, decode attention
over the pages and the online condensation of a group of cached tokens.

`run` computes each operator either through the library (`own` true) or in its plain form, elementary torch operations in
32 bits (64 for the importance scores, whose order decides the anchors).  A case names its operator in "op":

  pages   lca_page_update        block tables, free list and slot maps from the lengths of the requests
  write   lca_paged8_write       bf16 rows -> e4m3 codes with one power-of-two scale for each (page, KV head)
  attend  lca_decode_attention_paged8
  update  lca_decode_update_paged8

Layout: token n of a sequence is row n of its own logical row space, representative j is row j (a row of tokens condensed
long ago), rows [n_rep, n_rep * g) are absent; block_table[b, x / P] names the page of row x.  Pages hold
[n_pages, n_kv_heads, P, d] codes, scales are [n_pages, n_kv_heads].
"""
import math

import torch

own = False

DEV = "cuda"
FP8 = torch.float8_e4m3fn
#: smallest scale a block is given (a block of zeros, or of values below 2^-92)
MIN_EXP = -100


# ------------------------------------------------------------------------------------------------------------- cases
def _attend(name, variant, batch, heads, kv, d_sem, d_pos, context, window, page, q_len, ragged, condensed):
    return dict(name=name, op="attend", variant=variant, batch=batch, heads=heads, kv=kv, d_sem=d_sem, d_pos=d_pos,
                context=context, window=window, group=64, page=page, q_len=q_len, ragged=ragged, condensed=condensed)


def listed():
    return [
        # one decode step of 64 running requests: a slot for each new token, a new page where one is full; the drafts are
        # rolled back afterwards, as a rejected speculation is
        dict(name="pages step 64", op="pages", batch=64, context=65536, window=4096, group=64, page=64, step=1),
        # admission of 64 prompts of ragged length (condensed caches of about 5000 rows), and their release
        dict(name="pages prompt 64", op="pages", batch=64, context=65536, window=4096, group=64, page=64, step=0),
        # the row of one new token for each of 64 sequences, 512 + 64 wide latents
        dict(name="write step mla 64", op="write", variant="mla", batch=64, kv=1, d_sem=512, d_pos=64, rows=1, page=64, ragged=False),
        # the same for 8 KV heads of 128, small pages, 96 sequences
        dict(name="write step gqa 96", op="write", variant="gqa", batch=96, kv=8, d_sem=128, d_pos=128, rows=1, page=16, ragged=False),
        # condensed prompts into the cache: 64 sequences of 5056 rows
        dict(name="write prompt mla 64", op="write", variant="mla", batch=64, kv=1, d_sem=512, d_pos=64, rows=5056, page=64, ragged=False),
        # ragged prompts, odd lengths, 8 KV heads, pages of 32 rows
        dict(name="write prompt gqa 9", op="write", variant="gqa", batch=9, kv=8, d_sem=128, d_pos=128, rows=4999, page=32, ragged=True),
        # decode of 64 sequences with 65536 tokens of context each, 128 heads over one latent cache
        _attend("attend mla 64x64K", "mla", 64, 128, 1, 512, 64, 65536, 4096, 64, 1, False, True),
        # a single request, 16 heads: latency of one short decode step
        _attend("attend mla 1x32K h16", "mla", 1, 16, 1, 512, 64, 32768, 2048, 64, 1, False, True),
        # 64 sequences, 32 query heads on 8 KV heads
        _attend("attend gqa 64x64K", "gqa", 64, 32, 8, 128, 128, 65536, 4096, 64, 1, False, True),
        # four draft tokens at once over uncondensed ragged caches in small pages
        _attend("attend gqa 12x9K q4", "gqa", 12, 32, 8, 128, 128, 9001, 0, 16, 4, True, False),
        # the earliest 64 cached tokens of each of 64 sequences become one representative
        dict(name="update mla 64", op="update", variant="mla", batch=64, heads=128, kv=1, d_sem=512, d_pos=64, context=65536,
             window=4096, group=64, page=64, due=1.0),
        # 8 KV heads, groups of 32, only part of the sequences due
        dict(name="update gqa 48", op="update", variant="gqa", batch=48, heads=32, kv=8, d_sem=128, d_pos=128, context=20000,
             window=1024, group=32, page=16, due=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pages", "write", "attend", "attend", "update"])
    variant = rng.choice(["mla", "gqa"])
    page = rng.choice([16, 32, 64])
    if op == "pages":
        return dict(op=op, batch=_log(rng, 1, 300), context=_log(rng, 5000, 60000), window=64 * rng.randint(1, 64), group=64,
                    page=page, step=rng.choice([0, 1, 1, 2, 5]))
    kv, d_sem, d_pos = (1, 512, 64) if variant == "mla" else (rng.choice([1, 2, 4, 8]), 128, 128)
    if op == "write":
        rows = rng.choice([1, _log(rng, 2, 3000)])
        return dict(op=op, variant=variant, batch=_log(rng, 1, 400 if rows == 1 else 24), kv=kv, d_sem=d_sem, d_pos=d_pos, rows=rows,
                    page=page, ragged=rows > 1)
    if op == "update":
        return dict(op=op, variant=variant, batch=_log(rng, 1, 80), heads=kv * rng.choice([1, 4, 16]), kv=kv, d_sem=d_sem, d_pos=d_pos,
                    context=_log(rng, 4000, 40000), window=64 * rng.randint(1, 32), group=64, page=page, due=rng.choice([1.0, 0.3]))
    condensed = rng.random() < 0.5
    context = _log(rng, 4500, 120000) if condensed else _log(rng, 1, 20000)
    rows = 4096 + context // 64 if condensed else context
    batch = max(1, min(_log(rng, 1, 64), 200000 // rows))
    heads = rng.choice([16, 32, 40, 64, 128]) if variant == "mla" else kv * rng.choice([1, 2, 4, 7, 8, 16])
    q_len = rng.choice([1, 1, 1, 2, 3, 7]) if heads // kv <= 32 else 1
    c = _attend("", variant, batch, heads, kv, d_sem, d_pos, context, 64 * rng.randint(4, 64) if condensed else 0, page, q_len,
                rng.random() < 0.7, condensed)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
def _cdiv(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _lengths(c, g):
    """(n_rep, n_tok) of every sequence, int32: a context condensed in groups with a window, or not condensed at all."""
    B, L = c["batch"], c["context"]
    n_tok = torch.full((B,), L, device=DEV)
    if c.get("ragged", True):
        n_tok = n_tok - (torch.rand(B, generator=g, device=DEV) * 0.6 * L).long()
        n_tok[0] = L
    n_rep = ((n_tok - c["window"]) // c["group"]).clamp(min=0) if c.get("condensed", True) else torch.zeros_like(n_tok)
    return n_rep.int(), n_tok.int()


def _tables(n_rep, n_tok, group, page, g):
    """(block_table, n_pages): pages of a shuffled pool for every row that is present, -1 elsewhere."""
    B = n_tok.numel()
    width = max(1, _cdiv(int(n_tok.max()), page))
    e = torch.arange(width, device=DEV)
    used = (e < ((n_rep.long() + page - 1) // page)[:, None]) | ((e >= (n_rep.long() * group // page)[:, None]) & (e < ((n_tok.long() + page - 1) // page)[:, None]))
    n = int(used.sum())
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    table[used] = torch.randperm(n, generator=g, device=DEV).int()
    return table, max(n, 1)


def _most_rows(c):
    """Rows that a sequence of a condensed case has at most: representatives, window and the rest of a group."""
    return min(c["context"], c["context"] // c["group"] + c["window"] + c["group"])


def _most_pages(c):
    return _cdiv(_most_rows(c), c["page"]) + 2


def _codes(shape, g):
    """e4m3 codes of N(0, 60^2) values, drawn in pieces."""
    out = torch.empty(shape, dtype=torch.uint8, device=DEV)
    flat = out.view(-1)
    for s in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - s)
        flat[s:s + n] = (torch.randn(n, generator=g, device=DEV) * 60).clamp_(-448, 448).to(FP8).view(torch.uint8)
    return out


def _scales(n_pages, kv, g):
    return torch.exp2(-torch.randint(5, 8, (n_pages, kv), generator=g, device=DEV).float())


def _cache(c, n_pages, g):
    kv, P = c["kv"], c["page"]
    s = dict(pages_sem=_codes((n_pages, kv, P, c["d_sem"]), g), pages_pos=_codes((n_pages, kv, P, c["d_pos"]), g),
             scale_sem=_scales(n_pages, kv, g))
    s["scale_pos"] = _scales(n_pages, kv, g) if c["variant"] == "gqa" else None
    return s


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = dict(case=c)
    if c["op"] == "pages":
        n_rep, n_tok = _lengths(c, g)
        P, B = c["page"], c["batch"]
        s["n_rep"], s["n_tok"] = n_rep, n_tok
        if c["step"]:
            s["after"] = n_tok + c["step"]
            table, n = _tables(n_rep, n_tok, c["group"], P, g)
            wide = torch.full((B, _cdiv(int(n_tok.max()) + c["step"], P)), -1, dtype=torch.int32, device=DEV)
            wide[:, :table.shape[1]] = table
            cap = B * (_most_pages(c) + 2 + c["step"] // P)
            spare = cap - n
            s.update(table=wide, held_rep=n_rep.clone(), held_tok=n_tok.clone(), n_pages=cap, n_rows=B * c["step"])
            s["free"] = torch.zeros(cap, dtype=torch.int32, device=DEV)
            s["free"][:spare] = n + torch.randperm(spare, generator=g, device=DEV).int()
            s["n_free"] = torch.tensor([spare], dtype=torch.int32, device=DEV)
        else:
            cap = B * _most_pages(c)
            s.update(table=torch.full((B, _cdiv(int(n_tok.max()), P)), -1, dtype=torch.int32, device=DEV), n_pages=cap,
                     held_rep=torch.zeros_like(n_rep), held_tok=torch.zeros_like(n_tok), n_rows=B * _most_rows(c))
            s["free"] = torch.randperm(cap, generator=g, device=DEV).int()
            s["n_free"] = torch.tensor([cap], dtype=torch.int32, device=DEV)
            s["zero"] = torch.zeros_like(n_tok)
        s["slots"] = torch.empty(s["n_rows"], dtype=torch.int32, device=DEV)
        s["offsets"] = torch.empty(B + 1, dtype=torch.int32, device=DEV)
        s["status"] = torch.empty(1, dtype=torch.int32, device=DEV)
        return s
    if c["op"] == "write":
        B, P, kv = c["batch"], c["page"], c["kv"]
        if c["rows"] == 1:          # one new row in a page of its own sequence, at any place of the page
            n_pages = B + 3
            slots = torch.randperm(n_pages, generator=g, device=DEV)[:B] * P + torch.randint(0, P, (B,), generator=g, device=DEV)
        else:
            lens = torch.full((B,), c["rows"], device=DEV)
            if c["ragged"]:
                lens = (lens * (0.3 + 0.7 * torch.rand(B, generator=g, device=DEV))).long().clamp(min=1)
            need = _cdiv(c["rows"], P)
            n_pages = B * need
            pages = torch.randperm(n_pages, generator=g, device=DEV).view(B, need)
            x = torch.arange(c["rows"], device=DEV)
            all_slots = pages.gather(1, (x // P).expand(B, -1)) * P + x % P
            slots = all_slots[x < lens[:, None]]
        s.update(_cache(c, n_pages, g))
        s["slots"] = slots.int()
        T = slots.numel()
        gain = torch.exp(0.5 * torch.randn((T, 1, 1), generator=g, device=DEV))
        s["rows_sem"] = (torch.randn((T, kv, c["d_sem"]), generator=g, device=DEV) * gain).bfloat16()
        s["rows_pos"] = (torch.randn((T, kv, c["d_pos"]), generator=g, device=DEV) * gain).bfloat16()
        return s
    if c["op"] == "update":
        n_rep, n_tok = _lengths(c, g)
        due = torch.rand(c["batch"], generator=g, device=DEV) < c["due"]
        R = c["window"] + c["group"]
        n_tok = torch.where(due, n_rep * c["group"] + R, torch.minimum(n_tok, n_rep * c["group"] + R - 1)).int()
        s.update(n_rep=n_rep, n_tok=n_tok)
        s["table"], s["n_pages"] = _tables(n_rep, n_tok, c["group"], c["page"], g)
        s.update(_cache(c, s["n_pages"], g))
        dk = c["d_pos"] + (c["d_sem"] if c["variant"] == "mla" else 0)
        s["qbar"] = torch.randn((c["batch"], c["kv"], dk), generator=g, device=DEV) * 0.3
        s["rep_sem"] = torch.zeros((c["batch"], c["kv"], c["d_sem"]), dtype=torch.bfloat16, device=DEV)
        s["rep_pos"] = torch.zeros((c["batch"], c["kv"], c["d_pos"]), dtype=torch.bfloat16, device=DEV)
        return s
    n_rep, n_tok = _lengths(c, g)
    s.update(n_rep=n_rep, n_tok=n_tok)
    s["table"], n_pages = _tables(n_rep, n_tok, c["group"], c["page"], g)
    s.update(_cache(c, n_pages, g))
    lead = (c["batch"], c["q_len"], c["heads"])
    s["q_sem"] = torch.randn(lead + (c["d_sem"],), generator=g, device=DEV).bfloat16() if c["variant"] == "mla" else None
    s["q_pos"] = torch.randn(lead + (c["d_pos"],), generator=g, device=DEV).bfloat16()
    return s


def _scale_of(c):
    return 1.0 / math.sqrt(192.0 if c["variant"] == "mla" else c["d_pos"])


# ------------------------------------------------------------------------------------------------------ plain forms
def _ranges_rank(table, starts, stops):
    """For the ranges [starts[k][b], stops[k][b]) of table columns, in the order (b, k, column): a mask [B, width] of the
    columns that are in one, and the rank of each such column in that order.  Ranges of one row do not overlap."""
    B, width = table.shape
    e = torch.arange(width, device=table.device)
    mask = torch.zeros((B, width), dtype=torch.bool, device=table.device)
    rank = torch.zeros((B, width), dtype=torch.int64, device=table.device)
    lens = [(b - a).clamp(min=0) for a, b in zip(starts, stops)]
    base = torch.cumsum(sum(lens), 0) - sum(lens)
    for a, b, n in zip(starts, stops, lens):
        m = (e >= a[:, None]) & (e < b[:, None])
        rank = torch.where(m, base[:, None] + e - a[:, None], rank)
        mask |= m
        base = base + n
    return mask, rank, int(sum(lens).sum())


def _plain_pages(s, n_rep, n_tok, table, free, n_free, held_rep, held_tok, n_rows):
    """One table update; every argument a new tensor that is changed in place.  Returns (slots, offsets, status)."""
    c = s["case"]
    P, gr = c["page"], c["group"]
    B, width = table.shape
    r0, t0, r1, t1 = (x.long() for x in (held_rep, held_tok, n_rep, n_tok))
    a0, b0, c0 = (r0 + P - 1) // P, r0 * gr // P, (t0 + P - 1) // P
    a1, b1, c1 = (r1 + P - 1) // P, r1 * gr // P, (t1 + P - 1) // P
    mx, mn = torch.maximum, torch.minimum
    done = t1 == 0
    gone, grank, n_gone = _ranges_rank(table, [a1, mx(b0, a1), mx(mx(b0, c1), mx(b1, a1))], [a0, mn(c0, b1), c0])
    need, nrank, n_need = _ranges_rank(table, [a0, mx(a0, c0), mx(b1, c0)], [torch.where(done, a0, mn(a1, b0)), a1, c1])
    first_tok = mx(t0, r1 * gr)
    reps, toks = (r1 - r0).clamp(min=0), (t1 - first_tok).clamp(min=0)
    rows = reps + toks
    offsets = torch.zeros(B + 1, dtype=torch.int64, device=table.device)
    offsets[1:] = torch.cumsum(rows, 0)
    slots = torch.full((n_rows,), -1, dtype=torch.int64, device=table.device)
    status = torch.zeros(1, dtype=torch.int32, device=table.device)
    have = int(n_free) + n_gone
    if n_need > have:
        status.fill_(n_need - have)
        return slots.int(), offsets.int(), status
    free[int(n_free) + n_gone - 1 - grank[gone]] = table[gone]
    table[gone] = -1
    table[need] = free[have - 1 - nrank[need]]
    n_free.fill_(have - n_need)
    held_rep.copy_(n_rep)
    held_tok.copy_(n_tok)
    i = torch.arange(int(offsets[-1]), device=table.device)
    b = torch.searchsorted(offsets[1:], i, right=True)
    k = i - offsets[b]
    x = torch.where(k < reps[b], r0[b] + k, first_tok[b] + k - reps[b])
    slots[:i.numel()] = table[b, x // P].long() * P + x % P
    return slots.int(), offsets.int(), status


def _pow2_scale(amax):
    """2^e, e the smallest integer with amax <= 448 * 2^e, not below MIN_EXP; amax >= 0 finite."""
    m, e = torch.frexp(amax)                            # amax = m * 2^e, 0.5 <= m < 1, and 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(amax > 0, e, torch.full_like(e, MIN_EXP)).clamp(min=MIN_EXP)
    return torch.ldexp(torch.ones_like(m), e)


def _finite_abs(x):
    x = x.abs()
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x))


def _plain_write(s):
    c = s["case"]
    P, kv, T = c["page"], c["kv"], s["slots"].numel()
    slots = s["slots"].long()
    page, off = slots // P, slots % P
    head = torch.ones(T, dtype=torch.bool, device=slots.device)        # first row of a run inside one page
    head[1:] = page[1:] != page[:-1]
    run = torch.cumsum(head, 0) - 1
    n = int(run[-1]) + 1
    run_page, run_off = page[head], off[head]
    parts = [("sem", s["rows_sem"].float()), ("pos", s["rows_pos"].float())]
    amax = {}
    for k, x in parts:
        block = torch.zeros((n, P, kv), device=slots.device)                # a run has each place of its page once at most
        block[run, off] = _finite_abs(x).amax(-1)
        amax[k] = block.amax(1)
    if c["variant"] == "mla":
        amax["sem"] = amax["pos"] = torch.maximum(amax["sem"], amax["pos"])
    out = {}
    for k, x in parts:
        scale = s["scale_pos"] if k == "pos" and c["variant"] == "gqa" else s["scale_sem"]
        old = scale[run_page].clone()
        new = _pow2_scale(amax[k])
        new = torch.where((run_off > 0)[:, None], torch.maximum(new, old), new)
        pages = s["pages_" + k].view(FP8)
        # rows that the page holds already are rounded again where its scale has grown
        grown = ((run_off > 0)[:, None] & (new > old)).nonzero()
        if grown.numel():
            r, h = grown[:, 0], grown[:, 1]
            block = pages[run_page[r], h].float()
            again = (block * (old / new)[r, h][:, None, None]).clamp(-448, 448).to(FP8)
            keep = torch.arange(P, device=slots.device)[None, :, None] < run_off[r][:, None, None]
            s["pages_" + k][run_page[r], h] = torch.where(keep, again.view(torch.uint8), s["pages_" + k][run_page[r], h])
        out[k] = (run_page, new, scale)
        q = (x / new[run][:, :, None]).clamp(-448, 448).to(FP8)
        s["pages_" + k][page[:, None], torch.arange(kv, device=slots.device)[None], off[:, None]] = q.view(torch.uint8)
    for run_page, new, scale in out.values():
        scale[run_page] = new
    return _write_outputs(s)


def _write_outputs(s):
    r = dict(sem=s["pages_sem"].view(FP8), pos=s["pages_pos"].view(FP8), scale_sem=s["scale_sem"])
    if s["scale_pos"] is not None:
        r["scale_pos"] = s["scale_pos"]
    return r


def _gather_rows(s, x, which):
    """Values [B, kv, R, d] of the logical rows x [B, R] (rows outside the table or on no page read page 0)."""
    c = s["case"]
    P = c["page"]
    page = s["table"].gather(1, (x // P).clamp(max=s["table"].shape[1] - 1)).long().clamp(min=0)
    v = s["pages_" + which].view(FP8)[page, :, x % P]                       # [B, R, kv, d]
    scale = s["scale_pos"] if which == "pos" and c["variant"] == "gqa" else s["scale_sem"]
    return (v.float() * scale[page][..., None]).transpose(1, 2)


def _plain_attend(s):
    c = s["case"]
    B, Q, H, kv, gr = c["batch"], c["q_len"], c["heads"], c["kv"], c["group"]
    n_rep, n_tok = s["n_rep"].long(), s["n_tok"].long()
    rows = n_rep + n_tok - n_rep * gr
    i = torch.arange(int(rows.max()), device=DEV)
    x = torch.where(i < n_rep[:, None], i, i + (n_rep * (gr - 1))[:, None])    # row of the i-th present row
    present = i < rows[:, None]
    x = torch.where(present, x, torch.zeros_like(x))
    pos, sem = _gather_rows(s, x, "pos"), _gather_rows(s, x, "sem")
    rep = H // kv
    q = s["q_pos"].float().view(B, Q, kv, rep, c["d_pos"]).permute(0, 2, 1, 3, 4).reshape(B, kv, Q * rep, c["d_pos"])
    logit = q @ pos.transpose(2, 3)
    if c["variant"] == "mla":
        q = s["q_sem"].float().view(B, Q, kv, rep, c["d_sem"]).permute(0, 2, 1, 3, 4).reshape(B, kv, Q * rep, c["d_sem"])
        logit = logit + q @ sem.transpose(2, 3)
    logit = logit * _scale_of(c)
    t = torch.arange(Q, device=DEV).repeat_interleave(rep)
    seen = present[:, None] & (x[:, None] < (n_tok[:, None] - Q + 1 + t)[..., None])       # [B, Q * rep, R]
    logit = torch.where(seen[:, None], logit, torch.full_like(logit, -math.inf))
    m = logit.amax(-1, keepdim=True)
    p = torch.exp(logit - torch.where(torch.isfinite(m), m, torch.zeros_like(m)))
    l = p.sum(-1, keepdim=True)
    out = (p @ torch.where(present[:, None, :, None], sem, torch.zeros_like(sem))) / torch.where(l > 0, l, torch.ones_like(l))
    lse = (m + torch.log(l))[..., 0]
    back = lambda v, d: v.view(B, kv, Q, rep, d).permute(0, 2, 1, 3, 4).reshape(B, Q, H, d)  # noqa: E731
    return dict(out=back(out, c["d_sem"]).bfloat16(), lse=back(lse[..., None], 1)[..., 0].contiguous())


def _plain_update(s):
    c = s["case"]
    B, gr = c["batch"], c["group"]
    n_rep, n_tok = s["n_rep"].long(), s["n_tok"].long()
    due = n_tok - n_rep * gr >= c["window"] + gr
    x = (n_rep * gr)[:, None] + torch.arange(gr, device=DEV)
    pos, sem = _gather_rows(s, x, "pos"), _gather_rows(s, x, "sem")           # [B, kv, g, d]
    key = torch.cat([sem, pos], -1) if c["variant"] == "mla" else pos
    score = (key.double() * s["qbar"].double()[:, :, None]).sum(-1) * _scale_of(c)
    anchor = score.argmax(-1)
    w = torch.exp((score - score.amax(-1, keepdim=True)).float())
    w = w / w.sum(-1, keepdim=True)
    pooled = (w[..., None] * sem).sum(2).bfloat16()
    picked = pos.gather(2, anchor[..., None, None].expand(-1, -1, 1, pos.shape[-1]))[:, :, 0].bfloat16()
    d = due[:, None, None]
    return dict(rep_sem=torch.where(d, pooled, s["rep_sem"]), rep_pos=torch.where(d, picked, s["rep_pos"]),
                anchor=torch.where(due[:, None], anchor, torch.full_like(anchor, -1)).int(), n_rep=(s["n_rep"] + due.int()))


# ---------------------------------------------------------------------------------------------------------- one pass
def _handle(s):
    """Parameters, cache descriptor, outputs and workspace that a user's program keeps beside its cache."""
    from paper_2604_12452_b200 import binding as B
    c = s["case"]
    h = s["handle"] = dict(B=B)
    if c["op"] == "pages":
        h["p"] = B.make_params("mla", c["batch"], 1, 16, 1, 512, 64, c["group"], c["window"], 1.0)
        h["cache"] = B.paged8_cache(None, None, None, None, s["table"], page_size=c["page"], n_pages=s["n_pages"])
        return h
    h["p"] = B.make_params(c["variant"], c["batch"], 1, c.get("heads", c["kv"]), c["kv"], c["d_sem"], c["d_pos"],
                           c.get("group", 64), c.get("window", 0), _scale_of(c))
    h["cache"] = B.paged8_cache(s["pages_sem"], s["pages_pos"], s["scale_sem"], s["scale_pos"], s.get("table"))
    if c["op"] == "attend":
        h["out"] = torch.empty((c["batch"], c["q_len"], c["heads"], c["d_sem"]), dtype=torch.bfloat16, device=DEV)
        h["lse"] = torch.empty((c["batch"], c["q_len"], c["heads"]), dtype=torch.float32, device=DEV)
        h["ws"] = B.workspace_paged8(h["p"], h["cache"], c["q_len"], DEV)
    if c["op"] == "update":
        h["anchor"] = torch.empty((c["batch"], c["kv"]), dtype=torch.int32, device=DEV)
        h["n_rep"] = torch.empty_like(s["n_rep"])
        h["ws"] = B.workspace(h["p"], B.LCA_WS_UPDATE, DEV)
    return h


def _own(s):
    c = s["case"]
    h = s.get("handle") or _handle(s)
    B = h["B"]
    if c["op"] == "pages":
        state = (s["held_rep"], s["held_tok"], s["free"], s["n_free"])
        if c["step"]:
            B.page_update(h["p"], h["cache"], s["n_rep"], s["after"], *state, s["slots"], s["offsets"], s["status"])
            B.page_update(h["p"], h["cache"], s["n_rep"], s["n_tok"], *state, None, None, s["status"])
        else:
            B.page_update(h["p"], h["cache"], s["n_rep"], s["n_tok"], *state, s["slots"], s["offsets"], s["status"])
            B.page_update(h["p"], h["cache"], s["zero"], s["zero"], *state, None, None, s["status"])
        return dict(slots=s["slots"], offsets=s["offsets"], table=s["table"], free=s["free"], n_free=s["n_free"], status=s["status"])
    if c["op"] == "write":
        B.paged8_write(h["p"], h["cache"], s["rows_sem"], s["rows_pos"], s["slots"])
        return _write_outputs(s)
    if c["op"] == "attend":
        B.decode_attention_paged8(h["p"], h["cache"], s["q_sem"], s["q_pos"], s["n_rep"], s["n_tok"], out=h["out"], lse=h["lse"], ws=h["ws"])
        return dict(out=h["out"], lse=h["lse"])
    B.decode_update_paged8(h["p"], h["cache"], None, None, s["n_rep"], s["n_tok"], h["n_rep"], s["rep_sem"], s["rep_pos"],
                           qbar=s["qbar"], anchor=h["anchor"], ws=h["ws"])
    return dict(rep_sem=s["rep_sem"], rep_pos=s["rep_pos"], anchor=h["anchor"], n_rep=h["n_rep"])


def run(state):
    if own:
        return _own(state)
    s, op = state, state["case"]["op"]
    if op == "pages":
        table, free, n_free, hr, ht = (s[k].clone() for k in ("table", "free", "n_free", "held_rep", "held_tok"))
        first = s["after"] if s["case"]["step"] else s["n_tok"]
        slots, offsets, _ = _plain_pages(s, s["n_rep"], first, table, free, n_free, hr, ht, s["n_rows"])
        back = (s["n_rep"], s["n_tok"]) if s["case"]["step"] else (s["zero"], s["zero"])
        _, _, status = _plain_pages(s, *back, table, free, n_free, hr, ht, 0)
        return dict(slots=slots, offsets=offsets, table=table, free=free, n_free=n_free, status=status)
    return dict(write=_plain_write, attend=_plain_attend, update=_plain_update)[op](s)


# -------------------------------------------------------------------------------------------------------------- work
def _rows(c):
    """Expected number of rows of a sequence (ragged lengths are 0.4 to 1 times the context)."""
    L = c["context"] * (0.7 if c.get("ragged", True) and c["batch"] > 1 else 1.0)
    if not c.get("condensed", True) or L < c["window"] + c["group"]:
        return L
    m = (L - c["window"]) // c["group"]
    return m + L - m * c["group"]


def work(case):
    c = case
    B = c["batch"]
    if c["op"] == "pages":
        rows = B * c["step"] if c["step"] else B * _rows(c)
        pages = rows / c["page"]
        # lengths and counters of both calls, slots out, each changed table entry and free-list entry written twice
        return dict(bytes=4 * (2 * 6 * B + rows + 4 * pages), flops=0)
    width = c["kv"] * (c["d_sem"] + c["d_pos"])
    if c["op"] == "write":
        T = B * c["rows"] * (0.65 if c["ragged"] else 1.0)
        return dict(bytes=T * (3 * width + 4) + T / c["page"] * c["kv"] * 4, flops=3 * T * width)
    if c["op"] == "update":
        n = B * c["due"] * c["group"]
        return dict(bytes=n * width + B * c["kv"] * (c["d_sem"] + c["d_pos"]) * 4, flops=4 * n * width)
    rows = B * _rows(c)
    dk = c["d_pos"] + (c["d_sem"] if c["variant"] == "mla" else 0)
    q = B * c["q_len"] * c["heads"]
    return dict(bytes=rows * width + rows / c["page"] * c["kv"] * 8 + q * (dk + c["d_sem"]) * 2 + q * 4,
                flops=2 * rows * c["q_len"] * c["heads"] * (dk + c["d_sem"]))


# -------------------------------------------------------------------------------------------- 64-bit definitions
def _exact_pages(s):
    """The update one request and one page at a time, on Python lists."""
    c = s["case"]
    P, gr = c["page"], c["group"]
    table = s["table"].cpu().tolist()
    free, top = s["free"].cpu().tolist(), int(s["n_free"])
    held = list(zip(s["held_rep"].cpu().tolist(), s["held_tok"].cpu().tolist()))

    def present(r, t):
        return set(range(_cdiv(r, P))) | set(range(r * gr // P, _cdiv(t, P)))

    def update(target):
        nonlocal top
        gone = [(b, e) for b, (h, n) in enumerate(zip(held, target)) for e in sorted(present(*h) - present(*n))]
        for b, e in reversed(gone):
            free[top] = table[b][e]
            table[b][e] = -1
            top += 1
        slots, offsets = [], [0]
        for b, (h, n) in enumerate(zip(held, target)):
            for e in sorted(present(*n) - present(*h)):
                top -= 1
                table[b][e] = free[top]
            for x in list(range(h[0], n[0])) + list(range(max(h[1], n[0] * gr), n[1])):
                slots.append(table[b][x // P] * P + x % P)
            offsets.append(len(slots))
        held[:] = target
        return slots, offsets

    first = s["after"] if c["step"] else s["n_tok"]
    reps = s["n_rep"].cpu().tolist()
    slots, offsets = update(list(zip(reps, first.cpu().tolist())))
    update(list(zip(reps, s["n_tok"].cpu().tolist())) if c["step"] else [(0, 0)] * c["batch"])
    t = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    slots += [-1] * (s["n_rows"] - len(slots))
    return dict(slots=t(slots), offsets=t(offsets), table=t(table), free=t(free), n_free=t([top]), status=t([0]))


def _round_e4m3(x):
    """Nearest e4m3 value of each 64-bit x (ties to even mantissa, saturating), from the format's definition."""
    a = x.abs().clamp(max=448.0)
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))
    e = torch.where(torch.ldexp(torch.ones_like(a), e) > a.clamp(min=2.0 ** -6), e - 1, e)
    step = torch.exp2(e - 3)
    return torch.copysign(torch.round(a / step) * step, x)          # torch.round: ties to even


def _exact_write(s):
    c = s["case"]
    P, kv = c["page"], c["kv"]
    slots = s["slots"].long()
    page, off = slots // P, slots % P
    sem, pos = s["pages_sem"].view(FP8).double(), s["pages_pos"].view(FP8).double()
    res = dict(sem=sem, pos=pos, scale_sem=s["scale_sem"].double())
    if s["scale_pos"] is not None:
        res["scale_pos"] = s["scale_pos"].double()
    groups = [[("sem", s["rows_sem"]), ("pos", s["rows_pos"])]] if c["variant"] == "mla" else [[("sem", s["rows_sem"])], [("pos", s["rows_pos"])]]
    for parts in groups:
        scale = res["scale_" + parts[0][0]]
        top = torch.zeros_like(scale)
        first = torch.full((scale.shape[0],), P, device=slots.device)   # first row written in each page, P: none
        for o in reversed(range(P)):                                # the rows at place o of their pages: each page once
            at = off == o
            for _, x in parts:
                top[page[at]] = torch.maximum(top[page[at]], x[at].double().abs().amax(-1))
            first[page[at]] = o
        want = torch.full_like(top, 2.0 ** MIN_EXP)
        for e in range(MIN_EXP, 121):
            want = torch.where(top > 448 * want, 2 * want, want)
        touched, opened = (first < P)[:, None], (first == 0)[:, None]
        new = torch.where(opened, want, torch.maximum(want, scale))
        new = torch.where(touched, new, scale)
        for k, x in parts:
            old = res[k]
            again = _round_e4m3(old * (scale / new)[:, :, None, None])
            keep = (torch.arange(P, device=slots.device) < torch.where(first < P, first, 0)[:, None])[:, None, :, None] & (new > scale)[:, :, None, None]
            res[k] = torch.where(keep, again, old)
            res[k][page, :, off] = _round_e4m3(x.double() / new[page][:, :, None])
        res["scale_" + parts[0][0]] = new
    return res


def _exact_rows(s, b, x, which):
    c = s["case"]
    P = c["page"]
    page = s["table"][b, x // P].long()
    scale = s["scale_pos"] if which == "pos" and c["variant"] == "gqa" else s["scale_sem"]
    return (s["pages_" + which].view(FP8)[page, :, x % P].double() * scale[page].double()[..., None]).transpose(0, 1)


def _exact_attend(s):
    c = s["case"]
    Q, H, kv = c["q_len"], c["heads"], c["kv"]
    rep = H // kv
    out = torch.zeros((c["batch"], Q, H, c["d_sem"]), dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], Q, H), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(c["batch"]):
        r, t = int(s["n_rep"][b]), int(s["n_tok"][b])
        for j in range(Q):
            last = t - Q + 1 + j                                    # rows below `last` are seen
            x = torch.cat([torch.arange(min(r, max(last, 0)), device=DEV), torch.arange(r * c["group"], max(last, r * c["group"]), device=DEV)])
            if not x.numel():
                continue
            v = _exact_rows(s, b, x, "sem")                         # [kv, R, d]
            k = _exact_rows(s, b, x, "pos")
            q = s["q_pos"][b, j].double().view(kv, rep, -1)
            if c["variant"] == "mla":
                k = torch.cat([v, k], -1)
                q = torch.cat([s["q_sem"][b, j].double().view(kv, rep, -1), q], -1)
            z = torch.einsum("hqd,hrd->hqr", q, k) * _scale_of(c)
            lse[b, j] = torch.logsumexp(z, -1).reshape(H)
            out[b, j] = torch.einsum("hqr,hrd->hqd", torch.softmax(z, -1), v).reshape(H, -1)
    return dict(out=out, lse=lse)


def _exact_update(s):
    c = s["case"]
    gr, kv = c["group"], c["kv"]
    res = dict(rep_sem=s["rep_sem"].double(), rep_pos=s["rep_pos"].double(),
               anchor=torch.full((c["batch"], kv), -1, dtype=torch.int32, device=DEV), n_rep=s["n_rep"].clone())
    for b in range(c["batch"]):
        r, t = int(s["n_rep"][b]), int(s["n_tok"][b])
        if t - r * gr < c["window"] + gr:
            continue
        x = torch.arange(r * gr, (r + 1) * gr, device=DEV)
        v, k = _exact_rows(s, b, x, "sem"), _exact_rows(s, b, x, "pos")
        full = torch.cat([v, k], -1) if c["variant"] == "mla" else k
        z = torch.einsum("hgd,hd->hg", full, s["qbar"][b].double()) * _scale_of(c)
        top = z.argmax(-1)
        res["rep_sem"][b] = torch.einsum("hg,hgd->hd", torch.softmax(z, -1), v)
        res["rep_pos"][b] = k[torch.arange(kv, device=DEV), top]
        res["anchor"][b] = top.int()
        res["n_rep"][b] += 1
    return res


def exact(case, seed):
    s = prepare(case, seed)
    return dict(pages=_exact_pages, write=_exact_write, attend=_exact_attend, update=_exact_update)[case["op"]](s)
