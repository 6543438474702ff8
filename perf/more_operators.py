"""Measured cases of a speculative decode step on a paged 4-bit cache: rows quantised as they are written and read back,
decode attention over the pages, the online condensation of a group, rotary positions of queries and keys, and the
verification of drafted tokens against the target's probabilities.

`run` computes each operator either through the library (`own` true) or in its plain form, elementary torch operations in
32 bits (64 for angles, for sums of probabilities and for the importance scores, whose order decides the anchors).  A case
names its operator in "op":

  store   lca_paged4_write, then lca_paged4_read of the same rows
  read    lca_paged4_read
  attend  lca_decode_attention_paged4
  update  lca_decode_update_paged4
  rope    lca_rope
  verify  lca_verify_drafts

The 4-bit format: a value is  code * 2^(exponent of its row - shift of its block), blocks of 32 columns.  Codes have a sign
and one of the magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6.  Eight of them fill a 32-bit word: value i has its magnitude's index in
bits 4 i .. 4 i + 2, and its sign in bit 8 i + 7 (i < 4) or 8 (i - 4) + 3.  The exponent is a byte, 127 more than its value,
for each row and KV head (latent and rope key of MLA share it); shifts are four bits, two blocks to a byte, 0 to 14, and 15
says that the block's values are NaN.  The scale of a block is the smallest power of two with max|x| <= 6 * scale over its
finite elements, the row's exponent that of its largest block, and no shift is above 14.
Row space and tables are those of the paged 8-bit cache: token n of a sequence is row n, representative j row j, rows
[n_rep, n_rep * g) are absent, block_table[b, x / P] names the page of row x.
"""
import math

import torch

own = False

DEV = "cuda"
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
SIGN_BIT = (7, 15, 23, 31, 3, 11, 19, 27)
#: exponent of a row of zeros, or of values below it
MIN_EXP = -94
MAX_SHIFT, NAN_SHIFT = 14, 15


# ------------------------------------------------------------------------------------------------------------- cases
def _cache(op, variant, batch, kv, d_sem, d_pos, page, **more):
    return dict(op=op, variant=variant, batch=batch, kv=kv, d_sem=d_sem, d_pos=d_pos, page=page, **more)


def _context(context, window, group=64, ragged=False, condensed=True):
    return dict(context=context, window=window, group=group, ragged=ragged, condensed=condensed)


def listed():
    return [
        # the row of one new token for each of 64 sequences, 512 + 64 wide latents, quantised and read back
        dict(name="store step mla 64", **_cache("store", "mla", 64, 1, 512, 64, 64, rows=1, ragged=False)),
        # ragged prompts of odd lengths, 8 KV heads of 128, pages of 32 rows
        dict(name="store prompt gqa 9", **_cache("store", "gqa", 9, 8, 128, 128, 32, rows=4999, ragged=True)),
        # the condensed caches of 64 sequences back to bf16, to hand them to another server
        dict(name="read prompt mla 64", **_cache("read", "mla", 64, 1, 512, 64, 64, rows=5056, ragged=False)),
        # a single request with three drafts, 16 heads: latency of one short decode step
        dict(name="attend mla 1x32K h16 q4", **_cache("attend", "mla", 1, 1, 512, 64, 64, heads=16, q_len=4, **_context(32768, 2048))),
        # 64 sequences with 65536 tokens of context each, 32 query heads on 8 KV heads
        dict(name="attend gqa 64x64K", **_cache("attend", "gqa", 64, 8, 128, 128, 64, heads=32, q_len=1, **_context(65536, 4096))),
        # the same contexts, 128 heads over one latent cache
        dict(name="attend mla 64x64K", **_cache("attend", "mla", 64, 1, 512, 64, 64, heads=128, q_len=1, **_context(65536, 4096))),
        # the earliest 64 cached tokens of each of 64 sequences become one representative
        dict(name="update mla 64", **_cache("update", "mla", 64, 1, 512, 64, 64, heads=128, due=1.0, **_context(65536, 4096))),
        # 8 KV heads, groups of 32, part of the sequences due
        dict(name="update gqa 48", **_cache("update", "gqa", 48, 8, 128, 128, 16, heads=32, due=0.5, **_context(20000, 1024, 32))),
        # four tokens of each of 64 sequences: the last 64 of 192 columns of 128 heads, and the rope key behind the latent
        dict(name="rope step mla 256", op="rope", tokens=256, heads=128, kv=1, d=64, rot=64, before=128, interleaved=True,
             scaled=True, inverse=False, far=131072),
        # a prompt's queries and keys as they lie in a fused projection
        dict(name="rope prompt gqa 32768", op="rope", tokens=32768, heads=32, kv=8, d=128, rot=128, before=0, interleaved=False,
             scaled=False, inverse=False, far=32768),
        # a single request with seven drafts
        dict(name="verify 1x7 32001", op="verify", batch=1, drafts=7, vocab=32001, type="bf16", greedy_draft=False, ragged=False),
        # 64 requests with four drafts each
        dict(name="verify 64x4 128000", op="verify", batch=64, drafts=4, vocab=128000, type="fp32", greedy_draft=False, ragged=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "read", "attend", "attend", "attend", "update", "rope", "verify"])
    if op == "rope":
        d = rng.choice([64, 64, 128])
        rot = rng.choice([d, d, d // 2])
        mla = rng.random() < 0.5
        kv = 1 if mla else rng.choice([1, 2, 4, 8])
        heads = rng.choice([16, 40, 128]) if mla else kv * rng.choice([1, 4, 7])
        return dict(op=op, tokens=_log(rng, 1, 8000), heads=heads, kv=kv, d=d, rot=rot, before=rng.choice([0, 64, 128]) if mla else 0,
                    interleaved=rng.random() < 0.5, scaled=rng.random() < 0.5, inverse=rng.random() < 0.3, far=_log(rng, 100, 1000000))
    if op == "verify":
        return dict(op=op, batch=_log(rng, 1, 64), drafts=rng.randint(1, 8), vocab=_log(rng, 50, 128000), type=rng.choice(["fp32", "bf16"]),
                    greedy_draft=rng.random() < 0.3, ragged=rng.random() < 0.5)
    page = rng.choice([16, 32, 64])
    if rng.random() < 0.5:
        kv, (d_sem, d_pos), variant = 1, rng.choice([(512, 64), (512, 64), (128, 64)]), "mla"
    else:
        kv, (d_sem, d_pos), variant = rng.choice([1, 2, 4, 8]), rng.choice([(128, 128), (128, 128), (64, 64)]), "gqa"
    if op in ("store", "read"):
        rows = rng.choice([1, _log(rng, 2, 3000)])
        return _cache(op, variant, _log(rng, 1, 400 if rows == 1 else 24), kv, d_sem, d_pos, page, rows=rows, ragged=rows > 1)
    if op == "update":
        return _cache(op, variant, _log(rng, 1, 64), kv, d_sem, d_pos, page, heads=kv * rng.choice([1, 4, 16]), due=rng.choice([1.0, 0.3]),
                      **_context(_log(rng, 4000, 40000), 64 * rng.randint(1, 32)))
    condensed = rng.random() < 0.5
    context = _log(rng, 4500, 120000) if condensed else _log(rng, 1, 20000)
    rows = 4096 + context // 64 if condensed else context
    batch = max(1, min(_log(rng, 1, 64), 200000 // rows))
    heads = rng.choice([16, 32, 40, 64, 128]) if variant == "mla" else kv * rng.choice([1, 2, 4, 7, 8, 16])
    q_len = rng.choice([1, 1, 2, 3, 7]) if heads // kv <= 32 else 1
    return _cache(op, variant, batch, kv, d_sem, d_pos, page, heads=heads, q_len=q_len,
                  **_context(context, 64 * rng.randint(4, 64) if condensed else 0, 64, rng.random() < 0.7, condensed))


# ------------------------------------------------------------------------------------------------------------ inputs
def _cdiv(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _lengths(c, g):
    """(n_rep, n_tok) of every sequence, int32: a context condensed in groups with a window, or not condensed at all."""
    B, L = c["batch"], c["context"]
    n_tok = torch.full((B,), L, device=DEV)
    if c["ragged"]:
        n_tok = n_tok - (torch.rand(B, generator=g, device=DEV) * 0.6 * L).long()
        n_tok[0] = L
    n_rep = ((n_tok - c["window"]) // c["group"]).clamp(min=0) if c["condensed"] else torch.zeros_like(n_tok)
    return n_rep.int(), n_tok.int()


def _tables(n_rep, n_tok, group, page, g):
    """(block_table, n_pages): pages of a shuffled pool for every row that is present, -1 elsewhere."""
    B = n_tok.numel()
    e = torch.arange(max(1, _cdiv(int(n_tok.max()), page)), device=DEV)
    r, t = n_rep.long()[:, None], n_tok.long()[:, None]
    used = (e < (r + page - 1) // page) | ((e >= r * group // page) & (e < (t + page - 1) // page))
    n = int(used.sum())
    table = torch.full((B, e.numel()), -1, dtype=torch.int32, device=DEV)
    table[used] = torch.randperm(n, generator=g, device=DEV).int()
    return table, max(n, 1)


def _words(shape, g):
    """Packed codes of values N(0, 2^2): words taken at random from a pool of quantised ones."""
    pool = _pack(_codes(_randn(g, 1 << 17, 8) * 2))[:, 0]
    out = torch.empty(shape, dtype=torch.int32, device=DEV)
    flat = out.view(-1)
    for s in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - s)
        flat[s:s + n] = pool[torch.randint(0, pool.numel(), (n,), generator=g, device=DEV)]
    return out


def _pages(c, n_pages, g):
    """A pool of pages with rows of unit scale, whose blocks differ by factors of up to four."""
    kv, P = c["kv"], c["page"]
    s = {}
    for k in ("sem", "pos"):
        d = c["d_" + k]
        s["pages_" + k] = _words((n_pages, kv, P, d // 8), g).view(torch.uint8)
        lo, hi = (torch.randint(0, 3, (n_pages, kv, P, d // 64), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2))
        s["shift_" + k] = lo | (hi << 4)
        s["exp_" + k] = torch.randint(125, 128, (n_pages, kv, P), generator=g, device=DEV, dtype=torch.uint8)
    if c["variant"] == "mla":
        s["exp_pos"] = None
    return s


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = dict(case=c)
    if c["op"] == "rope":
        T, H, kv, d, rot, before = (c[k] for k in ("tokens", "heads", "kv", "d", "rot", "before"))
        if before:                  # MLA: columns without positions in front of a head's rotated ones, the key behind a latent
            s["q"] = _randn(g, T, H, before + d).bfloat16()[:, :, before:]
            s["k"] = _randn(g, T, 1, 512 + d).bfloat16()[:, :, 512:] if kv == 1 else _randn(g, T, kv, d).bfloat16()
        else:                       # queries, keys and values of one projection
            qkv = _randn(g, T, H + 2 * kv, d).bfloat16()
            s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + kv]
        s["positions"] = torch.randint(0, c["far"], (T,), generator=g, device=DEV, dtype=torch.int32)
        i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
        f = 10000.0 ** (-2 * i / rot)
        s["factor"] = 1.0
        if c["scaled"]:             # fast columns as they are, slow ones with their positions divided by 32, a ramp between them
            turns = 4096 * f / (2 * math.pi)
            keep = ((turns - 1) / 31).clamp(0, 1)
            f = f * keep + f / 32 * (1 - keep)
            s["factor"] = 0.1 * math.log(32) + 1
        s["freqs"] = f
        return s
    if c["op"] == "verify":
        B, K, V = c["batch"], c["drafts"], c["vocab"]
        dt = torch.float32 if c["type"] == "fp32" else torch.bfloat16
        z = _randn(g, B, K + 1, V) * 2.5
        s["target"] = torch.softmax(z, -1).to(dt)
        q = torch.softmax(z[:, :K] + _randn(g, B, K, V) * 0.7, -1)
        if c["greedy_draft"]:
            s["draft"], s["tokens"] = None, q.argmax(-1).int()
        else:
            s["draft"] = q.to(dt)
            e = -torch.log(torch.rand((B, K, V), generator=g, device=DEV).clamp(min=1e-30))
            s["tokens"] = (q / e).argmax(-1).int()
        s["u_accept"] = torch.rand((B, K), generator=g, device=DEV)
        s["u_sample"] = torch.rand((B,), generator=g, device=DEV)
        s["n_draft"] = torch.randint(0, K + 1, (B,), generator=g, device=DEV, dtype=torch.int32) if c["ragged"] else None
        s["n_tok"] = torch.randint(K + 1, 5000, (B,), generator=g, device=DEV, dtype=torch.int32)
        return s
    if c["op"] in ("store", "read"):
        B, P = c["batch"], c["page"]
        if c["rows"] == 1:          # one new row in a page of its own sequence, at any place of the page
            n_pages = B + 3
            slots = torch.randperm(n_pages, generator=g, device=DEV)[:B] * P + torch.randint(0, P, (B,), generator=g, device=DEV)
        else:
            lens = torch.full((B,), c["rows"], device=DEV)
            if c["ragged"]:
                spread = (torch.arange(1, B + 1, device=DEV) * 0.6180339887) % 1.0          # the same rows in all for every seed
                lens = (lens * (0.3 + 0.7 * spread)).long().clamp(min=1)[torch.randperm(B, generator=g, device=DEV)]
            need = _cdiv(c["rows"], P)
            n_pages = B * need
            pages = torch.randperm(n_pages, generator=g, device=DEV).view(B, need)
            x = torch.arange(c["rows"], device=DEV)
            slots = (pages.gather(1, (x // P).expand(B, -1)) * P + x % P)[x < lens[:, None]]
        s.update(_pages(c, n_pages, g))
        s["slots"] = slots.int()
        T = slots.numel()
        if c["op"] == "store":      # rows of different size, columns of different size
            for k in ("sem", "pos"):
                d = c["d_" + k]
                gain = torch.exp(0.5 * _randn(g, T, 1, 1)) * torch.exp(0.5 * _randn(g, c["kv"], d))
                s["rows_" + k] = (_randn(g, T, c["kv"], d) * gain).bfloat16()
        return s
    n_rep, n_tok = _lengths(c, g)
    if c["op"] == "update":
        due = torch.rand(c["batch"], generator=g, device=DEV) < c["due"]
        R = c["window"] + c["group"]
        n_tok = torch.where(due, n_rep * c["group"] + R, torch.minimum(n_tok, n_rep * c["group"] + R - 1)).int()
    s.update(n_rep=n_rep, n_tok=n_tok)
    s["table"], n_pages = _tables(n_rep, n_tok, c["group"], c["page"], g)
    s.update(_pages(c, n_pages, g))
    if c["op"] == "update":
        dk = c["d_pos"] + (c["d_sem"] if c["variant"] == "mla" else 0)
        s["qbar"] = _randn(g, c["batch"], c["kv"], dk) * 0.3
        s["rep_sem"] = torch.zeros((c["batch"], c["kv"], c["d_sem"]), dtype=torch.bfloat16, device=DEV)
        s["rep_pos"] = torch.zeros((c["batch"], c["kv"], c["d_pos"]), dtype=torch.bfloat16, device=DEV)
        return s
    lead = (c["batch"], c["q_len"], c["heads"])
    s["q_sem"] = _randn(g, *lead, c["d_sem"]).bfloat16() if c["variant"] == "mla" else None
    s["q_pos"] = _randn(g, *lead, c["d_pos"]).bfloat16()
    return s


def _scale_of(c):
    return 1.0 / math.sqrt(192.0 if c["variant"] == "mla" else c["d_pos"])


# ------------------------------------------------------------------------------------------------------ plain forms
def _codes(x):
    """Nearest code of each value: magnitude index, and 8 more where the value is negative.  Ties go to the even index."""
    a = x.abs()
    m = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5).int()
    return m + 8 * (x < 0).int()


def _pack(codes):
    """Codes [..., n] -> words [..., n / 8] (int32)."""
    c = codes.view(codes.shape[:-1] + (-1, 8)).long()
    at = torch.arange(8, device=codes.device)
    w = (((c & 7) << (4 * at)) | ((c >> 3) << torch.tensor(SIGN_BIT, device=codes.device))).sum(-1)
    return (w - ((w >> 31) << 32)).int()


def _unpack(pages):
    """Bytes [..., d / 2] -> values of the codes [..., d], fp32."""
    w = pages.view(torch.int32)[..., None]
    m = (w >> (4 * torch.arange(8, device=w.device, dtype=torch.int32))) & 7
    sign = (w >> torch.tensor(SIGN_BIT, device=w.device, dtype=torch.int32)) & 1
    e, f = m >> 1, m & 1
    v = torch.where(e > 0, torch.ldexp(2.0 + f, e - 2), 0.5 * f)
    return torch.where(sign > 0, -v, v).flatten(-2)


def _exponent_of(s, which):
    return s["exp_sem"] if s["exp_" + which] is None else s["exp_" + which]


def _values(s, which, at):
    """Values that the rows `at` (an index into [n_pages, kv, P]) of a pool stand for, fp32 [..., d]."""
    sh = s["shift_" + which][at].int()
    sh = torch.stack([sh & 15, sh >> 4], -1).flatten(-2)
    e = _exponent_of(s, which)[at].int()[..., None] - 127 - sh
    scale = torch.where(sh == NAN_SHIFT, torch.full((), math.nan, device=DEV), torch.ldexp(torch.ones_like(e, dtype=torch.float32), e))
    v = _unpack(s["pages_" + which][at])
    return (v.view(v.shape[:-1] + (-1, 32)) * scale[..., None]).flatten(-2)


def _block_exponents(x):
    """Smallest e with max|x| <= 6 * 2^e over the finite elements of each block of 32 columns; far below where it is 0."""
    a = x.view(x.shape[:-1] + (-1, 32)).abs()
    a = torch.where(torch.isfinite(a), a, torch.zeros_like(a)).amax(-1)
    m, e = torch.frexp(a)                                # a = m * 2^e, 0.5 <= m < 1, and 6 = 0.75 * 2^3
    return torch.where(a > 0, torch.where(m > 0.75, e - 2, e - 3), torch.full_like(e, -1000))


def _plain_write(s):
    c = s["case"]
    P, kv = c["page"], c["kv"]
    slots = s["slots"].long()
    page, off, head = (slots // P)[:, None], (slots % P)[:, None], torch.arange(kv, device=DEV)[None]
    x = {k: s["rows_" + k].float() for k in ("sem", "pos")}
    e = {k: _block_exponents(v) for k, v in x.items()}
    top = {k: v.amax(-1).clamp(min=MIN_EXP) for k, v in e.items()}
    if c["variant"] == "mla":
        top["sem"] = top["pos"] = torch.maximum(top["sem"], top["pos"])
    for k, v in x.items():
        block = v.view(v.shape[:-1] + (-1, 32))
        shift = (top[k][..., None] - e[k]).clamp(max=MAX_SHIFT)
        scale = torch.ldexp(torch.ones_like(shift, dtype=torch.float32), top[k][..., None] - shift)
        codes = _codes((block / scale[..., None]).flatten(-2))
        shift = torch.where(torch.isnan(block).any(-1), torch.full_like(shift, NAN_SHIFT), shift).byte()
        s["pages_" + k][page, head, off] = _pack(codes).view(torch.uint8)
        s["shift_" + k][page, head, off] = shift[..., 0::2] | (shift[..., 1::2] << 4)
        if s["exp_" + k] is not None:
            s["exp_" + k][page, head, off] = (top[k] + 127).byte()


def _plain_read(s):
    P = s["case"]["page"]
    slots = s["slots"].long()
    at = ((slots // P)[:, None], torch.arange(s["case"]["kv"], device=DEV)[None], (slots % P)[:, None])
    return dict(sem=_values(s, "sem", at).bfloat16(), pos=_values(s, "pos", at).bfloat16())


def _plain_store(s):
    _plain_write(s)
    return _plain_read(s)


def _gather_rows(s, x, which):
    """Values [B, kv, R, d] of the logical rows x [B, R] (rows outside the table or on no page read page 0)."""
    c = s["case"]
    P = c["page"]
    page = s["table"].gather(1, (x // P).clamp(max=s["table"].shape[1] - 1)).long().clamp(min=0)
    return _values(s, which, (page[:, None], torch.arange(c["kv"], device=DEV)[None, :, None], (x % P)[:, None]))


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
    split = lambda q, d: q.float().view(B, Q, kv, rep, d).permute(0, 2, 1, 3, 4).reshape(B, kv, Q * rep, d)  # noqa: E731
    logit = split(s["q_pos"], c["d_pos"]) @ pos.transpose(2, 3)
    if c["variant"] == "mla":
        logit = logit + split(s["q_sem"], c["d_sem"]) @ sem.transpose(2, 3)
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
    gr = c["group"]
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


def _plain_rope(s):
    c = s["case"]
    rot = c["rot"]
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos = (torch.cos(angle) * s["factor"]).float()[:, None]
    sin = (torch.sin(angle) * (-s["factor"] if c["inverse"] else s["factor"])).float()[:, None]

    def turn(x):
        y = x.float()
        a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if c["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
        u, v = a * cos - b * sin, a * sin + b * cos
        r = torch.stack([u, v], -1).flatten(-2) if c["interleaved"] else torch.cat([u, v], -1)
        return torch.cat([r, y[..., rot:]], -1).bfloat16()
    return dict(q=turn(s["q"]), k=turn(s["k"]))


def _plain_verify(s):
    c = s["case"]
    B, K = c["batch"], c["drafts"]
    tok = s["tokens"].long()
    n = s["n_draft"].long() if c["ragged"] else torch.full((B,), K, device=DEV)
    p = s["target"][:, :K].gather(2, tok[..., None])[..., 0].double()
    q = torch.ones_like(p) if s["draft"] is None else s["draft"].gather(2, tok[..., None])[..., 0].double()
    i = torch.arange(K, device=DEV)
    ok = (s["u_accept"].double() * q < p) & (i < n[:, None])
    taken = torch.cumprod(ok.long(), 1).sum(1)
    rejected = taken < n
    b = torch.arange(B, device=DEV)
    row = s["target"][b, taken].double()
    at = taken.clamp(max=K - 1)
    if s["draft"] is None:
        minus = torch.zeros_like(row).scatter_(1, tok[b, at][:, None], math.inf)
    else:
        minus = s["draft"][b, at].double()
    rest = torch.where(rejected[:, None], (row - minus).clamp(min=0), row)
    rest = torch.where((rest.sum(1) > 0)[:, None], rest, row)
    cum = torch.cumsum(rest, 1)
    hit = (cum > s["u_sample"].double()[:, None] * cum[:, -1:]) & (rest > 0)
    last = rest.shape[1] - 1 - (rest > 0).int().flip(1).argmax(1)
    new = torch.where(hit.any(1), hit.int().argmax(1), last)
    out = torch.where(i < taken[:, None], s["tokens"], torch.full_like(s["tokens"], -1))
    out = torch.cat([out, torch.full_like(out[:, :1], -1)], 1)
    out[b, taken] = new.int()
    return dict(accepted=taken.int(), tokens=out, n_tok=(s["n_tok"] - (n - taken).int()))


# ---------------------------------------------------------------------------------------------------------- one pass
def _handle(s):
    """Parameters, cache descriptor, outputs and workspace that a user's program keeps beside its cache."""
    from paper_2604_12452_b200 import binding as B
    c = s["case"]
    h = s["handle"] = dict(B=B)
    if c["op"] == "rope":
        h["q"] = torch.empty((c["tokens"], c["heads"], c["d"]), dtype=torch.bfloat16, device=DEV)
        h["k"] = torch.empty((c["tokens"], c["kv"], c["d"]), dtype=torch.bfloat16, device=DEV)
        return h
    if c["op"] == "verify":
        h["accepted"] = torch.empty(c["batch"], dtype=torch.int32, device=DEV)
        h["tokens"] = torch.empty((c["batch"], c["drafts"] + 1), dtype=torch.int32, device=DEV)
        h["n_tok"] = torch.empty(c["batch"], dtype=torch.int32, device=DEV)
        return h
    h["p"] = B.make_params(c["variant"], c["batch"], 1, c.get("heads", c["kv"]), c["kv"], c["d_sem"], c["d_pos"],
                           c.get("group", 64), c.get("window", 0), _scale_of(c))
    h["cache"] = B.paged4_cache(s["pages_sem"], s["pages_pos"], s["shift_sem"], s["shift_pos"], s["exp_sem"], s["exp_pos"], s.get("table"))
    if c["op"] in ("store", "read"):
        T = s["slots"].numel()
        h["sem"] = torch.empty((T, c["kv"], c["d_sem"]), dtype=torch.bfloat16, device=DEV)
        h["pos"] = torch.empty((T, c["kv"], c["d_pos"]), dtype=torch.bfloat16, device=DEV)
    if c["op"] == "attend":
        h["out"] = torch.empty((c["batch"], c["q_len"], c["heads"], c["d_sem"]), dtype=torch.bfloat16, device=DEV)
        h["lse"] = torch.empty((c["batch"], c["q_len"], c["heads"]), dtype=torch.float32, device=DEV)
        h["ws"] = B.workspace_paged4(h["p"], h["cache"], c["q_len"], DEV)
    if c["op"] == "update":
        h["anchor"] = torch.empty((c["batch"], c["kv"]), dtype=torch.int32, device=DEV)
        h["n_rep"] = torch.empty_like(s["n_rep"])
        h["ws"] = B.workspace(h["p"], B.LCA_WS_UPDATE, DEV)
    return h


def _own(s):
    c = s["case"]
    h = s.get("handle") or _handle(s)
    B = h["B"]
    if c["op"] == "rope":
        B.rope(s["q"], s["k"], s["positions"], s["freqs"], interleaved=c["interleaved"], inverse=c["inverse"], factor=s["factor"],
               q_out=h["q"], k_out=h["k"])
        return dict(q=h["q"], k=h["k"])
    if c["op"] == "verify":
        B.verify_drafts(s["target"], s["draft"], s["tokens"], s["u_accept"], s["u_sample"], n_draft=s["n_draft"], n_tok=s["n_tok"],
                        accepted=h["accepted"], out=h["tokens"], n_tok_out=h["n_tok"])
        return dict(accepted=h["accepted"], tokens=h["tokens"], n_tok=h["n_tok"])
    if c["op"] in ("store", "read"):
        if c["op"] == "store":
            B.paged4_write(h["p"], h["cache"], s["rows_sem"], s["rows_pos"], s["slots"])
        B.paged4_read(h["p"], h["cache"], s["slots"], h["sem"], h["pos"])
        return dict(sem=h["sem"], pos=h["pos"])
    if c["op"] == "attend":
        B.decode_attention_paged4(h["p"], h["cache"], s["q_sem"], s["q_pos"], s["n_rep"], s["n_tok"], out=h["out"], lse=h["lse"], ws=h["ws"])
        return dict(out=h["out"], lse=h["lse"])
    B.decode_update_paged4(h["p"], h["cache"], None, None, s["n_rep"], s["n_tok"], h["n_rep"], s["rep_sem"], s["rep_pos"],
                           qbar=s["qbar"], anchor=h["anchor"], ws=h["ws"])
    return dict(rep_sem=s["rep_sem"], rep_pos=s["rep_pos"], anchor=h["anchor"], n_rep=h["n_rep"])


def run(state):
    if own:
        return _own(state)
    return dict(store=_plain_store, read=_plain_read, attend=_plain_attend, update=_plain_update, rope=_plain_rope,
                verify=_plain_verify)[state["case"]["op"]](state)


# -------------------------------------------------------------------------------------------------------------- work
def _rows(c):
    """Expected number of rows of a sequence (ragged lengths are 0.4 to 1 times the context)."""
    L = c["context"] * (0.7 if c["ragged"] and c["batch"] > 1 else 1.0)
    if not c["condensed"] or L < c["window"] + c["group"]:
        return L
    m = (L - c["window"]) // c["group"]
    return m + L - m * c["group"]


def work(case):
    c = case
    if c["op"] == "rope":
        n = c["tokens"] * (c["heads"] + c["kv"]) * c["d"]
        return dict(bytes=4 * n + 4 * c["tokens"] + 4 * c["rot"], flops=3 * n)
    if c["op"] == "verify":
        size = 4 if c["type"] == "fp32" else 2
        rows = 1 if c["greedy_draft"] else 2                    # the target's row, and the drafter's where a draft is rejected
        return dict(bytes=c["batch"] * (rows * c["vocab"] * size + c["drafts"] * (12 + 2 * size) + 16), flops=3 * c["batch"] * c["vocab"])
    B, width = c["batch"], c["kv"] * (c["d_sem"] + c["d_pos"])
    held = width / 2 + width / 64 + (1 if c["variant"] == "mla" else 2) * c["kv"]          # bytes of a cached row
    if c["op"] in ("store", "read"):
        T = B * c["rows"] * (0.65 if c["ragged"] else 1.0)
        return dict(bytes=T * (held + 2 * width * (2 if c["op"] == "store" else 1) + 4), flops=2 * T * width)
    if c["op"] == "update":
        n = B * c["due"] * c["group"]
        return dict(bytes=n * held + B * c["kv"] * (c["d_sem"] + c["d_pos"]) * 4, flops=4 * n * width)
    rows = B * _rows(c)
    dk = c["d_pos"] + (c["d_sem"] if c["variant"] == "mla" else 0)
    q = B * c["q_len"] * c["heads"]
    return dict(bytes=rows * held + q * (dk + c["d_sem"]) * 2 + q * 4, flops=2 * rows * c["q_len"] * c["heads"] * (dk + c["d_sem"]))


# -------------------------------------------------------------------------------------------- 64-bit definitions
def _exact_rows(s, which, page, off):
    """Values of the rows at (page, off), [kv, n, d] in 64 bits, bit by bit from the format's definition."""
    raw = s["pages_" + which][page, :, off].transpose(0, 1).long()            # [kv, n, d / 2] bytes
    d = 2 * raw.shape[-1]
    v = torch.empty(raw.shape[:-1] + (d,), dtype=torch.float64, device=DEV)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
    bit = lambda i: (raw[..., i // 8::4] >> (i % 8)) & 1  # noqa: E731          bit i of each word
    for i in range(8):
        m = level[bit(4 * i) + 2 * bit(4 * i + 1) + 4 * bit(4 * i + 2)]
        v[..., i::8] = m * (1 - 2 * bit(8 * i + 7 if i < 4 else 8 * i - 29)).double()
    shift = s["shift_" + which][page, :, off].transpose(0, 1).long()
    e = s["exp_sem" if s["exp_" + which] is None else "exp_" + which][page, :, off].transpose(0, 1).double() - 127
    for j in range(d // 32):
        sh = (shift[..., j // 2] >> (4 * (j % 2))) & 15
        v[..., 32 * j:32 * j + 32] *= torch.where(sh == 15, math.nan, torch.exp2(e - sh.double()))[..., None]
    return v


def _exact_read(s):
    page, off = (s["slots"].long() // s["case"]["page"], s["slots"].long() % s["case"]["page"])
    return {k: _exact_rows(s, k, page, off).transpose(0, 1) for k in ("sem", "pos")}


def _exact_store(s):
    """What the format makes of each row, without packing it."""
    c = s["case"]
    level = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
    step = torch.arange(MIN_EXP, 127, device=DEV).double()
    scale, top = {}, {}
    for k in ("sem", "pos"):
        x = s["rows_" + k].double()
        amax = x.reshape(x.shape[:-1] + (-1, 32)).abs().amax(-1)
        scale[k] = torch.searchsorted(6 * torch.exp2(step), amax.contiguous()) + MIN_EXP         # first e with 6 * 2^e >= amax
        top[k] = scale[k].amax(-1, keepdim=True)
    if c["variant"] == "mla":
        top["sem"] = top["pos"] = torch.maximum(top["sem"], top["pos"])
    res = {}
    for k in ("sem", "pos"):
        e = torch.exp2(torch.maximum(scale[k], top[k] - MAX_SHIFT).double()).repeat_interleave(32, -1)
        a = s["rows_" + k].double() / e
        hi = torch.searchsorted(level, a.abs().clamp(max=6.0)).clamp(min=1, max=7)
        lo = hi - 1
        up, down = level[hi] - a.abs(), a.abs() - level[lo]
        pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        res[k] = torch.copysign(level[pick], a) * e
    return res


def _exact_sequence(s, b, x, which):
    P = s["case"]["page"]
    return _exact_rows(s, which, s["table"][b, x // P].long(), x % P)


def _exact_attend(s):
    c = s["case"]
    Q, H, kv = c["q_len"], c["heads"], c["kv"]
    rep = H // kv
    out = torch.zeros((c["batch"], Q, H, c["d_sem"]), dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], Q, H), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(c["batch"]):
        r, t = int(s["n_rep"][b]), int(s["n_tok"][b])
        every = torch.cat([torch.arange(r, device=DEV), torch.arange(r * c["group"], max(t, r * c["group"]), device=DEV)])
        if not every.numel():
            continue
        v_all, k_all = _exact_sequence(s, b, every, "sem"), _exact_sequence(s, b, every, "pos")
        for j in range(Q):
            n = int((every < t - Q + 1 + j).sum())                  # rows that query j sees: the first n
            if not n:
                continue
            v, k = v_all[:, :n], k_all[:, :n]                       # [kv, n, d]
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
        v, k = _exact_sequence(s, b, x, "sem"), _exact_sequence(s, b, x, "pos")
        full = torch.cat([v, k], -1) if c["variant"] == "mla" else k
        z = torch.einsum("hgd,hd->hg", full, s["qbar"][b].double()) * _scale_of(c)
        top = z.argmax(-1)
        res["rep_sem"][b] = torch.einsum("hg,hgd->hd", torch.softmax(z, -1), v)
        res["rep_pos"][b] = k[torch.arange(kv, device=DEV), top]
        res["anchor"][b] = top.int()
        res["n_rep"][b] += 1
    return res


def _exact_rope(s):
    """A pair of columns as a complex number, times factor * e^(+-i angle)."""
    c = s["case"]
    rot, n = c["rot"], c["rot"] // 2
    angle = s["positions"].double()[:, None, None] * s["freqs"]
    turn = torch.polar(torch.full_like(angle, s["factor"]), -angle if c["inverse"] else angle)
    cols = torch.arange(rot, device=DEV)
    first, second = (cols[0::2], cols[1::2]) if c["interleaved"] else (cols[:n], cols[n:])
    res = {}
    for k in ("q", "k"):
        y = s[k].double()
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        res[k] = y
    return res


def _exact_verify(s):
    """One request and one draft at a time."""
    c = s["case"]
    B, K = c["batch"], c["drafts"]
    accepted, tokens, lengths = [], [], []
    drafts, n_tok = s["tokens"].cpu().tolist(), s["n_tok"].cpu().tolist()
    u, us = s["u_accept"].double().cpu().tolist(), s["u_sample"].double().cpu().tolist()
    for b in range(B):
        n = int(s["n_draft"][b]) if c["ragged"] else K
        out, rest = [], None
        for i in range(n):
            x = drafts[b][i]
            q = 1.0 if s["draft"] is None else float(s["draft"][b, i, x])
            if u[b][i] * q < float(s["target"][b, i, x]):
                out.append(x)
                continue
            rest = s["target"][b, i].double()
            if s["draft"] is None:
                rest = rest.clone()
                rest[x] = 0
            else:
                rest = (rest - s["draft"][b, i].double()).clamp(min=0)
            if not float(rest.sum()) > 0:
                rest = s["target"][b, i].double()
            break
        if rest is None:
            rest = s["target"][b, len(out)].double()
        some = rest.nonzero()[:, 0]                             # tokens that can be drawn, in order
        cum = torch.cumsum(rest[some], 0)
        k = int(torch.searchsorted(cum, cum[-1:] * us[b], right=True))
        accepted.append(len(out))
        lengths.append(n_tok[b] - (n - len(out)))
        tokens.append(out + [int(some[min(k, some.numel() - 1)])] + [-1] * (K - len(out)))
    t = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(accepted=t(accepted), tokens=t(tokens), n_tok=t(lengths))


def exact(case, seed):
    s = prepare(case, seed)
    return dict(store=_exact_store, read=_exact_read, attend=_exact_attend, update=_exact_update, rope=_exact_rope,
                verify=_exact_verify)[case["op"]](s)
