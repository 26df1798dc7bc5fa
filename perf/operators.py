"""The operators of the 8-bit paged cache and of beam search, case by case: inputs, plain forms, library calls, 64-bit values.

A case's ``op`` says which operator it is:

* ``attend``: a few new tokens attend over a paged cache held in 8 bits, one scale per 16 tokens, layer, sequence and KV head
  (K and V apart);
* ``append``: rows are rounded to 8 bits and written into the pages, next to tokens that share their block;
* ``fork``: the sequences of a batch become copies of a list of parents (beam search's reordering of the cache);
* ``compact``: live pages move to the lowest page numbers;
* ``beam``: the best continuations over beams and vocabulary.

``own`` picks the library's calls instead of the plain forms.
"""
import math

import torch

own = False

BLOCK = 16  # tokens that share a scale
NEG = float("-inf")


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # one short sequence at the smallest shape: what a single call costs
        dict(name="attend one short", op="attend", layers=1, seqs=1, hq=4, hkv=2, d=64, lo=190, hi=190, rows=1, page=16, fmt="e4m3", dtype="f32"),
        # a long prompt's cache, one new token, one layer: the decode step of a single stream
        dict(name="attend one long", op="attend", layers=1, seqs=1, hq=32, hkv=8, d=128, lo=16384, hi=16384, rows=1, page=64, fmt="int8", dtype="bf16"),
        # eight streams of uneven length, one layer
        dict(name="attend ragged batch", op="attend", layers=1, seqs=8, hq=32, hkv=8, d=128, lo=2048, hi=16384, rows=1, page=64, fmt="e4m3", dtype="bf16"),
        # drafted tokens checked in one call, eight query heads to a KV head, uneven long sequences
        dict(name="attend drafted tokens", op="attend", layers=1, seqs=6, hq=64, hkv=8, d=128, lo=20001, hi=32768, rows=4, page=128, fmt="int8", dtype="bf16"),
        # all layers of a single-precision cache at once
        dict(name="attend fp32 layers", op="attend", layers=8, seqs=3, hq=32, hkv=8, d=128, lo=3000, hi=4096, rows=1, page=32, fmt="int8", dtype="f32"),
        # decoding: every sequence of a large batch writes its new token, some blocks have to be rescaled
        dict(name="append one token", op="append", layers=1, seqs=96, hkv=8, d=128, lo=200, hi=5000, new_lo=1, new_hi=1, page=64, fmt="int8", dtype="bf16", pick=False, of=1),
        # what eviction kept of a 16k prompt goes straight from the prompt's rows into the cache
        dict(name="append kept rows", op="append", layers=16, seqs=1, hkv=8, d=128, lo=0, hi=0, new_lo=1000, new_hi=1024, page=64, fmt="e4m3", dtype="bf16", pick=True, of=16),
        # whole prompts of uneven length, single precision, behind cached prefixes
        dict(name="append prompts", op="append", layers=4, seqs=4, hkv=8, d=128, lo=0, hi=300, new_lo=4000, new_hi=8192, page=32, fmt="int8", dtype="f32", pick=False, of=1),
        # beam search's step: every layer's table follows the parents, open pages are copied
        dict(name="fork beams", op="fork", layers=32, groups=4, beams=8, hkv=8, d=128, lo=1500, hi=4096, page=64, fmt="int8"),
        # a pool with holes after sequences have left
        dict(name="compact pool", op="compact", layers=32, seqs=24, hkv=8, d=128, lo=200, hi=2500, page=64, fmt="e4m3"),
        dict(name="beam small", op="beam", seqs=1, beams=4, vocab=32000, n_out=4, dtype="bf16", finished=False),
        dict(name="beam large", op="beam", seqs=16, beams=8, vocab=128256, n_out=16, dtype="f32", finished=True),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "append", "fork", "compact", "beam"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 5, 8])
    fmt = rng.choice(["int8", "e4m3"])
    page = rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "attend":
        seqs = _log_between(rng, 1, 24)
        layers = rng.choice([1, 1, 2, 4])
        group, rows = rng.choice([1, 2, 3, 4, 7, 8]), rng.choice([1, 1, 1, 2, 3, 5, 8, 16])
        hi = _log_between(rng, 1, min(32768, 190000 // (seqs * layers * max(1, group * rows // 32))))
        return dict(op=op, layers=layers, seqs=seqs, hq=hkv * group, hkv=hkv, d=d, lo=rng.randint(1, hi), hi=hi, rows=rows, page=page, fmt=fmt, dtype=dtype)
    if op == "append":
        seqs = _log_between(rng, 1, 48)
        layers = rng.choice([1, 2, 4])
        new = _log_between(rng, 1, min(8192, 120000 // (seqs * layers)))
        pick = rng.random() < 0.4
        return dict(op=op, layers=layers, seqs=seqs, hkv=hkv, d=d, lo=0, hi=_log_between(rng, 1, 600), new_lo=rng.randint(1, new), new_hi=new,
                    page=page, fmt=fmt, dtype=dtype, pick=pick, of=rng.randint(1, max(1, min(16, 260000 // (seqs * layers * new)))) if pick else 1)
    if op == "fork":
        hi = _log_between(rng, 20, 4096)
        return dict(op=op, layers=_log_between(rng, 1, 32), groups=_log_between(rng, 1, 4), beams=rng.randint(2, 8), hkv=hkv, d=d,
                    lo=rng.randint(1, hi), hi=hi, page=page, fmt=fmt)
    if op == "compact":
        hi = _log_between(rng, 30, 2500)
        return dict(op=op, layers=_log_between(rng, 1, 32), seqs=_log_between(rng, 4, 24), hkv=hkv, d=d, lo=rng.randint(1, hi), hi=hi, page=page, fmt=fmt)
    return dict(op=op, seqs=_log_between(rng, 1, 16), beams=rng.randint(1, 8), vocab=_log_between(rng, 500, 128256), n_out=rng.choice([1, 2, 5, 8, 16]),
                dtype=dtype, finished=rng.random() < 0.5)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _code_dtype(fmt):
    return torch.int8 if fmt == "int8" else torch.float8_e4m3fn


def _scale_of(amax, fmt):
    """The scale of a block from its largest magnitude (fp32 in, fp32 out)."""
    if fmt == "int8":
        s = (amax.double() / 127.0).float()
    else:
        m, e = torch.frexp(amax)
        s = torch.ldexp(torch.ones_like(amax), (e - 9 + (m > 0.875)).clamp(min=-126))
    return torch.where(amax > 0, s.clamp(min=2.0 ** -126), torch.zeros_like(s))


def _round(x, s, fmt):
    """Codes of ``x`` (fp64) at scale ``s`` (fp32): the nearest value of the format, ties to even."""
    q = x / torch.where(s > 0, s, torch.ones_like(s)).double()
    if fmt == "int8":
        return q.round().clamp(-127, 127).to(torch.int8)
    return q.float().to(torch.float8_e4m3fn)


def _ints(gen, lo, hi, n):
    """``n`` lengths between lo and hi; where there is room for both, the ends are among them."""
    x = torch.randint(lo, hi + 1, (n,), generator=gen, device="cuda")
    x[0] = hi
    return x


def _pool(case, gen, n_pages):
    """A pool of ``n_pages`` pages full of rounded values, and one page more that no table names."""
    h, ps, d, fmt = case["hkv"], case["page"], case["d"], case["fmt"]
    st = {}
    for g in ("k", "v"):
        x = torch.randn((n_pages + 1, h, ps // BLOCK, BLOCK, d), generator=gen, device="cuda")
        x *= torch.exp(torch.randn((1, h, 1, 1, d), generator=gen, device="cuda") * 0.5)  # channels differ in size
        s = _scale_of(x.abs().amax((-1, -2)), fmt)
        codes = torch.empty(x.shape, dtype=_code_dtype(fmt), device="cuda")
        for i in range(0, n_pages + 1, 512):
            codes[i:i + 512] = _round(x[i:i + 512].double(), s[i:i + 512, ..., None, None], fmt)
        st[g + "_codes"], st[g + "_scale"] = codes.view(n_pages + 1, h, ps, d), s
    return st


def _tables(case, gen, lens, max_pages, n_pages):
    """Tables whose pages lie anywhere in the pool; -1 behind a sequence's last page."""
    ps = case["page"]
    used = (lens + ps - 1) // ps
    col = torch.arange(max_pages, device="cuda")
    live = col[None] < used[:, None]
    order = torch.randperm(n_pages, generator=gen, device="cuda")
    rank = live.reshape(-1).cumsum(0).reshape(live.shape) - 1
    pages = torch.where(live, order[rank.clamp(min=0)], torch.full_like(rank, -1)).int()
    ref = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda")
    ref.index_add_(0, pages[live].long(), torch.ones_like(pages[live]))
    return pages, ref


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op = case["op"]
    st = {"case": case}
    if op == "beam":
        rows, v = case["seqs"] * case["beams"], case["vocab"]
        st["logits"] = (torch.randn((rows, v), generator=gen, device="cuda") * 2.5).to(_dtype(case))
        st["score"] = -torch.rand((rows,), generator=gen, device="cuda") * 4.0 - 0.5
        st["finished"] = torch.rand((rows,), generator=gen, device="cuda") < 0.15 if case["finished"] else None
        st["eos"] = v // 3
        if own:
            from paper_2507_06517_b200.pipeline import SpindleKVBeamSelect
            st["handle"] = SpindleKVBeamSelect(case["seqs"], case["beams"], v, case["n_out"])
        return st
    ps, fmt, n_l = case["page"], case["fmt"], case["layers"]
    if op == "fork":
        seqs = case["groups"] * case["beams"]
        lens = _ints(gen, case["lo"], case["hi"], case["groups"])
        lens = lens.repeat_interleave(case["beams"]).repeat(n_l)                       # beams of a group are of one age
        max_pages = -(-case["hi"] // ps) + 1
        open_pages = n_l * seqs
        shared = n_l * case["groups"] * max_pages
        n_pages = shared + 3 * open_pages
        st.update(_pool(case, gen, n_pages))
        # beams of a group share its full pages and own the open one
        glens = lens.view(n_l, case["groups"], case["beams"])[:, :, 0].reshape(-1)
        gpages, _ = _tables(case, gen, (glens // ps) * ps, max_pages, n_pages)
        pages = gpages.view(n_l, case["groups"], 1, max_pages).expand(-1, -1, case["beams"], -1).reshape(n_l * seqs, max_pages).contiguous()
        taken = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
        taken[gpages[gpages >= 0].long()] = True
        free = (~taken[:n_pages]).nonzero().view(-1)
        free = free[torch.randperm(len(free), generator=gen, device="cuda")]
        part = lens % ps != 0
        at = torch.arange(n_l * seqs, device="cuda")[part]
        pages[at, (lens // ps)[part]] = free[: len(at)].int()
        ref = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda")
        ref.index_add_(0, pages[pages >= 0].long(), torch.ones_like(pages[pages >= 0]))
        st["parent"] = (torch.randint(0, case["beams"], (case["groups"], case["beams"]), generator=gen, device="cuda")
                        + torch.arange(case["groups"], device="cuda")[:, None] * case["beams"]).view(-1).int()
    else:
        seqs = case["seqs"]
        if op == "append":
            start = _ints(gen, case["lo"], case["hi"], n_l * seqs)
            new = _ints(gen, case["new_lo"], case["new_hi"], n_l * seqs)
            lens = start + new
            top = case["hi"] + case["new_hi"]
        else:
            lens = _ints(gen, case["lo"], case["hi"], n_l * seqs)
            top = case["hi"]
        max_pages = -(-top // ps) + 1
        n_pages = n_l * seqs * (-(-top // ps)) + 1                             # room for every sequence at its longest
        st.update(_pool(case, gen, n_pages))
        pages, ref = _tables(case, gen, lens, max_pages, n_pages)
    st["pages"], st["lens"], st["page_ref"] = pages.view(n_l, seqs, max_pages), lens.view(n_l, seqs).int().contiguous(), ref
    if op == "compact":
        st["pages_saved"], st["ref_saved"] = st["pages"].clone(), st["page_ref"].clone()
    if op == "attend":
        shape = (n_l, seqs, case["hq"], case["rows"], case["d"])
        st["q"] = torch.randn(shape, generator=gen, device="cuda").to(_dtype(case))
    if op == "append":
        st["start"] = start.view(n_l, seqs).int().contiguous()
        n = case["new_hi"] * case["of"]  # rows to pick from
        shape = (n_l, seqs, case["hkv"], n, case["d"])
        grow = torch.exp(torch.randn((n_l, seqs, 1, 1, 1), generator=gen, device="cuda") * 0.5)
        for g in ("K", "V"):
            st[g] = (torch.randn(shape, generator=gen, device="cuda") * grow).to(_dtype(case))
        st["idx"] = None
        if case["pick"]:  # ascending positions, as eviction leaves them: [layer][head][sequence * n + i]
            order = torch.rand((n_l, case["hkv"], seqs, n), generator=gen, device="cuda").argsort(-1)[..., : case["new_hi"]].sort(-1).values
            idx = torch.zeros((n_l, case["hkv"], seqs, n), dtype=torch.int32, device="cuda")
            idx[..., : case["new_hi"]] = order.int()
            st["idx"] = idx.view(n_l, case["hkv"], seqs * n)
    if own:
        from paper_2507_06517_b200.pipeline import SpindleKVPagedCache
        st["handle"] = SpindleKVPagedCache.over({g: st[g][:-1] for g in ("k_codes", "v_codes", "k_scale", "v_scale", "page_ref")},
                                                st["pages"], st["lens"], n_q_heads=case.get("hq"))
    return st


# ---- plain forms -------------------------------------------------------------------------------------------------

def _values(st, g, page):
    """Values of whole pages: ``page`` [...] -> [..., heads, page tokens, d], fp32."""
    codes, scale = st[g + "_codes"], st[g + "_scale"]
    x = codes.view(torch.uint8)[page].view(codes.dtype).float()
    return x * scale[page].repeat_interleave(BLOCK, -1)[..., None]


def _plain_attend(st):
    c, q = st["case"], st["q"].float()
    n_l, b, hq, r, d = q.shape
    h, ps = c["hkv"], c["page"]
    page = st["pages"].long().clamp(min=0)

    def rows(g):  # [L, B, H, tokens, d]
        return _values(st, g, page).permute(0, 1, 3, 2, 4, 5).reshape(n_l, b, h, -1, d)

    k = rows("k")
    s = (q.view(n_l, b, h, (hq // h) * r, d) @ k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    del k
    last = st["lens"][:, :, None] - (r - 1) + torch.arange(r, device="cuda")                 # tokens that row i sees
    seen = torch.arange(s.shape[-1], device="cuda") < last.repeat(1, 1, hq // h)[:, :, None, :, None]
    s = torch.where(seen, s, torch.full_like(s, NEG))
    m = s.amax(-1, keepdim=True)
    p = torch.where(seen, (s - torch.where(m > NEG, m, torch.zeros_like(m))).exp(), torch.zeros_like(s))
    den = p.sum(-1, keepdim=True)
    o = (p @ rows("v")) / torch.where(den > 0, den, torch.ones_like(den))
    return o.view(n_l, b, hq, r, d).to(st["q"].dtype)


def _plain_append(st):
    c = st["case"]
    fmt, ps, h, d = c["fmt"], c["page"], c["hkv"], c["d"]
    start, lens, pages = st["start"].long(), st["lens"].long(), st["pages"].long()
    n_l, b = start.shape
    n_blocks = (c["new_hi"] + BLOCK - 1) // BLOCK + 1
    blk = (start // BLOCK)[..., None] + torch.arange(n_blocks, device="cuda")                # [L, B, blocks]
    pos = blk[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")                        # [L, B, blocks, 16]
    is_new = (pos >= start[..., None, None]) & (pos < lens[..., None, None])
    is_old = pos < start[..., None, None]
    touched = is_new.any(-1)                                                                 # [L, B, blocks]
    spare = st["page_ref"].shape[0] - 1
    per = ps // BLOCK
    page = torch.gather(pages, 2, (blk // per).clamp(max=pages.shape[2] - 1))
    page = torch.where(touched, page, torch.full_like(page, spare))                          # blocks without a new token end up in the spare page
    inner = blk % per
    heads = torch.arange(h, device="cuda")
    where = (page[:, :, None], heads[None, None, :, None], inner[:, :, None])                # -> [L, B, H, blocks]
    row = (pos - start[..., None, None]).clamp(0, st["K"].shape[3] - 1)[:, :, None].expand(-1, -1, h, -1, -1)
    if st["idx"] is not None:
        idx = st["idx"].view(n_l, h, b, -1).permute(0, 2, 1, 3).long()
        row = torch.gather(idx, 3, row.reshape(n_l, b, h, -1)).view(row.shape)
    li, bi = torch.arange(n_l, device="cuda").view(-1, 1, 1, 1, 1), torch.arange(b, device="cuda").view(1, -1, 1, 1, 1)
    new, old = is_new[:, :, None, :, :, None], is_old[:, :, None, :, :, None]
    out = []
    for g in ("k", "v"):
        codes, scale = st[g + "_codes"], st[g + "_scale"]
        blocks = codes.view(torch.uint8).view(-1, h, per, BLOCK, d)
        x = st[g.upper()][li, bi, heads.view(1, 1, -1, 1, 1), row].float()                   # [L, B, H, blocks, 16, d]
        amax = torch.where(new, x.abs(), torch.zeros_like(x)).amax((-1, -2))
        had = scale[where]
        s = torch.maximum(_scale_of(amax, fmt), torch.where(is_old[:, :, None, :, 0], had, torch.zeros_like(had)))[..., None, None]
        was = blocks[where]
        rescaled = was.view(codes.dtype).double() * had[..., None, None].double()
        both = _round(torch.where(new, x.double(), rescaled), s, fmt).view(torch.uint8)
        blocks[where] = torch.where(new | old, both, was)
        scale[where] = s[..., 0, 0]
        out += [codes[:-1], scale[:-1]]
    return out


def _take_free(ref, count_before, wanted):
    """The page for each wanted slot: the lowest free page for the first slot, and so on."""
    free = ref[:-1] == 0
    nth = free.cumsum(0) - 1
    table = torch.full((ref.shape[0],), -1, dtype=torch.int64, device=ref.device)
    at = torch.where(free, nth, torch.full_like(nth, ref.shape[0] - 1))
    table.scatter_(0, at, torch.where(free, torch.arange(ref.shape[0] - 1, device=ref.device), torch.full_like(nth, -1)))
    return torch.where(wanted, table[count_before], torch.full_like(count_before, -1))


def _plain_fork(st):
    c, ps = st["case"], st["case"]["page"]
    pages, lens, ref, parent = st["pages"], st["lens"], st["page_ref"], st["parent"].long()
    n_l, n, max_pages = pages.shape
    children = torch.zeros(n, dtype=torch.int64, device="cuda").index_add_(0, parent, torch.ones_like(parent))
    same = parent[:, None] == parent[None, :]
    first = ~torch.tril(same, -1).any(1)
    col = torch.arange(max_pages, device="cuda")
    old_len = lens.long()
    live = col < ((old_len + ps - 1) // ps)[..., None]
    is_open = (col == (old_len // ps)[..., None]) & live
    new_len = old_len[:, parent]
    wants = (new_len % ps != 0) & ~first
    slot = (wants.view(-1).long().cumsum(0) - wants.view(-1).long()).view(n_l, n)
    fresh = _take_free(ref, slot, wants)                                                     # [L, N]
    # references: every entry counts once per child; an open page goes to its first child, the others get copies
    delta = torch.where(is_open, (children.clamp(max=1) - 1)[None, :, None], (children - 1)[None, :, None])
    spare = ref.shape[0] - 1
    ref.index_add_(0, torch.where(live, pages.long(), torch.full_like(delta, spare)).view(-1), torch.where(live, delta, torch.zeros_like(delta)).view(-1).int())
    ref.index_fill_(0, torch.where(wants, fresh, torch.full_like(fresh, spare)).view(-1), 1)
    ref[spare] = 0
    open_col = (new_len // ps).clamp(max=max_pages - 1)
    src = torch.where(wants, torch.gather(pages[:, parent], 2, open_col[..., None])[..., 0].long(), torch.full_like(fresh, spare))
    taken = pages[:, parent]
    use = live[:, parent]
    entry = torch.where((col == open_col[..., None]) & wants[..., None], fresh[..., None].int(), taken)
    pages.copy_(torch.where(use, entry, pages))
    lens.copy_(new_len)
    # the copied page's blocks that hold tokens
    dst = torch.where(wants, fresh, torch.full_like(fresh, spare)).view(-1)
    filled = ((new_len % ps + BLOCK - 1) // BLOCK).view(-1)
    keep = (torch.arange(ps // BLOCK, device="cuda") < filled[:, None])[:, None, :]
    out = [pages, lens, ref[:-1]]
    for g in ("k", "v"):
        codes, scale = st[g + "_codes"], st[g + "_scale"]
        blocks = codes.view(torch.uint8).view(-1, c["hkv"], ps // BLOCK, BLOCK, c["d"])
        blocks[dst] = torch.where(keep[..., None, None], blocks[src.view(-1)], blocks[dst])
        scale[dst] = torch.where(keep, scale[src.view(-1)], scale[dst])
        out += [codes[:-1].view(torch.int8), scale[:-1]]
    return out


def _plain_compact(st):
    c = st["case"]
    st["pages"].copy_(st["pages_saved"])
    st["page_ref"].copy_(st["ref_saved"])
    pages, ref = st["pages"], st["page_ref"]
    spare = ref.shape[0] - 1
    page = torch.arange(spare, device="cuda")
    live = ref[:-1] > 0
    n_live = live.sum()
    hole = ~live & (page < n_live)
    moves = live & (page >= n_live)
    nth_hole = hole.long().cumsum(0) - 1
    holes = torch.full((spare + 1,), spare, dtype=torch.int64, device="cuda")
    holes.scatter_(0, torch.where(hole, nth_hole, torch.full_like(page, spare)), torch.where(hole, page, torch.full_like(page, spare)))
    to = torch.where(moves, holes[(moves.long().cumsum(0) - 1).clamp(min=0)], page)
    lens = st["lens"].long()
    used = torch.arange(pages.shape[2], device="cuda") < ((lens + c["page"] - 1) // c["page"])[..., None]
    pages.copy_(torch.where(used, to[pages.long().clamp(min=0)].int(), pages))
    moving = moves.nonzero().view(-1)
    out = [pages, n_live.int().view(1)]
    for g in ("k", "v"):
        codes, scale = st[g + "_codes"], st[g + "_scale"]
        raw = codes.view(torch.uint8)
        raw[to[moving]] = raw[moving]
        scale[to[moving]] = scale[moving]
        out += [codes[:-1].view(torch.int8), scale[:-1]]
    ref[to[moving]] = ref[moving]
    ref[moving] = 0
    return out + [ref[:-1]]


def _plain_beam(st):
    c = st["case"]
    n, w, v, k = c["seqs"], c["beams"], c["vocab"], c["n_out"]
    x = st["logits"].double()
    m = x.amax(-1, keepdim=True)
    lse = (x - m).exp().sum(-1, keepdim=True).log() + m
    total = x - lse + st["score"].double()[:, None]
    if st["finished"] is not None:  # a finished beam goes on as itself alone
        alone = torch.full_like(total, NEG)
        alone[:, st["eos"]] = st["score"].double()
        total = torch.where(st["finished"][:, None], alone, total)
    total = total.view(n, w * v)
    best = total.topk(k, -1)
    edge = best.values[:, -1:]
    tied = torch.where(total == edge, torch.arange(w * v, device="cuda"), torch.full((1,), w * v, device="cuda")).topk(k, -1, largest=False).values
    at = torch.cat([torch.where(best.values > edge, best.indices, torch.full_like(best.indices, w * v)), tied], -1).sort(dim=-1).values
    val = torch.where(at < w * v, total.gather(1, at.clamp(max=w * v - 1)), torch.full_like(at, NEG, dtype=torch.float64))
    # by falling value, then by rising index: places that stand for nothing last
    order = torch.sort(torch.where(at < w * v, val, torch.full_like(val, -1e300)), dim=-1, descending=True, stable=True).indices[:, :k]
    at, val = at.gather(1, order), val.gather(1, order)
    parent = at // v + torch.arange(n, device="cuda")[:, None] * w
    return [val.float(), parent.int(), (at % v).int()]


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(st):
    op = st["case"]["op"]
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "fork": _plain_fork, "compact": _plain_compact, "beam": _plain_beam}[op](st)
    h = st["handle"]
    if op == "attend":
        return h.attend(st["q"], max_len=st["case"]["hi"])
    if op == "append":
        h.append(st["K"], st["V"], st["start"], idx=st["idx"], max_new=st["case"]["new_hi"])
        return [st["k_codes"][:-1], st["k_scale"][:-1], st["v_codes"][:-1], st["v_scale"][:-1]]
    if op == "fork":
        h.fork(st["parent"])
        return [st["pages"], st["lens"], st["page_ref"][:-1], st["k_codes"][:-1].view(torch.int8), st["k_scale"][:-1],
                st["v_codes"][:-1].view(torch.int8), st["v_scale"][:-1]]
    if op == "compact":
        st["pages"].copy_(st["pages_saved"])
        st["page_ref"].copy_(st["ref_saved"])
        n_live = h.compact()
        return [st["pages"], n_live, st["k_codes"][:-1].view(torch.int8), st["k_scale"][:-1], st["v_codes"][:-1].view(torch.int8),
                st["v_scale"][:-1], st["page_ref"][:-1]]
    return list(h.run(st["logits"], st["score"], finished=st["finished"], eos=st["eos"]))


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def _mean_len(lo, hi):
    return 0.5 * (lo + hi)


def work(case):
    op = case["op"]
    if op == "beam":
        rows = case["seqs"] * case["beams"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": rows * case["vocab"] * size * (0.85 if case["finished"] else 1.0), "flops": 3.0 * rows * case["vocab"]}
    h, d, ps = case["hkv"], case["d"], case["page"]
    token = 2 * h * (d + 4.0 / BLOCK)                      # bytes of a cached token, K and V
    if op == "attend":
        units = case["layers"] * case["seqs"]
        tokens = units * _mean_len(case["lo"], case["hi"])
        q = units * case["hq"] * case["rows"] * d * (2 if case["dtype"] == "bf16" else 4)
        return {"bytes": tokens * token + 2 * q, "flops": 4.0 * tokens * case["hq"] * case["rows"] * d}
    if op == "append":
        tokens = case["layers"] * case["seqs"] * _mean_len(case["new_lo"], case["new_hi"])
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": tokens * (2 * h * d * size + token + (4 * h if case["pick"] else 0)), "flops": 4.0 * tokens * h * d}
    if op == "fork":
        units = case["layers"] * case["groups"] * case["beams"]
        copies = units * (1 - 1 / case["beams"]) ** case["beams"]  # sequences whose parent an earlier one has taken
        return {"bytes": 2 * copies * token * ps / 2 + units * 8.0 * (case["lo"] + case["hi"]) / 2 / ps, "flops": 0}
    pages, room = (case["layers"] * case["seqs"] * x / ps for x in (_mean_len(case["lo"], case["hi"]) + ps / 2, case["hi"]))
    moved = pages * max(0.0, 1 - pages / room)            # live pages behind the first `pages` ones
    return {"bytes": 2 * moved * token * ps + 8.0 * pages + 4.0 * room, "flops": 0}


# ---- in 64 bits, from the definitions ----------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op in ("fork", "compact"):
        return None
    if op == "beam":
        n, w = case["seqs"], case["beams"]
        rows = []
        for i in range(n):
            cand = []
            for j in range(w):
                r = i * w + j
                if st["finished"] is not None and bool(st["finished"][r]):
                    cand.append(st["score"][r:r + 1].double())
                else:
                    x = st["logits"][r].double()
                    cand.append(st["score"][r].double() + x - torch.logsumexp(x, 0))
            rows.append(torch.cat(cand).sort(descending=True).values[: case["n_out"]])
        if any(len(r) < case["n_out"] for r in rows):
            return None
        return [torch.stack(rows), None, None]
    if op == "attend":
        q = st["q"].double()
        out = torch.zeros_like(q)
        n_l, b, hq, rows, d = q.shape
        g = hq // case["hkv"]
        for li in range(n_l):
            for s in range(b):
                n = int(st["lens"][li, s])
                pg = st["pages"][li, s, : -(-n // case["page"])].long()

                def tokens(which):
                    y = st[which + "_codes"].view(torch.uint8)[pg].view(_code_dtype(case["fmt"])).double()
                    y = y.unflatten(2, (-1, BLOCK)) * st[which + "_scale"][pg].double()[..., None, None]
                    return y.flatten(2, 3).transpose(0, 1).flatten(1, 2)[:, :n]              # [H, n, d]

                k, v = tokens("k"), tokens("v")
                for r in range(rows):
                    m = n - (rows - 1 - r)
                    if m > 0:
                        a = torch.softmax(torch.einsum("hgd,htd->hgt", q[li, s, :, r].view(-1, g, d), k[:, :m]) / math.sqrt(d), -1)
                        out[li, s, :, r] = torch.einsum("hgt,htd->hgd", a, v[:, :m]).reshape(hq, d)
        return out
    # append: only the scales are computed numbers that stand for themselves
    out = {g: st[g + "_scale"].double() for g in ("k", "v")}
    for li in range(case["layers"]):
        for s in range(case["seqs"]):
            a, e = int(st["start"][li, s]), int(st["lens"][li, s])
            table = st["pages"][li, s].tolist()
            for blk in range(a // BLOCK, (e - 1) // BLOCK + 1):
                lo, hi = max(a, blk * BLOCK), min(e, (blk + 1) * BLOCK)
                pg, inner = table[blk * BLOCK // case["page"]], blk % (case["page"] // BLOCK)
                for g in ("k", "v"):
                    src = st[g.upper()][li, s]
                    if st["idx"] is None:
                        rows = src[:, lo - a:hi - a].double()
                    else:
                        n = src.shape[1]
                        at = st["idx"][li, :, s * n + lo - a:s * n + hi - a].long()
                        rows = torch.gather(src, 1, at[..., None].expand(-1, -1, src.shape[2])).double()
                    top = rows.abs().amax((1, 2))
                    if case["fmt"] == "int8":
                        sc = top / 127
                    else:
                        sc = torch.exp2(torch.floor(torch.log2(top / 448)))                # within a step of the least power of two,
                        for _ in range(2):                                                  # whatever log2 rounds to
                            sc = torch.where(448 * sc < top, 2 * sc, sc)
                            sc = torch.where(448 * sc >= 2 * top, sc / 2, sc)
                    if lo > blk * BLOCK:
                        sc = torch.maximum(sc, out[g][pg, :, inner])
                    out[g][pg, :, inner] = sc
    return [None, out["k"][:-1], None, out["v"][:-1]]
