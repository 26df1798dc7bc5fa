"""The operators around the paged cache, case by case: inputs, plain forms, library calls, 64-bit values.

A case's ``op`` says which operator it is:

* ``prompt``: the causal attention of a prompt (or of the last rows of one) over its keys and values, grouped heads, packed or padded
  sequences of different lengths;
* ``rotate``: rows take their position's rotation on the way into the 8-bit pages, queries beside them;
* ``logits``: penalties for repeated tokens, biases and grammar masks ahead of beam selection.

``own`` picks the library's calls instead of the plain forms.
"""
import math

import torch

own = False

BLOCK = 16  # tokens of a page that share a scale
NEG = float("-inf")
ROPE_BASE = 10000.0


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # one short prompt at the smallest shape: what a single call costs
        dict(name="prompt one short", op="prompt", layers=1, seqs=1, hq=4, hkv=2, d=64, lo=190, hi=190, rows=0, packed=False, dtype="bf16"),
        # one prompt, one layer: the ordinary call
        dict(name="prompt 4k", op="prompt", layers=1, seqs=1, hq=32, hkv=8, d=128, lo=4096, hi=4096, rows=0, packed=False, dtype="bf16"),
        # a long prompt
        dict(name="prompt 16k", op="prompt", layers=1, seqs=1, hq=32, hkv=8, d=128, lo=16384, hi=16384, rows=0, packed=False, dtype="bf16"),
        # a batch of prompts of uneven length behind one another
        dict(name="prompt packed", op="prompt", layers=1, seqs=9, hq=32, hkv=8, d=128, lo=300, hi=4095, rows=0, packed=True, dtype="bf16"),
        # the last few rows of long prompts: keys have to be split over the device
        dict(name="prompt last rows", op="prompt", layers=1, seqs=2, hq=32, hkv=8, d=128, lo=12000, hi=16001, rows=33, packed=False, dtype="bf16"),
        # single precision, padded batch
        dict(name="prompt fp32", op="prompt", layers=1, seqs=2, hq=32, hkv=8, d=128, lo=1500, hi=4001, rows=0, packed=False, dtype="f32"),
        # decoding: every sequence of a large batch rotates its new key and queries and writes the token
        dict(name="rotate one token", op="rotate", layers=1, seqs=96, hq=32, hkv=8, d=128, lo=200, hi=5000, new_lo=1, new_hi=1, page=64, fmt="int8",
             dtype="bf16", pick=False, of=1),
        # prompts of uneven length: keys and queries for the prompt's attention, codes for the cache
        dict(name="rotate prompts", op="rotate", layers=1, seqs=4, hq=32, hkv=8, d=128, lo=0, hi=100, new_lo=3500, new_hi=8192, page=64, fmt="int8",
             dtype="bf16", pick=False, of=1),
        # what eviction kept of a prompt, rotated at the positions that the rows had
        dict(name="rotate kept rows", op="rotate", layers=16, seqs=1, hq=0, hkv=8, d=128, lo=0, hi=0, new_lo=1000, new_hi=1024, page=64, fmt="e4m3",
             dtype="f32", pick=True, of=8),
        # one search of a few beams
        dict(name="logits few rows", op="logits", rows=4, vocab=32000, hist=300, bias=4, mask=True, pad=0, dtype="bf16"),
        # a batch with an odd vocabulary and no alignment of its rows
        dict(name="logits odd rows", op="logits", rows=37, vocab=50257, hist=2500, bias=0, mask=True, pad=0, dtype="bf16"),
        # a large batch with long histories
        dict(name="logits large", op="logits", rows=128, vocab=128256, hist=16384, bias=64, mask=True, pad=64, dtype="f32"),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "prompt", "rotate", "rotate", "logits"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "prompt":
        seqs, layers = _log_between(rng, 1, 16), rng.choice([1, 1, 1, 2])
        hq = hkv * rng.choice([1, 2, 3, 4, 7, 8])
        rows = rng.choice([0, 0, 0, 1, 2, 5, 17, 64, 300])
        # pairs of the padded batch, of all heads: what the plain form holds
        most = (2 ** 32.5 if dtype == "bf16" else 2 ** 30) / (seqs * layers * max(hq, 4))
        hi = _log_between(rng, max(rows, 1), max(rows, min(16384, int(math.sqrt(most) if not rows else most / max(rows, 64)))))
        return dict(op=op, layers=layers, seqs=seqs, hq=hq, hkv=hkv, d=d, lo=rng.randint(max(rows, 1), hi), hi=hi, rows=rows,
                    packed=rng.random() < 0.5, dtype=dtype)
    if op == "rotate":
        seqs, layers = _log_between(rng, 1, 48), rng.choice([1, 2, 4])
        new = _log_between(rng, 1, min(8192, 30000 // (seqs * layers)))
        pick = rng.random() < 0.35
        return dict(op=op, layers=layers, seqs=seqs, hq=0 if pick else hkv * rng.choice([0, 1, 3, 4, 8]), hkv=hkv, d=d, lo=0, hi=_log_between(rng, 1, 600),
                    new_lo=rng.randint(1, new), new_hi=new, page=rng.choice([16, 32, 64, 128]), fmt=rng.choice(["int8", "e4m3"]), dtype=dtype, pick=pick,
                    of=rng.randint(1, max(1, min(8, 120000 // (seqs * layers * new)))) if pick else 1)
    return dict(op=op, rows=_log_between(rng, 1, 128), vocab=_log_between(rng, 500, 128256), hist=rng.choice([0, _log_between(rng, 1, 16384)]),
                bias=rng.choice([0, 1, 7, 64]), mask=rng.random() < 0.6, pad=rng.choice([0, 1, 8, 64]), dtype=dtype)


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
    """``n`` lengths between lo and hi, hi among them."""
    x = torch.randint(lo, hi + 1, (n,), generator=gen, device="cuda")
    x[0] = hi
    return x


def _angles(positions, d):
    """Angles of ``positions`` for every pair of elements, fp64."""
    freq = ROPE_BASE ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    return positions.double()[..., None] * freq


def _prepare_prompt(case, gen, st):
    n_l, b, hq, hkv, d = (case[k] for k in ("layers", "seqs", "hq", "hkv", "d"))
    # spread evenly between lo and hi, in an order of the seed's
    lens = torch.linspace(case["hi"], case["lo"], b, device="cuda", dtype=torch.float64).round().long()[torch.randperm(b, generator=gen, device="cuda")]
    n_rows = lens.clone() if case["rows"] == 0 else torch.full_like(lens, case["rows"])
    st["lens"], st["n_rows"] = lens.int(), n_rows.int()
    host_lens, host_rows = lens.tolist(), n_rows.tolist()
    channels = torch.exp(torch.randn((hkv, 1, d), generator=gen, device="cuda") * 0.3)

    def rows_of(h, each, most):  # [L, B, H, most, d], or [L, T, H, d]
        shape = (n_l, sum(each), h, d) if case["packed"] else (n_l, b, h, most, d)
        return torch.randn(shape, generator=gen, device="cuda")

    q = rows_of(hq, host_rows, max(host_rows))
    k, v = rows_of(hkv, host_lens, case["hi"]), rows_of(hkv, host_lens, case["hi"])
    cu = [torch.cat([torch.zeros_like(x[:1]), x.cumsum(0).int()]).int() for x in (st["lens"], st["n_rows"])]
    if case["packed"]:
        st["cu"], st["cu_rows"] = cu
        k *= channels.transpose(0, 1)
        first = cu[0][:-1].long()
        k[:, first] *= 3.0                                       # a sequence's first key draws more than its share
    else:
        k *= channels
        k[:, :, :, 0] *= 3.0
    st["q"], st["k"], st["v"] = (x.to(_dtype(case)) for x in (q, k, v))
    st["out"] = torch.zeros_like(st["q"])
    total = sum(host_rows) if case["packed"] else b * max(host_rows)
    st["lse"] = torch.zeros((n_l, hq, total), dtype=torch.float32, device="cuda")
    st["max_rows"] = max(host_rows)
    if own:
        from paper_2507_06517_b200 import binding as B
        from paper_2507_06517_b200.pipeline import SpindleKVPromptAttention
        if case["packed"]:
            keys, rows = (B.Batch(n_l, b, max(x), sum(x), c) for x, c in ((host_lens, st["cu"]), (host_rows, st["cu_rows"])))
        else:
            keys, rows = (B.Batch(n_l, b, max(h), b * max(h), None, None if min(h) == max(h) else x[None].expand(n_l, b).contiguous())
                          for h, x in ((host_lens, st["lens"]), (host_rows, st["n_rows"])))
        st["handle"] = SpindleKVPromptAttention(keys, hq, hkv, d, _dtype(case), rows=rows)


def _prepare_rotate(case, gen, st):
    n_l, b, h, d, ps, fmt = (case[k] for k in ("layers", "seqs", "hkv", "d", "page", "fmt"))
    start = _ints(gen, case["lo"], case["hi"], n_l * b)
    lens = start + _ints(gen, case["new_lo"], case["new_hi"], n_l * b)
    top = case["hi"] + case["new_hi"]
    max_pages = -(-top // ps) + 1
    n_pages = n_l * b * (-(-top // ps)) + 1
    for g in ("k", "v"):                                         # a pool full of rounded values, and one page more that no table names
        x = torch.randn((n_pages + 1, h, ps // BLOCK, BLOCK, d), generator=gen, device="cuda")
        s = _scale_of(x.abs().amax((-1, -2)), fmt)
        codes = torch.empty(x.shape, dtype=_code_dtype(fmt), device="cuda")
        for i in range(0, n_pages + 1, 512):
            codes[i:i + 512] = _round(x[i:i + 512].double(), s[i:i + 512, ..., None, None], fmt)
        st[g + "_codes"], st[g + "_scale"] = codes.view(n_pages + 1, h, ps, d), s
    used = (lens + ps - 1) // ps
    live = torch.arange(max_pages, device="cuda") < used[:, None]
    order = torch.randperm(n_pages, generator=gen, device="cuda")
    rank = live.reshape(-1).cumsum(0).reshape(live.shape) - 1
    pages = torch.where(live, order[rank.clamp(min=0)], torch.full_like(rank, -1)).int()
    ref = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda")
    ref.index_add_(0, pages[live].long(), torch.ones_like(pages[live]))
    st["pages"], st["page_ref"] = pages.view(n_l, b, max_pages), ref
    st["lens"], st["start"] = lens.view(n_l, b).int().contiguous(), start.view(n_l, b).int().contiguous()
    n = case["new_hi"] * case["of"]
    grow = torch.exp(torch.randn((n_l, b, 1, 1, 1), generator=gen, device="cuda") * 0.5)
    for g in ("K", "V"):
        st[g] = (torch.randn((n_l, b, h, n, d), generator=gen, device="cuda") * grow).to(_dtype(case))
    st["Q"] = torch.randn((n_l, b, case["hq"], n, d), generator=gen, device="cuda").to(_dtype(case)) if case["hq"] else None
    st["K_out"] = None if case["pick"] else torch.zeros_like(st["K"])
    st["Q_out"] = torch.zeros_like(st["Q"]) if case["hq"] else None
    st["idx"] = None
    if case["pick"]:                                             # ascending positions, as eviction leaves them: [layer][head][sequence * n + i]
        order = torch.rand((n_l, h, b, n), generator=gen, device="cuda").argsort(-1)[..., : case["new_hi"]].sort(-1).values
        idx = torch.zeros((n_l, h, b, n), dtype=torch.int32, device="cuda")
        idx[..., : case["new_hi"]] = order.int()
        st["idx"] = idx.view(n_l, h, b * n)
    # where row 0 stands: the token's own place, or what a sequence had before eviction shortened it
    ahead = torch.randint(0, 2000, (n_l, b), generator=gen, device="cuda")
    st["first_pos"] = (ahead if case["pick"] else st["start"] + ahead).int().contiguous()
    angle = _angles(torch.arange(case["hi"] + 2000 + n, device="cuda"), d)
    st["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()                         # [positions, d / 2, 2]
    if own:
        from paper_2507_06517_b200.pipeline import SpindleKVPagedCache
        st["handle"] = SpindleKVPagedCache.over({g: st[g][:-1] for g in ("k_codes", "v_codes", "k_scale", "v_scale", "page_ref")}, st["pages"], st["lens"],
                                                n_q_heads=case["hq"] or None)


def _prepare_logits(case, gen, st):
    n, v = case["rows"], case["vocab"]
    wide = torch.randn((n, v + case["pad"]), generator=gen, device="cuda") * 2.5
    st["logits"] = wide.to(_dtype(case))[:, :v]
    st["out"] = torch.zeros_like(wide, dtype=_dtype(case))[:, :v]
    most = max(case["hist"], 1)
    # words follow a steep distribution: few of them make up most of a text
    st["history"] = (torch.rand((n, most), generator=gen, device="cuda") ** 4 * v).int().clamp(max=v - 1)
    st["history_lens"] = torch.randint(case["hist"] // 3, case["hist"] + 1, (n,), generator=gen, device="cuda").int()
    st["history_lens"][0] = case["hist"]
    st["n_prompt"] = (st["history_lens"].float() * torch.rand((n,), generator=gen, device="cuda")).int()
    st["repetition"] = 1.0 + torch.rand((n,), generator=gen, device="cuda") * 0.5
    st["presence"] = torch.rand((n,), generator=gen, device="cuda")
    st["frequency"] = torch.rand((n,), generator=gen, device="cuda") * 0.25
    st["bias_token"] = st["bias_value"] = st["allowed"] = None
    if case["bias"]:
        st["bias_token"] = torch.rand((n, v), generator=gen, device="cuda").topk(case["bias"], -1).indices.int()
        st["bias_value"] = torch.randn((n, case["bias"]), generator=gen, device="cuda") * 5.0
    if case["mask"]:                                             # a grammar allows a tenth of the tokens, or all but a few
        share = torch.where(torch.rand((n, 1), generator=gen, device="cuda") < 0.5, 0.1, 0.98)
        words = -(-v // 32)
        bits = torch.rand((n, words, 32), generator=gen, device="cuda") < share[..., None]
        word = (bits.long() << torch.arange(32, device="cuda")).sum(-1)
        st["allowed"] = torch.where(word >= 2 ** 31, word - 2 ** 32, word).int()             # bit t % 32 of word t / 32
    if own:
        from paper_2507_06517_b200.pipeline import SpindleKVLogits
        st["handle"] = SpindleKVLogits(n, v)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    st = {"case": case}
    {"prompt": _prepare_prompt, "rotate": _prepare_rotate, "logits": _prepare_logits}[case["op"]](case, gen, st)
    return st


# ---- plain forms -------------------------------------------------------------------------------------------------

def _places(cu, n):
    """Rows of a packed tensor that the padded places [sequence, i] stand for."""
    return (cu[:-1].long()[:, None] + torch.arange(n, device="cuda")).clamp(max=int(2 ** 31 - 1))


def _plain_prompt(st):
    c = st["case"]
    n_l, b, hq, h, d = (c[k] for k in ("layers", "seqs", "hq", "hkv", "d"))
    g, n, r = hq // h, c["hi"], st["max_rows"]
    q, k, v = st["q"], st["k"], st["v"]
    if c["packed"]:
        at, at_rows = _places(st["cu"], n).clamp(max=k.shape[1] - 1), _places(st["cu_rows"], r).clamp(max=q.shape[1] - 1)
        q, k, v = (x[:, i].transpose(2, 3) for x, i in ((q, at_rows), (k, at), (v, at)))     # [L, B, H, rows, d]
    q, k, v = q.float(), k.float(), v.float()
    s = q.reshape(n_l, b, h, g * r, d) @ k.transpose(-1, -2)
    s = s.view(n_l, b, h, g, r, n).mul_(1.0 / math.sqrt(d))
    i, j = torch.arange(r, device="cuda")[:, None], torch.arange(n, device="cuda")
    lens, n_rows = st["lens"].long()[:, None, None], st["n_rows"].long()[:, None, None]
    hidden = (j > lens - n_rows + i) | (j >= lens)                                           # [B, r, n]
    s.masked_fill_(hidden[None, :, None, None], NEG)
    m = s.amax(-1, keepdim=True)
    s.sub_(torch.where(m > NEG, m, torch.zeros_like(m))).exp_()
    den = s.sum(-1, keepdim=True)
    o = (s.view(n_l, b, h, g * r, n) @ v).view(n_l, b, h, g, r, d) / torch.where(den > 0, den, torch.ones_like(den))
    o, lse = o.view(n_l, b, hq, r, d).to(st["q"].dtype), (den.log() + m).view(n_l, b, hq, r)
    if c["packed"]:
        t = torch.arange(st["q"].shape[1], device="cuda")
        seq = torch.searchsorted(st["cu_rows"][1:].long(), t, right=True)
        place = seq * r + t - st["cu_rows"].long()[seq]
        return [o.permute(0, 1, 3, 2, 4).reshape(n_l, b * r, hq, d)[:, place], lse.transpose(1, 2).reshape(n_l, hq, b * r)[:, :, place]]
    there = torch.arange(r, device="cuda") < st["n_rows"][:, None]                           # [B, r]
    o = torch.where(there[None, :, None, :, None], o, st["out"])
    lse = torch.where(there[None, :, None], lse, torch.zeros_like(lse))
    return [o, lse.transpose(1, 2).reshape(n_l, hq, b * r)]


def _rotated(x, pos, table):
    """Rows ``x`` [..., d] at positions ``pos`` [...]: fp32, each operation rounded by itself, then the rows' type."""
    a, b = x.float().chunk(2, -1)
    c, s = table[pos].unbind(-1)
    return torch.cat([a * c - b * s, b * c + a * s], -1).to(x.dtype)


def _plain_rotate(st):
    c = st["case"]
    fmt, ps, h, d = c["fmt"], c["page"], c["hkv"], c["d"]
    start, lens, pages = st["start"].long(), st["lens"].long(), st["pages"].long()
    n_l, b = start.shape
    n = st["K"].shape[3]
    at = st["first_pos"].long()[:, :, None, None] + torch.arange(n, device="cuda")           # [L, B, 1, n]
    k = _rotated(st["K"], at, st["rope"])
    n_blocks = (c["new_hi"] + BLOCK - 1) // BLOCK + 1
    blk = (start // BLOCK)[..., None] + torch.arange(n_blocks, device="cuda")                # [L, B, blocks]
    pos = blk[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")                        # [L, B, blocks, 16]
    is_new = (pos >= start[..., None, None]) & (pos < lens[..., None, None])
    is_old = pos < start[..., None, None]
    touched = is_new.any(-1)
    spare = st["page_ref"].shape[0] - 1
    per = ps // BLOCK
    page = torch.gather(pages, 2, (blk // per).clamp(max=pages.shape[2] - 1))
    page = torch.where(touched, page, torch.full_like(page, spare))
    heads = torch.arange(h, device="cuda")
    where = (page[:, :, None], heads[None, None, :, None], (blk % per)[:, :, None])          # -> [L, B, H, blocks]
    row = (pos - start[..., None, None]).clamp(0, n - 1)[:, :, None].expand(-1, -1, h, -1, -1)
    if st["idx"] is not None:
        idx = st["idx"].view(n_l, h, b, -1).permute(0, 2, 1, 3).long()
        row = torch.gather(idx, 3, row.reshape(n_l, b, h, -1)).view(row.shape)
    li, bi = torch.arange(n_l, device="cuda").view(-1, 1, 1, 1, 1), torch.arange(b, device="cuda").view(1, -1, 1, 1, 1)
    new, old = is_new[:, :, None, :, :, None], is_old[:, :, None, :, :, None]
    out = []
    for g, rows in (("k", k), ("v", st["V"])):
        codes, scale = st[g + "_codes"], st[g + "_scale"]
        blocks = codes.view(torch.uint8).view(-1, h, per, BLOCK, d)
        x = rows[li, bi, heads.view(1, 1, -1, 1, 1), row].float()                            # [L, B, H, blocks, 16, d]
        amax = torch.where(new, x.abs(), torch.zeros_like(x)).amax((-1, -2))
        had = scale[where]
        s = torch.maximum(_scale_of(amax, fmt), torch.where(is_old[:, :, None, :, 0], had, torch.zeros_like(had)))[..., None, None]
        was = blocks[where]
        rescaled = was.view(codes.dtype).double() * had[..., None, None].double()
        both = _round(torch.where(new, x.double(), rescaled), s, fmt).view(torch.uint8)
        blocks[where] = torch.where(new | old, both, was)
        scale[where] = s[..., 0, 0]
        out += [codes[:-1], scale[:-1]]
    there = (torch.arange(n, device="cuda") < (lens - start)[..., None])[:, :, None, :, None]
    if st["K_out"] is not None:
        out.append(torch.where(there, k, st["K_out"]))
    if st["Q"] is not None:
        out.append(torch.where(there, _rotated(st["Q"], at, st["rope"]), st["Q_out"]))
    return out


def _plain_logits(st):
    x = st["logits"].float()
    n, v = x.shape
    at = torch.arange(st["history"].shape[1], device="cuda")
    said = at < st["history_lens"][:, None]
    zeros = torch.zeros((n, v), dtype=torch.int32, device="cuda")
    token = st["history"].long()
    seen = zeros.scatter_add(1, token, said.int()) > 0
    count = zeros.scatter_add(1, token, (said & (at >= st["n_prompt"][:, None])).int())
    rep = st["repetition"][:, None]
    z = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    z = torch.where(count > 0, z - (st["frequency"][:, None] * count.float() + st["presence"][:, None]), z)
    if st["bias_token"] is not None:
        z = z.scatter_add(1, st["bias_token"].long(), st["bias_value"])
    if st["allowed"] is not None:
        t = torch.arange(v, device="cuda")
        z = torch.where(st["allowed"][:, t // 32] >> (t % 32) & 1 > 0, z, torch.full_like(z, NEG))
    return z.to(st["logits"].dtype)


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(st):
    op = st["case"]["op"]
    if not own:
        return {"prompt": _plain_prompt, "rotate": _plain_rotate, "logits": _plain_logits}[op](st)
    h = st["handle"]
    if op == "prompt":
        return [h.run(st["q"], st["k"], st["v"], out=st["out"], lse=st["lse"]), st["lse"]]
    if op == "rotate":
        h.append_rotated(st["K"], st["V"], st["rope"], start=st["start"], first_pos=st["first_pos"], idx=st["idx"], max_new=st["case"]["new_hi"], K_out=st["K_out"],
                         Q=st["Q"], Q_out=st["Q_out"])
        return [st["k_codes"][:-1], st["k_scale"][:-1], st["v_codes"][:-1], st["v_scale"][:-1]] + [st[x] for x in ("K_out", "Q_out") if st[x] is not None]
    return h.adjust(st["logits"], out=st["out"], history=st["history"], history_lens=st["history_lens"], n_prompt=st["n_prompt"], repetition=st["repetition"],
                    presence=st["presence"], frequency=st["frequency"], bias_token=st["bias_token"], bias_value=st["bias_value"], allowed=st["allowed"])


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def _mean_len(lo, hi):
    return 0.5 * (lo + hi)


def work(case):
    op = case["op"]
    size = 2 if case["dtype"] == "bf16" else 4
    if op == "logits":
        n, v = case["rows"], case["vocab"]
        return {"bytes": n * (2.0 * v * size + (v / 8 if case["mask"] else 0) + 4 * case["hist"] * 2 / 3 + 8 * case["bias"]), "flops": 4.0 * n * v}
    h, hq, d = case["hkv"], case["hq"], case["d"]
    if op == "prompt":
        units = case["layers"] * case["seqs"]
        keys = case["hi"] if case["seqs"] == 1 else _mean_len(case["lo"], case["hi"])
        if case["rows"]:
            rows, pairs = case["rows"], case["rows"] * (keys - (case["rows"] - 1) / 2)
        else:                                                    # mean of n (n + 1) / 2
            spread = 0 if case["seqs"] == 1 else (case["hi"] - case["lo"]) ** 2 / 12
            rows, pairs = keys, (keys * keys + spread + keys) / 2
        return {"bytes": units * (2.0 * rows * hq * d * size + 2.0 * keys * h * d * size + 4 * rows * hq), "flops": 4.0 * units * pairs * hq * d}
    tokens = case["layers"] * case["seqs"] * _mean_len(case["new_lo"], case["new_hi"])
    token = 2 * h * (d + 4.0 / BLOCK) + 2 * h * d * size + (4 * h if case["pick"] else h * d * size) + 2 * hq * d * size
    return {"bytes": tokens * token, "flops": 3.0 * tokens * (h + hq) * d + 4.0 * tokens * h * d}


# ---- in 64 bits, from the definitions ----------------------------------------------------------------------------

def _exact_prompt(case, st):
    n_l, b, hq, h = (case[k] for k in ("layers", "seqs", "hq", "hkv"))
    out, lse = st["out"].double(), st["lse"].double()
    lens, n_rows = st["lens"].tolist(), st["n_rows"].tolist()
    for li in range(n_l):
        for s in range(b):
            n, r = lens[s], n_rows[s]
            for head in range(hq):
                if case["packed"]:
                    k0, r0 = sum(lens[:s]), sum(n_rows[:s])
                    q, k, v = st["q"][li, r0:r0 + r, head], st["k"][li, k0:k0 + n, head // (hq // h)], st["v"][li, k0:k0 + n, head // (hq // h)]
                    o, at = out[li, r0:r0 + r, head], r0
                else:
                    q, k, v = st["q"][li, s, head, :r], st["k"][li, s, head // (hq // h), :n], st["v"][li, s, head // (hq // h), :n]
                    o, at = out[li, s, head, :r], s * st["max_rows"]
                a = q.double() @ k.double().T / math.sqrt(case["d"])
                a = a + torch.full((r, n), NEG, dtype=torch.float64, device="cuda").triu(n - r + 1)
                lse[li, head, at:at + r] = torch.logsumexp(a, -1)
                o.copy_(torch.softmax(a, -1) @ v.double())
    return [out, lse]


def _turned(x, pos):
    """Rows as complex numbers, each times e^(i angle)."""
    a, b = x.double().chunk(2, -1)
    z = torch.complex(a, b) * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), _angles(pos, x.shape[-1]))
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "prompt":
        return _exact_prompt(case, st)
    if case["op"] == "logits":
        z = st["logits"].double()
        for i in range(case["rows"]):
            said = st["history"][i, : int(st["history_lens"][i])].long()
            n = torch.bincount(said[int(st["n_prompt"][i]):], minlength=case["vocab"])
            seen = torch.bincount(said, minlength=case["vocab"]) > 0
            rep = st["repetition"][i].double()
            z[i] = torch.where(seen, torch.where(z[i] > 0, z[i] / rep, z[i] * rep), z[i])
            z[i] -= st["frequency"][i].double() * n + st["presence"][i].double() * (n > 0)
            if case["bias"]:
                z[i, st["bias_token"][i].long()] += st["bias_value"][i].double()
            if case["mask"]:
                bit = (st["allowed"][i].long()[:, None] >> torch.arange(32, device="cuda")) & 1
                z[i, bit.reshape(-1)[: case["vocab"]] == 0] = NEG
        return z
    if case["pick"]:
        return None
    # codes and scales stand for rounded values; the rotated rows are computed numbers
    out = [None, None, None, None]
    n = st["K"].shape[3]
    at = st["first_pos"].long()[:, :, None, None] + torch.arange(n, device="cuda")
    there = (torch.arange(n, device="cuda") < (st["lens"] - st["start"])[..., None])[:, :, None, :, None]
    for x in ("K", "Q"):
        if st[x + "_out"] is not None:
            out.append(torch.where(there, _turned(st[x], at), torch.zeros((), dtype=torch.float64, device="cuda")))
    return out
