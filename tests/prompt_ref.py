"""Plain float64 form of the prompt's attention, one (layer, sequence, head) at a time, and the errors that its roundings allow."""
import math

import torch

NEG = float("-inf")


def spans(batch):
    """``[(layer, seq, first row, rows)]`` of a batch, rows numbered along a packed tensor or within a sequence."""
    out = []
    cu = None if batch.cu_seqlens is None else batch.cu_seqlens.tolist()
    ll = None if batch.layer_lens is None else batch.layer_lens.tolist()
    for layer in range(batch.n_layers):
        for s in range(batch.n_seqs):
            if cu is not None:
                out.append((layer, s, cu[s], cu[s + 1] - cu[s]))
            else:
                out.append((layer, s, 0, batch.max_len if ll is None else ll[layer][s]))
    return out


def of_head(t, batch, layer, s, first, n, head):
    return t[layer, first:first + n, head] if batch.cu_seqlens is not None else t[layer, s, head, :n]


def attend(q, k, v, keys, rows, scale=0.0):
    """float64 ``(out, lse, bound)`` laid out like q and [L, Hq, T]; NaN where there is no row.  ``bound``: how far an output may be off."""
    packed = rows.cu_seqlens is not None
    hq, h, d = q.shape[2], k.shape[2], q.shape[-1]
    scale = scale or 1.0 / math.sqrt(d)
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    lse = torch.full((rows.n_layers, hq, rows.total_len), math.nan, dtype=torch.float64, device=q.device)
    half = torch.finfo(q.dtype).eps / 2
    bf = q.dtype == torch.bfloat16
    for (layer, s, r0, r), (_, _, k0, n) in zip(spans(rows), spans(keys)):
        for head in range(hq):
            if r == 0:
                continue
            qq = of_head(q, rows, layer, s, r0, r, head).double()
            kk = of_head(k, keys, layer, s, k0, n, head // (hq // h)).double()
            vv = of_head(v, keys, layer, s, k0, n, head // (hq // h)).double()
            col = r0 if packed else s * rows.max_len
            o = torch.zeros((r, d), dtype=torch.float64, device=q.device)
            e, lg = torch.zeros_like(o), torch.full((r,), NEG, dtype=torch.float64, device=q.device)
            if n:
                hidden = torch.ones((r, n), dtype=torch.bool, device=q.device).triu(n - r + 1)
                x = (qq @ kk.T * scale).masked_fill(hidden, NEG)
                m = x.amax(-1, keepdim=True)
                m = torch.where(m > NEG, m, torch.zeros_like(m))
                p = (x - m).exp()
                l = p.sum(-1, keepdim=True)
                w = p / torch.where(l > 0, l, torch.ones_like(l))
                o = w @ vv
                lg = torch.logsumexp(x, -1)
                # A score: products of d factors added up d / 16 at a time (fp32: six such sums, and 2^-22 for what is left out), each step losing
                # 2^-23 of what it adds to at most, then 2^-23 of itself in the exponent; a power is right to 2^-22, a sum of n to (n / 128 + 8) 2^-24.
                big = (qq.abs() @ kk.abs().T * scale).masked_fill(hidden, 0.0).amax(-1, keepdim=True)
                delta = big * (d / 16 * (1 if bf else 6) + 4) * 2.0 ** -23 + (n / 128 + 24) * 2.0 ** -23
                # the weights' rounding (bf16: half a step each), the sums of n products, 128 at a time, and the result's rounding
                weigh = (half if bf else 2.0 ** -22) + 2 * delta + (n / 16) * (1 if bf else 6) * 2.0 ** -23
                e = weigh * (w @ vv.abs()) + half * o.abs() + 1e-38
            if packed:
                out[layer, r0:r0 + r, head], bound[layer, r0:r0 + r, head] = o, e
            else:
                out[layer, s, head, :r], bound[layer, s, head, :r] = o, e
            lse[layer, head, col:col + r] = lg
    return out, lse, bound
