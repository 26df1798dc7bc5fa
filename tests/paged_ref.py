"""Plain float64 / python-integer forms of the 8-bit paged cache and of beam selection, for the tests: one step at a time, no torch."""
import numpy as np

BLOCK = 16

# every E4M3 magnitude by code 0 .. 126 (127 is a NaN): exponent bias 7, three fraction bits
_E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def decode(codes, fmt):
    """Bytes -> float64."""
    if fmt == "int8":
        return codes.view(np.int8).astype(np.float64)
    u = codes.view(np.uint8)
    mag = np.concatenate([_E4M3, [np.nan]])[u & 127]
    return np.where(u & 128, -mag, mag)


def encode(q, fmt):
    """float64 quotients -> bytes: nearest, ties to even."""
    if fmt == "int8":
        return np.clip(np.rint(q), -127, 127).astype(np.int8).view(np.uint8)
    mag = np.minimum(np.abs(q), 448.0)
    lo = np.clip(np.searchsorted(_E4M3, mag, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    mid = (_E4M3[lo] + _E4M3[hi]) / 2
    up = (mag > mid) | ((mag == mid) & (lo % 2 == 1))
    return (np.where(up, hi, lo) | np.where(np.signbit(q), 128, 0)).astype(np.uint8)


def scale_of(amax, fmt):
    """float64 amax (the largest of fp32 numbers) -> the block's scale, as the fp32 number it is."""
    if not np.isfinite(amax):
        return np.float32(np.nan)
    if amax == 0:
        return np.float32(0)
    if fmt == "int8":
        return max(np.float32(amax / 127.0), np.float32(2.0 ** -126))
    k = -126
    while 448.0 * 2.0 ** k < amax:
        k += 1
    return np.float32(2.0 ** k)


class RefCache:
    """Pool and table on the host, with the operators one step at a time."""

    def __init__(self, k_codes, v_codes, k_scale, v_scale, page_ref, pages, lens, fmt):
        self.codes = {"k": k_codes.view(np.uint8).copy(), "v": v_codes.view(np.uint8).copy()}
        self.scale = {"k": k_scale.copy(), "v": v_scale.copy()}
        self.ref, self.pages, self.lens, self.fmt = page_ref.copy(), pages.copy(), lens.copy(), fmt
        self.n_pages, self.heads, self.ps, self.d = k_codes.shape
        self.n_layers, self.n_seqs, self.max_pages = pages.shape

    def units(self):
        return [(l, s) for l in range(self.n_layers) for s in range(self.n_seqs)]

    def free(self):
        return [i for i in range(self.n_pages) if self.ref[i] == 0]

    def count(self, n):
        return -(-int(n) // self.ps)

    # -- append ----------------------------------------------------------------------------------
    def append(self, start, K, V, idx=None, idx_seq=0):
        for l, s in self.units():
            a, e = int(start[l, s]), int(self.lens[l, s])
            if a < 0 or a >= e:
                continue
            for h in range(self.heads):
                for g, X in (("k", K), ("v", V)):
                    for blk in range(a // BLOCK, (e - 1) // BLOCK + 1):
                        lo, hi = max(a, blk * BLOCK), min(e, (blk + 1) * BLOCK)
                        rows = np.zeros((hi - lo, self.d))
                        for i in range(lo, hi):
                            r = i - a if idx is None else int(idx[l, h, s * idx_seq + i - a])
                            if 0 <= r < X.shape[3]:
                                rows[i - lo] = X[l, s, h, r]
                        self._write(g, int(self.pages[l, s, blk * BLOCK // self.ps]), h, blk, lo - blk * BLOCK, rows)

    def _write(self, g, page, h, blk, first, rows):
        b = blk % (self.ps // BLOCK)
        codes = self.codes[g][page, h, b * BLOCK:(b + 1) * BLOCK]
        was = self.scale[g][page, h, b] if first else np.float32(0)
        new = scale_of(np.nan if np.isnan(rows).any() else np.abs(rows).max(), self.fmt)
        s = np.float32(np.nan) if np.isnan(was) or np.isnan(new) else max(was, new)
        self.scale[g][page, h, b] = s
        if np.isnan(s) or s == 0:
            if np.isnan(s):
                codes[:first] = 0
            codes[first:first + len(rows)] = 0
            return
        if first and s > was:
            codes[:first] = encode(decode(codes[:first], self.fmt) * np.float64(was) / np.float64(s), self.fmt)
        codes[first:first + len(rows)] = encode(rows / np.float64(s), self.fmt)

    # -- pages -----------------------------------------------------------------------------------
    def copy_blocks(self, src, dst, tokens):
        n = -(-tokens // BLOCK)
        for g in "kv":
            self.codes[g][dst, :, :n * BLOCK] = self.codes[g][src, :, :n * BLOCK]
            self.scale[g][dst, :, :n] = self.scale[g][src, :, :n]

    def resize(self, new_lens):
        """``start``, or None when nothing was done."""
        need = []
        for l, s in self.units():
            old, new = int(self.lens[l, s]), int(new_lens[l, s])
            if new < 0 or new > self.max_pages * self.ps:
                return None
            upto = min(old, new)
            copy = upto % self.ps != 0 and self.ref[self.pages[l, s, upto // self.ps]] > 1
            need.append((l, s, old, new, max(self.count(new) - self.count(old), 0), copy))
        free = self.free()
        if sum(n[4] + n[5] for n in need) > len(free):
            return None
        start = np.zeros_like(self.lens)
        ref = self.ref.copy()
        for l, s, old, new, grow, copy in need:
            for i in range(grow):
                p = free.pop(0)
                self.pages[l, s, self.count(old) + i] = p
                ref[p] = 1
            if copy:
                p, at = free.pop(0), min(old, new) // self.ps
                self.copy_blocks(self.pages[l, s, at], p, min(old, new) % self.ps)
                ref[self.pages[l, s, at]] -= 1
                self.pages[l, s, at] = p
                ref[p] = 1
            for i in range(self.count(new), self.count(old)):
                ref[self.pages[l, s, i]] -= 1
            self.lens[l, s] = new
            start[l, s] = min(old, new)
        self.ref = ref
        return start

    def fork(self, parent):
        first = {}
        for i, p in enumerate(parent):
            if not -1 <= p < self.n_seqs:
                return False
            if p >= 0:
                first.setdefault(int(p), i)
        copies = [(l, i) for l in range(self.n_layers) for i, p in enumerate(parent)
                  if p >= 0 and first[int(p)] != i and self.lens[l, p] % self.ps]
        free = self.free()
        if len(copies) > len(free):
            return False
        fresh = dict(zip(copies, free))
        pages, lens = self.pages.copy(), self.lens.copy()
        for l in range(self.n_layers):
            for i, p in enumerate(parent):
                n = int(lens[l, p]) if p >= 0 else 0
                self.lens[l, i] = n
                for c in range(self.count(n)):
                    self.pages[l, i, c] = pages[l, p, c]
                if (l, i) in fresh:
                    self.copy_blocks(pages[l, p, n // self.ps], fresh[l, i], n % self.ps)
                    self.pages[l, i, n // self.ps] = fresh[l, i]
        self.recount()
        return True

    def recount(self):
        self.ref[:] = 0
        for l, s in self.units():
            for c in range(self.count(self.lens[l, s])):
                self.ref[self.pages[l, s, c]] += 1

    def compact(self):
        live = [i for i in range(self.n_pages) if self.ref[i] > 0]
        holes = [i for i in range(len(live)) if self.ref[i] == 0]
        to = {i: i for i in live}
        for src, dst in zip([i for i in live if i >= len(live)], holes):
            to[src] = dst
            self.copy_blocks(src, dst, self.ps)
        for l, s in self.units():
            for c in range(self.count(self.lens[l, s])):
                self.pages[l, s, c] = to[int(self.pages[l, s, c])]
        self.recount()
        return len(live)

    # -- attention -------------------------------------------------------------------------------
    def rows(self, g, l, s):
        """float64 ``[heads, len, d]`` of one sequence, and which of its tokens lie on pages of the pool."""
        n = int(self.lens[l, s])
        out, there = np.zeros((self.heads, n, self.d)), np.ones(n, dtype=bool)
        for t in range(0, n, BLOCK):
            e, p, b = min(t + BLOCK, n), int(self.pages[l, s, t // self.ps]), t % self.ps // BLOCK
            if not 0 <= p < self.n_pages:
                there[t:e] = False
                continue
            out[:, t:e] = decode(np.ascontiguousarray(self.codes[g][p, :, b * BLOCK:b * BLOCK + e - t]), self.fmt) \
                * self.scale[g][p, :, b].astype(np.float64)[:, None, None]
        return out, there

    def attend(self, q, scale=None):
        """``q`` float64 ``[L, B, Hq, rows, d]`` -> output, sum of weight * |value|, and the largest sum of |q_i k_i| * scale per row."""
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        out, mag, top = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:4])
        hn, rows = q.shape[2] // self.heads, q.shape[3]
        for l, s in self.units():
            (k, there), (v, _) = self.rows("k", l, s), self.rows("v", l, s)
            n = k.shape[1]
            for h in range(q.shape[2]):
                for r in range(rows):
                    m = n - rows + 1 + r
                    sel = np.flatnonzero(there[:max(m, 0)])
                    if not len(sel):
                        continue
                    kk, vv = k[h // hn][sel], v[h // hn][sel]
                    x = kk @ q[l, s, h, r] * scale
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    out[l, s, h, r], mag[l, s, h, r] = w @ vv, w @ np.abs(vv)
                    top[l, s, h, r] = (np.abs(kk) @ np.abs(q[l, s, h, r])).max() * abs(scale)
        return out, mag, top


def beam(logits, score, n_beams, n_out, finished=None, eos=0):
    """float64 logits ``[rows, vocab]`` -> (score, parent, token), each ``[seqs, n_out]``."""
    rows, vocab = logits.shape
    total = np.full((rows, vocab), -np.inf)
    for r in range(rows):
        if not np.isfinite(score[r]):
            continue
        if finished is not None and finished[r]:
            total[r, eos] = score[r]
            continue
        m = logits[r].max()
        if np.isnan(m) or np.isinf(m):
            continue
        total[r] = score[r] + (logits[r] - (m + np.log(np.exp(logits[r] - m).sum())))
    n = rows // n_beams
    out = np.zeros((n, n_out)), np.zeros((n, n_out), dtype=np.int64), np.zeros((n, n_out), dtype=np.int64)
    for s in range(n):
        flat = total[s * n_beams:(s + 1) * n_beams].reshape(-1)
        best = np.lexsort((np.arange(len(flat)), -flat))[:n_out]
        out[0][s], out[1][s], out[2][s] = flat[best], s * n_beams + best // vocab, best % vocab
    return out
