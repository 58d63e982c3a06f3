"""The paged 8-bit KV cache by its definition, in numpy and 64 bits: tables, pages, attention.  Written apart from the library and
from perf/operators.py; what a pass may read is worked out from positions."""
import numpy as np

PAGE = 64


def to_bf16(x):
    """Nearest even bf16 of float32 values, as float32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), r, x).astype(np.float32)


def e4m3(y):
    """Nearest even e4m3 of |y| <= 448, float64."""
    a = np.abs(y)
    e = np.where(a > 0, np.frexp(np.where(a > 0, a, 1.0))[1] - 1, -6)
    step = np.ldexp(1.0, np.maximum(e, -6) - 3)
    return np.rint(y / step) * step


def page_values(x):
    """A complete page [64][heads][head_dim] as what its 8 bits stand for; rows of NaN stay, and set no scale."""
    out = np.empty(x.shape, np.float64)
    for h in range(x.shape[1]):
        top = np.nanmax(np.abs(np.where(np.isfinite(x[:, h]), x[:, h], 0.0)).astype(np.float64))
        e = 0
        if top > 0:
            e = int(np.frexp(top)[1]) - 12
            while top > 448.0 * 2.0 ** e:
                e += 1
            e = max(e, -100)
        with np.errstate(invalid="ignore"):
            out[:, h] = e4m3(x[:, h].astype(np.float64) / 2.0 ** e) * 2.0 ** e
    return out


class Kv8Model:
    def __init__(self, n_layers, hq, hkv, hd, max_batch, max_seq, n_pages=0):
        self.hq, self.hkv, self.hd, self.max_seq = hq, hkv, hd, max_seq
        self.n_pages = n_pages or max_batch * (max_seq // PAGE)
        self.free = list(range(self.n_pages))[::-1]
        self.table = [[] for _ in range(max_batch)]
        self.len, self.hot, self.base = [0] * max_batch, [0] * max_batch, [0] * max_batch
        self.k = np.zeros((n_layers, max_batch, max_seq, hkv, hd), np.float32)
        self.v = np.zeros_like(self.k)

    def reserve(self, start, new, rows, max_new, max_len):
        """Returns (slots, sequences, positions) of the rows, and the sequences refused."""
        B = len(start)
        slots, seqs, poss = np.full(rows, -1), np.full(rows, -1), np.zeros(rows, int)
        at, plan = 0, []
        for b in range(B):
            n = min(max(new[b], 0), rows)
            s = start[b]
            ok = 0 <= s <= max_len and 0 <= new[b] <= min(max_new, rows) and s + new[b] <= max_len and s <= self.len[b]
            ok = ok and (s % PAGE == 0 or s // PAGE >= self.hot[b] or self.base[b] // PAGE * PAGE < s <= self.base[b]) and at + n <= rows
            plan.append([at, s, new[b] if ok else 0, ok])
            at += n
        pages = lambda b: -(-(plan[b][1] + plan[b][2]) // PAGE) if plan[b][3] else len(self.table[b])   # noqa: E731
        given = []
        for b in range(B):
            given += self.table[b][pages(b):]
        self.free += given[::-1]
        short = False
        for b in range(B):
            p = plan[b]
            need = pages(b) - len(self.table[b])
            if need > 0 and (short or need > len(self.free)):
                short, p[2], p[3] = True, 0, False
                continue
            if need <= 0:
                self.table[b] = self.table[b][:pages(b)]
            for _ in range(need):
                self.table[b].append(self.free.pop())
            if p[3]:
                first, last = p[1] // PAGE, (p[1] + max(p[2], 1) - 1) // PAGE
                ring = first >= self.hot[b]
                kept = self.base[b] // PAGE * PAGE < p[1] <= self.base[b]
                if kept or (min(max_new, rows) > PAGE and p[1] % PAGE and p[2]):
                    self.base[b] = p[1]
                elif p[1] < self.base[b]:
                    self.base[b] = first * PAGE
                if p[2]:
                    self.hot[b] = max(min(self.hot[b], first), last - 1)
                elif p[1] % PAGE == 0 or ring:
                    self.hot[b] = min(self.hot[b], first)
                self.len[b] = p[1] + p[2]
            for i in range(p[2]):
                ps = p[1] + i
                slots[p[0] + i], seqs[p[0] + i], poss[p[0] + i] = self.table[b][ps // PAGE] * PAGE + ps % PAGE, b, ps
        self.plan, self.seqs, self.poss = plan, seqs, poss
        return slots, seqs, poss, sum(not p[3] for p in plan)

    def append(self, layer, k, v):
        k, v = to_bf16(k), to_bf16(v)
        bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))
        k, v = np.where(bad[..., None], np.nan, k), np.where(bad[..., None], 0.0, v)
        for r, (b, p) in enumerate(zip(self.seqs, self.poss)):
            if b >= 0:
                self.k[layer, b, p], self.v[layer, b, p] = k[r], v[r]

    def _cold(self, layer, b, pages):
        cat = lambda x: np.concatenate([page_values(x[layer, b, p * PAGE:(p + 1) * PAGE]) for p in range(pages)] + [np.zeros((0, self.hkv, self.hd))])   # noqa: E731
        return cat(self.k), cat(self.v)

    def read(self, layer, seq, pos):
        out = np.zeros((2, len(seq), self.hkv, self.hd))
        for b in set(int(x) for x in seq):
            if not 0 <= b < len(self.len):
                continue
            whole = self.len[b] // PAGE
            k8, v8 = self._cold(layer, b, whole)
            for r in np.nonzero(np.asarray(seq) == b)[0]:
                p = int(pos[r])
                if 0 <= p < self.len[b]:
                    out[0, r] = k8[p] if p < whole * PAGE else self.k[layer, b, p]
                    out[1, r] = v8[p] if p < whole * PAGE else self.v[layer, b, p]
        return out

    def attend(self, layer, q, limits=None, scale=0.0):
        """(result, sum of p |v|, largest sum of |q k| times scale) per row and head, float64."""
        R, G = q.shape[0], self.hq // self.hkv
        scale = scale or self.hd ** -0.5
        out, mag, prod = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
        for b, (row0, s, n, ok) in enumerate(self.plan):
            if not n:
                continue
            k8, v8 = self._cold(layer, b, self.len[b] // PAGE)
            for i in range(n):
                r = row0 + i
                lim = min(max(int(limits[r]), 0), self.len[b]) if limits is not None else s + i + 1
                if lim == 0:
                    continue
                own = (lim - 1) // PAGE
                cut = own * PAGE if own >= s // PAGE else lim
                kk = np.concatenate([k8[:cut], self.k[layer, b, cut:lim].astype(np.float64)])
                vv = np.concatenate([v8[:cut], self.v[layer, b, cut:lim].astype(np.float64)])
                qq = q[r].astype(np.float64).reshape(self.hkv, G, self.hd)
                sc = np.einsum("hgd,lhd->hgl", qq, kk) * scale
                with np.errstate(invalid="ignore"):
                    p = np.exp(sc - sc.max(-1, keepdims=True))
                    p /= p.sum(-1, keepdims=True)
                out[r] = np.einsum("hgl,lhd->hgd", p, vv).reshape(self.hq, self.hd)
                mag[r] = np.einsum("hgl,lhd->hgd", p, np.abs(vv)).reshape(self.hq, self.hd)
                prod[r] = (np.einsum("hgd,lhd->hgl", np.abs(qq), np.abs(kk)) * scale).max(-1).reshape(self.hq)
        return out, mag, prod

    def tolerance(self, dtype, out, mag, prod):
        """How far a correct kernel's result may be from attend()'s, elementwise.  mag: sum of p |v|.
        scores: head_dim products and as many sums in fp32, half a step (2^-24) of at most sum |q k| each; a score off by d
            changes every weight by at most 2 d of itself (its own term and the sum's).  The exponent's argument has up to three
            roundings more and the exponential is good to 2^-22.
        sums over keys: at most max_seq / 8 + 64 of them behind each other in any order of tiles, half a step each, for the
            weights' sum and for the result.
        bf16: each weight is rounded once (2^-9 of the value's power of two, so at most 2^-8 of it), and the result."""
        h = 2.0 ** -24
        score = (self.hd + 3) * h * prod[..., None] + 2.0 ** -22
        keys = 2 * (self.max_seq / 8 + 64) * h
        t = (2 * score + keys) * 2 * mag + h * np.abs(out)
        return t + 2.0 ** -8 * (mag + np.abs(out)) if dtype == "bf16" else t
