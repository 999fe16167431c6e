"""Plain implementations of the paged 8-bit cache's operators, sequence by sequence, for the tests: codes in the stated fp32 arithmetic (numpy), attention in
64 bits, the bookkeeping as a loop over rows and pages."""
import numpy as np
import torch

from paper_2408_01890_b200 import binding as lb

BLOCK = 16


def top(dtype):
    return np.float32(127.0 if dtype == lb.S8 else 448.0)


def encode(y, dtype):
    """fp32 values in units of the scale -> code values (as fp32)."""
    t = torch.from_numpy(np.ascontiguousarray(y, dtype=np.float32))
    if dtype == lb.S8:
        return t.round().clamp(-127, 127).numpy()
    return t.clamp(-448, 448).to(torch.float8_e4m3fn).float().numpy()


class Mirror:
    """What a layer's pool should hold: codes (as values) and scales of every page, on the host."""

    def __init__(self, layer):
        self.layer = layer
        kw = layer.r if layer.kind == lb.CACHE_SHARED else layer.d
        n, H, P = layer.n_pages, layer.Hkv, layer.page_tokens
        self.codes = [np.zeros((n, H, P, w), np.float32) for w in (kw, layer.d)]
        self.scales = np.zeros((n, H, P // BLOCK, 2), np.float32)
        self.load()

    def load(self):
        l = self.layer
        k = l.k.float()
        if l.kind == lb.CACHE_SHARED:
            k = k.transpose(3, 4).flatten(2, 3)
        self.codes = [k.cpu().numpy().copy(), l.v.float().cpu().numpy().copy()]
        self.scales = l.scales.cpu().numpy().copy()

    def append(self, table, rows, first, counts):
        """rows: (k or k', v) fp32 numpy [B,n,H,w]; table, first, counts: host lists."""
        l, P = self.layer, self.layer.page_tokens
        for b in range(len(first)):
            end = first[b] + counts[b]
            blk = first[b] // BLOCK
            while counts[b] > 0 and blk * BLOCK < end:
                lo, hi = max(first[b], blk * BLOCK), min(end, (blk + 1) * BLOCK)
                page, at = table[b][blk * BLOCK // P], blk * BLOCK % P
                blk += 1
                if not 0 <= page < l.n_pages:
                    continue
                old = slice(at, at + lo % BLOCK)
                new = slice(at + lo % BLOCK, at + lo % BLOCK + hi - lo)
                for i in (0, 1):
                    x = rows[i][b, lo - first[b]:hi - first[b]].transpose(1, 0, 2)     # [H, rows, w]
                    codes, scale = self.codes[i], self.scales[page, :, at // BLOCK, i]
                    for h in range(l.Hkv):
                        amax = np.max(np.abs(x[h])) if np.all(np.isfinite(x[h])) else np.float32(np.nan)
                        s = np.float32(amax) / top(l.dtype)
                        if lo % BLOCK:
                            held = scale[h]
                            s = np.float32(np.nan) if np.isnan(s) or np.isnan(held) else max(s, held)
                            if not s == held:
                                codes[page, h, old] = encode(codes[page, h, old] * (held / s), l.dtype) if s > 0 else 0
                        codes[page, h, new] = encode(x[h] / s, l.dtype) if s > 0 else 0
                        scale[h] = s

    def rows(self, b_table, n, i):
        """[H, n, w] values of the first n positions, in 64 bits."""
        P = self.layer.page_tokens
        out = []
        for pos in range(n):
            page, at = b_table[pos // P], pos % P
            out.append(self.codes[i][page, :, at].astype(np.float64) * self.scales[page, :, at // BLOCK, i].astype(np.float64)[:, None])
        return np.stack(out, 1)


def softmax_v(a, V, G):
    """a [Hq, n] scores, V [Hkv, n, d], both fp64 -> o [Hq, d]"""
    p = np.exp(a - a.max(1, keepdims=True))
    return np.einsum("hn,hnd->hd", p / p.sum(1, keepdims=True), np.repeat(V, G, 0))


ACT = {lb.ACT_NONE: lambda x: x, lb.ACT_RELU: lambda x: np.maximum(x, 0), lb.ACT_SILU: lambda x: x / (1 + np.exp(-x))}


def shared_scores(prev, qp, KP, link):
    """prev [Hq, n], qp [Hq, r], KP [Hkv, n, r], all fp64 -> [Hq, n]"""
    f = lambda t: None if t is None else t.double().cpu().numpy()
    w1, w2, b1, b2 = f(link.w1), f(link.w2), f(link.b1), f(link.b2)
    D = np.einsum("hr,hnr->hn", qp, np.repeat(KP, len(qp) // len(KP), 0)) / np.sqrt(qp.shape[1])
    if link.integrate == lb.INTEGRATE_PLUS:
        return prev + D
    x = np.concatenate([prev, D]) if link.integrate == lb.INTEGRATE_CONCAT else prev
    y = w1.T @ x + (0 if b1 is None else b1[:, None])
    if link.ffn_layers == 2:
        y = w2.T @ ACT[link.act](y) + (0 if b2 is None else b2[:, None])
    return y if link.integrate == lb.INTEGRATE_CONCAT else y + D


class Book:
    """The bookkeeping on the host, row by row."""

    def __init__(self, B, max_pages, n_pages, P):
        self.P, self.n_pages, self.max_pages = P, n_pages, max_pages
        self.table = np.full((B, max_pages), -1, np.int64)
        self.lens = np.zeros(B, np.int64)
        self.recount()

    def recount(self):
        self.refs = np.bincount(self.table[self.table >= 0].ravel(), minlength=self.n_pages)

    def fork(self, parent):
        t, l = self.table.copy(), self.lens.copy()
        for i, q in enumerate(parent):
            ok = 0 <= q < len(l)
            self.table[i], self.lens[i] = (t[q], l[q]) if ok else (-1, 0)
        self.recount()

    def reserve(self, n_new):
        """Pairs (source, destination) to copy, or None where there are too few pages."""
        P, refs, table = self.P, self.refs.copy(), self.table.copy()
        moves, taken = [], []
        plan = []
        for b, (n, add) in enumerate(zip(self.lens, n_new)):
            add = max(0, add)
            have, need = -(-n // P), -(-(n + add) // P)
            if need > self.max_pages:
                return None
            if n % P and add:
                last = table[b, have - 1]
                if last >= 0 and refs[last] > 1:
                    refs[last] -= 1
                    plan.append((b, have - 1, last))
            plan += [(b, s, -1) for s in range(have, need)]
        free = [q for q in range(self.n_pages) if self.refs[q] == 0]
        if len(free) < len(plan):
            return None
        for (b, slot, src), page in zip(plan, free):
            table[b, slot] = page
            refs[page] = 1
            if src >= 0:
                moves.append((src, page))
        self.table, self.refs = table, refs
        return moves

    def compact(self):
        used = self.refs > 0
        n = used.sum()
        holes, movers = np.nonzero(~used[:n])[0], np.nonzero(used[n:])[0] + n
        to = np.arange(self.n_pages)
        to[movers] = holes
        self.table = np.where(self.table >= 0, to[self.table], -1)
        refs = self.refs.copy()
        refs[holes], refs[movers] = self.refs[movers], 0
        self.refs = refs
        return list(zip(movers, holes))
