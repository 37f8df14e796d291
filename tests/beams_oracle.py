"""Several continuations of a prompt, in float64 on the CPU from the definitions: pages by counting, beam selection by sorting every
candidate, attention row by row."""
import math

import torch

F64 = torch.float64


def blocks_of(n):
    return (n + 15) // 16


# ---- pages --------------------------------------------------------------------------------------------------------
class Pages:
    """refs, and tables as lists of rows: (entries, length)."""

    def __init__(self, refs):
        self.refs = list(refs)

    def fork(self, rows, parents):
        new = []
        for p in parents:
            t, n = rows[p] if 0 <= p < len(rows) else ([], 0)
            t = list(t[:blocks_of(n)])
            for b in t:
                self.refs[b] += 1
            new.append((t, n))
        return new

    def release(self, rows):
        for t, n in rows:
            for b in t[:blocks_of(n)]:
                self.refs[b] -= 1

    def grow(self, rows, new_lens):
        """(rows, moves, missing), changed in the order of the rows: the simplest statement of who keeps a block."""
        left, replace, want = list(self.refs), [], 0
        writers = {}
        for m, (t, n) in enumerate(rows):
            if n % 16 and new_lens[m] > n:
                writers.setdefault(t[n // 16], []).append(m)
        for m, (t, n) in enumerate(rows):
            b = t[n // 16] if n % 16 and new_lens[m] > n else None
            replace.append(b is not None and left[b] > 1 and not (len(writers[b]) == left[b] and writers[b][-1] == m))
            want += replace[-1] + max(0, blocks_of(new_lens[m]) - blocks_of(n))
        free = [b for b, r in enumerate(self.refs) if r <= 0]
        if want > len(free):
            return rows, [(-1, -1)] * len(rows), want - len(free)
        grown, moves, taken = [], [], iter(free)
        for m, (t, n) in enumerate(rows):
            t, move = list(t[:blocks_of(n)]), (-1, -1)
            if replace[m]:
                move = (t[n // 16], next(taken))
                t[n // 16] = move[1]
                self.refs[move[0]] -= 1
                self.refs[move[1]] = 1
            for _ in range(blocks_of(new_lens[m]) - blocks_of(n)):
                t.append(next(taken))
                self.refs[t[-1]] = 1
            grown.append((t, n))
            moves.append(move)
        return grown, moves, 0

    def compact(self, rows):
        n = sum(r > 0 for r in self.refs)
        pairs = list(zip([b for b, r in enumerate(self.refs) if r > 0 and b >= n], [b for b, r in enumerate(self.refs) if r <= 0 and b < n]))
        to = dict(pairs)
        remap = [to.get(b, b) if r > 0 else -1 for b, r in enumerate(self.refs)]
        refs = [0] * len(self.refs)
        for b, r in enumerate(self.refs):
            if r > 0:
                refs[remap[b]] = r
        self.refs = refs
        return [([remap[b] for b in t[:blocks_of(k)]], k) for t, k in rows], remap, pairs


def shared(rows, first):
    out = []
    for a, z in zip(first, first[1:]):
        k = 0
        while a < z and k < min(n // 16 for _, n in rows[a:z]) and len({t[k] for t, _ in rows[a:z]}) == 1:
            k += 1
        out.append(k)
    return out


# ---- beams --------------------------------------------------------------------------------------------------------
def select(logits, scores, beams, n_out, finished=None, end=-1):
    """(tokens, parents, scores float64, finished) of every group, flat."""
    rows, vocab = logits.shape
    out = ([], [], [], [])
    for g in range(0, rows, beams):
        cand = []
        for b in range(g, g + beams):
            s = float(scores[b])
            if finished is not None and finished[b]:
                v = torch.full((vocab,), -math.inf, dtype=F64)
                v[end] = s
            else:
                z = logits[b].double()
                most = z.max()
                v = s + (z - (most + torch.log(torch.exp(z - most).sum())))
            cand.append(torch.where(torch.isfinite(v), v, -math.inf))
        v, at = torch.sort(torch.cat(cand), descending=True, stable=True)
        for s, i in zip(v[:n_out].tolist(), at[:n_out].tolist()):
            p, t = g + i // vocab, i % vocab
            for lst, x in zip(out, (t, p, s, int(t == end or (finished is not None and bool(finished[p]))))):
                lst.append(x)
    return out


# ---- attention ----------------------------------------------------------------------------------------------------
def attend(q, k, v, tables, lens, row_table=None):
    """q [rows][H][dh], one layer's pools k, v [blocks][kv][16][dh] (any type): (out, bound), float64.

    The bound counts roundings, eps = 2^-24.  A score is a sum of dh products of q (scaled, one rounding) with K, accumulated in float: off by at
    most (dh + 8) eps S with S the largest sum of |q K| / sqrt(dh); a probability by twice that and the exponential's 2^-21, relatively.  Sums over n
    positions are chains of at most 3 n / 32 products of 32, and of the joins behind them."""
    rows, heads, dh = q.shape
    kv, eps = k.shape[1], 2.0 ** -24
    out, bound = torch.zeros(q.shape, dtype=F64), torch.zeros(q.shape, dtype=F64)
    for m in range(rows):
        n = int(lens[m]) + 1
        if n <= 0:
            continue
        t = tables[row_table[m] if row_table is not None else m]
        at = torch.arange(n)
        blk = t[at // 16].long()
        for h in range(heads):
            kk, vv = k[blk, h // (heads // kv), at % 16].double(), v[blk, h // (heads // kv), at % 16].double()
            x = q[m, h].double()
            z = kk @ x / math.sqrt(dh)
            p = torch.softmax(z, 0)
            out[m, h] = p @ vv
            s = float((kk.abs() @ x.abs()).max()) / math.sqrt(dh)
            bound[m, h] = (p @ vv.abs()) * (2 * (dh + 8) * eps * s + 2.0 ** -21 + (3 * n / 32 + 80) * eps)
    return out, bound
