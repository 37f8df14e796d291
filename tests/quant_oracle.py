"""The 8-bit cache, its attention, its eviction and the rotary embedding on their own, in float64 on the CPU, written from the
definitions: one position, one head at a time."""
import math

import torch

F64 = torch.float64
FLOOR = 2.0 ** -126


def f32(x):
    """A float64 tensor or number rounded to float32, as float64."""
    if isinstance(x, float):
        return float(torch.tensor(x, dtype=F64).float())
    return x.float().double()


# ---- bytes ------------------------------------------------------------------------------------------------------
def scale_for(largest, fmt):
    if not largest < math.inf:
        return math.nan
    if fmt == "int8":
        return max(FLOOR, f32(largest / 127.0))
    if largest == 0.0:
        return FLOOR
    m, e = math.frexp(largest)
    return max(FLOOR, 2.0 ** (e - 9 if m <= 0.875 else e - 8))


def rounded(x, scale, fmt):
    """The bytes' own values nearest to x / scale (float64)."""
    if scale != scale:
        return torch.zeros_like(x)
    y = x / scale
    if fmt == "int8":
        return torch.round(y).clamp(-127, 127)
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -40)))
    e = torch.where(torch.exp2(e) > y.abs(), e - 1, e)
    step = torch.exp2(torch.clamp(e, min=-6) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


class Cache:
    """One layer: own values k, v [blocks][heads][16][dh] (float64) and scales [blocks][heads][2]."""

    def __init__(self, k, v, scales, fmt):
        self.k, self.v, self.scales, self.fmt = k, v, scales, fmt

    @classmethod
    def of(cls, kv, layer=0):
        """A copy of a device cache's layer."""
        fmt = "int8" if kv.k.dtype == torch.int8 else "e4m3"
        return cls(kv.k[layer].cpu().double(), kv.v[layer].cpu().double().transpose(-1, -2).contiguous(), kv.scales[layer].cpu().double(), fmt)

    def copy(self):
        return Cache(self.k.clone(), self.v.clone(), self.scales.clone(), self.fmt)

    def value(self, which, blk, head, off):
        return f32((self.v if which else self.k)[blk, head, off] * self.scales[blk, head, which])

    def gather(self, which, table, head, n):
        """The floats of positions 0..n-1: [n][dh]."""
        pool = self.v if which else self.k
        blk = table[torch.arange(n) // 16].long()
        return f32(pool[blk, head, torch.arange(n) % 16] * self.scales[blk, head, which][:, None])


def append(c, k, v, lens, tables, row_table=None):
    """In place.  k, v [rows][heads][dh] float64."""
    n, wide = len(lens), tables.shape[1]
    row = 0
    while row < n:
        pos, seq = lens[row], row_table[row] if row_table is not None else row
        end = row + 1
        while end < n and pos >= 0 and (row_table[end] if row_table is not None else end) == seq and lens[end] == pos + end - row and lens[end] // 16 == pos // 16:
            end += 1
        m, row = row, end
        if pos < 0 or pos // 16 >= wide:
            continue
        blk = int(tables[seq, pos // 16])
        if not 0 <= blk < c.k.shape[0]:
            continue
        off = pos % 16
        for which, new, pool in ((0, k, c.k), (1, v, c.v)):
            for h in range(pool.shape[1]):
                x = new[m:end, h]
                big = float(x.abs().max()) if bool(torch.isfinite(x).all()) else math.inf
                s, was = scale_for(big, c.fmt), float(c.scales[blk, h, which])
                if off:
                    s = math.nan if s != s or was != was else max(s, was)
                    if s != was:
                        pool[blk, h, :off] = rounded(f32(pool[blk, h, :off] * was), s, c.fmt) if was == was else 0.0
                pool[blk, h, off:off + end - m] = rounded(x, s, c.fmt)
                c.scales[blk, h, which] = s


def attention(c, q, lens, tables, row_table=None):
    """q [rows][H][dh] float64.  (result [rows][H][dh], probabilities per row [H][positions], bound [rows][H][dh] on what a
    float computation may be off by)."""
    rows, H, dh = q.shape
    heads = c.k.shape[1]
    out, bound, probs = torch.zeros_like(q), torch.zeros_like(q), []
    for m in range(rows):
        n = lens[m] + 1
        seq = row_table[m] if row_table is not None else m
        mine = torch.zeros(H, max(n, 0), dtype=F64)
        slack = torch.zeros(H, dtype=F64)
        for h in range(H):
            if n <= 0:
                continue
            kk, vv = c.gather(0, tables[seq], h // (H // heads), n), c.gather(1, tables[seq], h // (H // heads), n)
            z = (kk @ q[m, h]) / math.sqrt(dh)
            p = torch.softmax(z, 0)
            mine[h] = p
            out[m, h] = p @ vv
            # q in two fp16 pieces is 2^-22 off; a product sum of dh terms gathers 2^-24 each (a byte's value is exact, the float of byte times
            # scale is not formed); the score is multiplied twice and goes to exp2 relative to the maximum
            mass = float((kk.abs() @ q[m, h].abs()).max()) / math.sqrt(dh)
            dz = mass * (2.0 ** -22 + (dh + 8) * 2.0 ** -24) + 4 * float(z.abs().max()) * 2.0 ** -24
            # softmax: both sums move with the scores, exp2 is good to 2^-22, sums gather 2^-24 a term; the weights in two pieces
            slack[h] = 2 * dz + 2.0 ** -20 + 2 * (n + 32) * 2.0 ** -24
            bound[m, h] = float(slack[h]) * (p @ vv.abs()) + 1e-37
        probs.append((mine, slack))
    return out, probs, bound


def evict(c, lens, tables, weights, keep, recent, dst_tables=None):
    """In place in c (dst_tables or the sequence's own first blocks).  Returns (kept lists, new lengths)."""
    old = c.copy()
    kept, heads = [], c.k.shape[1]
    for b, n in enumerate(lens):
        mine = []
        for h in range(heads):
            if n <= keep:
                ids = list(range(n))
            else:
                w = [float(x) for x in weights[b, h, :n]]
                key = [math.inf if x != x else x for x in w]
                nan = [x != x for x in w]
                order = sorted(range(n - recent), key=lambda i: (not nan[i], -key[i], i))
                ids = sorted(order[:keep - recent]) + list(range(n - recent, n))
            mine.append(ids)
            if dst_tables is None and n <= keep:
                continue
            for slot in range((len(ids) + 15) // 16):
                part = ids[slot * 16:slot * 16 + 16]
                to = int((tables if dst_tables is None else dst_tables)[b, slot])
                for which in (0, 1):
                    pool, was = (old.v if which else old.k), old.scales
                    need = [FLOOR]
                    for p in part:
                        blk = int(tables[b, p // 16])
                        s, most = float(was[blk, h, which]), float(pool[blk, h, p % 16].abs().max())
                        need.append(s if c.fmt == "int8" and most >= 127 else scale_for(f32(most * s), c.fmt))
                    s = math.nan if any(x != x for x in need) else max(need)
                    for j, p in enumerate(part):
                        x = old.value(which, int(tables[b, p // 16]), h, p % 16)
                        (c.v if which else c.k)[to, h, j] = rounded(x, s, c.fmt)
                    c.scales[to, h, which] = s
        kept.append(mine)
    return kept, [min(n, keep) for n in lens]


# ---- rotary -----------------------------------------------------------------------------------------------------
def frequencies(rotary_dim, theta=10000.0, scaling="plain", factor=1.0, original=1, turns=(1.0, 4.0)):
    out = []
    for j in range(rotary_dim // 2):
        f = theta ** (-2.0 * j / rotary_dim)
        if scaling == "linear":
            f /= factor
        if scaling == "turns":
            w = (original * f / (2 * math.pi) - turns[0]) / (turns[1] - turns[0])
            w = min(1.0, max(0.0, w))
            f = f * w + f * (1 - w) / factor
        out.append(f)
    return torch.tensor(out, dtype=F64)


def rotary(x, positions, freqs, layout, amplitude=1.0, transpose=False):
    """x [rows][heads][dh] float64."""
    r = 2 * len(freqs)
    y = x.clone()
    w = positions.double()[:, None] * freqs[None]
    c, s = amplitude * torch.cos(w)[:, None], amplitude * torch.sin(w)[:, None] * (-1 if transpose else 1)
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if layout == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    ra, rb = a * c - b * s, a * s + b * c
    if layout == "half":
        y[..., :r // 2], y[..., r // 2:r] = ra, rb
    else:
        y[..., 0:r:2], y[..., 1:r:2] = ra, rb
    return y
