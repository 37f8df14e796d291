"""The 8-bit cache's attention where scales of V lie far apart: results are those of the definition, and none of a row's bits depends on what
another sequence holds or on what it does not attend."""
import pytest
import torch

import quant_oracle as Q
import test_gpu_quant as T
from paper_2407_20272_amd import binding as B

pytestmark = pytest.mark.gpu
F64 = torch.float64


def split_error(c, q, lens, tables, row_table=None):
    """What the weighted probabilities' two fp16 pieces may be off by beyond 2^-22 of themselves: [rows][H][dh].
    The smaller piece is a multiple of 2^-24, so a weighted probability is off by 2^-25 at most where that is more.  Weighted probabilities are kept in
    units of R / 2^14, and R is at most four times the largest (probability in a block) * (its scale): the scale is taken as the power of two above it, and so
    is the sum of the two logarithms.  So 2^-37 of that product for each byte."""
    out = torch.zeros_like(q)
    heads = c.k.shape[1]
    for m in range(q.shape[0]):
        n, seq = lens[m] + 1, row_table[m] if row_table is not None else m
        for h in range(q.shape[1] if n > 0 else 0):
            g = h // (q.shape[1] // heads)
            blk, off = tables[seq][torch.arange(n) // 16].long(), torch.arange(n) % 16
            p = torch.softmax(c.gather(0, tables[seq], g, n) @ q[m, h] / q.shape[2] ** 0.5, 0)
            out[m, h] = 2.0 ** -37 * float((p * c.scales[blk, g, 1]).max()) * c.v[blk, g, off].abs().sum(0)
    return out


def check(kv, layer, q, out, lens, tables, row_table=None):
    c = Q.Cache.of(kv, layer - 1)
    want, _, bound = Q.attention(c, q.double(), lens, tables, row_table)
    err = (out.cpu().double() - want).abs()
    bound = bound + split_error(c, q.double(), lens, tables, row_table)
    assert bool((err <= bound).all()), (float((err / bound).max()), float(err.max()))


def grow(kv, tables, blocks, factor):
    """Multiplies V's scales of the (sequence, logical block) pairs."""
    for b, i in blocks:
        kv.scales[:, int(tables[b, i]), :, 1] *= factor


RATIOS = [20, 45]


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("ratio", RATIOS)
def test_sequences_of_one_tile(fmt, ratio):
    """Rows of three sequences in one tile of prompt rows, the one with the largest V first."""
    owned = [70, 40, 130]
    tables, nb = T.tables_for(owned, 3)
    kv = T.filled(1, nb, 2, 64, fmt, 3)
    lens, rt = [69, 68, 39, 38, 129, 128], [0, 0, 1, 1, 2, 2]
    q = torch.randn(6, 4, 64, generator=T.gen(8))
    alone = T.attend(kv, 1, q.cuda(), lens, tables, rt)
    grow(kv, tables, [(0, i) for i in range(5)], 2.0 ** ratio)
    out = T.attend(kv, 1, q.cuda(), lens, tables, rt)
    check(kv, 1, q, out, lens, tables, rt)
    assert torch.equal(out[2:], alone[2:])
    grow(kv, tables, [(2, i) for i in range(9)], 2.0 ** -ratio)
    out = T.attend(kv, 1, q.cuda(), lens, tables, rt)
    check(kv, 1, q, out, lens, tables, rt)
    assert torch.equal(out[2:4], alone[2:4])


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("ratio", RATIOS)
@pytest.mark.parametrize("n", [100, 3000])
def test_later_positions_of_a_prompt(fmt, ratio, n):
    """A chunk whose last blocks hold large values: its earlier rows do not attend them."""
    lens = [n - 40 + j for j in range(40)]
    tables, nb = T.tables_for([n], 5)
    kv = T.filled(1, nb, 1, 64, fmt, 5)
    q = torch.randn(40, 2, 64, generator=T.gen(9))
    alone = T.attend(kv, 1, q.cuda(), lens, tables, [0] * 40)
    large = [(0, i) for i in range((n - 16) // 16, (n + 15) // 16)]
    first = large[0][1] * 16
    grow(kv, tables, large, 2.0 ** ratio)
    out = T.attend(kv, 1, q.cuda(), lens, tables, [0] * 40)
    check(kv, 1, q, out, lens, tables, [0] * 40)
    before = [m for m, p in enumerate(lens) if p < first]
    assert len(before) > 10 and torch.equal(out[before], alone[before])


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("ratio", RATIOS)
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("n,group", [(200, 1), (2000, 1), (1500, 3)])
def test_large_values_that_nearly_nothing_attends(fmt, ratio, shared, n, group):
    """Blocks with the largest V whose scores are about 60 / log 2 below the others', in the first step, a middle one and the last."""
    tables, nb = T.tables_for([n, n - 50], n)
    kv = T.filled(1, nb, 2, 64, fmt, n)
    q = torch.randn(1, 2, 1, 64, generator=T.gen(4)).expand(2, 2, group, 64) * 1.5      # (query heads alike, so that one K is far from all of them)
    q = q * (1 + torch.arange(group)[:, None] / 8)
    q = q.reshape(2, 2 * group, 64).contiguous()
    large = [(b, i) for b in (0, 1) for i in (0, n // 32, (n - 50 + 15) // 16 - 1)]
    top = 127.0 if fmt == "int8" else 448.0
    for b, i in large:
        blk = int(tables[b, i])
        for h in range(2):
            x = -q[b, h * group]
            k = (x / x.abs().max() * top)
            k = k.round().to(torch.int8) if fmt == "int8" else k.to(torch.float8_e4m3fn)
            kv.k.view(torch.int8)[0, blk, h] = k.view(torch.int8).cuda()[None]
            value = float(k.double() @ x.double()) / 8.0
            kv.scales[0, blk, h, 0] = 60.0 / value
    lens = [n - 1, n - 51]
    grow(kv, tables, large, 2.0 ** ratio)
    out = T.attend(kv, 1, q.cuda(), lens, tables, [0, 1] if shared else None)
    check(kv, 1, q, out, lens, tables, [0, 1] if shared else None)
    # the same again when the large blocks are what is attended
    for b, i in large:
        kv.scales[0, int(tables[b, i]), :, 0] *= 0.0
        kv.scales[0, int(tables[b, i]), :, 0] += 2.0 ** -126
    out = T.attend(kv, 1, q.cuda(), lens, tables, [0, 1] if shared else None)
    check(kv, 1, q, out, lens, tables, [0, 1] if shared else None)


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("lens", [[40, 300], [2500, 1200, -1, 0]])
def test_scales_of_every_size(fmt, shared, lens):
    """Every block's scale of V another power of two between 2^-126 and 2^100."""
    owned = [n + 1 for n in lens]
    tables, nb = T.tables_for(owned, 6)
    kv = T.filled(1, nb, 2, 64, fmt, 6)
    kv.scales[..., 1] = torch.exp2(torch.randint(-126, 101, kv.scales.shape[:-1], generator=T.gen(7)).float())
    q = torch.randn(len(lens), 4, 64, generator=T.gen(1))
    out = T.attend(kv, 1, q.cuda(), lens, tables, list(range(len(lens))) if shared else None)
    check(kv, 1, q, out, lens, tables, list(range(len(lens))) if shared else None)


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("n", [60, 300, 5000])
def test_values_next_to_the_largest_float(fmt, shared, n):
    """The sum of probabilities times values stays below the largest value."""
    tables, nb = T.tables_for([n], 2)
    kv = T.filled(1, nb, 1, 64, fmt, 2)
    kv.v.view(torch.int8)[:] = torch.full_like(kv.v.float(), 127.0 if fmt == "int8" else 448.0).to(kv.v.dtype).view(torch.int8)
    kv.scales[..., 1] = 2.6e36 if fmt == "int8" else 2.0 ** 119
    q = torch.randn(1, 8, 64, generator=T.gen(1))
    out = T.attend(kv, 1, q.cuda(), [n - 1], tables, [0] if shared else None)
    check(kv, 1, q, out, [n - 1], tables, [0] if shared else None)
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("n,shared", [(300, False), (300, True), (3000, False), (3000, True)])
def test_scores_of_any_size(fmt, n, shared):
    """Scores of 10^8 and more, beside small scales of V: the position with the largest one is the result, and has the attention."""
    tables, nb = T.tables_for([n], 2)
    kv = T.filled(1, nb, 1, 64, fmt, 2)
    kv.scales[..., 1] *= 2.0 ** -30
    q = torch.randn(1, 2, 64, generator=T.gen(1))
    q[0, 1] = q[0, 0] * 3.0
    c = Q.Cache.of(kv)
    z = c.gather(0, tables[0], 0, n) @ q[0, 0].double()
    top = z.topk(2)
    # (float scores: 2^-16 of the largest apart is far more than their errors, and e^(-z) of it is nothing)
    assert float(top.values[0] - top.values[1]) > 2.0 ** -16 * float(z.abs().max())
    best = int(top.indices[0])
    want = c.gather(1, tables[0], 0, n)[best]
    for size in (1e8, 1e12, 1e30):
        w = None if shared else torch.full((1, 1, n), 7.0, device="cuda")
        out = T.attend(kv, 1, (q * size).cuda(), [n - 1], tables, [0] if shared else None, weights=w).cpu().double()
        assert bool(((out[0] - want).abs() <= want.abs() * 2.0 ** -20 + 1e-37).all())
        if not shared:
            assert bool(((w[0, 0].cpu().double() - 2.0 * (torch.arange(n) == best)).abs() <= 2.0 ** -20).all())
