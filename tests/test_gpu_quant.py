"""The 8-bit cache, its attention and eviction, and the rotary embedding on their own, on the GPU against float64 (quant_oracle).

Bytes and scales are exact: every rounding is to the nearest of an exact quotient.  Floats have the bounds that quant_oracle derives."""
import math

import pytest
import torch

import quant_oracle as Q
from paper_2407_20272_amd import binding as B

pytestmark = pytest.mark.gpu
F64 = torch.float64
FORMATS = ["int8", "e4m3"]


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def tables_for(lens, seed, spare=2, width=0):
    """Shuffled blocks for lens[i] positions each, -1 behind them; (tables, num_blocks)."""
    need = [(n + 15) // 16 for n in lens]
    order = torch.randperm(sum(need) + spare, generator=gen(seed)).to(torch.int32)
    t, used = torch.full((len(lens), max(1, width, *need)), -1, dtype=torch.int32), 0
    for i, n in enumerate(need):
        t[i, :n] = order[used:used + n]
        used += n
    return t, sum(need) + spare


def filled(n_layers, num_blocks, heads, dh, fmt, seed):
    """A cache of random bytes and scales."""
    kv = B.QuantKV(n_layers, num_blocks, heads, dh, fmt)
    g = gen(seed)
    for pool in (kv.k, kv.v):
        x = torch.randn(pool.shape, generator=g) * (45 if fmt == "int8" else 120)
        x = x.round().clamp(-127, 127).to(torch.int8) if fmt == "int8" else x.clamp(-448, 448).to(torch.float8_e4m3fn)
        pool.view(torch.int8).copy_(x.view(torch.int8))
    s = torch.rand(kv.scales.shape, generator=g) + 0.3
    kv.scales.copy_(s / 50 if fmt == "int8" else torch.exp2(torch.round(torch.log2(s) * 2) - 7))
    return kv


def poison(kv, tables, lens, layer=0):
    """Bytes that are no number and scales that are NaN wherever no position of a sequence is."""
    nb = kv.num_blocks
    used = torch.zeros(nb, 16, dtype=torch.bool)
    for b, n in enumerate(lens):
        for p in range(n):
            used[int(tables[b, p // 16]), p % 16] = True
    k, v = kv.k[layer].view(torch.uint8), kv.v[layer].view(torch.uint8)
    hole = (~used).cuda()
    k[hole[:, None, :, None].expand_as(k)] = 0x7F
    v[hole[:, None, None, :].expand_as(v)] = 0x7F
    kv.scales[layer][(~used.any(1)).cuda()] = float("nan")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda") if not torch.is_tensor(x) else x.to(torch.int32).cuda()


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))


def assert_cache(kv, ref, layer=0):
    got = Q.Cache.of(kv, layer)
    assert same(got.scales, ref.scales)
    # (-0 and 0 are different bytes of one value; a block whose scale is NaN stands for nothing else)
    alive = ref.scales == ref.scales
    for name, x, y in (("k", got.k, ref.k), ("v", got.v, ref.v)):
        ok = (x == y) | ~alive[..., 0 if name == "k" else 1][:, :, None, None] | (x != x) & (y != y)
        assert bool(ok.all()), (name, (~ok).nonzero()[:5].tolist())


# ---- rotary ------------------------------------------------------------------------------------------------------
ROTARY = [
    # dtype, layout, head_dim, rotary_dim, heads, kv heads, rows
    (torch.bfloat16, "half", 128, 128, 32, 8, 1),
    (torch.bfloat16, "half", 128, 64, 5, 1, 37),
    (torch.bfloat16, "half", 80, 80, 3, 3, 9),          # halves of 40: pieces of eight
    (torch.bfloat16, "half", 80, 24, 3, 1, 9),          # halves of 12: element by element
    (torch.bfloat16, "interleaved", 64, 64, 4, 2, 300),
    (torch.bfloat16, "interleaved", 96, 40, 4, 2, 17),
    (torch.bfloat16, "interleaved", 66, 10, 2, 1, 5),
    (torch.float32, "half", 64, 64, 4, 4, 65),
    (torch.float32, "half", 30, 14, 3, 1, 7),
    (torch.float32, "half", 1024, 1024, 2, 1, 3),
    (torch.float32, "interleaved", 128, 128, 40, 10, 33),
    (torch.float32, "interleaved", 7, 6, 1, 1, 2),
]


def rotary_tolerance(x, y, layout, r, amplitude, dtype):
    """The angle's rounding to float (half a step of a number up to half a turn, times 2 pi: under 2^-23), sincospi (2^-23), amplitude, two
    products and a sum: under 2^-20 of the pair's magnitudes; then half a step of the type."""
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if layout == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    m = (a.abs() + b.abs()) * abs(amplitude) * 2.0 ** -20
    t = torch.zeros_like(x)
    if layout == "half":
        t[..., :r // 2], t[..., r // 2:r] = m, m
    else:
        t[..., 0:r:2], t[..., 1:r:2] = m, m
    return t + (y.abs() + t) * torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype,layout,dh,r,h,kv,rows", ROTARY)
def test_rotary(dtype, layout, dh, r, h, kv, rows, transpose):
    g = gen(rows + dh)
    scaling = ["plain", "linear", "turns"][(rows + r) % 3]
    amplitude = 1.0 if rows % 2 else -1.25
    kw = dict(theta=500000.0 if dh == 128 else 10000.0, scaling=scaling, factor=13.59)
    desc = B.make_rotary_desc(dh, r, layout=layout, original_context=8192, turns=(1.0, 4.0), amplitude=amplitude, **kw)
    freqs = B.ee_rotary_frequencies(desc)
    ref = Q.frequencies(r, original=8192, **kw)
    assert float(((freqs.cpu() - ref) / ref).abs().max()) < 2.0 ** -45
    pos = torch.randint(-5, 1000000, (rows,), generator=g)
    pos[0] = 0
    # q in rows that are part of wider ones, k in place, both in a buffer whose other elements stay
    wide = (h + kv) * dh + 16
    buf = torch.randn(rows, wide, generator=g).to(dtype).cuda()
    before = buf.clone()
    q, k = buf[:, :h * dh].unflatten(1, (h, dh)), buf[:, h * dh:(h + kv) * dh].unflatten(1, (kv, dh))
    q_out = torch.full((rows, h, dh), float("nan"), dtype=dtype, device="cuda")
    B.ee_rotary(desc, freqs, i32(pos), q, q_out, k, k, transpose=transpose)
    torch.cuda.synchronize()
    for x, y in ((before[:, :h * dh].unflatten(1, (h, dh)), q_out), (before[:, h * dh:(h + kv) * dh].unflatten(1, (kv, dh)), k)):
        x = x.cpu().double()
        want = Q.rotary(x, pos, ref, layout, amplitude, transpose)
        err = (y.cpu().double() - want).abs()
        assert bool((err <= rotary_tolerance(x, want, layout, r, amplitude, dtype)).all()), float(err.max())
        assert torch.equal(y[..., r:].cpu().double(), x[..., r:])
    assert torch.equal(buf[:, :h * dh], before[:, :h * dh]) and torch.equal(buf[:, (h + kv) * dh:], before[:, (h + kv) * dh:])


def test_rotary_of_a_fused_buffer_in_place():
    """q and k lie between each other's rows, both in place: the same results as apart, and V's rows stay."""
    dh, h, kv, rows = 64, 6, 2, 9
    desc = B.make_rotary_desc(dh)
    freqs = B.ee_rotary_frequencies(desc)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 7
    buf = torch.randn(rows, (h + 2 * kv) * dh, generator=gen(5)).cuda()
    before = buf.clone()

    def parts(x):
        return x[:, :h * dh].unflatten(1, (h, dh)), x[:, h * dh:(h + kv) * dh].unflatten(1, (kv, dh))
    q, k = parts(buf)
    q0, k0 = parts(before)
    q_out, k_out = torch.empty(rows, h, dh, device="cuda"), torch.empty(rows, kv, dh, device="cuda")
    B.ee_rotary(desc, freqs, pos, q0.contiguous(), q_out, k0.contiguous(), k_out)
    B.ee_rotary(desc, freqs, pos, q, q, k, k)
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(buf[:, (h + kv) * dh:], before[:, (h + kv) * dh:])


def test_rotary_addresses_off_sixteen_bytes():
    """The same results from an address that allows no wide loads."""
    desc = B.make_rotary_desc(64)
    freqs = B.ee_rotary_frequencies(desc)
    pos = torch.arange(5, dtype=torch.int32, device="cuda") * 100
    flat = torch.randn(5 * 3 * 64 + 1, device="cuda")
    x = flat[1:].view(5, 3, 64)
    a, b = torch.empty(5, 3, 64, device="cuda"), torch.empty(5, 3, 64, device="cuda")
    B.ee_rotary(desc, freqs, pos, x, a)
    B.ee_rotary(desc, freqs, pos, x.clone(), b)
    assert torch.equal(a, b)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient(layout):
    """The transposed rotation against differences of the rotation: it is linear, so differences are as exact as its floats."""
    desc = B.make_rotary_desc(16, 12, layout=layout, amplitude=1.5)
    freqs = B.ee_rotary_frequencies(desc)
    pos = torch.tensor([0, 3, 70000], dtype=torch.int32, device="cuda")
    g = gen(1)
    w = torch.randn(3, 2, 16, generator=g).cuda()                # the gradient of sum(w * out)
    grad = torch.empty_like(w)
    B.ee_rotary(desc, freqs, pos, w, grad, transpose=True)
    for m in range(3):
        for h in range(2):
            for c in range(16):
                x = torch.zeros(3, 2, 16, device="cuda")
                x[m, h, c] = 1.0
                y = torch.empty_like(x)
                B.ee_rotary(desc, freqs, pos, x, y)
                # each pair's two products, 2^-20 as above
                assert abs(float((w.double() * y.double()).sum()) - float(grad[m, h, c])) < 2.0 ** -18 * 1.5 * float(w.abs().max())


# ---- append and read ----------------------------------------------------------------------------------------------
def run_append(fmt, dtype, heads, dh, starts, rows, seed, magnitudes=None, rounds=1):
    """`rounds` appends of rows[i] positions to sequence i from starts[i] on; every byte of the pool against the oracle."""
    g = gen(seed)
    lens = [s + r * rounds for s, r in zip(starts, rows)]
    tables, nb = tables_for(lens, seed)
    kv = filled(2, nb, heads, dh, fmt, seed)
    ref, untouched = Q.Cache.of(kv, 1), Q.Cache.of(kv, 0)
    for step in range(rounds):
        row_table = [i for i, n in enumerate(rows) for _ in range(n)]
        pos = [starts[i] + step * n + j for i, n in enumerate(rows) for j in range(n)]
        wide = heads * dh + 2
        new = [torch.randn(len(pos), wide, generator=g) for _ in range(2)]
        if magnitudes:
            for x in new:
                x *= torch.tensor([magnitudes[(p + step) % len(magnitudes)] for p in pos])[:, None]
        new = [x.to(dtype).cuda()[:, :heads * dh].unflatten(1, (heads, dh)) for x in new]
        batch = B.make_batch(None, i32(pos), i32(tables), max(lens), i32(row_table))
        B.ee_kv_quant_append(kv, 2, new[0], new[1], batch)
        Q.append(ref, new[0].cpu().double(), new[1].cpu().double(), pos, tables, row_table)
    torch.cuda.synchronize()
    assert_cache(kv, ref, 1)
    assert_cache(kv, untouched, 0)
    return kv, ref, tables, lens


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,dh", [(1, 16), (3, 64), (2, 80), (5, 128), (2, 192), (1, 256)])
def test_append_chunks(fmt, dtype, heads, dh):
    run_append(fmt, dtype, heads, dh, starts=[0, 5, 16, 31, 100], rows=[33, 7, 16, 2, 1], seed=heads * dh)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_rows_of_many_sequences(fmt):
    """Single rows and short runs of 21 sequences next to each other, runs that end where another sequence's begins."""
    run_append(fmt, torch.bfloat16, 3, 64, starts=[(7 * i) % 40 for i in range(21)], rows=[1, 1, 1, 2, 1, 5, 1] * 3, seed=21)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_one_by_one(fmt):
    """40 positions, one a call, magnitudes going up and down: blocks whose scale grows again and again."""
    run_append(fmt, torch.float32, 2, 128, starts=[0, 13], rows=[1, 1], seed=5, rounds=40,
               magnitudes=[1.0, 1.7, 0.1, 2.9, 3.0, 10.0, 0.0, 50.0, 4.0, 1e-3, 700.0])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", [0.0, 1e-42, 1e-37, 1e-30, 1e30, 3e38])
def test_append_extreme_magnitudes(fmt, size):
    """Zeros, subnormal floats, and numbers whose products with 127 or 448 are no floats."""
    g = gen(3)
    tables, nb = tables_for([20], 3)
    kv = filled(1, nb, 2, 64, fmt, 3)
    ref = Q.Cache.of(kv)
    x = ((torch.rand(20, 2, 64, generator=g) * 2 - 1) * size).cuda()
    B.ee_kv_quant_append(kv, 1, x, x, B.make_batch(None, i32(range(20)), i32(tables), 20, i32([0] * 20)))
    Q.append(ref, x.cpu().double(), x.cpu().double(), list(range(20)), tables, [0] * 20)
    assert_cache(kv, ref)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_ties(fmt):
    """Quotients that lie exactly between two bytes go to the even one."""
    kv = B.QuantKV(1, 1, 1, 64, fmt)
    x = torch.zeros(1, 1, 64)
    top = 127.0 if fmt == "int8" else 448.0                      # scale 1
    x[0, 0, 0] = top
    half = torch.arange(1, 32).float() + 0.5 if fmt == "int8" else torch.tensor([17.0, 19.0, 21.0, 23.0, 25.0, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10])
    x[0, 0, 1:1 + len(half)] = half
    x[0, 0, 32:32 + len(half)] = -half
    ref = Q.Cache.of(kv)
    t = torch.zeros(1, 1, dtype=torch.int32)
    B.ee_kv_quant_append(kv, 1, x.cuda(), x.cuda(), B.make_batch(None, i32([0]), i32(t), 1))
    Q.append(ref, x.double(), x.double(), [0], t)
    assert float(ref.scales[0, 0, 0]) == 1.0
    assert_cache(kv, ref)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_skips_and_drops(fmt):
    """Padding rows, positions behind the table, blocks that are none: nothing is written for them."""
    kv = filled(1, 6, 2, 64, fmt, 9)
    tables = torch.tensor([[0, 1], [2, -1], [6, 3], [4, 5]], dtype=torch.int32)
    lens = [3, 20, 2, -1, 40, -7]
    rt = [0, 1, 2, 3, 3, 0]
    ref = Q.Cache.of(kv)
    x = torch.randn(6, 2, 64, generator=gen(2)).cuda()
    B.ee_kv_quant_append(kv, 1, x, -x, B.make_batch(None, i32(lens), i32(tables), 32, i32(rt)))
    Q.append(ref, x.cpu().double(), -x.cpu().double(), lens, tables, rt)
    assert_cache(kv, ref)
    B.ee_kv_quant_append(kv, 1, x[:0], x[:0], B.make_batch(None, i32(lens)[:0], i32(tables), 32))
    assert_cache(kv, ref)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_append_not_a_number(fmt, bad):
    """The block's scale is NaN from then on, its neighbours' are not, and the block's next first position starts anew."""
    tables = torch.tensor([[1, 0]], dtype=torch.int32)
    kv = filled(1, 2, 2, 64, fmt, 4)
    ref = Q.Cache.of(kv)
    g = gen(6)
    for pos in (0, 1, 2, 3, 16, 0):
        x = torch.randn(1, 2, 64, generator=g)
        if pos == 2:
            x[0, 1, 5] = bad
        B.ee_kv_quant_append(kv, 1, x.cuda(), x.cuda(), B.make_batch(None, i32([pos]), i32(tables), 32))
        Q.append(ref, x.double(), x.double(), [pos], tables)
        assert_cache(kv, ref)
        nan = kv.scales[0, 1, 1].isnan().all().item()
        assert nan == (pos in (2, 3, 16)) and not kv.scales[0, 1, 0].isnan().any()
    assert not kv.scales.isnan().any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,dh", [(1, 16), (3, 80), (2, 128), (2, 256)])
def test_read(fmt, dtype, heads, dh):
    """Runs, single positions, positions twice, descending ones, padding rows."""
    lens = [50, 17]
    tables, nb = tables_for(lens, 1)
    kv = filled(2, nb, heads, dh, fmt, dh)
    rows = [(0, p) for p in range(3, 40)] + [(1, 16), (1, 16), (0, 49), (0, 48), (1, 0), (0, -1), (1, 1), (1, 2), (0, 3)]
    k = torch.full((len(rows), heads, dh), float("nan"), dtype=dtype, device="cuda")
    v = k.clone()
    B.ee_kv_quant_read(kv, 2, B.make_batch(None, i32([p for _, p in rows]), i32(tables), 50, i32([s for s, _ in rows])), k, v)
    ref = Q.Cache.of(kv, 1)
    for m, (s, p) in enumerate(rows):
        for h in range(heads):
            for which, out in ((0, k), (1, v)):
                want = torch.zeros(dh, dtype=F64) if p < 0 else ref.value(which, int(tables[s, p // 16]), h, p % 16)
                assert torch.equal(out[m, h].cpu().double(), want.float().to(dtype).double()), (m, h, which)


# ---- attention ----------------------------------------------------------------------------------------------------
def attend(kv, layer, q, lens, tables, row_table=None, weights=None, w_in=None, max_context=None):
    ctx = max_context or max(1, max(lens) + 1)
    out = torch.full_like(q, float("nan"))
    ws = B.QuantWorkspace(kv, q.shape[1], len(lens), ctx, weights is not None)
    ws.buf.fill_(0xFF)
    B.ee_paged_attention_quant(kv, layer, q, B.make_batch(None, i32(lens), i32(tables), ctx, i32(row_table) if row_table is not None else None),
                               out, ws, w_in, weights)
    torch.cuda.synchronize()
    return out


def check_attention(fmt, dh, heads, group, lens, seed=0, width=0, row_table=None, sequences=None, q_scale=1.0, max_context=None):
    owned = sequences or [n + 1 for n in lens]
    tables, nb = tables_for(owned, seed, width=width)
    kv = filled(2, nb, heads, dh, fmt, seed)
    poison(kv, tables, owned, 1)
    q = torch.randn(len(lens), heads * group, dh, generator=gen(seed + 1)) * q_scale
    out = attend(kv, 2, q.cuda(), lens, tables, row_table, max_context=max_context)
    want, _, bound = Q.attention(Q.Cache.of(kv, 1), q.double(), lens, tables, row_table)
    err = (out.cpu().double() - want).abs()
    assert bool((err <= bound).all()), (float((err / bound).max()), float(err.max()))
    return kv, tables, q, out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh", [16, 48, 64, 80, 128, 176, 192, 240, 256])
def test_attention_head_dims(fmt, dh):
    check_attention(fmt, dh, heads=2, group=3, lens=[0, 70, 200], seed=dh)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,group", [(1, 1), (4, 2), (2, 7), (2, 16), (1, 17), (1, 40)])
def test_attention_groups(fmt, heads, group):
    check_attention(fmt, 64, heads, group, lens=[33, 5, 130], seed=group)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_lengths(fmt):
    """Block, step and part borders, a padded row, an empty batch."""
    check_attention(fmt, 128, 2, 4, lens=[0, 1, 14, 15, 16, 17, 62, 63, 64, 65, 255, 256, 257, -1, 511, 700], width=60)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [4000, 20011])
def test_attention_of_a_split_context(fmt, n):
    check_attention(fmt, 128, 2, 4, lens=[n], seed=n)
    check_attention(fmt, 64, 1, 1, lens=[n // 3, 12, n], seed=n + 1)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,group,rows", [(2, 2, 40), (1, 20, 9), (4, 1, 70), (16, 1, 5)])
def test_attention_of_a_ragged_batch(fmt, heads, group, rows):
    """Rows whose steps are dealt out: workgroups with pieces of several rows, rows with pieces in several workgroups, empty rows at the ends and
    between, rows of one position."""
    lens = torch.randint(0, 1500, (rows,), generator=gen(rows)).tolist()
    lens[0], lens[3], lens[4], lens[-1], lens[1] = -1, -1, 0, -1, 2000
    check_attention(fmt, 64, heads, group, lens, seed=rows, width=130)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,heads,group,rows,most", [(64, 32, 1, 36, 300), (128, 16, 2, 70, 130), (80, 64, 1, 17, 700), (32, 16, 17, 33, 70), (64, 33, 1, 33, 90)])
def test_attention_of_many_heads(fmt, dh, heads, group, rows, most):
    """Enough (row, K/V head) units that two share a workgroup (not with an odd number of heads), with and without weights."""
    lens = torch.randint(-1, most, (rows,), generator=gen(rows)).tolist()
    kv, tables, q, out = check_attention(fmt, dh, heads, group, lens, seed=rows, width=(most + 15) // 16, max_context=most)
    w = torch.full((rows, heads, most), 2.0, device="cuda")
    again = attend(kv, 2, q.cuda(), lens, tables, weights=w, max_context=most)
    assert torch.equal(again, out)
    _, probs, _ = Q.attention(Q.Cache.of(kv, 1), q.double(), lens, tables)
    for m, n in enumerate(lens):
        want = probs[m][0].view(heads, group, -1).sum(1)
        # each probability by its head's slack, the sum of the heads 2^-24 a term
        tol = (probs[m][0] * probs[m][1][:, None]).view(heads, group, -1).sum(1) + want * (group + 2) * 2.0 ** -24 + 1e-37
        assert bool(((w[m, :, :n + 1].cpu().double() - want).abs() <= tol).all()) and bool((w[m, :, n + 1:] == 2.0).all())


@pytest.mark.parametrize("shared", [False, True])
def test_attention_of_no_positions_at_all(shared):
    tables, nb = tables_for([2000, 2000], 1)
    kv = filled(1, nb, 2, 64, "int8", 1)
    q = torch.randn(2, 4, 64, generator=gen(1)).cuda()
    w = torch.full((2, 2, 2000), 3.0, device="cuda")
    out = attend(kv, 1, q, [-1, -1], tables, [0, 1] if shared else None, weights=None if shared else w, max_context=2000)
    assert torch.equal(out, torch.zeros_like(out)) and bool((w == 3.0).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shared", [False, True])
def test_attention_of_more_blocks_than_a_table_holds(fmt, shared):
    """Many heads, so that a workgroup walks a context of 18000 positions alone."""
    n, heads = 18000, 512
    tables, nb = tables_for([n], 2)
    kv = filled(1, nb, heads, 16, fmt, 2)
    q = torch.randn(1, heads, 16, generator=gen(3))
    out = attend(kv, 1, q.cuda(), [n - 1], tables, [0] if shared else None)
    few = [0, 1, 255, 256, 511]
    kv_few = Q.Cache.of(kv)
    part = Q.Cache(kv_few.k[:, few], kv_few.v[:, few], kv_few.scales[:, few], fmt)
    want, _, bound = Q.attention(part, q[:, few].double(), [n - 1], tables)
    assert bool(((out[:, few].cpu().double() - want).abs() <= bound).all())


def test_attention_replays_with_other_lengths():
    """One captured call, replayed as contexts grow: the work is divided by the lengths on the device."""
    heads, group, dh, room = 2, 2, 64, 2100
    tables, nb = tables_for([room, room, room], 5)
    kv = filled(1, nb, heads, dh, "int8", 5)
    q = torch.randn(3, heads * group, dh, generator=gen(6))
    qd, lens, tb = q.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"), i32(tables)
    out, weights = torch.empty_like(qd), torch.zeros(3, heads, room, device="cuda")
    batch, ws = B.make_batch(None, lens, tb, room), B.QuantWorkspace(kv, heads * group, 3, room, True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.ee_paged_attention_quant(kv, 1, qd, batch, out, ws, None, weights)
    for now in ([0, -1, 2000], [2099, 2098, 1024], [5, 1023, 64], [-1, -1, -1]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        w2 = torch.zeros_like(weights)
        eager = attend(kv, 1, qd, now, tables, weights=w2, max_context=room)
        assert torch.equal(out, eager)
        for m, n in enumerate(now):
            assert torch.equal(weights[m, :, :n + 1], w2[m, :, :n + 1])


def test_calls_on_two_streams():
    """Two chains of calls at once, each with buffers and a workspace of its own, give what they give alone."""
    chains = []
    for seed in (1, 2):
        lens = [1700, 40, 900]
        tables, nb = tables_for([n + 1 for n in lens], seed)
        kv = filled(1, nb, 2, 64, "e4m3", seed)
        q = torch.randn(3, 8, 64, generator=gen(seed)).cuda()
        out, w = torch.empty_like(q), torch.zeros(3, 2, 1701, device="cuda")
        batch, ws = B.make_batch(None, i32(lens), i32(tables), 1701), B.QuantWorkspace(kv, 8, 3, 1701, True)
        chains.append((kv, q, batch, out, ws, w))
    alone = []
    for kv, q, batch, out, ws, w in chains:
        B.ee_paged_attention_quant(kv, 1, q, batch, out, ws, None, w)
        torch.cuda.synchronize()
        alone.append((out.clone(), w.clone()))
    streams = [torch.cuda.Stream() for _ in chains]
    for _ in range(5):
        for (kv, q, batch, out, ws, w), st in zip(chains, streams):
            with torch.cuda.stream(st):
                B.ee_paged_attention_quant(kv, 1, q, batch, out, ws, None, w)
    torch.cuda.synchronize()
    for (_, _, _, out, _, w), (o, x) in zip(chains, alone):
        assert torch.equal(out, o) and torch.equal(w, x)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_scale", [0.0, 1e-20, 30.0, 1e4])
def test_attention_extreme_queries(fmt, q_scale):
    check_attention(fmt, 64, 2, 2, lens=[100, 300], q_scale=q_scale)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,heads,group", [(64, 2, 1), (128, 2, 4), (80, 1, 3), (256, 1, 8), (192, 1, 1)])
def test_attention_prompt_rows(fmt, dh, heads, group):
    """Chunks of several prompts, single rows among them, padding rows, a tile that holds the ends of several sequences."""
    spans = [(0, 37), (100, 20), (64, 1), (15, 2), (250, 70), (3, 3)]
    lens = [a + j for a, n in spans for j in range(n)] + [-1, -1]
    rt = [i for i, (_, n) in enumerate(spans) for _ in range(n)] + [0, 5]
    check_attention(fmt, dh, heads, group, lens, seed=dh, row_table=rt, sequences=[a + n for a, n in spans])


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_rows_in_any_order(fmt):
    lens = [5, 90, 3, 40, 6, 89, 200, 7]
    check_attention(fmt, 128, 2, 2, lens, row_table=[0, 1, 0, 2, 0, 1, 2, 0], sequences=[10, 100, 210])


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_long_prompt(fmt):
    """A few rows behind a long context: parts of the context are joined for prompt rows as well."""
    lens = [6000 + j for j in range(9)]
    check_attention(fmt, 64, 1, 2, lens, row_table=[0] * 9, sequences=[6009])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shared", [False, True])
def test_attention_not_a_number_stays_in_its_sequence(fmt, shared):
    owned = [200, 90, 130]
    tables, nb = tables_for(owned, 3)
    kv = filled(1, nb, 2, 64, fmt, 3)
    lens = [199, 198, 89, 88, 129] if shared else [199, 89, 129]
    rt = [0, 0, 1, 1, 2] if shared else None
    mine = rt or [0, 1, 2]
    q = torch.randn(len(lens), 4, 64, generator=gen(8)).cuda()
    good = attend(kv, 1, q, lens, tables, rt)
    for which in (0, 1):
        saved = kv.scales.clone()
        kv.scales[0, int(tables[1, 2]), :, which] = float("nan")
        out = attend(kv, 1, q, lens, tables, rt)
        kv.scales.copy_(saved)
        for m, s in enumerate(mine):
            if s == 1:
                assert out[m].isnan().all()
            else:
                assert torch.equal(out[m], good[m])
    q[0, 1] = float("inf")
    out = attend(kv, 1, q, lens, tables, rt)
    assert out[0, 1].isnan().all() and torch.equal(out[0, 0], good[0, 0]) and torch.equal(out[1:], good[1:])


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_bad_blocks_reach_nothing(fmt):
    """Block ids outside the pool and positions behind the table: the rows' own results are unspecified, the others' are not."""
    owned = [60, 60, 60]
    tables, nb = tables_for(owned, 4)
    kv = filled(1, nb, 2, 128, fmt, 4)
    q = torch.randn(3, 4, 128, generator=gen(9)).cuda()
    good = attend(kv, 1, q, [59, 59, 59], tables)
    bad = tables.clone()
    bad[1, 1], bad[1, 2] = -5, 1 << 30
    out = attend(kv, 1, q, [59, 59, 59], bad)
    assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
    out = attend(kv, 1, q, [59, 5000, 59], tables, max_context=64)
    assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,group,lens", [(2, 4, [0, 1, 63, 64, 500, -1]), (1, 20, [100, 3]), (2, 1, [5000]), (3, 2, [1500, 40]),
                                              (1, 18, [1400, -1, 3]), (2, 5, [1100, 64, 0, 1300])])
@pytest.mark.parametrize("where", ["apart", "in place", "from nothing"])
def test_attention_weights(fmt, heads, group, lens, where):
    tables, nb = tables_for([n + 1 for n in lens], 7)
    kv = filled(1, nb, heads, 64, fmt, 7)
    poison(kv, tables, [n + 1 for n in lens])
    q = torch.randn(len(lens), heads * group, 64, generator=gen(2))
    pitch = max(lens) + 4
    w_in = torch.rand(len(lens), heads, pitch, generator=gen(3)).cuda()
    before = w_in.clone()
    w_out = w_in if where == "in place" else torch.full_like(w_in, 7.0)
    left = w_out.clone()
    out = attend(kv, 1, q.cuda(), lens, tables, weights=w_out, w_in=None if where == "from nothing" else w_in)
    want, probs, bound = Q.attention(Q.Cache.of(kv), q.double(), lens, tables)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())
    for m, n in enumerate(lens):
        assert torch.equal(w_out[m, :, n + 1:], left[m, :, n + 1:])
        for h in range(heads if n >= 0 else 0):
            p, slack = probs[m][0][h * group:(h + 1) * group], probs[m][1][h * group:(h + 1) * group]
            base = before[m, h, :n + 1].cpu().double() if where != "from nothing" else torch.zeros(n + 1, dtype=F64)
            base[n] = 0.0
            total = base + p.sum(0)
            tol = (p * slack[:, None]).sum(0) + total * (group + 2) * 2.0 ** -24 + 1e-37
            assert bool(((w_out[m, h, :n + 1].cpu().double() - total).abs() <= tol).all()), (m, h)


def test_attention_of_the_last_blocks_of_a_large_pool():
    """Blocks beyond 4 GiB from the pool's start."""
    heads, dh = 8, 256
    nb = (5 << 30) // (heads * 16 * dh)
    kv = B.QuantKV(1, nb, heads, dh, "int8")
    lens = [20, 40]
    tables = torch.tensor([[nb - 1, 0, -1], [nb - 2, nb - 4, nb - 3]], dtype=torch.int32)
    x = torch.randn(62, heads, dh, generator=gen(1)).cuda()
    pos, rt = list(range(21)) + list(range(41)), [0] * 21 + [1] * 41
    B.ee_kv_quant_append(kv, 1, x, -x, B.make_batch(None, i32(pos), i32(tables), 48, i32(rt)))
    q = torch.randn(2, heads, dh, generator=gen(2))
    out = attend(kv, 1, q.cuda(), lens, tables)
    k, v = torch.empty_like(x), torch.empty_like(x)
    B.ee_kv_quant_read(kv, 1, B.make_batch(None, i32(pos), i32(tables), 48, i32(rt)), k, v)
    # half a step of a block's scale each way
    assert float((k - x).abs().max()) <= float(x.abs().max()) / 127 * 0.51 and torch.equal(v, -k)
    for m, rows in ((0, slice(0, 21)), (1, slice(21, 62))):
        z = torch.einsum("hd,nhd->hn", q[m].double(), k[rows].cpu().double()) / math.sqrt(dh)
        want = torch.einsum("hn,nhd->hd", torch.softmax(z, -1), v[rows].cpu().double())
        assert float((out[m].cpu().double() - want).abs().max()) < 1e-5 * float(v.abs().max())   # (a slip reads other blocks: order 1)


# ---- eviction -----------------------------------------------------------------------------------------------------
def run_evict(fmt, heads, dh, lens, keep, recent, seed, weights=None, apart=False, w_where="apart", extra=0):
    tables, nb = tables_for(lens, seed, spare=2 + (sum((min(n, keep) + 15) // 16 for n in lens) if apart else 0))
    kv = filled(2, nb, heads, dh, fmt, seed)
    pitch = max(max(lens), keep) + extra
    w = torch.rand(len(lens), heads, pitch, generator=gen(seed + 1)) if weights is None else weights
    dst = None
    if apart:
        free = [i for i in range(nb) if i not in set(tables.flatten().tolist())]
        dst = torch.full((len(lens), (keep + 15) // 16), -1, dtype=torch.int32)
        for b, n in enumerate(lens):
            for s in range((min(n, keep) + 15) // 16):
                dst[b, s] = free.pop()
    ref, other = Q.Cache.of(kv, 1), Q.Cache.of(kv, 0)
    kept_ref, lens_ref = Q.evict(ref, lens, tables, w, keep, recent, dst)
    wd = w.cuda()
    w_out = {"apart": torch.full((len(lens), heads, keep), 9.0, device="cuda"), "in place": wd, "none": None}[w_where]
    kept = torch.full((len(lens), heads, keep), 77, dtype=torch.int32, device="cuda")
    out_lens = torch.full((len(lens),), 77, dtype=torch.int32, device="cuda")
    ws = None if apart else B.QuantWorkspace(kv, 0, len(lens), keep, evicting=True)
    batch = B.make_batch(None, i32(lens), i32(tables), max(1, max(lens)))
    B.ee_kv_quant_evict(kv, 2, batch, wd, w_out, keep, recent, kept, out_lens, ws, i32(dst) if dst is not None else None)
    torch.cuda.synchronize()
    assert out_lens.tolist() == lens_ref
    for b in range(len(lens)):
        for h in range(heads):
            ids = kept_ref[b][h]
            assert kept[b, h].tolist() == ids + [-1] * (keep - len(ids)), (b, h)
            if w_out is not None:
                assert same(w_out[b, h, :len(ids)].cpu(), w[b, h, ids])
                rest = w[b, h, len(ids):] if w_where == "in place" else torch.full((keep - len(ids),), 9.0)
                assert same(w_out[b, h, len(ids):].cpu(), rest)
    # what holds a position, and every block that no sequence was moved to
    got, where = Q.Cache.of(kv, 1), tables if dst is None else dst
    moved = set()
    for b, n in enumerate(lens_ref):
        for p in range(n):
            blk = int(where[b, p // 16])
            moved.add(blk)
            for h in range(heads):
                for which in (0, 1):
                    assert same(got.value(which, blk, h, p % 16), ref.value(which, blk, h, p % 16)), (b, p, h, which)
    rest = [i for i in range(nb) if i not in moved]
    for x, y in ((got.k, ref.k), (got.v, ref.v), (got.scales, ref.scales)):
        assert torch.equal(x[rest], y[rest])
    assert_cache(kv, other, 0)
    return kv, kept


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("heads,dh,lens,keep,recent", [
    (2, 64, [40, 100, 17], 33, 5), (1, 128, [300, 256, 255, 0, 1], 256, 0), (3, 80, [50], 50, 10), (2, 16, [90, 20], 16, 16),
    (1, 192, [70], 1, 0), (1, 256, [40, 33], 31, 30), (1, 64, [2500, 1025], 1030, 100)])
def test_evict(fmt, apart, heads, dh, lens, keep, recent):
    run_evict(fmt, heads, dh, lens, keep, recent, seed=keep, apart=apart, extra=3)


@pytest.mark.parametrize("w_where", ["in place", "none"])
def test_evict_weights_in_place(w_where):
    run_evict("int8", 2, 64, [1300, 60, 2100], 900, 40, seed=3, w_where=w_where)


@pytest.mark.parametrize("kind", ["equal", "few", "signs", "not numbers", "recent only"])
def test_evict_order(kind):
    """Ties go to the lowest position, -0 is 0, NaN is the largest, infinities are numbers like others."""
    n, g = 200, gen(11)
    w = torch.rand(1, 2, n, generator=g)
    if kind == "equal":
        w[:] = 0.25
    if kind == "few":
        w = torch.randint(0, 3, (1, 2, n), generator=g).float()
    if kind == "signs":
        w = torch.randint(-2, 3, (1, 2, n), generator=g).float() * torch.where(torch.rand(1, 2, n, generator=g) < 0.5, -1.0, 1.0)
    if kind == "not numbers":
        w[0, 0, 30:40] = float("nan")
        w[0, 0, 50:60] = -float("nan")
        w[0, 1, 70:90] = float("inf")
        w[0, 1, 90:120] = -float("inf")
        w[0, 1, 120:130] = 1e-45
    run_evict("e4m3", 2, 64, [n], 70, 70 if kind == "recent only" else 15, seed=5, weights=w)


@pytest.mark.parametrize("w_where", ["in place", "apart"])
def test_evict_a_long_context(w_where):
    """More positions than keys are held at once, with ties on both sides of that border."""
    w = torch.randint(0, 4, (1, 1, 30000), generator=gen(4)).float()
    run_evict("int8", 1, 16, [30000], 20000, 100, seed=1, weights=w, w_where=w_where)


@pytest.mark.parametrize("fmt", FORMATS)
def test_evict_what_append_wrote_stays_as_it_is(fmt):
    """Nothing to evict into other blocks: what append wrote comes out with the same values."""
    kv, ref, tables, lens = run_append(fmt, torch.float32, 2, 64, [0, 0], [100, 47], seed=8)
    w = torch.rand(2, 2, 100, device="cuda")
    extra = filled(2, 2 * kv.num_blocks, 2, 64, fmt, 1)
    extra.k.view(torch.int8)[:, :kv.num_blocks] = kv.k.view(torch.int8)
    extra.v.view(torch.int8)[:, :kv.num_blocks] = kv.v.view(torch.int8)
    extra.scales[:, :kv.num_blocks] = kv.scales
    dst = torch.arange(14, dtype=torch.int32).view(2, 7) + kv.num_blocks
    kept, out = torch.zeros(2, 2, 100, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    B.ee_kv_quant_evict(extra, 2, B.make_batch(None, i32(lens), i32(tables), 100), w, None, 100, 0, kept, out, None, i32(dst))
    got = Q.Cache.of(extra, 1)
    for b, n in enumerate(lens):
        for h in range(2):
            for which in (0, 1):
                assert torch.equal(got.gather(which, dst[b], h, n), ref.gather(which, tables[b], h, n))


@pytest.mark.parametrize("fmt", FORMATS)
def test_evict_a_block_that_is_not_a_number(fmt):
    """Positions of a NaN block make the blocks they move to NaN, no others."""
    lens = [64]
    tables, nb = tables_for(lens, 2)
    kv = filled(1, nb, 1, 64, fmt, 2)
    kv.scales[0, int(tables[0, 2]), 0, 0] = float("nan")
    w = torch.ones(1, 1, 64)
    w[0, 0, :20] = 0.0
    kept, out = torch.zeros(1, 1, 44, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ee_kv_quant_evict(kv, 1, B.make_batch(None, i32(lens), i32(tables), 64), w.cuda(), None, 44, 0, kept, out,
                        B.QuantWorkspace(kv, 0, 1, 44, evicting=True))
    nan = [kv.scales[0, int(tables[0, s]), 0, 0].isnan().item() for s in range(3)]
    assert nan == [True, True, False]          # positions 20..35, 36..51, 52..63; the bad block held 32..47
    assert not kv.scales[0, :, :, 1].isnan().any()


# ---- together -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("captured", [False, True])
def test_a_run_of_them_together(fmt, captured):
    """A prompt chunk, then decode steps with rotary positions, append and attention that sums its weights, and an eviction whenever a
    sequence reaches its budget: every step against the oracle on the same cache.  Captured: each step is a graph that is
    recorded once and replayed, with the library's eager calls between replays."""
    heads, group, dh, n_seq, budget, keep = 2, 3, 64, 2, 48, 32
    g = gen(4)
    kv = filled(1, 12, heads, dh, fmt, 4)
    tables = torch.randperm(12, generator=g).to(torch.int32)[:8].view(2, 4)
    desc = B.make_rotary_desc(dh, 48, scaling="linear", factor=2.0)
    freqs, fr = B.ee_rotary_frequencies(desc), Q.frequencies(48, scaling="linear", factor=2.0)
    ref = Q.Cache.of(kv)
    chunk = [20, 31]
    rt = [i for i, n in enumerate(chunk) for _ in range(n)]
    pos = [p for n in chunk for p in range(n)]
    x = torch.randn(2, len(pos), heads, dh, generator=g).cuda()
    B.ee_kv_quant_append(kv, 1, x[0], x[1], B.make_batch(None, i32(pos), i32(tables), budget, i32(rt)))
    Q.append(ref, x[0].cpu().double(), x[1].cpu().double(), pos, tables, rt)
    assert_cache(kv, ref)
    # the step's buffers
    tb, slot, place = i32(tables), i32(chunk), i32(chunk)
    q, k, v = (torch.zeros(n_seq, n, dh, device="cuda") for n in (heads * group, heads, heads))
    qr, kr, out = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(q)
    weights = torch.zeros(n_seq, heads, budget, device="cuda")
    w_ref = torch.zeros(n_seq, heads, budget, dtype=F64)
    batch = B.make_batch(None, slot, tb, budget)
    ws = B.QuantWorkspace(kv, heads * group, n_seq, budget, True)
    ws_e = B.QuantWorkspace(kv, 0, n_seq, keep, evicting=True)
    kept, lens_out = torch.zeros(n_seq, heads, keep, dtype=torch.int32, device="cuda"), torch.zeros(n_seq, dtype=torch.int32, device="cuda")

    def step():
        B.ee_rotary(desc, freqs, place, q, qr, k, kr)
        B.ee_kv_quant_append(kv, 1, kr, v, batch)
        B.ee_paged_attention_quant(kv, 1, qr, batch, out, ws, weights, weights)

    side, graph = torch.cuda.Stream(), None
    slots, places = list(chunk), list(chunk)
    for t in range(40):
        new = [torch.randn(y.shape, generator=g) for y in (q, k, v)]
        for y, z in zip((q, k, v), new):
            y.copy_(z)
        slot.copy_(torch.tensor(slots, dtype=torch.int32))
        place.copy_(torch.tensor(places, dtype=torch.int32))
        if not captured:
            with torch.cuda.stream(side):
                side.wait_stream(torch.cuda.default_stream())
                step()
            torch.cuda.default_stream().wait_stream(side)
        else:
            if graph is None:
                torch.cuda.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step()
            graph.replay()
        torch.cuda.synchronize()
        # append is exact from the keys the rotation left; attention from the cache that append left
        kd, qd = kr.cpu().double(), qr.cpu().double()
        for got, src in ((kd, new[1]), (qd, new[0])):
            want = Q.rotary(src.double(), torch.tensor(places), fr, "half")
            assert bool(((got - want).abs() <= rotary_tolerance(src.double(), want, "half", 48, 1.0, torch.float32)).all())
        Q.append(ref, kd, new[2].double(), slots, tables)
        assert_cache(kv, ref)
        want, probs, bound = Q.attention(ref, qd, slots, tables)
        assert bool(((out.cpu().double() - want).abs() <= bound).all()), t
        for b in range(n_seq):
            for h in range(heads):
                p = probs[b][0][h * group:(h + 1) * group].sum(0)
                w_ref[b, h, :slots[b]] += p[:-1]
                w_ref[b, h, slots[b]] = p[-1]
                err = (weights[b, h, :slots[b] + 1].cpu().double() - w_ref[b, h, :slots[b] + 1]).abs()
                # every step adds its own slack, 2^-14 at most here
                assert bool((err <= (t + 1) * 2.0 ** -14 * (1e-3 + w_ref[b, h, :slots[b] + 1])).all())
        slots, places = [n + 1 for n in slots], [n + 1 for n in places]
        if max(slots) == budget:
            w_now = weights.cpu()
            slot.copy_(torch.tensor(slots, dtype=torch.int32))
            B.ee_kv_quant_evict(kv, 1, B.make_batch(None, slot, tb, budget), weights, weights, keep, 8, kept, lens_out, ws_e)
            ids, slots = Q.evict(ref, slots, tables, w_now, keep, 8)
            assert lens_out.tolist() == slots and max(slots) <= keep
            for b in range(n_seq):
                for h in range(heads):
                    assert kept[b, h].tolist() == ids[b][h] + [-1] * (keep - len(ids[b][h]))
                    w_ref[b, h, :len(ids[b][h])] = w_ref[b, h, ids[b][h]].clone()
            # (E4M3: a rebuilt block may hold the same values under half the scale)
            got = Q.Cache.of(kv)
            for b in range(n_seq):
                for h in range(heads):
                    for which in (0, 1):
                        assert torch.equal(got.gather(which, tables[b], h, slots[b]), ref.gather(which, tables[b], h, slots[b]))
            ref = got


def test_results_repeat_bit_for_bit():
    lens = [3000, 700, 64, 1500]
    tables, nb = tables_for([n + 1 for n in lens], 6)
    kv = filled(1, nb, 4, 128, "int8", 6)
    q = torch.randn(4, 16, 128, generator=gen(1)).cuda()
    first = attend(kv, 1, q, lens, tables)
    for _ in range(3):
        assert torch.equal(attend(kv, 1, q, lens, tables), first)


def test_profile_names_the_calls():
    kv = filled(1, 4, 2, 64, "int8", 1)
    tables, x = torch.tensor([[0, 1]], dtype=torch.int32), torch.randn(1, 2, 64, device="cuda")
    batch = B.make_batch(None, i32([3]), i32(tables), 32)
    desc = B.make_rotary_desc(64)
    freqs = B.ee_rotary_frequencies(desc)
    B.ee_profile_read()
    B.ee_profile_enable(True)
    try:
        B.ee_rotary(desc, freqs, i32([3]), x, torch.empty_like(x))
        B.ee_kv_quant_append(kv, 1, x, x, batch)
        B.ee_paged_attention_quant(kv, 1, x, batch, torch.empty_like(x), B.QuantWorkspace(kv, 2, 1, 32))
        B.ee_kv_quant_read(kv, 1, batch, torch.empty_like(x), torch.empty_like(x))
    finally:
        B.ee_profile_enable(False)
    assert [(n, l) for n, l, _ in B.ee_profile_read()] == [("other", 0), ("kv_fill", 1), ("attention", 1), ("other", 1)]
