"""The 8-bit cache at the borders of what its calls take: the largest floats, rows of no sequence."""
import math

import pytest
import torch

import quant_oracle as Q
import test_gpu_quant as T
from paper_2407_20272_amd import binding as B

pytestmark = pytest.mark.gpu
LARGEST = torch.finfo(torch.float32).max


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("later", [False, True])
def test_the_largest_float(fmt, later):
    """It is cached as a float next to it, in a block of its own and where a block's scale grows to it, and stays one when it is moved."""
    tables, nb = T.tables_for([20], 1)
    kv = T.filled(1, nb, 1, 64, fmt, 1)
    x = torch.randn(20, 1, 64, generator=T.gen(1)) * 1e30
    x[3, 0, 5], x[3, 0, 6], x[17, 0, 63] = LARGEST, -LARGEST, -LARGEST
    calls = [list(range(3)), list(range(3, 20))] if later else [list(range(20))]
    for rows in calls:
        B.ee_kv_quant_append(kv, 1, x[rows].cuda(), -x[rows].cuda(), B.make_batch(None, T.i32(rows), T.i32(tables), 20, T.i32([0] * len(rows))))

    def check(places):
        k, v = torch.empty(20, 1, 64, device="cuda"), torch.empty(20, 1, 64, device="cuda")
        B.ee_kv_quant_read(kv, 1, B.make_batch(None, T.i32(range(20)), T.i32(tables if places is None else places), 20, T.i32([0] * 20)), k, v)
        for got, want in ((k, x), (v, -x)):
            got = got.cpu()
            assert bool(torch.isfinite(got).all())
            # half a step of the block's scale; 1e30 is far less than that
            step = LARGEST / 127 if fmt == "int8" else 2.0 ** 120 * 32
            assert bool(((got.double() - want.double()).abs() <= step * 0.51).all())
            assert abs(float(got[3, 0, 5]) / float(want[3, 0, 5]) - 1) < (2.0 ** -20 if fmt == "int8" else 2.0 ** -4)
    check(None)
    # all of it into other blocks, with one position more than stays
    free = [i for i in range(nb) if i not in tables.flatten().tolist()]
    dst = torch.tensor([free[:2]], dtype=torch.int32)
    kept, lens = torch.zeros(1, 1, 20, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ee_kv_quant_evict(kv, 1, B.make_batch(None, T.i32([20]), T.i32(tables), 20), torch.ones(1, 1, 20, device="cuda"), None, 20, 0, kept, lens, None, T.i32(dst))
    assert kept[0, 0].tolist() == list(range(20))
    check(dst)


def some_of(kv, q, out, lens, tables, rows, heads, row_table=None):
    """A few rows and K/V heads (one query head each) against the definition."""
    c = Q.Cache.of(kv)
    part = Q.Cache(c.k[:, heads], c.v[:, heads], c.scales[:, heads], c.fmt)
    seq = [row_table[m] if row_table is not None else m for m in rows]
    want, probs, bound = Q.attention(part, q[rows][:, heads].double(), [lens[m] for m in rows], tables, seq)
    assert bool(((out[rows][:, heads].cpu().double() - want).abs() <= bound).all())
    return probs


def test_attention_of_tens_of_thousands_of_sequences():
    heads, rows, most = 32, 33001, 40
    kv = T.filled(1, 50, heads, 16, "int8", 1)
    tables = torch.randint(0, 50, (rows, 3), generator=T.gen(2), dtype=torch.int32)       # (reading shares blocks)
    lens = torch.randint(-1, most, (rows,), generator=T.gen(3)).tolist()
    q = torch.randn(rows, heads, 16, generator=T.gen(4))
    w = torch.full((rows, heads, most), 2.0, device="cuda")
    out = T.attend(kv, 1, q.cuda(), lens, tables, weights=w, max_context=most)
    some = [0, 1, 32767, 32768, 32769, 33000] + [m for m in range(40, 33000, 1500)]
    probs = some_of(kv, q, out, lens, tables, some, [0, 17, 31])
    for m, (p, slack) in zip(some, probs):
        n = lens[m] + 1
        assert bool(((w[m, [0, 17, 31], :n].cpu().double() - p).abs() <= p * slack[:, None] + p * 2.0 ** -22 + 1e-37).all())
        assert bool((w[m, :, n:] == 2.0).all())


def test_attention_of_a_long_prompt_chunk():
    """More rows than 8191 of 128 heads: 282 tiles."""
    heads, chunk = 128, [3000, 5, 6000]
    tables, nb = T.tables_for(chunk, 1)
    kv = T.filled(1, nb, heads, 16, "e4m3", 1)
    lens, rt = [p for n in chunk for p in range(n)], [i for i, n in enumerate(chunk) for _ in range(n)]
    q = torch.randn(len(lens), heads, 16, generator=T.gen(4))
    out = T.attend(kv, 1, q.cuda(), lens, tables, rt)
    some_of(kv, q, out, lens, tables, [0, 1, 2999, 3000, 3004, 3005, 8190, 8191, 8192, 9004], [0, 64, 127], rt)


def test_append_and_read_of_more_rows_than_one_launch_has():
    """2^24 + 5 sequences of a block each."""
    rows, dh = (1 << 24) + 5, 16
    kv = B.QuantKV(1, rows, 1, dh, "int8")
    tables = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")[:, None]
    lens = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(16)
    x = torch.randint(-127, 128, (rows, 1, dh), dtype=torch.int32, device="cuda").to(torch.bfloat16)
    x[:, 0, 0] = 127.0                                   # the scale is 1: everything comes back as it was
    batch = B.make_batch(None, lens, tables, 16)
    B.ee_kv_quant_append(kv, 1, x, -x, batch)
    k, v = torch.zeros_like(x), torch.zeros_like(x)
    B.ee_kv_quant_read(kv, 1, batch, k, v)
    assert torch.equal(k, x) and torch.equal(v, -x)


def test_rotary_of_more_rows_than_one_launch_has():
    rows = (1 << 27) + 9
    desc = B.make_rotary_desc(2)
    freqs = B.ee_rotary_frequencies(desc)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    x = torch.tensor([1.0, 0.0], dtype=torch.bfloat16, device="cuda").repeat(rows).view(rows, 1, 2)
    B.ee_rotary(desc, freqs, pos, x, x)
    for m in (0, 1, 1000, (1 << 27) - 9, (1 << 27) - 8, 1 << 27, rows - 1):
        want = torch.stack([torch.cos(pos[m].double()), torch.sin(pos[m].double())])
        assert bool(((x[m, 0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20).all()), m


def test_rotary_of_more_pieces_than_one_launch_has():
    """A row of 65536 query and 65536 key heads of 1024 channels, of which two are rotated: element by element."""
    desc = B.make_rotary_desc(1024, 2)
    freqs = B.ee_rotary_frequencies(desc)
    pos = torch.tensor([3], dtype=torch.int32, device="cuda")
    q, k = (torch.full((1, 65536, 1024), float(n), device="cuda") for n in (1, 2))
    q_out, k_out = torch.zeros_like(q), torch.zeros_like(k)
    B.ee_rotary(desc, freqs, pos, q, q_out, k, k_out)
    c, s = math.cos(3.0), math.sin(3.0)
    for out, n in ((q_out, 1.0), (k_out, 2.0)):
        assert bool((out[..., 2:] == n).all())
        assert bool(((out[..., 0].double() - n * (c - s)).abs() <= n * 2.0 ** -20).all()) and bool(((out[..., 1].double() - n * (c + s)).abs() <= n * 2.0 ** -20).all())


@pytest.mark.parametrize("fmt", T.FORMATS)
def test_rows_of_no_sequence(fmt):
    """Entries of row_table outside the batch: appending drops the row, no sequence's positions change, and reading is of nothing."""
    kv = T.filled(1, 6, 2, 64, fmt, 9)
    tables = torch.tensor([[0, 1], [2, 3], [4, 5], [0, 0], [0, 0], [0, 0]], dtype=torch.int32)
    lens, rt = [3, 4, 5, 18, 0, 2], [-1, 0, 6, 1 << 30, 2, -(1 << 31)]
    ref = Q.Cache.of(kv)
    x = torch.randn(6, 2, 64, generator=T.gen(2)).cuda()
    batch = B.make_batch(None, T.i32(lens), T.i32(tables), 32, T.i32(rt))
    B.ee_kv_quant_append(kv, 1, x, -x, batch)
    there = [0 <= s < 6 for s in rt]
    Q.append(ref, x.cpu().double(), -x.cpu().double(), [n if ok else -1 for n, ok in zip(lens, there)], tables, [s if ok else 0 for s, ok in zip(rt, there)])
    T.assert_cache(kv, ref)
    k, v = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    B.ee_kv_quant_read(kv, 1, batch, k, v)
    for m, ok in enumerate(there):
        for out, which in ((k, 0), (v, 1)):
            for h in range(2):
                want = ref.value(which, int(tables[rt[m], lens[m] // 16]), h, lens[m] % 16) if ok else torch.zeros(64, dtype=torch.float64)
                assert torch.equal(out[m, h].cpu().double(), want)
