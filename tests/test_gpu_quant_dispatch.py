"""Every way in which the 8-bit cache's attention divides its work: whole contexts, dealt-out ones, and both in one call, around the borders between them.
A few rows and K/V heads of each call against the definition, with the sums of their weights."""
import pytest
import torch

import quant_oracle as Q
import test_gpu_quant as T
from paper_2407_20272_amd import binding as B

pytestmark = pytest.mark.gpu
BLOCKS = 700


def shared_blocks(rows, most, seed):
    """Tables that take their blocks from a small pool (reading shares them)."""
    return torch.randint(0, BLOCKS, (rows, (most + 15) // 16), generator=T.gen(seed), dtype=torch.int32)


def check(kv, q, out, lens, tables, rows, heads, w=None, base=None):
    G = q.shape[1] // kv.head[0]
    pick = [h * G + g for h in heads for g in range(G)]
    c = Q.Cache.of(kv)
    part = Q.Cache(c.k[:, heads], c.v[:, heads], c.scales[:, heads], c.fmt)
    want, probs, bound = Q.attention(part, q[rows][:, pick].double(), [lens[m] for m in rows], tables, rows)
    got = out[rows][:, pick].cpu().double()
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())
    if w is None:
        return
    for m, (p, slack) in zip(rows, probs):
        n = lens[m] + 1
        total = p.view(len(heads), G, -1).sum(1)
        tol = (p * slack[:, None]).view(len(heads), G, -1).sum(1)
        if n:
            total[:, :-1] += base[m][heads][:, :n - 1].double()
        tol = tol + total * (G + 2) * 2.0 ** -24 + 1e-37
        mine = w[m][heads].cpu().double()
        assert bool(((mine[:, :n] - total).abs() <= tol).all()) and torch.equal(mine[:, n:], base[m][heads][:, n:].double()), m


def run(fmt, dh, kv_heads, G, lens, most, rows, heads, weights):
    kv = T.filled(1, BLOCKS, kv_heads, dh, fmt, 1)
    tables = shared_blocks(len(lens), most, 2)
    q = torch.randn(len(lens), kv_heads * G, dh, generator=T.gen(3))
    w = base = None
    if weights:
        base = torch.rand(len(lens), kv_heads, most, generator=T.gen(4))
        w = base.clone().cuda()
    out = T.attend(kv, 1, q.cuda(), lens, tables, weights=w, w_in=w, max_context=most)
    for m, n in enumerate(lens):
        if n < 0:
            assert bool((out[m] == 0).all())
    check(kv, q, out, lens, tables, rows, heads, w, base)


def lengths(rows, low, high, seed):
    return torch.randint(low, high, (rows,), generator=T.gen(seed)).tolist()


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("heads,G,rows", [(64, 1, 33), (33, 1, 64), (32, 17, 33)])
@pytest.mark.parametrize("most", [2000, 8192, 8193, 20000])
def test_many_rows_and_heads(fmt, weights, heads, G, rows, most):
    """2048 (row, K/V head) pairs and more: whole contexts, two heads a workgroup or one, and beside them a few long ones where there may be such.  Contexts of
    8192 and 8193 positions are either side of the border."""
    lens = lengths(rows, -1, 70, rows)
    lens[2], lens[5], lens[rows - 1], lens[7], lens[8] = most - 1, min(most, 8193) - 1, min(most, 8192) - 1, -1, 0
    run(fmt, 16, heads, G, lens, most, [0, 2, 5, 7, 8, 20, rows - 1], [0, 1, heads - 1], weights)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("rows,G,most", [(1023, 1, 1100), (1024, 1, 1100), (1025, 1, 1100), (512, 17, 1100), (513, 17, 1100), (1024, 2, 9000), (1025, 1, 9000), (2500, 3, 9000), (1100, 17, 8500)])
def test_rows_around_what_is_dealt_out_at_once(weights, rows, G, most):
    """1024 tiles of rows are dealt out in a launch: all of them, one less, one more, several launches; with long contexts in the first and last ones."""
    lens = lengths(rows, -1, 130, rows)
    some = [0, 1, 3, 500, 511, 512 % rows, rows - 2, rows - 1]
    lens[0], lens[1], lens[3], lens[rows - 2], lens[rows - 1] = -1, most - 1, 1025, -1, most - 3
    if rows > 1024:
        lens[1023], lens[1024] = most - 2, min(8191, most - 1)
        some += [1023, 1024]
    run("int8", 16, 1, G, lens, most, some, [0], weights)


@pytest.mark.parametrize("all_long", [False, True])
def test_only_long_or_only_short_contexts(all_long):
    """A call that may hold both."""
    lens = lengths(40, 8192, 9000, 1) if all_long else lengths(40, -1, 8192, 1)
    run("e4m3", 16, 64, 1, lens, 9000, [0, 13, 39], [0, 63], True)


def test_replays_on_both_sides_of_the_border():
    """One captured call whose contexts grow past 8192 positions and shrink again."""
    rows, heads, most = 33, 64, 9000
    kv = T.filled(1, BLOCKS, heads, 16, "int8", 1)
    tables = shared_blocks(rows, most, 2)
    q = torch.randn(rows, heads, 16, generator=T.gen(3)).cuda()
    lens, tb, out = torch.zeros(rows, dtype=torch.int32, device="cuda"), T.i32(tables), torch.empty_like(q)
    w = torch.zeros(rows, heads, most, device="cuda")
    batch, ws = B.make_batch(None, lens, tb, most), B.QuantWorkspace(kv, heads, rows, most, True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.ee_paged_attention_quant(kv, 1, q, batch, out, ws, None, w)
    for now in ([8190] * rows, [8192] * rows, lengths(rows, -1, 9000, 5), [8191] * rows, [-1] * rows, lengths(rows, 7000, 9000, 6)):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        w2 = torch.zeros_like(w)
        eager = T.attend(kv, 1, q, now, tables, weights=w2, max_context=most)
        assert torch.equal(out, eager)
        for m, n in enumerate(now):
            assert torch.equal(w[m, :, :n + 1], w2[m, :, :n + 1])
