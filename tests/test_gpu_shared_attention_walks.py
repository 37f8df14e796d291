"""Attention of rows with common leading blocks where a wavefront walks many steps: it holds the blocks of 32 of them at a time.  Against float64, with the bound of beams_oracle.

A workgroup's eight wavefronts take its steps (32 positions each) in turn.  128 K/V heads leave two workgroups a head, so a tile of a group has half of its steps in each: 33 steps a wavefront are
2 * 8 * 33 of the tile.  The heads repeat a few that are drawn, and the oracle sees those."""
import pytest
import torch

import beams_oracle as O
from paper_2407_20272_amd import binding as B
from test_gpu_shared_attention import Case, gen, i32

pytestmark = pytest.mark.gpu

HEADS, DH, WAVES = 128, 64, 8
WIDTHS = [("bf16", 16), ("bf16", 32), ("bf16", 48), ("fp32", 16), ("fp32", 32)]


def walk(c, groups, row_table=None):
    """The case's attention with its K/V heads repeated to 128 of them: each like the oracle's."""
    kv = c.k.shape[2]
    more = HEADS // kv
    cfg = c.cfg.with_(d_model=HEADS * DH, n_heads=HEADS)
    k, v = (x.cuda().repeat(1, 1, more, 1, 1) for x in (c.k, c.v))
    q = c.q.repeat(1, more, 1).cuda()
    desc, rows = B.make_desc(cfg), len(c.lens)
    batch = B.make_batch(None, i32(c.lens), c.tables.cuda(), c.max_context, None if row_table is None else i32(row_table))
    first, shared = groups
    out = torch.full(q.shape, 77.0, device="cuda")
    ws = B.SharedWorkspace(desc, q.shape[1], rows, len(shared), c.max_context)
    B.ee_paged_attention_shared(desc, B.PagedKV.of(cfg, k, v), 1, q, batch, B.make_prefix_groups(i32(first), i32(shared), max(shared)), out, ws)
    out = out.cpu().view(rows, more, c.heads, DH)
    assert all(torch.equal(out[:, 0], out[:, i]) for i in range(1, more))
    c.check(out[:, 0], row_table=row_table)


def own_positions(rows, steps):
    """Positions of each row, so that their steps are 2 * 8 * `steps` together; last blocks of every filling."""
    each, over = divmod(2 * WAVES * steps, rows)
    return [32 * (each + (i < over)) - (i * 5) % 32 for i in range(rows)]


@pytest.mark.parametrize("steps", [32, 33, 65, 100])
@pytest.mark.parametrize("dtype,columns", WIDTHS)
def test_rows_of_their_own(dtype, columns, steps):
    """Steps of one row after the other: the blocks at a renewal are partly filled, and what lies behind their positions is NaN or Inf."""
    c = Case(dtype, DH, 2, 2, [(0, own_positions(columns, steps))], seed=steps)
    walk(c, (c.first, c.shared))


@pytest.mark.parametrize("steps", [33, 66])
@pytest.mark.parametrize("dtype,columns", WIDTHS)
def test_shared_blocks(dtype, columns, steps):
    """Steps that all rows attend, and the rows' own behind them; one row that ends before."""
    group = 4
    shared = 4 * WAVES * steps - 13
    rows = [shared * 16 + 1 + (i * 11) % 70 for i in range(columns // group)]
    rows[1] = 45
    c = Case(dtype, DH, group, 1, [(shared, rows)], seed=steps)
    walk(c, (c.first, c.shared))


@pytest.mark.parametrize("dtype,columns", WIDTHS)
def test_positions_of_a_sequence(dtype, columns):
    """Rows of chunks: several positions of each of four sequences, whose first blocks are the same."""
    steps = 40
    a_row = 2 * WAVES * steps * 32 // columns
    sequences = [a_row + 64 + 90 + 7 * i for i in range(4)]
    c = Case(dtype, DH, 2, 2, [(5, sequences)], seed=9)
    row_table = [i * 4 // columns for i in range(columns)]
    c.lens = [sequences[s] - 1 - i % (columns // 4) for i, s in enumerate(row_table)]
    c.lens[3] = -1
    c.q = torch.randn((columns, 2, DH), generator=gen(10))
    walk(c, ([0, columns], [5]), row_table)


@pytest.mark.parametrize("dtype,columns", WIDTHS)
def test_whole_tiles(dtype, columns):
    """More rows than are dealt out: a workgroup has all steps of a tile, one of which is long."""
    n, kv = 1104 // columns, 8
    groups = [(0, [32 * (WAVES * 70 // columns) - i % 19 for i in range(columns)])] + [(0, [1 + i % 3] * columns) for i in range(n)]
    Case(dtype, DH, kv, kv, groups, seed=columns).check()


def test_a_graph_of_long_walks():
    """Captured and replayed, with other queries."""
    c = Case("bf16", DH, 2, 2, [(0, own_positions(48, 40))], seed=3)
    more = HEADS // 2
    cfg = c.cfg.with_(d_model=HEADS * DH, n_heads=HEADS)
    cache = B.PagedKV.of(cfg, *(x.cuda().repeat(1, 1, more, 1, 1) for x in (c.k, c.v)))
    desc, q = B.make_desc(cfg), c.q.repeat(1, more, 1).cuda()
    batch, groups = B.make_batch(None, i32(c.lens), c.tables.cuda(), c.max_context), B.make_prefix_groups(i32([0, 48]), i32([0]), 0)
    out, ws = torch.zeros(q.shape, device="cuda"), B.SharedWorkspace(desc, HEADS, 48, 1, c.max_context)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.ee_paged_attention_shared(desc, cache, 1, q, batch, groups, out, ws)
    for i in range(3):
        c.q = torch.randn(c.q.shape, generator=gen(30 + i))
        q.copy_(c.q.repeat(1, more, 1))
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        c.check(out.cpu().view(48, more, 2, DH)[:, -1])
