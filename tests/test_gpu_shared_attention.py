"""Attention of rows with common leading blocks, on the GPU against float64 row by row; the bound is derived in beams_oracle."""
import math

import pytest
import torch

import beams_oracle as O
from paper_2407_20272_amd import binding as B
from paper_2407_20272_amd import workloads as W

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """groups: (shared blocks, positions of each row); a row's blocks are its group's shared ones, then its own."""

    def __init__(self, dtype, dh, heads, kv, groups, seed=0, layers=1, layer=1, spare=2, poison=True):
        g = gen(seed)
        self.heads, self.groups, self.layer = heads, groups, layer
        lens = [n for _, rows in groups for n in rows]
        need = sum(s for s, _ in groups) + sum(max(0, O.blocks_of(n) - s) for s, rows in groups for n in rows)
        blocks = need + spare
        order = torch.randperm(blocks, generator=g).to(torch.int32)
        wide = max([1] + [max(s, O.blocks_of(n)) for s, rows in groups for n in rows])
        self.tables, used, m = torch.full((max(1, len(lens)), wide), -1, dtype=torch.int32), 0, 0
        seen = torch.zeros(blocks, 16, dtype=torch.bool)
        first = [0]
        for s, rows in groups:
            common = order[used:used + s]
            used += s
            for n in rows:
                extra = max(0, O.blocks_of(n) - s)
                self.tables[m, :s] = common
                self.tables[m, s:s + extra] = order[used:used + extra]
                used += extra
                for p in range(0, n, 16):
                    seen[int(self.tables[m, p // 16]), :min(16, n - p)] = True
                m += 1
            first.append(m)
        cfg = W.CONFIGS[0].with_(n_layers=layers, d_model=kv * dh, n_heads=kv, head_dim=dh, dtype=dtype)
        self.cfg, self.desc = cfg, B.make_desc(cfg)
        shape = (layers, blocks, kv, 16, dh)
        self.k, self.v = (torch.randn(shape, generator=g).to(cfg.torch_dtype) for _ in range(2))
        if poison:   # slots that hold no position
            hole = ~seen
            for x, bad in ((self.k, math.nan), (self.v, math.inf)):
                x.permute(0, 1, 3, 2, 4)[:, hole] = bad
        self.q = torch.randn((len(lens), heads, dh), generator=g) * 1.3
        self.lens = [n - 1 for n in lens]
        self.first, self.shared = first, [s for s, _ in groups]
        self.max_context = max([1] + lens)

    def run(self, max_shared=None, shared=None, first=None, row_table=None, max_context=None, ws=None):
        cache = B.PagedKV.of(self.cfg, self.k.cuda(), self.v.cuda())
        batch = B.make_batch(None, i32(self.lens), self.tables.cuda(), max_context or self.max_context, None if row_table is None else i32(row_table))
        shared, first = self.shared if shared is None else shared, self.first if first is None else first
        groups = B.make_prefix_groups(i32(first), i32(shared), max([0] + shared) if max_shared is None else max_shared)
        out = torch.full(self.q.shape, 77.0, device="cuda")
        ws = ws or B.SharedWorkspace(self.desc, self.heads, len(self.lens), max(1, len(shared)), max_context or self.max_context)
        ws.buf.fill_(255)
        B.ee_paged_attention_shared(self.desc, cache, self.layer, self.q.cuda(), batch, groups, out, ws)
        return out.cpu()

    def check(self, out=None, rows=None, **kw):
        out = self.run(**kw) if out is None else out
        want, bound = O.attend(self.q, self.k[self.layer - 1], self.v[self.layer - 1], self.tables, self.lens, kw.get("row_table"))
        rows = range(len(self.lens)) if rows is None else rows
        for m in rows:
            err = (out[m].double() - want[m]).abs()
            assert bool((err <= bound[m]).all()), (m, self.lens[m], float((err / bound[m].clamp(min=1e-30)).max()))
        return out


HEADS = [("bf16", 128, 4, 4), ("bf16", 64, 4, 2), ("bf16", 128, 8, 1), ("bf16", 64, 5, 5), ("bf16", 128, 14, 2), ("fp32", 64, 6, 2), ("fp32", 128, 2, 2), ("fp32", 64, 8, 1)]


@pytest.mark.parametrize("dtype,dh,heads,kv", HEADS)
def test_groups_of_all_kinds(dtype, dh, heads, kv):
    """One row alone, beams inside their first blocks, an odd number of shared blocks, rows that end in or before the shared blocks, and rows without a position."""
    Case(dtype, dh, heads, kv, [(0, [1]), (1, [17, 18, 40]), (3, [48, 49, 64, 65, 90]), (2, [33, 5, 32, 0, 31, 100]), (0, [3, 0, 16]), (7, [120] * 9), (1, [16])]).check()


@pytest.mark.parametrize("dtype,dh,heads,kv", HEADS)
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 130])
def test_many_rows_of_one_group(dtype, dh, heads, kv, rows):
    Case(dtype, dh, heads, kv, [(5, [80 + (i * 7) % 45 for i in range(rows)])], seed=rows).check()


@pytest.mark.parametrize("heads,kv", [(16, 1), (17, 1), (33, 1), (64, 1), (70, 1), (48, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_heads_over_one(dtype, heads, kv):
    Case(dtype, 64, heads, kv, [(2, [33, 40, 32]), (0, [20])]).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_contexts_in_parts(dtype):
    """Contexts that several workgroups share, beside short ones, and results that repeat bit for bit."""
    c = Case(dtype, 64, 4, 2, [(200, [3210, 3300, 3201, 3205]), (3, [50, 49]), (0, [2000]), (150, [100, 2400, 2401])])
    a = c.check()
    assert torch.equal(a, c.run())
    c.check(max_context=8000 if c.tables.shape[1] * 16 >= 8000 else c.tables.shape[1] * 16)


def test_one_long_document():
    c = Case("bf16", 128, 8, 2, [(900, [14400 + 1 + i for i in range(12)])])
    c.check()


def test_fewer_shared_than_there_are():
    """What is said to be shared is only how it is read: any smaller number, or none, gives the same attention."""
    c = Case("bf16", 128, 4, 4, [(6, [97, 120, 130]), (4, [70, 66])])
    for shared in ([5, 2], [0, 0], [1, 4]):
        c.check(shared=shared, max_shared=6)
    c.check(max_shared=3)
    c.check(max_shared=0)
    c.check(shared=[-3, 4], max_shared=4)
    c.check(shared=[6, 100000], max_shared=4)


def test_rows_of_no_group():
    c = Case("bf16", 64, 2, 2, [(1, [20, 21]), (2, [40, 45, 50]), (0, [7])])
    out = c.check(first=[0, 2, 4], shared=[1, 2], rows=range(4))
    assert bool((out[4:] == 77).all())
    out = c.check(first=[2, 5], shared=[2], rows=range(2, 5))
    assert bool((out[:2] == 77).all() and (out[5:] == 77).all())
    out = c.run(first=[0], shared=[])
    assert bool((out == 77).all())
    c.check(first=[0, 2, 2, 5, 6], shared=[1, 3, 2, 0])      # an empty group


def test_row_table():
    """Rows of a chunk share a sequence, and sequences share their first blocks."""
    c = Case("bf16", 128, 4, 2, [(3, [60, 75]), (2, [50])])
    row_table = [0, 0, 0, 1, 1, 2, 2]
    c.lens = [57, 58, 59, 73, 74, 48, 49]
    c.q = torch.randn((7, 4, 128), generator=gen(5))
    c.check(first=[0, 5, 7], row_table=row_table)
    c.lens[1], c.lens[5] = -1, 3
    c.check(first=[0, 5, 7], row_table=row_table)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_one_row_cached_stays_with_it(dtype, bad):
    """An Inf or NaN among one row's own positions reaches no other row."""
    c = Case(dtype, 64, 4, 4, [(2, [40, 41, 42, 20, 50])])
    for which in (c.k, c.v):
        old = which.clone()
        which[0, int(c.tables[1, 2]), :, 5] = bad      # row 1's own third block
        out = c.check(rows=[0, 2, 3, 4])
        if which is c.v or bad != -math.inf:
            assert not bool(torch.isfinite(out[1]).all())
        which.copy_(old)
    c.v[0, int(c.tables[0, 1]), :, 9] = bad            # position 25 of the shared blocks: row 3 ends before it
    out = c.check(rows=[3])
    assert not bool(torch.isfinite(out[[0, 1, 2, 4]]).all(-1).any())


def test_large_and_small_values():
    c = Case("bf16", 128, 4, 4, [(3, [60, 61, 64])], poison=False)
    c.q *= 200                                        # softmax of one position
    c.check()
    c.q *= 0.0
    c.check()
    c.q = torch.randn(c.q.shape, generator=gen(2)) * 1e-3
    c.k = (c.k.float() * 1e20).to(torch.bfloat16)
    c.q = c.q * 1e-18
    c.check()
    c.v = (c.v.float() * 1e36).to(torch.bfloat16)
    c.check()
    c.v = (c.v.float() * 1e-37).to(torch.bfloat16)
    c.v = (c.v.float() * 1e-37).to(torch.bfloat16)
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("score", [1e31, -1e31, 3e37, -3e37])
def test_scores_far_out(dtype, score):
    """Scores that are floats, however far out: the softmax of one position is 1, that of equal ones an equal share."""
    c = Case(dtype, 64, 2, 2, [(1, [17, 33, 50]), (0, [1, 20])], poison=False)
    c.q = torch.full(c.q.shape, 2.0 ** 40)
    c.k = torch.full(c.k.shape, score / 2.0 ** 40 / 8).to(c.k.dtype)      # (64 products over sqrt(64): the score)
    out = c.run()
    for m, n in enumerate(c.lens):
        at = torch.arange(n + 1)
        v = c.v[0, c.tables[m][at // 16].long(), :, at % 16].double().mean(0)
        assert bool(((out[m].double() - v).abs() <= 2e-5).all())      # (a sum of 50 values below 6, and its 50: 100 roundings of 6 * 2^-24 / 2 are 1.8e-5)


@pytest.mark.parametrize("groups,rows", [(64, 2), (65, 1), (70, 3), (513, 1), (600, 2), (4096, 1)])
def test_many_groups(groups, rows):
    c = Case("bf16", 64, 2, 2, [(i % 3, [i % 3 * 16 + 1 + (i * 7 + r) % 30 for r in range(rows)]) for i in range(groups)])
    c.check()


@pytest.mark.parametrize("groups,rows,shared,own", [(100, 2, 20, 90), (3, 400, 30, 20), (2, 600, 70, 5), (512, 2, 4, 40)])
def test_many_rows_dealt_out_or_not(groups, rows, shared, own):
    """Around the numbers of rows, groups and tiles up to which steps are dealt out."""
    c = Case("bf16", 64, 2, 1, [(shared - i % 2, [(shared - i % 2) * 16 + 1 + (i + r * 11) % own for r in range(rows)]) for i in range(groups)])
    a = c.check()
    assert torch.equal(a, c.run())


def test_layers_and_a_larger_workspace():
    c = Case("fp32", 128, 4, 2, [(2, [40, 50]), (0, [300])], layers=3, layer=2)
    ws = B.SharedWorkspace(c.desc, 4, 50, 20, 16000)
    c.check(ws=ws)


def test_far_blocks():
    """Blocks whose elements lie beyond 2^32 bytes and 2^31 values."""
    kv, dh, blocks = 32, 128, 36000                   # 4.7 GB a pool
    cfg = W.CONFIGS[0].with_(n_layers=1, d_model=kv * dh, n_heads=kv, head_dim=dh, dtype="bf16")
    k, v = (torch.empty((1, blocks, kv, 16, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = [35999, 35990, 33000, 5]
    small = []
    for x in (k, v):
        y = torch.randn((4, kv, 16, dh), generator=gen(3)).to(torch.bfloat16)
        x[0, ids] = y.cuda()
        small.append(y)
    q = torch.randn((2, kv, dh), generator=gen(4))
    lens = [47, 55]
    near = torch.tensor([[0, 1, 2, -1], [0, 1, 2, 3]], dtype=torch.int32)
    far = torch.tensor([[35999, 35990, 33000, -1], [35999, 35990, 33000, 5]], dtype=torch.int32)
    desc = B.make_desc(cfg)
    out = torch.zeros(q.shape, device="cuda")
    B.ee_paged_attention_shared(desc, B.PagedKV.of(cfg, k, v), 1, q.cuda(), B.make_batch(None, i32(lens), far.cuda(), 56),
                                B.make_prefix_groups(i32([0, 2]), i32([2]), 2), out, B.SharedWorkspace(desc, kv, 2, 1, 56))
    want, bound = O.attend(q, small[0], small[1], near, lens)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())


def test_agrees_with_the_decode_attention():
    """The same rows through ee_paged_attention_decode."""
    c = Case("bf16", 128, 6, 6, [(4, [70, 80, 66]), (0, [33])])
    out = c.check()
    cache = B.PagedKV.of(c.cfg, c.k.cuda(), c.v.cuda())
    other = torch.zeros(c.q.shape, device="cuda")
    B.ee_paged_attention_decode(c.desc, cache, 1, c.q.cuda(), B.make_batch(None, i32(c.lens), c.tables.cuda(), c.max_context), other)
    c.check(other.cpu())


def test_captured_on_another_stream():
    c = Case("bf16", 64, 4, 4, [(120, [1925, 1930, 1990]), (2, [33, 40])])
    cache = B.PagedKV.of(c.cfg, c.k.cuda(), c.v.cuda())
    lens, tables, q = i32(c.lens), c.tables.cuda(), c.q.cuda()
    batch, groups = B.make_batch(None, lens, tables, c.max_context), B.make_prefix_groups(i32(c.first), i32(c.shared), 120)
    out, ws = torch.zeros(c.q.shape, device="cuda"), B.SharedWorkspace(c.desc, 4, 5, 2, c.max_context)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.ee_paged_attention_shared(c.desc, cache, 1, q, batch, groups, out, ws)
    for i in range(4):
        c.q = torch.randn(c.q.shape, generator=gen(20 + i))
        q.copy_(c.q)
        out.fill_(3.0)
        ws.buf.fill_(i)
        g.replay()
        torch.cuda.synchronize()
        c.check(out.cpu())


def test_ids_that_are_no_block():
    """Such a row's result is unspecified; the others' are theirs."""
    c = Case("bf16", 64, 4, 4, [(1, [30, 31, 40])])
    c.tables[1, 1] = 1 << 30
    out = c.run()
    c.tables[1, 1] = 0          # (for the oracle, which has no such row)
    c.check(out, rows=[0, 2])
