"""Pages that sequences share, on the GPU against counting on the CPU: every result is a whole number or a copy, so everything is equal."""
import random

import pytest
import torch

import beams_oracle as O
from paper_2407_20272_amd import binding as B
from paper_2407_20272_amd import workloads as W

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """A pool and tables on the device, and the same in lists."""

    def __init__(self, num_blocks, rows, wide, seed=0):
        """(-7 behind a row's blocks: nothing there is read or written)"""
        self.r, self.n, self.wide = random.Random(seed), num_blocks, wide
        self.refs = torch.zeros(num_blocks, dtype=torch.int32, device="cuda")
        self.pool = B.PagePool.of(self.refs, rows)
        self.sets = []
        for _ in range(2):
            t = torch.full((rows, wide), -7, dtype=torch.int32, device="cuda")
            self.sets.append(B.PageTables(t, torch.zeros(rows, dtype=torch.int32, device="cuda")))
        self.o, self.rows = O.Pages([0] * num_blocks), [([], 0)] * rows
        self.moves = torch.full((rows, 2), 5, dtype=torch.int32, device="cuda")
        self.missing = i32([9])

    def check(self, which=0):
        assert self.refs.tolist() == self.o.refs
        tables, lens = self.sets[which].block_tables.tolist(), self.sets[which].lens.tolist()
        assert lens == [n for _, n in self.rows]
        for t, (want, _) in zip(tables, self.rows):
            assert t[:len(want)] == want

    def grow(self, new, which=0):
        B.ee_kv_pages_grow(self.pool, self.sets[which], i32(new), self.moves, self.missing)
        new = [min(n, 16 * self.wide) for n in new]
        self.rows, moves, missing = self.o.grow(self.rows, new)
        assert [tuple(m) for m in self.moves.tolist()] == moves
        assert self.missing.item() == missing
        self.check(which)
        if not missing:   # the positions are cached: as a caller does
            lens = [max(a, n) for a, (_, n) in zip(new, self.rows)]
            self.sets[which].lens.copy_(i32(lens))
            self.rows = [(t, n) for (t, _), n in zip(self.rows, lens)]
        return missing

    def fork(self, parents, release, src=0):
        B.ee_kv_pages_fork(self.pool, self.sets[src], i32(parents), self.sets[1 - src], release=release)
        new = self.o.fork(self.rows, parents)
        if release:
            self.o.release(self.rows)
            assert self.sets[src].lens.tolist() == [0] * len(self.rows)
        old, self.rows = self.rows, new
        self.check(1 - src)
        return old


@pytest.mark.parametrize("num_blocks,rows,seed", [(40, 3, 0), (1000, 8, 1), (1024, 33, 2), (2500, 70, 3), (5000, 300, 4), (16384, 40, 5), (16385, 40, 6), (20000, 1024, 7), (40000, 1500, 8),
                                                  (9000, 1025, 9)])
def test_a_long_beam_search(num_blocks, rows, seed):
    """Prompts of all lengths, then steps that fork rows at random and grow them, packing on the way; a search that finds no room changes nothing."""
    b = Both(num_blocks, rows, 60, seed)
    room = num_blocks // (2 * rows)
    assert b.grow([b.r.choice([0, 1, 15, 16, 17, b.r.randint(0, 16 * max(1, min(20, room)))]) for _ in range(rows)]) == 0
    at, short = 0, 0
    for step in range(24 if rows < 500 else 8):
        parents = [b.r.randrange(rows) if b.r.random() < 0.6 else m for m in range(rows)]
        if step == 7:
            parents[0] = -1
            parents[-1] = rows
        b.fork(parents, True, at)
        at = 1 - at
        short += b.grow([n + b.r.choice([0, 1, 1, 1, 3, 17]) if n < 16 * 50 else n for _, n in b.rows], at) > 0
        if step % 9 == 5:
            remap, moves, count = torch.empty(num_blocks, dtype=torch.int32, device="cuda"), torch.empty((num_blocks, 2), dtype=torch.int32, device="cuda"), i32([0])
            B.ee_kv_pages_compact(b.pool, b.sets[at], remap, moves, count)
            b.rows, want, pairs = b.o.compact(b.rows)
            assert remap.tolist() == want and count.item() == len(pairs)
            assert [tuple(m) for m in moves.tolist()] == pairs + [(-1, -1)] * (num_blocks - len(pairs))
            b.check(at)
        first = sorted(b.r.sample(range(rows + 1), min(3, rows)))
        first = [0] + first + [rows]
        out = torch.empty(len(first) - 1, dtype=torch.int32, device="cuda")
        B.ee_kv_pages_shared(b.sets[at], i32(first), out)
        assert out.tolist() == O.shared(b.rows, first)
    B.ee_kv_pages_release(b.pool, b.sets[at])
    assert b.refs.tolist() == [0] * num_blocks and b.sets[at].lens.tolist() == [0] * rows
    B.ee_kv_pages_release(b.pool, b.sets[at])   # rows without blocks give nothing up
    assert b.refs.tolist() == [0] * num_blocks


@pytest.mark.parametrize("spare", [0, 20000])
def test_all_or_nothing(spare):
    """(With a pool beyond what one workgroup looks through, most of it taken.)"""
    b = Both(10 + spare, 4, 8)
    if spare:
        taken = b.r.sample(range(10 + spare), spare)
        for i in taken:
            b.o.refs[i] = 1
        b.refs.copy_(i32(b.o.refs))
    assert b.grow([30, 30, 0, 5]) == 0
    b.fork([0, 0, 1, 3], False)
    assert b.grow([31, 31, 40, 6], 1) == 0       # rows 0 and 1 move (the parents keep theirs), row 2 moves and adds one, row 3 moves
    assert b.grow([31, 31, 128, 128], 1) > 0
    assert b.grow([32, 32, 40, 16], 1) == 0      # room in what they have
    b2 = Both(1, 1, 1)
    assert b2.grow([16]) == 0 and b2.grow([16]) == 0
    assert b2.grow([500]) == 0                   # beyond the table: no more blocks
    assert b2.sets[0].block_tables.tolist() == [[0]]


def test_who_keeps_a_block():
    """Of the rows that alone refer to a block the last that writes keeps it; where others refer to it too, all move."""
    b = Both(64, 5, 4)
    assert b.grow([20, 0, 0, 0, 0]) == 0
    b.fork([0, 0, 0, 0, 0], True)
    assert b.grow([21, 21, 20, 21, 21], 1) == 0          # row 2 does not write: four move
    assert sum(m[0] >= 0 for m in b.moves.tolist()) == 4
    c = Both(64, 5, 4)
    assert c.grow([20, 0, 0, 0, 0]) == 0
    c.fork([0, 0, 0, 0, 0], True)
    assert c.grow([21] * 5, 1) == 0
    assert [m[0] >= 0 for m in c.moves.tolist()] == [True] * 4 + [False]


def test_empty_calls():
    pool = B.PagePool(3, 0)
    none = B.PageTables(torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    missing = i32([4])
    B.ee_kv_pages_fork(pool, none, e, none, release=True)
    B.ee_kv_pages_release(pool, none)
    B.ee_kv_pages_grow(pool, none, e, e.view(0, 2), missing)
    assert missing.item() == 0
    out = i32([3, 3])
    B.ee_kv_pages_shared(none, i32([0, 0, 0]), out)
    assert out.tolist() == [0, 0]
    remap, moves, count = i32([7] * 3), i32([[7, 7]] * 3), i32([7])
    B.ee_kv_pages_compact(pool, None, remap, moves, count)
    assert remap.tolist() == [-1] * 3 and count.item() == 0 and moves.tolist() == [[-1, -1]] * 3


def test_entries_that_are_no_block():
    """A table with entries outside the pool: nothing outside is read or counted."""
    refs = torch.zeros(8, dtype=torch.int32, device="cuda")
    pool = B.PagePool.of(refs, 4)
    t = B.PageTables(i32([[-5, 99], [3, 1 << 30]]), i32([30, 100]))
    d = B.PageTables(torch.zeros((2, 2), dtype=torch.int32, device="cuda"), i32([0, 0]))
    B.ee_kv_pages_fork(pool, t, i32([0, 1]), d)
    assert refs.tolist() == [0, 0, 0, 1, 0, 0, 0, 0] and d.block_tables.tolist() == t.block_tables.tolist() and d.lens.tolist() == [30, 32]
    moves, missing = i32([[0, 0]] * 2), i32([0])
    B.ee_kv_pages_grow(pool, d, i32([31, 32]), moves, missing)
    assert moves.tolist() == [[-1, -1]] * 2 and missing.item() == 0
    B.ee_kv_pages_release(pool, d)
    assert refs.tolist() == [0] * 8


# ---- contents -----------------------------------------------------------------------------------------------------
def pools(kind, layers, blocks, kv, dh, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if kind in ("fp32", "bf16"):
        cfg = W.CONFIGS[0].with_(n_layers=layers, d_model=kv * dh, n_heads=kv, head_dim=dh, dtype=kind)
        c = B.PagedKV(cfg, blocks)
        for p in (c.k, c.v):
            p.copy_(torch.randn(p.shape, generator=g, device="cuda"))
        return c, lambda *a: B.ee_kv_copy(B.make_desc(cfg), c, *a), [c.k, c.v]
    c = B.QuantKV(layers, blocks, kv, dh, kind)
    for p in (c.k, c.v):
        p.view(torch.int8).copy_(torch.randint(-128, 128, p.shape, generator=g, device="cuda", dtype=torch.int8))
    c.scales.copy_(torch.randn(c.scales.shape, generator=g, device="cuda"))
    return c, lambda *a: B.ee_kv_quant_copy(c, *a), [c.k.view(torch.int8), c.v.view(torch.int8), c.scales]


@pytest.mark.parametrize("kind,layers,kv,dh", [("fp32", 2, 3, 64), ("bf16", 3, 5, 128), ("int8", 2, 1, 16), ("e4m3", 4, 3, 80), ("int8", 1, 7, 128)])
def test_copies(kind, layers, kv, dh):
    blocks = 50
    _, copy, tensors = pools(kind, layers, blocks, kv, dh, 3)
    was = [t.clone() for t in tensors]
    moves = [(3, 4), (-1, -1), (3, 5), (6, 6), (10, 49), (50, 2), (2, 50), (1 << 30, 7), (0, 48)]
    copy(i32(moves))
    for t, w in zip(tensors, was):
        for a, b in [(3, 4), (3, 5), (10, 49), (0, 48)]:
            w[:, b] = w[:, a]
        assert torch.equal(t, w)
    copy(i32([(20, 30), (21, 31), (22, 32)]), i32([2]))
    for t, w in zip(tensors, was):
        w[:, 30], w[:, 31] = w[:, 20].clone(), w[:, 21].clone()
        assert torch.equal(t, w)
    for count in (0, -3):
        copy(i32([(20, 40)]), i32([count]))
    copy(torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    for t, w in zip(tensors, was):
        assert torch.equal(t, w)


def test_many_copies():
    """More moves than are gathered at a time, most of them none."""
    blocks = 6000
    _, copy, tensors = pools("int8", 1, blocks, 1, 16, 4)
    r = random.Random(1)
    half = list(range(blocks))
    r.shuffle(half)
    pairs = [(half[2 * i], half[2 * i + 1]) if i % 3 else (-1, -1) for i in range(blocks // 2)]
    was = [t.clone() for t in tensors]
    copy(i32(pairs))
    src, dst = (torch.tensor([p[i] for p in pairs if p[0] >= 0], device="cuda") for i in (0, 1))
    for t, w in zip(tensors, was):
        w[:, dst] = w[:, src]
        assert torch.equal(t, w)


def test_far_blocks():
    """Byte offsets beyond 2^32."""
    c, copy, tensors = pools("bf16", 1, 2, 1, 64, 0)
    cfg = c.cfg.with_(d_model=32 * 128, n_heads=32, head_dim=128)
    k = torch.empty((1, 40000, 32, 16, 128), dtype=torch.bfloat16, device="cuda")   # 5.2 GB
    k[0, 39990].normal_()
    big = B.PagedKV.of(cfg, k, k)
    B.ee_kv_copy(B.make_desc(cfg), big, i32([[39990, 39999], [39990, 7]]))
    assert torch.equal(k[0, 39999], k[0, 39990]) and torch.equal(k[0, 7], k[0, 39990])


def test_captured_and_on_another_stream():
    """One beam step in a graph, replayed: the counts go on from where they are."""
    b = Both(200, 6, 8, 3)
    b.grow([40, 17, 16, 5, 0, 33])
    parents, new = i32([0, 0, 1, 2, 3, 5]), i32([41, 41, 18, 17, 6, 34])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.ee_kv_pages_fork(b.pool, b.sets[0], parents, b.sets[1])
            B.ee_kv_pages_grow(b.pool, b.sets[1], new, b.moves, b.missing)
            b.sets[1].lens.copy_(new)
            B.ee_kv_pages_release(b.pool, b.sets[1])
    before = b.refs.clone()
    want = None
    for _ in range(4):
        b.sets[1].block_tables.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        got = (b.sets[1].block_tables.clone(), b.moves.clone(), b.missing.item())
        want = want or got
        assert torch.equal(b.refs, before) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[2] == 0
    o = O.Pages(b.o.refs)
    rows, moves, _ = o.grow(o.fork(b.rows, parents.tolist()), new.tolist())
    assert [tuple(m) for m in want[1].tolist()] == moves
    for t, (r, _) in zip(want[0].tolist(), rows):
        assert t[:len(r)] == r
