"""Beam selection and the reordering of states, on the GPU against every candidate sorted in float64.

Tokens, rows and flags are equal.  A score is formed in double and rounded once; the sum's exponentials are floats (of an argument off by 2^-24 of itself):
log-sum-exp is off by at most (2 + d) 2^-23 for logits d below the largest that count, and these are at most 20 here (e^-20 counts nothing):
|error| <= 22 * 2^-23 + |score| 2^-24."""
import math
import random

import pytest
import torch

import beams_oracle as O
from paper_2407_20272_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF = torch.float32, torch.bfloat16


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def run(logits, scores, beams, n_out, finished=None, end=-1, ws=None):
    """The call on device copies (logits as they are)."""
    groups = len(scores) // beams
    t, p, f = (torch.full((groups * n_out,), -9, dtype=torch.int32, device="cuda") for _ in range(3))
    s = torch.full((groups * n_out,), math.nan, device="cuda")
    ws = ws or B.BeamWorkspace(groups, beams, logits.shape[1], n_out)
    B.ee_beam_select(logits.cuda() if not logits.is_cuda else logits, scores.cuda(), beams, t, p, s, ws,
                     finished=None if finished is None else finished.int().cuda(), finished_out=f, end_token=end)
    return t.tolist(), p.tolist(), s.cpu(), f.tolist()


def check(logits, scores, beams, n_out, finished=None, end=-1):
    got = run(logits, scores, beams, n_out, finished, end)
    want = O.select(logits.cpu(), scores, beams, n_out, finished, end)
    assert got[0] == want[0] and got[1] == want[1] and got[3] == want[3]
    s = torch.tensor(want[2], dtype=torch.float64)
    fine = torch.isfinite(s)
    assert torch.equal(torch.isfinite(got[2]), fine) and bool((got[2][~fine] == -math.inf).all())
    assert bool(((got[2].double() - s).abs()[fine] <= 22 * 2.0 ** -23 + s.abs()[fine] * 2.0 ** -24).all())
    return got


@pytest.mark.parametrize("groups,beams,vocab,n_out,dtype", [
    (1, 1, 1, 1, F32), (1, 1, 2, 2, BF), (3, 2, 5, 7, F32), (1, 4, 2048, 4, F32), (2, 5, 4095, 10, F32), (2, 3, 4097, 6, BF), (7, 4, 32000, 8, BF),
    (1, 128, 333, 128, F32), (2, 1, 200, 128, F32), (1, 64, 5000, 128, BF), (3, 8, 33333, 33, F32), (1, 2, 150001, 32, F32), (40, 1, 100, 1, F32),
    (1, 3, 17000, 100, F32)])
def test_random(groups, beams, vocab, n_out, dtype):
    g = gen(vocab + beams)
    logits = (torch.randn((groups * beams, vocab), generator=g) * 3).to(dtype)
    scores = torch.randn(groups * beams, generator=g) * 2 - 15
    check(logits, scores, beams, n_out)
    end = vocab // 2
    finished = torch.rand(groups * beams, generator=g) < 0.4
    check(logits, scores, beams, n_out, finished, end)
    check(logits, scores, beams, n_out, None, end)
    check(logits, scores, beams, n_out, torch.ones(groups * beams, dtype=torch.bool), 0)   # all done: one candidate each, and -inf


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("pad,off", [(0, 0), (1, 0), (3, 1), (5, 7), (8, 8)])
def test_strides_and_alignment(dtype, pad, off):
    g = gen(5)
    big = (torch.randn((6, 9001 + pad + off), generator=g) * 2).to(dtype).cuda()
    check(big[:, off:off + 9001], torch.randn(6, generator=g), 3, 6)


def test_rows_that_are_alike():
    """Equal rows with equal scores: of equal candidates the lower row, whatever the rows' alignment."""
    g = gen(6)
    row = torch.randn(10007, generator=g)
    big = torch.empty((8, 10009), device="cuda")
    big[:, 1:10008] = row.cuda()
    check(big[:, 1:10008], torch.full((8,), -3.0), 4, 16)


@pytest.mark.parametrize("vocab,n_out", [(50, 16), (4096, 16), (40000, 40), (20000, 128), (3000, 32)])
@pytest.mark.parametrize("what", ["equal", "zeros", "steps", "two"])
def test_equal_logits(vocab, n_out, what):
    """More equal values than are put in order at a time: the lowest tokens of the lowest rows."""
    g = gen(7)
    logits = {"equal": torch.full((4, vocab), 1.25), "zeros": torch.zeros((4, vocab)), "steps": torch.randint(0, 3, (4, vocab), generator=g).float(),
              "two": torch.randn((2, vocab), generator=g).repeat(2, 1).round()}[what]
    if what == "zeros":
        logits[:, ::3] = -0.0
    check(logits, torch.tensor([-1.0, -1.0, -2.0, -1.0]) if what != "two" else torch.full((4,), -1.0), 2, n_out)


def test_masks():
    g = gen(8)
    inf = math.inf
    logits = torch.randn((12, 9000), generator=g)
    logits[0] = -inf                                  # a row without a token
    logits[1, :] = -inf
    logits[1, 8999] = 0.5                             # one token left
    logits[2, 5000:] = -inf                           # chunks without a token
    logits[3, 77] = inf                               # rows that are no distribution
    logits[4, 4500] = math.nan
    logits[5] = math.nan
    logits[6] = torch.finfo(F32).min                  # the lowest value is one like others
    logits[7, 10:] = torch.finfo(F32).min
    logits[8:12] = -inf                               # a group with nothing
    scores = torch.randn(12, generator=g)
    for n_out in (1, 8, 40, 128):
        check(logits, scores, 4, n_out)
        check(logits, scores, 2, n_out)
    logits[8, 3] = 1.0
    logits[11, 8998] = 1.0
    check(logits, scores, 4, 6)
    check(logits.to(BF), scores, 4, 6)


def test_scores_that_are_none():
    """The first step of a search: one beam of each group stands for all."""
    g = gen(9)
    logits = torch.randn((8, 700), generator=g)
    scores = torch.tensor([0.0, -math.inf, -math.inf, -math.inf, math.nan, 1.0, math.inf, -2.0])
    check(logits, scores, 4, 4)
    check(logits, scores, 4, 8, torch.tensor([0, 0, 1, 0, 1, 0, 1, 0], dtype=torch.bool), 5)


def test_large_scores():
    """Scores next to each other where floats are far apart: compared before they are rounded."""
    g = gen(10)
    logits = torch.randn((4, 3000), generator=g)
    got = check(logits, torch.tensor([-1e6, -1e6, -1e6, -1e6]), 4, 8)
    assert len(set(got[2].tolist())) < 8
    check(logits * 1e4, torch.zeros(4), 4, 8)
    check(logits * 1e30, torch.zeros(4), 4, 8)


@pytest.mark.parametrize("beams,vocab,n_out", [(57, 105147, 114), (128, 20000, 128), (64, 32000, 128), (20, 9000, 32)])
@pytest.mark.parametrize("spread", [0.1, 3.0, 200.0])
def test_unlike_beams(beams, vocab, n_out, spread):
    """Where few beams have all the best candidates, and more of them than are kept at hand; and where all are alike."""
    g = gen(beams)
    logits = torch.randn((beams, vocab), generator=g) * 2
    check(logits, torch.randn(beams, generator=g) * spread, beams, n_out)
    finished = torch.rand(beams, generator=g) < 0.3
    check(logits[:, :vocab - 1].contiguous(), -torch.arange(beams).float() * spread, beams, n_out, finished, 7)


@pytest.mark.parametrize("beams,vocab,n_out", [(4, 2048, 4), (4, 32000, 8), (64, 32000, 128), (128, 128256, 128)])
@pytest.mark.parametrize("others", [-1e9, -3e38, -math.inf])
def test_a_first_step(beams, vocab, n_out, others):
    """All beams of a group alike, and only the first of them counts."""
    g = gen(beams + vocab)
    logits = (torch.randn((1, vocab), generator=g) * 3).expand(beams, vocab).contiguous()
    scores = torch.full((beams,), others)
    scores[0] = 0.0
    check(logits, scores, beams, n_out)


@pytest.mark.parametrize("beams,vocab,n_out", [(1, 50, 33), (4, 4096, 128), (5, 40000, 33), (64, 32000, 128)])
def test_scores_that_hide_the_logits(beams, vocab, n_out):
    """Scores so large that all of a row's are one double: the order within the row is that of the logits, and the rows' is theirs."""
    g = gen(vocab)
    logits = torch.randn((beams, vocab), generator=g)
    t, p, _, _ = run(logits, torch.full((beams,), -3e38), beams, n_out)
    assert p == [0] * n_out and t == torch.sort(logits[0], descending=True, stable=True)[1][:n_out].tolist()
    scores = torch.full((beams,), -1e20)
    scores[-1] = 1e20
    t, p, _, _ = run(logits, scores, beams, n_out)
    assert p == [beams - 1] * n_out and t == torch.sort(logits[-1], descending=True, stable=True)[1][:n_out].tolist()


@pytest.mark.parametrize("beams,vocab,n_out,dtype", [(128, 270001, 32, F32), (128, 128256, 20, BF), (125, 540001, 40, BF), (128, 794625, 32, BF)])
@pytest.mark.parametrize("spread", [0.0, 40.0])
def test_more_lists_than_are_looked_at_first(beams, vocab, n_out, dtype, spread):
    """Vocabularies whose chunks, over all beams, are up to 12416 lists; of beams that are alike, and of one in front."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    logits = (torch.randn((beams, vocab), generator=g, device="cuda") * 3).to(dtype)
    logits[:, ::7919] += torch.rand((beams, len(range(0, vocab, 7919))), generator=g, device="cuda").to(dtype)
    scores = -torch.linspace(0, 1, beams) * spread
    t, p, s, _ = run(logits, scores, beams, n_out)
    every = logits.double()
    every = every - torch.logsumexp(every, 1, keepdim=True) + scores.cuda().double()[:, None]
    # of equal scores the lower index first: bf16 logits meet within a beam
    least = torch.topk(every.flatten(), n_out)[0][-1]
    at = torch.nonzero(every.flatten() >= least).flatten()
    order = sorted(at.tolist(), key=lambda i: (-float(every.flatten()[i]), i))[:n_out]
    del every
    assert [b * vocab + x for b, x in zip(p, t)] == order


def test_a_workspace_of_larger_sizes_and_repeats():
    g = gen(11)
    ws = B.BeamWorkspace(9, 40, 20000, 128)
    for groups, beams, vocab, n_out in [(9, 40, 20000, 32), (2, 3, 500, 3), (9, 40, 20000, 128), (1, 40, 9000, 33)]:
        logits, scores = torch.randn((groups * beams, vocab), generator=g), torch.randn(groups * beams, generator=g)
        a = run(logits, scores, beams, n_out, ws=ws)
        b = run(logits, scores, beams, n_out, ws=ws)
        want = O.select(logits, scores, beams, n_out)
        assert a[0] == b[0] == want[0] and a[1] == want[1] and torch.equal(a[2], b[2])


def test_captured():
    g = gen(12)
    logits, scores = torch.randn((8, 5000), generator=g).cuda(), torch.randn(8, generator=g).cuda()
    t, p = (torch.zeros(16, dtype=torch.int32, device="cuda") for _ in range(2))
    s, state, out = torch.zeros(16, device="cuda"), torch.randn((8, 100), generator=g).cuda(), torch.zeros((16, 100), device="cuda")
    ws = B.BeamWorkspace(2, 4, 5000, 8)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        B.ee_beam_select(logits, scores, 4, t, p, s, ws)
        B.ee_reorder_rows(state, p, out)
    for i in range(4):
        logits.copy_(torch.randn((8, 5000), generator=g))
        graph.replay()
        torch.cuda.synchronize()
        want = O.select(logits.cpu(), scores.cpu(), 4, 8)
        assert t.tolist() == want[0] and p.tolist() == want[1]
        assert torch.equal(out, state[p.long()])


@pytest.mark.parametrize("dtype,shape,cut", [(torch.float32, (100,), 0), (torch.int32, (7,), 0), (torch.bfloat16, (33,), 0), (torch.uint8, (5,), 3), (torch.float64, (4, 70), 0),
                                             (torch.bfloat16, (20000,), 4), (torch.uint8, (16385,), 1), (torch.float32, (1,), 0), (torch.int32, (5000,), 12)])
def test_reorder(dtype, shape, cut):
    r = random.Random(3)
    size = math.prod(shape)
    x = (torch.randn((9, size + cut), generator=gen(1)) * 50).to(dtype).cuda()
    out = torch.zeros((14, size + cut), dtype=dtype, device="cuda")
    parents = [r.randrange(9) for _ in range(14)]
    parents[3], parents[13] = -1, 9
    a, b = (x, out) if not cut else (x[:, :size], out[:, cut:])
    a, b = a.view(9, *shape) if not cut else a, b.view(14, *shape) if not cut else b
    B.ee_reorder_rows(a, torch.tensor(parents, dtype=torch.int32, device="cuda"), b)
    for m, p in enumerate(parents):
        assert torch.equal(b[m], a[p] if 0 <= p < 9 else torch.zeros_like(b[m]))
    if cut:
        assert not bool(out[:, :cut].any())
