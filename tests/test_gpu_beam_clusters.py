"""Beam selection where scores lie in clusters: the join's bound is then moved up in several turns, with candidates above all of what a turn looks at.  Checked as in test_gpu_beam."""
import pytest
import torch

from test_gpu_beam import BF, F32, check, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beams,vocab,n", [(64, 32000, 128), (16, 9000, 32), (57, 33000, 114), (8, 2000, 100)])
@pytest.mark.parametrize("wide,spread", [(1.0, 0.1), (3.0, 30.0), (6.0, 0.1), (6.0, 30.0), (20.0, 3.0)])
def test_logits_far_apart(beams, vocab, n, wide, spread):
    g = gen(int(wide * 7 + spread * 3))
    check(torch.randn((beams, vocab), generator=g) * wide, torch.randn(beams, generator=g) * spread - 20, beams, n)


@pytest.mark.parametrize("beams,vocab,n", [(24, 20000, 20), (24, 20000, 33), (64, 32000, 128), (5, 9000, 60)])
@pytest.mark.parametrize("above", [1, 0.25, 0.9])
@pytest.mark.parametrize("blob", [0.01, 1e-4])
def test_a_few_above_many_alike(beams, vocab, n, above, blob):
    """Fewer than are asked for far above all others, and these near each other."""
    g = gen(n)
    logits = torch.randn((2 * beams, vocab), generator=g) * blob
    for i in range(1 if above == 1 else int(above * n)):
        logits[i % (2 * beams), 37 * i + 5] = 4.0 + 8.0 * float(torch.rand(1, generator=g))
    check(logits, torch.full((2 * beams,), -3.0), beams, n)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("live", [1, 8, 16, 40])
@pytest.mark.parametrize("others", [-1e9, -1e4])
def test_some_beams_live(live, others, dtype):
    g = gen(live)
    scores = torch.full((64,), others)
    scores[torch.randperm(64, generator=g)[:live]] = -torch.rand(live, generator=g) * 30
    check((torch.randn((64, 32000), generator=g) * 3).to(dtype), scores, 64, 128, torch.rand(64, generator=g) < 0.2, 9)
