"""A workspace of a beam selection serves smaller calls too, whatever chunks their rows are divided into."""
import itertools

import pytest
import torch

import beams_oracle as O
from paper_2407_20272_amd import binding as B


def size(groups, beams, vocab, n):
    return B.lib().ee_beam_select_bytes(groups, beams, vocab, n)


def needed(groups, beams, vocab, n):
    """What a call keeps: 16 bytes of every chunk, and its n best of 8 bytes; chunks of 16384 values where more than 32 come back, else of 4096, or 8192 beyond 1536 of them."""
    rows, up = groups * beams, lambda x: (x + 255) // 256 * 256
    each = 16384 if n > 32 else 4096 if rows * -(-vocab // 4096) <= 1536 else 8192
    pieces = rows * -(-vocab // each)
    return up(pieces * 16) + up(pieces * n * 8)


SWEEPS = [
    [(g, 4, 32000, n) for n in (4,) for g in range(1, 120)],
    [(g, 4, 32000, 8) for g in range(30, 70)],
    [(g, 4, 50000, 8) for g in range(1, 60)],
    [(32, 8, v, 16) for v in range(24000, 25200, 31)] + [(32, 8, v, 16) for v in range(25200, 300000, 4093)],
    [(1, 128, v, 32) for v in range(40000, 60000, 257)],
    [(1, b, 128256, 20) for b in range(1, 129)],
    [(12, b, 65537, 128) for b in range(1, 129)],
    [(g, 1, 4097, 32) for g in range(700, 1600, 7)],
    [(g, 128, 4096, 33) for g in range(1, 40)],
    [(49, 4, 32000, n) for n in range(1, 129)],
    [(48, 4, 32000, n) for n in range(1, 129)],
    [(200, 100, 16385, n) for n in range(1, 129)],
]


@pytest.mark.parametrize("sweep", range(len(SWEEPS)))
def test_sizes_never_fall(sweep):
    sizes = [size(*x) for x in SWEEPS[sweep]]
    assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))
    assert all(b >= needed(*x) for x, b in zip(SWEEPS[sweep], sizes))


def test_sizes_cover_what_smaller_calls_need():
    some = list(itertools.product((1, 5, 47, 48, 49, 96), (1, 4, 64), (1000, 4097, 24576, 24577, 32000, 100003), (1, 4, 32, 33, 128)))
    for x in some:
        for y in some:
            if all(b <= a for a, b in zip(x, y)):
                assert size(*x) >= needed(*y), (x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("large,small", [((49, 4, 32000, 4), (48, 4, 32000, 4)), ((95, 4, 32000, 4), (48, 4, 32000, 4)), ((32, 8, 24577, 16), (32, 8, 24576, 16)),
                                         ((49, 4, 32000, 40), (48, 4, 32000, 32)), ((30, 4, 50000, 8), (29, 4, 50000, 8))])
def test_a_smaller_call_in_it(large, small):
    ws = B.BeamWorkspace(*large)
    ws.buf.fill_(255)
    for groups, beams, vocab, n in (small, large, small):
        g = torch.Generator().manual_seed(vocab + groups)
        logits, scores = torch.randn((groups * beams, vocab), generator=g) * 3, torch.randn(groups * beams, generator=g)
        tokens, parents = (torch.full((groups * n,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
        B.ee_beam_select(logits.cuda(), scores.cuda(), beams, tokens, parents, torch.zeros(groups * n, device="cuda"), ws)
        want = O.select(logits, scores, beams, n)
        assert tokens.tolist() == want[0] and parents.tolist() == want[1]
