"""A beam search with everything that belongs to it: selection, reordering, pages and the attention over them, against a search that
keeps every hypothesis as a list of tokens and computes its attention anew in float64."""
import math

import pytest
import torch

import beams_oracle as O
from paper_2407_20272_amd import binding as B
from paper_2407_20272_amd import workloads as W

pytestmark = pytest.mark.gpu
F64 = torch.float64


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Model:
    """A layer that attends tokens' keys and values, and a head on what comes out: float tables by token and a position's phase."""

    def __init__(self, vocab, heads, kv, dh, dtype, seed):
        g = torch.Generator()
        g.manual_seed(seed)
        t = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.k, self.v = (torch.randn((vocab, kv, dh), generator=g).to(t) for _ in range(2))
        self.q = torch.randn((vocab, heads, dh), generator=g)
        self.head = torch.randn((heads * dh, vocab), generator=g) * 0.5
        self.vocab, self.heads, self.kv, self.dh = vocab, heads, kv, dh

    def logits(self, tokens):
        """Of the position after `tokens`, float64."""
        t = torch.tensor(tokens)
        k, v, q = self.k[t].double(), self.v[t].double(), self.q[tokens[-1]].double()
        out = torch.empty((self.heads, self.dh), dtype=F64)
        for h in range(self.heads):
            g = h // (self.heads // self.kv)
            out[h] = torch.softmax(k[:, g] @ q[h] / math.sqrt(self.dh), 0) @ v[:, g]
        return out.flatten() @ self.head.double()


def plain_search(model, prompts, beams, steps, end):
    """(tokens behind the prompt, score, ended) of every beam after each step, and how near the nearest choice was."""
    hyps = [[(list(p), 0.0 if b == 0 else -math.inf, False) for b in range(beams)] for p in prompts]
    told, nearest = [], math.inf
    for _ in range(steps):
        for i, group in enumerate(hyps):
            cand = []
            for b, (t, s, ended) in enumerate(group):
                if ended:
                    cand.append((-s, b * model.vocab + end, t + [end], True))
                elif s > -math.inf:
                    lp = torch.log_softmax(model.logits(t), 0)
                    cand += [(-(s + x), b * model.vocab + j, t + [j], j == end) for j, x in enumerate(lp.tolist())]
            cand.sort()
            nearest = min([nearest] + [y[0] - x[0] for x, y in zip(cand[:beams], cand[1:beams + 1])])
            hyps[i] = [(t, -s, e) for s, _, t, e in cand[:beams]]
        told.append([[(t[len(p):], s, e) for t, s, e in group] for group, p in zip(hyps, prompts)])
    return told, nearest


@pytest.mark.parametrize("dtype,cache_kind", [("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("beams,lens,steps", [(4, [37, 16, 50], 24), (1, [5], 5), (7, [31, 33], 20)])
def test_search(dtype, cache_kind, beams, lens, steps):
    vocab, heads, kv, dh, end = 40, 4, 2, 64, 3
    m = Model(vocab, heads, kv, dh, dtype, 1)
    g = torch.Generator()
    g.manual_seed(2)
    prompts = [torch.randint(4, vocab, (n,), generator=g).tolist() for n in lens]
    told, nearest = plain_search(m, prompts, beams, steps, end)
    assert nearest > 1e-4   # no choice hangs on a rounding

    groups, rows, wide = len(lens), len(lens) * beams, 16
    blocks = 8 * rows + 20
    cfg = W.CONFIGS[0].with_(n_layers=1, d_model=kv * dh, n_heads=kv, head_dim=dh, dtype=cache_kind)
    desc, cache = B.make_desc(cfg), B.PagedKV(cfg, blocks, fill=math.nan)
    pool = B.PagePool(blocks, rows)

    def tables(n):
        return B.PageTables(torch.full((n, wide), -1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"))

    prompt_rows, sets = tables(groups), [tables(rows), tables(rows)]
    kd, vd, qd, head = m.k.cuda(), m.v.cuda(), m.q.cuda(), m.head.cuda()
    moves, missing = torch.zeros((rows, 2), dtype=torch.int32, device="cuda"), i32([0])

    def cache_tokens(t, row, pos, tokens):
        """Writes tokens' keys and values at (row, pos)."""
        blk = t.block_tables[row.long(), (pos // 16).long()].long()
        cache.k[0, blk, :, (pos % 16).long()] = kd[tokens.long()]
        cache.v[0, blk, :, (pos % 16).long()] = vd[tokens.long()]

    # the prompts, all but their last token, and their beams
    B.ee_kv_pages_grow(pool, prompt_rows, i32([n - 1 for n in lens]), torch.zeros((groups, 2), dtype=torch.int32, device="cuda"), missing)
    prompt_rows.lens.copy_(i32([n - 1 for n in lens]))
    cache_tokens(prompt_rows, i32([i for i, n in enumerate(lens) for _ in range(n - 1)]), i32([p for n in lens for p in range(n - 1)]),
                 i32([t for p in prompts for t in p[:-1]]))
    at = 0
    B.ee_kv_pages_fork(pool, prompt_rows, i32([i for i in range(groups) for _ in range(beams)]), sets[0], release=True)
    tokens = i32([p[-1] for p in prompts for _ in range(beams)])
    scores = torch.tensor([0.0 if b == 0 else -math.inf for _ in prompts for b in range(beams)], device="cuda")
    finished = torch.zeros(rows, dtype=torch.int32, device="cuda")
    first, shared = i32([i * beams for i in range(groups + 1)]), torch.zeros(groups, dtype=torch.int32, device="cuda")
    history = torch.full((rows, steps), -1, dtype=torch.int32, device="cuda")
    ws, bws = B.SharedWorkspace(desc, heads, rows, groups, 16 * wide), B.BeamWorkspace(groups, beams, vocab, beams)
    out = torch.zeros((rows, heads, dh), device="cuda")
    parents, new_scores, new_finished, new_tokens = (torch.zeros(rows, dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int32, torch.int32))
    row_ids = torch.arange(rows, dtype=torch.int32, device="cuda")
    for step in range(steps):
        t = sets[at]
        B.ee_kv_pages_grow(pool, t, t.lens + 1, moves, missing)
        B.ee_kv_copy(desc, cache, moves)
        cache_tokens(t, row_ids, t.lens, tokens)
        B.ee_kv_pages_shared(B.PageTables(t.block_tables, t.lens + 1), first, shared)
        batch = B.make_batch(None, t.lens, t.block_tables, 16 * wide)
        B.ee_paged_attention_shared(desc, cache, 1, qd[tokens.long()].contiguous(), batch, B.make_prefix_groups(first, shared, wide), out, ws)
        t.lens.add_(1)
        logits = out.view(rows, -1) @ head
        B.ee_beam_select(logits, scores, beams, new_tokens, parents, new_scores, bws, finished=finished, finished_out=new_finished, end_token=end)
        new_history = torch.full_like(history, -1)
        B.ee_reorder_rows(history, parents, new_history)
        history = new_history
        history[:, step] = new_tokens
        B.ee_kv_pages_fork(pool, t, parents, sets[1 - at], release=True)
        at = 1 - at
        scores.copy_(new_scores)
        finished.copy_(new_finished)
        tokens = new_tokens.clone()
        assert missing.item() == 0
        want = [h for group in told[step] for h in group]
        assert history[:, :step + 1].tolist() == [h[0] for h in want]
        assert finished.tolist() == [int(h[2]) for h in want]
        assert max(abs(a - h[1]) for a, h in zip(scores.tolist(), want)) < 1e-3
    used = {int(b) for row, n in zip(sets[at].block_tables.tolist(), sets[at].lens.tolist()) for b in row[:O.blocks_of(n)]}
    assert {i for i, r in enumerate(pool.refs.tolist()) if r > 0} == used
    B.ee_kv_pages_release(pool, sets[at])
    assert not bool(pool.refs.any())
