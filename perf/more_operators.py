"""Performance cases of decoding several continuations of a prompt: beam selection, pages of a cache that are shared, and the
attention of rows with a long common prefix.

    listed()             the named cases
    draw(rng)            one more case of the same ranges
    prepare(case, seed)  what a serving program holds before the call
    run(state)           one pass and its outputs: plain torch, or with `own` the library's entry points
    work(case)           bytes and operations no implementation of the pass can do without
    exact(case, seed)    the same outputs in float64

A case names its operator in "op":
    attention   ee_paged_attention_shared: one position of every row over a float cache, rows in groups whose first blocks are the same
    select      ee_beam_select over the beams of every group and the vocabulary, and ee_reorder_rows of two states by what it chose
    fork        ee_kv_pages_fork of every prompt into beams, ee_kv_pages_grow for the next positions, ee_kv_copy (or ee_kv_quant_copy) of
                the blocks that are no longer shared, ee_kv_pages_shared, and ee_kv_pages_release of the beams
    compact     ee_kv_pages_compact of a pool with holes, and the copy of the blocks that it moves

Sizes are a case's own: rows of a group, shared lengths and tails run evenly from ..._min to ..._max, tails in an order the seed decides.
"""
import math

import torch

own = False
DEVICE = "cuda"
BLOCK = 16


# ----------------------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # The first steps of one beam search over a short prompt on the 7B shape: nothing but latency.
        dict(name="attention_beams_short", op="attention", groups=1, rows_min=4, rows_max=4, shared_min=96, shared_max=96, tail_min=1,
             tail_max=12, padding=0, heads=32, kv_heads=32, head_dim=128, dtype="bf16"),
        # Eight beam searches of four beams over prompts of the headline length.
        dict(name="attention_beams_7b", op="attention", groups=8, rows_min=4, rows_max=4, shared_min=512, shared_max=512, tail_min=1,
             tail_max=64, padding=0, heads=32, kv_heads=32, head_dim=128, dtype="bf16"),
        # Conversations that start with one long instruction, grouped K/V heads.
        dict(name="attention_instruction_b64", op="attention", groups=1, rows_min=64, rows_max=64, shared_min=2000, shared_max=2000, tail_min=100,
             tail_max=900, padding=0, heads=32, kv_heads=8, head_dim=128, dtype="bf16"),
        # A dozen questions about one very long document.
        dict(name="attention_document_100k", op="attention", groups=1, rows_min=12, rows_max=12, shared_min=100000, shared_max=100000,
             tail_min=10, tail_max=200, padding=0, heads=32, kv_heads=8, head_dim=128, dtype="bf16"),
        # Groups of all sizes on a float cache, some of them alone, rows of a padded batch at the end.
        dict(name="attention_fp32_ragged", op="attention", groups=7, rows_min=1, rows_max=9, shared_min=0, shared_max=300, tail_min=1,
             tail_max=150, padding=3, heads=12, kv_heads=4, head_dim=64, dtype="fp32"),
        # One beam search over a small vocabulary.
        dict(name="select_b1_w4", op="select", groups=1, beams=4, n_out=4, vocab=2048, dtype="fp32", pad=0, finished=0.0, masked=0.0,
             steps=16, width=256),
        # A batch of beam searches on the 7B shape: twice the beams come back, so that those that end can be put aside.
        dict(name="select_b32_w4", op="select", groups=32, beams=4, n_out=8, vocab=32000, dtype="bf16", pad=0, finished=0.1, masked=0.0,
             steps=100, width=4096),
        # A large odd vocabulary, rows padded to a multiple, some beams done, most tokens forbidden by a grammar.
        dict(name="select_b16_w8_odd", op="select", groups=16, beams=8, n_out=16, vocab=100003, dtype="fp32", pad=61, finished=0.2, masked=0.7,
             steps=500, width=4096),
        # One search as wide as they get.
        dict(name="select_b1_w64", op="select", groups=1, beams=64, n_out=128, vocab=32000, dtype="fp32", pad=0, finished=0.05, masked=0.0,
             steps=60, width=1024),
        # One prompt becomes four beams on a small float model.
        dict(name="fork_b1_w4", op="fork", prompts=1, beams=4, len_min=30, len_max=30, new=1, layers=4, kv_heads=4, head_dim=64,
             cache="fp32", spare=8),
        # Eight prompts become four beams each in a part of a 7B cache.
        dict(name="fork_b8_w4", op="fork", prompts=8, beams=4, len_min=100, len_max=600, new=1, layers=8, kv_heads=32, head_dim=128,
             cache="bf16", spare=40),
        # A pool of the 8-bit cache with holes everywhere, put together again.
        dict(name="compact_e4m3", op="compact", rows=40, len_min=50, len_max=800, holes=0.6, layers=8, kv_heads=8, head_dim=128, cache="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "select", "select", "fork", "compact"])
    if op == "attention":
        kv, dh, dtype = rng.choice([1, 2, 4, 5, 8, 8, 16, 32]), rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "fp32"])
        group = rng.choice([1, 2, 3, 4, 7, 8]) if kv <= 8 else 1
        groups = _log_int(rng, 1, 16)
        rows_max = _log_int(rng, 1, max(1, 128 // groups))
        rows = groups * rows_max
        # what the plain form holds, and no more bytes or products than the listed document
        room = min(4.8e8 / (kv * dh * rows), 4e9 / (rows * kv * group * dh))
        token = kv * 2 * dh * (2 if dtype == "bf16" else 4)
        shared = _log_int(rng, 16, max(16, min(60000, int(0.8 * room), int(3e8 / (groups * token)))))
        tail = _log_int(rng, 1, max(1, min(2000, int(0.2 * room), int(0.8e8 / (rows * token)))))
        return dict(op=op, groups=groups, rows_min=rng.randint(1, rows_max), rows_max=rows_max, shared_min=rng.choice([0, shared // 2, shared]),
                    shared_max=shared, tail_min=rng.randint(1, tail), tail_max=tail, padding=rng.choice([0, 0, 1, 5]), heads=kv * group,
                    kv_heads=kv, head_dim=dh, dtype=dtype)
    if op == "select":
        beams = _log_int(rng, 1, 64)
        groups = _log_int(rng, 1, max(1, 128 // beams))
        vocab = _log_int(rng, 500, min(150000, 12000000 // (beams * groups)))
        return dict(op=op, groups=groups, beams=beams, n_out=rng.choice([beams, 2 * beams]), vocab=vocab, dtype=rng.choice(["bf16", "fp32"]),
                    pad=rng.choice([0, 0, 1, 29]), finished=rng.choice([0.0, 0.0, 0.3]), masked=rng.choice([0.0, 0.0, 0.9]),
                    steps=_log_int(rng, 1, 500), width=_log_int(rng, 16, 4096))
    kv, dh, layers = rng.choice([1, 2, 4, 5, 8, 8, 16, 32]), rng.choice([64, 128, 128]), rng.randint(1, 8)
    cache = rng.choice(["bf16", "fp32", "int8", "e4m3"])
    blocks = max(8, min(1200, int(9e7 / (layers * kv * dh * BLOCK))))
    if op == "fork":
        prompts, beams = _log_int(rng, 1, 8), _log_int(rng, 1, 8)
        new = rng.choice([1, 1, 1, _log_int(rng, 2, 40)])
        most = max(1, (blocks - prompts * beams * (new // BLOCK + 2)) * BLOCK // prompts)
        len_max = _log_int(rng, 16, max(16, min(4000, most)))
        return dict(op=op, prompts=prompts, beams=beams, len_min=rng.randint(0, len_max), len_max=len_max, new=new, layers=layers,
                    kv_heads=kv, head_dim=dh, cache=cache, spare=rng.randint(0, 20))
    rows = _log_int(rng, 1, 64)
    holes = round(rng.uniform(0.0, 0.8), 2)
    len_max = _log_int(rng, 16, max(16, min(4000, int(blocks * (1 - holes)) * BLOCK // rows)))
    return dict(op=op, rows=rows, len_min=rng.randint(0, len_max), len_max=len_max, holes=holes, layers=layers, kv_heads=kv,
                head_dim=dh, cache=cache)


# ----------------------------------------------------------------------------------------------------------------
# what a case says about sizes (the same for every seed)
# ----------------------------------------------------------------------------------------------------------------
def _even(n, lo, hi):
    return [lo + (i * (hi - lo)) // max(1, n - 1) for i in range(n)]


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _sizes(case):
    """Rows of every group, its shared blocks, and the tails of all rows."""
    rows = _even(case["groups"], case["rows_min"], case["rows_max"])
    shared = [n // BLOCK for n in _even(case["groups"], case["shared_min"], case["shared_max"])]
    return rows, shared, _even(sum(rows), case["tail_min"], case["tail_max"])


def _block_bytes(case):
    """Bytes of one block of all layers, K and V."""
    size = {"fp32": 4, "bf16": 2, "int8": 1, "e4m3": 1}[case["cache"]]
    scales = 8 if size == 1 else 0
    return case["layers"] * case["kv_heads"] * (2 * BLOCK * case["head_dim"] * size + scales)


def work(case):
    if case["op"] == "attention":
        rows, shared, tails = _sizes(case)
        size = 2 if case["dtype"] == "bf16" else 4
        cached = sum(s * BLOCK for s in shared) + sum(tails)
        attended = sum(r * s * BLOCK for r, s in zip(rows, shared)) + sum(tails)
        b = cached * case["kv_heads"] * 2 * case["head_dim"] * size + 2 * sum(rows) * case["heads"] * case["head_dim"] * 4
        return {"bytes": b + 4 * (sum(shared) + sum(map(_blocks, tails))), "flops": 4 * case["heads"] * case["head_dim"] * attended}
    if case["op"] == "select":
        rows, outs = case["groups"] * case["beams"], case["groups"] * case["n_out"]
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": rows * case["vocab"] * size + 2 * outs * 4 * (case["steps"] + case["width"]) + 16 * outs + 8 * rows, "flops": 4 * rows * case["vocab"]}
    if case["op"] == "fork":
        lens = _even(case["prompts"], case["len_min"], case["len_max"])
        copied = sum(case["beams"] for n in lens if n % BLOCK)
        entries = sum(map(_blocks, lens)) * (1 + case["beams"])
        return {"bytes": 2 * copied * _block_bytes(case) + 8 * entries + 8 * len(lens) * (1 + case["beams"]), "flops": 4 * entries}
    lens = _even(case["rows"], case["len_min"], case["len_max"])
    live = sum(map(_blocks, lens))
    pool = _pool(case)
    moved = live * max(0, pool - live) / pool   # as many live blocks as lie behind the live ones' number, about
    return {"bytes": 2 * moved * _block_bytes(case) + 4 * pool * 4 + 8 * live, "flops": 4 * pool}


def _pool(case):
    """Blocks of the pool of a compaction."""
    return max(1, math.ceil(sum(map(_blocks, _even(case["rows"], case["len_min"], case["len_max"]))) / (1 - case["holes"]))) + 1


# ----------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------
def _generators(seed):
    host, dev = torch.Generator(), torch.Generator(device=DEVICE)
    host.manual_seed(int(seed))
    dev.manual_seed(int(seed))
    return host, dev


def _int32(values):
    return torch.tensor(values, dtype=torch.int32).to(DEVICE)


def _randn(shape, dev, dtype):
    return torch.randn(shape, generator=dev, device=DEVICE, dtype=torch.float32 if dtype == torch.float32 else torch.bfloat16)


def _cache(s, num_blocks, layers, dev):
    """Pools of random values: float [layers][blocks][heads][16][dh], or bytes with scales (V [layers][blocks][heads][dh][16])."""
    c = s["case"]
    kind, kv, dh = c.get("cache", c.get("dtype")), c["kv_heads"], c["head_dim"]
    shape = (layers, num_blocks, kv, BLOCK, dh)
    if kind in ("fp32", "bf16"):
        t = torch.float32 if kind == "fp32" else torch.bfloat16
        s["k"], s["v"] = _randn(shape, dev, t), _randn(shape, dev, t)
        return
    for name, dims in (("k", shape), ("v", (layers, num_blocks, kv, dh, BLOCK))):
        b = torch.randint(-120 if kind == "int8" else 0, 120, dims, generator=dev, device=DEVICE, dtype=torch.int8)   # (as e4m3: 0 to 240)
        s[name] = b if kind == "int8" else b.view(torch.float8_e4m3fn)
    s["scales"] = torch.exp2(torch.randint(-10, -4, (layers, num_blocks, kv, 2), generator=dev, device=DEVICE).float())


def _prepare_attention(s, host, dev):
    c = s["case"]
    rows, shared, tails = _sizes(c)
    tails = [tails[i] for i in torch.randperm(len(tails), generator=host).tolist()]
    need = sum(shared) + sum(map(_blocks, tails))
    pool = need + 3
    order = torch.randperm(pool, generator=host).to(torch.int32)
    wide = max(1, max(s + _blocks(t) for n, s, i in zip(rows, shared, range(len(rows))) for t in tails[sum(rows[:i]):sum(rows[:i]) + n]))
    n_rows = len(tails) + c["padding"]
    tables, lens, used, m = torch.full((n_rows, wide), -1, dtype=torch.int32), [], 0, 0
    for n, blocks in zip(rows, shared):
        common = order[used:used + blocks]
        used += blocks
        for _ in range(n):
            own_blocks = _blocks(tails[m])
            tables[m, :blocks] = common
            tables[m, blocks:blocks + own_blocks] = order[used:used + own_blocks]
            used += own_blocks
            lens.append(blocks * BLOCK + tails[m] - 1)
            m += 1
    first = [sum(rows[:i]) for i in range(len(rows))] + [n_rows]   # (padded rows belong to the last group)
    s.update(tables=tables.to(DEVICE), lens=_int32(lens + [-1] * c["padding"]), first=_int32(first), shared=_int32(shared),
             max_shared=max(shared), max_context=max(lens) + 1)
    _cache(s, pool, 1, dev)
    s["q"] = torch.randn((n_rows, c["heads"], c["head_dim"]), generator=dev, device=DEVICE).mul_(1.5)
    s["out"] = torch.empty_like(s["q"])


def _prepare_select(s, host, dev):
    c = s["case"]
    rows, outs = c["groups"] * c["beams"], c["groups"] * c["n_out"]
    t = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    z = torch.randn((rows, c["vocab"] + c["pad"]), generator=dev, device=DEVICE).mul_(3.0)
    if c["masked"]:
        z.masked_fill_(torch.rand(z.shape, generator=dev, device=DEVICE) < c["masked"], -math.inf)
    s["logits"] = z.to(t)[:, :c["vocab"]]
    s["scores"] = torch.randn(rows, generator=dev, device=DEVICE).mul_(1.5).sub_(20.0)
    s["finished"] = (torch.rand(rows, generator=dev, device=DEVICE) < c["finished"]).int() if c["finished"] else None
    s["end"] = 2
    s["history"] = torch.randint(0, c["vocab"], (rows, c["steps"]), generator=dev, device=DEVICE, dtype=torch.int32)
    s["hidden"] = torch.randn((rows, c["width"]), generator=dev, device=DEVICE)
    for name in ("tokens", "parents", "finished_out"):
        s[name] = torch.zeros(outs, dtype=torch.int32, device=DEVICE)
    s["scores_out"] = torch.zeros(outs, device=DEVICE)
    s["history_out"] = torch.zeros((outs, c["steps"]), dtype=torch.int32, device=DEVICE)
    s["hidden_out"] = torch.zeros((outs, c["width"]), device=DEVICE)


def _prepare_fork(s, host, dev):
    c = s["case"]
    lens = _even(c["prompts"], c["len_min"], c["len_max"])
    lens = [lens[i] for i in torch.randperm(len(lens), generator=host).tolist()]
    used, beams = sum(map(_blocks, lens)), c["prompts"] * c["beams"]
    pool = used + beams * (c["new"] // BLOCK + 2) + c["spare"]
    order, at = torch.randperm(pool, generator=host).to(torch.int32), 0
    wide = _blocks(max(lens) + c["new"])
    tables = torch.full((len(lens), wide), -1, dtype=torch.int32)
    for i, n in enumerate(lens):
        tables[i, :_blocks(n)] = order[at:at + _blocks(n)]
        at += _blocks(n)
    refs = torch.zeros(pool, dtype=torch.int32)
    refs[order[:used].long()] = 1
    s.update(refs=refs.to(DEVICE), tables=tables.to(DEVICE), lens=_int32(lens), parents=_int32([i for i in range(len(lens)) for _ in range(c["beams"])]),
             new_lens=_int32([n + c["new"] for n in lens for _ in range(c["beams"])]), first=_int32([i * c["beams"] for i in range(len(lens) + 1)]))
    s["beam_tables"] = torch.full((beams, wide), -1, dtype=torch.int32, device=DEVICE)
    s["beam_lens"] = torch.zeros(beams, dtype=torch.int32, device=DEVICE)
    s["moves"] = torch.full((beams, 2), -1, dtype=torch.int32, device=DEVICE)
    s["missing"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    s["shared"] = torch.zeros(len(lens), dtype=torch.int32, device=DEVICE)
    _cache(s, pool, c["layers"], dev)


def _prepare_compact(s, host, dev):
    c = s["case"]
    lens = _even(c["rows"], c["len_min"], c["len_max"])
    lens = [lens[i] for i in torch.randperm(len(lens), generator=host).tolist()]
    pool, used = _pool(c), sum(map(_blocks, lens))
    order, at = torch.randperm(pool, generator=host).to(torch.int32), 0
    tables = torch.full((len(lens), max(1, _blocks(max(lens)))), -1, dtype=torch.int32)
    for i, n in enumerate(lens):
        tables[i, :_blocks(n)] = order[at:at + _blocks(n)]
        at += _blocks(n)
    refs = torch.zeros(pool, dtype=torch.int32)
    refs[order[:used].long()] = 1
    s.update(refs_before=refs.to(DEVICE), tables_before=tables.to(DEVICE), lens=_int32(lens))
    s["refs"], s["tables"] = s["refs_before"].clone(), s["tables_before"].clone()
    s["remap"] = torch.full((pool,), -1, dtype=torch.int32, device=DEVICE)
    s["moves"] = torch.full((pool, 2), -1, dtype=torch.int32, device=DEVICE)
    s["n_moves"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    _cache(s, pool, c["layers"], dev)


def prepare(case, seed):
    host, dev = _generators(seed)
    s = dict(case=case)
    {"attention": _prepare_attention, "select": _prepare_select, "fork": _prepare_fork, "compact": _prepare_compact}[case["op"]](s, host, dev)
    if own:
        s["handle"] = _handle(s)
    return s


# ----------------------------------------------------------------------------------------------------------------
# the library's calls
# ----------------------------------------------------------------------------------------------------------------
def _handle(s):
    """The records a program keeps beside its cache, its tables and its workspaces."""
    from paper_2407_20272_amd import binding as B
    from paper_2407_20272_amd import workloads as W
    c, h = s["case"], dict(B=B)
    if c["op"] == "select":
        h["ws"] = B.BeamWorkspace(c["groups"], c["beams"], c["vocab"], c["n_out"])
        return h
    kind = c.get("cache", c.get("dtype"))
    if kind in ("fp32", "bf16"):
        cfg = W.CONFIGS[0].with_(n_layers=s["k"].shape[0], d_model=c["kv_heads"] * c["head_dim"], n_heads=c["kv_heads"], head_dim=c["head_dim"], dtype=kind)
        h["desc"], h["cache"] = B.make_desc(cfg), B.PagedKV.of(cfg, s["k"], s["v"])
    else:
        h["cache"] = B.QuantKV.of(s["k"], s["v"], s["scales"])
    if c["op"] == "attention":
        h["batch"] = B.make_batch(None, s["lens"], s["tables"], s["max_context"])
        h["groups"] = B.make_prefix_groups(s["first"], s["shared"], s["max_shared"])
        h["ws"] = B.SharedWorkspace(h["desc"], c["heads"], len(s["lens"]), c["groups"], s["max_context"])
        return h
    h["pool"] = B.PagePool.of(s["refs"], max_rows=max(len(s["lens"]), len(s.get("beam_lens", ()))))
    h["tables"] = B.PageTables(s["tables"], s["lens"])
    if c["op"] == "fork":
        h["beams"] = B.PageTables(s["beam_tables"], s["beam_lens"])
    return h


def _copy(h, moves, count=None):
    B = h["B"]
    if "desc" in h:
        B.ee_kv_copy(h["desc"], h["cache"], moves, count)
    else:
        B.ee_kv_quant_copy(h["cache"], moves, count)


def _run_own(s):
    c, h = s["case"], s["handle"]
    B = h["B"]
    if c["op"] == "attention":
        B.ee_paged_attention_shared(h["desc"], h["cache"], 1, s["q"], h["batch"], h["groups"], s["out"], h["ws"])
        return {"out": s["out"]}
    if c["op"] == "select":
        B.ee_beam_select(s["logits"], s["scores"], c["beams"], s["tokens"], s["parents"], s["scores_out"], h["ws"], finished=s["finished"],
                         finished_out=s["finished_out"], end_token=s["end"])
        B.ee_reorder_rows(s["history"], s["parents"], s["history_out"])
        B.ee_reorder_rows(s["hidden"], s["parents"], s["hidden_out"])
        return {n: s[n] for n in ("tokens", "parents", "scores_out", "finished_out", "history_out", "hidden_out")}
    pools = {n: s[n] for n in ("k", "v", "scales") if n in s}
    if c["op"] == "fork":
        B.ee_kv_pages_fork(h["pool"], h["tables"], s["parents"], h["beams"])
        B.ee_kv_pages_grow(h["pool"], h["beams"], s["new_lens"], s["moves"], s["missing"])
        _copy(h, s["moves"])
        s["beam_lens"].copy_(s["new_lens"])       # (a program does so when the positions are cached)
        B.ee_kv_pages_shared(h["beams"], s["first"], s["shared"])
        B.ee_kv_pages_release(h["pool"], h["beams"])
        return {**pools, **{n: s[n] for n in ("refs", "beam_tables", "beam_lens", "moves", "missing", "shared")}}
    s["refs"].copy_(s["refs_before"])
    s["tables"].copy_(s["tables_before"])
    B.ee_kv_pages_compact(h["pool"], h["tables"], s["remap"], s["moves"], s["n_moves"])
    _copy(h, s["moves"], s["n_moves"])
    return {**pools, **{n: s[n] for n in ("refs", "tables", "remap", "moves", "n_moves")}}


# ----------------------------------------------------------------------------------------------------------------
# the plain form
# ----------------------------------------------------------------------------------------------------------------
def _attention(s):
    c = s["case"]
    n, h, kv, dh = len(s["lens"]), c["heads"], c["kv_heads"], c["head_dim"]
    blk = s["tables"].clamp(min=0).long()
    ctx = blk.shape[1] * BLOCK
    seen = torch.arange(ctx, device=DEVICE)[None, :] <= s["lens"][:, None]                       # [n][ctx]
    k = s["k"][0][blk].float().transpose(1, 2).reshape(n, kv, ctx, dh)
    z = torch.matmul(s["q"].view(n, kv, h // kv, dh), k.transpose(-1, -2).contiguous()).div_(math.sqrt(dh))
    del k
    z = torch.where(seen[:, None, None, :], z, -math.inf)
    e = torch.where(seen[:, None, None, :], torch.exp(z - z.amax(-1, keepdim=True)), 0.0)
    total = e.sum(-1, keepdim=True)
    v = s["v"][0][blk].float().transpose(1, 2).reshape(n, kv, ctx, dh)
    v = torch.where(seen[:, None, :, None], v, 0.0)
    out = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    return {"out": out.reshape(n, h, dh)}


def _select(s):
    c = s["case"]
    g, w, vocab, n = c["groups"], c["beams"], c["vocab"], c["n_out"]
    z = s["logits"].double()                       # next to a border 32 bits would choose by their rounding
    most = z.amax(-1, keepdim=True)
    lse = most + torch.log(torch.exp(z - most).sum(-1, keepdim=True))
    score = s["scores"].double()[:, None] + (z - lse)
    if s["finished"] is not None:
        done = s["finished"][:, None] != 0
        ends = torch.arange(vocab, device=DEVICE)[None, :] == s["end"]
        score = torch.where(done, torch.where(ends, s["scores"].double()[:, None], -math.inf), score)
    score = torch.where(torch.isfinite(score), score, -math.inf)
    best, at = torch.sort(score.view(g, w * vocab), dim=-1, descending=True, stable=True)
    best, at = best[:, :n], at[:, :n]
    parents = (at // vocab + torch.arange(g, device=DEVICE)[:, None] * w).reshape(-1)
    tokens = (at % vocab).reshape(-1)
    finished = tokens == s["end"]
    if s["finished"] is not None:
        finished = finished | (s["finished"][parents] != 0)
    return {"tokens": tokens.int(), "parents": parents.int(), "scores_out": best.reshape(-1).float(), "finished_out": finished.int(),
            "history_out": s["history"][parents], "hidden_out": s["hidden"][parents]}


def _copied(s, src, dst, there):
    """Blocks src -> dst of all layers, where there is one."""
    a, b = src[there].long(), dst[there].long()
    for name in ("k", "v", "scales"):
        if name in s:
            x = s[name].view(torch.int8) if s[name].dtype == torch.float8_e4m3fn else s[name]
            x[:, b] = x[:, a]


def _fork(s):
    c = s["case"]
    refs, wide, pool = s["refs"], s["tables"].shape[1], len(s["refs"])
    parents, entry = s["parents"].long(), torch.arange(s["tables"].shape[1], device=DEVICE)[None, :]
    # fork
    lens = s["lens"][parents]
    has = entry < ((lens + BLOCK - 1) // BLOCK)[:, None]
    s["beam_tables"].copy_(torch.where(has, s["tables"][parents], s["beam_tables"]))
    s["beam_lens"].copy_(lens)
    t = s["beam_tables"]
    refs.scatter_add_(0, torch.where(has, t, 0).flatten().long(), has.flatten().int())
    # grow
    old, new = (lens + BLOCK - 1) // BLOCK, (s["new_lens"] + BLOCK - 1) // BLOCK
    at = (lens // BLOCK)[:, None]
    writes = (lens % BLOCK > 0) & (s["new_lens"] > lens)
    last = torch.gather(t, 1, at.clamp(max=wide - 1).long())[:, 0]
    row = torch.arange(len(lens), device=DEVICE)
    named = torch.where(writes, last, pool).long()
    claims = torch.zeros(pool + 1, dtype=torch.int32, device=DEVICE).scatter_add_(0, named, writes.int())
    latest = torch.full((pool + 1,), -1, dtype=torch.int64, device=DEVICE).scatter_reduce_(0, named, row, "amax")
    count = torch.cat([refs, refs.new_zeros(1)])[named]
    replace = writes & (count > 1) & ~((claims[named] == count) & (latest[named] == row))
    fresh = (entry >= old[:, None]) & (entry < new[:, None])
    wants = fresh | ((entry == at) & replace[:, None])
    rank = torch.cumsum(wants.flatten(), 0) - 1
    free = torch.argsort((refs > 0).int(), stable=True)
    missing = (rank[-1] + 1 - (refs <= 0).sum()).clamp(min=0)
    wants, replace = wants & (missing == 0), replace & (missing == 0)
    block = free[rank.clamp(min=0, max=pool - 1)].view(wants.shape).int()
    s["moves"][:, 0] = torch.where(replace, last, -1)
    s["moves"][:, 1] = torch.where(replace, torch.gather(block, 1, at.clamp(max=wide - 1).long())[:, 0], -1)
    t.copy_(torch.where(wants, block, t))
    refs.scatter_add_(0, torch.where(replace, last, 0).long(), -replace.int())
    refs.scatter_add_(0, torch.where(wants, block, 0).flatten().long(), wants.flatten().int())
    s["missing"].copy_(missing.view(1).int())
    _copied(s, s["moves"][:, 0], s["moves"][:, 1], replace)
    # leading blocks that a prompt's beams share
    same = t.view(c["prompts"], c["beams"], wide)
    same = ((same == same[:, :1]).all(1) & (entry < (s["new_lens"] // BLOCK).view(c["prompts"], c["beams"]).amin(1)[:, None])).int()
    s["shared"].copy_(torch.cumprod(same, 1).sum(1).int())
    # release
    has = entry < new[:, None]
    refs.scatter_add_(0, torch.where(has, t, 0).flatten().long(), -has.flatten().int())
    s["beam_lens"].zero_()
    return {**{n: s[n] for n in ("k", "v", "scales") if n in s}, **{n: s[n] for n in ("refs", "beam_tables", "beam_lens", "moves", "missing", "shared")}}


def _compact(s):
    pool = len(s["refs"])
    s["refs"].copy_(s["refs_before"])
    s["tables"].copy_(s["tables_before"])
    live = s["refs"] > 0
    ids = torch.arange(pool, device=DEVICE)
    n_live = live.sum()
    goes, takes = live & (ids >= n_live), ~live & (ids < n_live)
    src = torch.argsort((~goes).int(), stable=True)
    dst = torch.argsort((~takes).int(), stable=True)
    n = goes.sum()
    there = ids < n
    s["moves"].copy_(torch.where(there[:, None], torch.stack([src, dst], 1), -1).int())
    s["n_moves"].copy_(n.view(1).int())
    remap = torch.where(live, ids, -1)
    remap = torch.cat([remap, remap.new_zeros(1)]).scatter_(0, torch.where(there, src, pool), dst)[:pool]
    s["remap"].copy_(remap.int())
    has = torch.arange(s["tables"].shape[1], device=DEVICE)[None, :] < ((s["lens"] + BLOCK - 1) // BLOCK)[:, None]
    s["tables"].copy_(torch.where(has, s["remap"][torch.where(has, s["tables"], 0).long()], s["tables"]))
    moved = torch.where(there, s["refs"][src], 0)
    s["refs"].copy_(torch.where(goes, 0, s["refs"]))
    s["refs"].scatter_add_(0, torch.where(there, dst, 0), moved)
    _copied(s, src, dst, there)
    return {**{n: s[n] for n in ("k", "v", "scales") if n in s}, **{n: s[n] for n in ("refs", "tables", "remap", "moves", "n_moves")}}


def run(state):
    if own:
        return _run_own(state)
    return {"attention": _attention, "select": _select, "fork": _fork, "compact": _compact}[state["case"]["op"]](state)


# ----------------------------------------------------------------------------------------------------------------
# float64, row by row from the definitions
# ----------------------------------------------------------------------------------------------------------------
def _exact_attention(s):
    c = s["case"]
    h, kv, dh = c["heads"], c["kv_heads"], c["head_dim"]
    out = torch.zeros((len(s["lens"]), h, dh), dtype=torch.float64, device=DEVICE)
    for m, last in enumerate(s["lens"].tolist()):
        if last < 0:
            continue
        blk = s["tables"][m, :last // BLOCK + 1].long()
        for g in range(kv):
            k = s["k"][0, blk, g].double().reshape(-1, dh)[:last + 1]
            v = s["v"][0, blk, g].double().reshape(-1, dh)[:last + 1]
            heads = slice(g * (h // kv), (g + 1) * (h // kv))
            out[m, heads] = torch.softmax(s["q"][m, heads].double() @ k.t() / math.sqrt(dh), -1) @ v
    return {"out": out}


def _exact_select(s):
    c = s["case"]
    g, w, vocab, n = c["groups"], c["beams"], c["vocab"], c["n_out"]
    scores, tokens, parents = [], [], []
    done = s["finished"].cpu().tolist() if s["finished"] is not None else [0] * (g * w)
    base = s["scores"].cpu().double().tolist()
    for i in range(g):
        found = []
        for b in range(i * w, i * w + w):
            if done[b]:
                found.append((-base[b], b, s["end"]))
                continue
            z = s["logits"][b].double()
            lp = z - torch.logsumexp(z, 0)
            top = torch.topk(lp, min(vocab, n + 64))
            found += [(-(base[b] + v), b, t) for v, t in zip(top.values.tolist(), top.indices.tolist()) if math.isfinite(v)]
        found.sort()
        if len(found) < n:
            return None
        scores += [-f[0] for f in found[:n]]
        parents += [f[1] for f in found[:n]]
        tokens += [f[2] for f in found[:n]]
    at = torch.tensor(parents, device=DEVICE)
    ended = [int(t == s["end"] or done[p] != 0) for t, p in zip(tokens, parents)]
    return {"tokens": _int32(tokens), "parents": _int32(parents), "scores_out": torch.tensor(scores, dtype=torch.float64, device=DEVICE),
            "finished_out": _int32(ended), "history_out": s["history"][at], "hidden_out": s["hidden"][at].double()}


def _moved(s, pairs):
    """The pools with blocks of `pairs` copied, as values."""
    out = {}
    for name in ("k", "v", "scales"):
        if name in s:
            x = s[name].clone()
            raw, was = (x.view(torch.int8), s[name].view(torch.int8)) if x.dtype == torch.float8_e4m3fn else (x, s[name])
            for a, b in pairs:
                raw[:, b] = was[:, a]
            out[name] = x
    return out


def _exact_fork(s):
    c = s["case"]
    refs, tables, lens = s["refs"].tolist(), s["tables"].tolist(), s["lens"].tolist()
    beams = [(list(tables[p]), lens[p]) for p in s["parents"].tolist()]
    for t, n in beams:
        for b in t[:_blocks(n)]:
            refs[b] += 1
    new_lens = s["new_lens"].tolist()
    replaced, want = [False] * len(beams), 0
    left = list(refs)
    for i, (t, n) in enumerate(beams):
        if n % BLOCK and new_lens[i] > n and left[t[n // BLOCK]] > 1:   # the rows behind may still want it; the last one may keep it
            replaced[i] = True
            left[t[n // BLOCK]] -= 1
            want += 1
        want += max(0, _blocks(new_lens[i]) - _blocks(n))
    free = [b for b, r in enumerate(refs) if r <= 0]
    missing = max(0, want - len(free))
    moves, taken = [], iter(free)
    for i, (t, n) in enumerate(beams):
        pair = [-1, -1]
        if not missing:
            if replaced[i]:
                pair = [t[n // BLOCK], next(taken)]
                t[n // BLOCK] = pair[1]
            for e in range(_blocks(n), _blocks(new_lens[i])):
                t[e] = next(taken)
        moves.append(pair)
    shared = []
    for p in range(c["prompts"]):
        mine = beams[p * c["beams"]:(p + 1) * c["beams"]]
        k = 0
        full = min(new_lens[p * c["beams"]:(p + 1) * c["beams"]]) // BLOCK
        while k < full and len({t[k] for t, _ in mine}) == 1:
            k += 1
        shared.append(k)
    table = s["beam_tables"].cpu()
    for i, (t, n) in enumerate(beams):
        k = _blocks(new_lens[i])
        table[i, :k] = torch.tensor(t[:k], dtype=torch.int32)
    after = s["refs"].tolist()                     # the beams are released: what there was before
    return {**_moved(s, [m for m in moves if m[0] >= 0]), "refs": _int32(after), "beam_tables": table.to(DEVICE), "beam_lens": torch.zeros_like(s["beam_lens"]),
            "moves": _int32(moves), "missing": _int32([missing]), "shared": _int32(shared)}


def _exact_compact(s):
    refs, tables, lens = s["refs_before"].tolist(), s["tables_before"].tolist(), s["lens"].tolist()
    n = sum(r > 0 for r in refs)
    pairs = list(zip([b for b, r in enumerate(refs) if r > 0 and b >= n], [b for b, r in enumerate(refs) if r <= 0 and b < n]))
    to = {a: b for a, b in pairs}
    remap = [-1 if r <= 0 else to.get(b, b) for b, r in enumerate(refs)]
    after = [0] * len(refs)
    for b, r in enumerate(refs):
        if r > 0:
            after[remap[b]] = r
    moves = [list(p) for p in pairs] + [[-1, -1]] * (len(refs) - len(pairs))
    tables = [[remap[b] if e < _blocks(n) else b for e, b in enumerate(t)] for t, n in zip(tables, lens)]
    return {**_moved(s, pairs), "refs": _int32(after), "tables": _int32(tables), "remap": _int32(remap), "moves": _int32(moves), "n_moves": _int32([len(pairs)])}


def exact(case, seed):
    global own
    was, own = own, False   # inputs only: no handle of the library's
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"attention": _exact_attention, "select": _exact_select, "fork": _exact_fork, "compact": _exact_compact}[case["op"]](s)
