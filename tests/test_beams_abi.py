"""Refusals of the entry points for several continuations of a prompt, on the host (nothing is launched), and what their workspace sizes promise."""
import ctypes as C

import pytest

from paper_2407_20272_amd import binding as B

P = 4096   # an aligned address nobody reads
Q = 1 << 30
FAR = 1 << 33
INVALID, SHAPE, UNSUPPORTED, WORKSPACE, OK = B.EE_ERR_INVALID_ARG, B.EE_ERR_SHAPE, B.EE_ERR_UNSUPPORTED, B.EE_ERR_WORKSPACE, B.EE_OK


def ref(x):
    return C.byref(x) if x is not None else None


def tables(at=P, lens=FAR, rows=4, blocks=8):
    return B.ee_page_tables(at, lens, rows, blocks)


def desc(**kw):
    d = dict(n_layers=2, d_model=256, n_heads=4, head_dim=64, d_ffn=1024, vocab=2048, dtype=B.EE_BF16, rms_eps=1e-5, rope_theta=1e4, exit_every=1,
             logit_scale=4.0, conf_mode=0)
    d.update(kw)
    return B.ee_model_desc(**d)


# ---- pages ----------------------------------------------------------------------------------------------------------
def fork(refs=P, n=10, src=tables(), parents=2 * FAR, dst=tables(3 * FAR, 4 * FAR), release=0):
    return B.lib().ee_kv_pages_fork(refs, n, ref(src), parents, ref(dst), release, None)


def release(refs=P, n=10, t=tables()):
    return B.lib().ee_kv_pages_release(refs, n, ref(t), None)


def grow(refs=P, n=10, t=tables(), new=2 * FAR, moves=3 * FAR, missing=4 * FAR, ws=P, size=1 << 30):
    return B.lib().ee_kv_pages_grow(refs, n, ref(t), new, moves, missing, ws, size, None)


def compact(refs=P, n=10, t=tables(), remap=2 * FAR, moves=3 * FAR, count=4 * FAR, ws=P, size=1 << 30):
    return B.lib().ee_kv_pages_compact(refs, n, ref(t), remap, moves, count, ws, size, None)


def shared(t=tables(), first=2 * FAR, groups=3, out=3 * FAR):
    return B.lib().ee_kv_pages_shared(ref(t), first, groups, out, None)


@pytest.mark.parametrize("call", [fork, release, grow, compact])
def test_pools_that_are_refused(call):
    assert call(refs=None) == INVALID and call(refs=P + 2) == INVALID
    assert call(n=0) == INVALID and call(n=-1) == INVALID and call(n=(1 << 23) + 1) == UNSUPPORTED


@pytest.mark.parametrize("call,name", [(fork, "src"), (fork, "dst"), (release, "t"), (grow, "t"), (compact, "t"), (shared, "t")])
def test_tables_that_are_refused(call, name):
    for bad, rc in [(tables(at=None), INVALID), (tables(lens=None), INVALID), (tables(at=P + 1), INVALID), (tables(lens=FAR + 2), INVALID),
                    (tables(rows=-1), INVALID), (tables(rows=1 << 21), UNSUPPORTED), (tables(blocks=0), INVALID), (tables(blocks=1 << 24), UNSUPPORTED), (tables(rows=1 << 12, blocks=(1 << 18) + 1), UNSUPPORTED)]:
        assert call(**{name: bad}) == rc, B.ee_last_error()
    if call is not compact:
        assert call(**{name: None}) == INVALID


def test_fork_refuses():
    assert fork(parents=None) == INVALID and fork(parents=2 * FAR + 1) == INVALID and fork(release=2) == INVALID
    assert fork(dst=tables(3 * FAR, 4 * FAR, 4, 7)) == SHAPE
    assert fork(dst=tables()) == INVALID and "overlap" in B.ee_last_error()
    assert fork(dst=tables(P + 4 * 8 * 4 - 4, 4 * FAR)) == INVALID
    assert fork(dst=tables(3 * FAR, FAR + 8)) == INVALID and fork(dst=tables(FAR - 64, 4 * FAR)) == INVALID
    assert fork(parents=3 * FAR + 4) == INVALID
    assert fork(src=tables(rows=0), dst=tables(rows=0), parents=None) == OK


def test_grow_and_compact_refuse():
    for name in ("new", "moves", "missing"):
        assert grow(**{name: None}) == INVALID and grow(**{name: 2 * FAR + 2}) == INVALID
    assert grow(moves=2 * FAR + 8) == INVALID and grow(moves=FAR) == INVALID and grow(missing=FAR + 4) == INVALID and grow(missing=2 * FAR) == INVALID
    for name in ("remap", "moves", "count"):
        assert compact(**{name: None}) == INVALID and compact(**{name: 2 * FAR + 2}) == INVALID
    assert compact(remap=P + 8) == INVALID and compact(moves=2 * FAR + 4) == INVALID and compact(moves=P - 16) == INVALID
    for call in (grow, compact):
        assert call(ws=None) == WORKSPACE and call(ws=P + 64) == WORKSPACE and call(size=100) == WORKSPACE


def test_shared_refuses():
    assert shared(groups=-1) == INVALID and shared(first=None) == INVALID and shared(out=None) == INVALID and shared(first=2 * FAR + 1) == INVALID
    assert shared(out=2 * FAR + 12) == INVALID
    assert shared(groups=0, first=None, out=None) == OK


def test_copies_refuse():
    L = B.lib()

    def plain(d=desc(), c=B.ee_kv_cache(P, P, 10, 16), moves=P, n=3, count=None):
        return L.ee_kv_copy(ref(d), ref(c), moves, n, count, None)

    def quant(c=B.ee_quant_cache(P, P, P, 2, 8, 16, 4, 64, B.EE_QUANT_INT8), moves=P, n=3, count=None):
        return L.ee_kv_quant_copy(ref(c), moves, n, count, None)

    for call in (plain, quant):
        assert call(c=None) == INVALID and call(moves=None) == INVALID and call(moves=P + 2) == INVALID and call(count=P + 1) == INVALID and call(n=-1) == INVALID
        assert call(n=0, moves=None) == OK
    assert plain(d=None) == INVALID and plain(d=desc(head_dim=32, n_heads=8)) == UNSUPPORTED and plain(c=B.ee_kv_cache(P, P, 10, 32)) == UNSUPPORTED
    assert plain(c=B.ee_kv_cache(P + 8, P, 10, 16)) == INVALID and plain(c=B.ee_kv_cache(P, P + 2, 10, 16)) == INVALID
    assert quant(c=B.ee_quant_cache(P, P, P, 2, 8, 16, 4, 72, B.EE_QUANT_INT8)) == UNSUPPORTED


def test_page_workspaces():
    L = B.lib()
    assert L.ee_kv_pages_bytes(0, 4) == 0 and L.ee_kv_pages_bytes((1 << 23) + 1, 4) == 0 and L.ee_kv_pages_bytes(5, -1) == 0 and L.ee_kv_pages_bytes(5, 1 << 21) == 0
    last = 0
    for n in list(range(1, 4000, 37)) + [1 << 20, 1 << 23]:
        now = L.ee_kv_pages_bytes(n, 10)
        assert now >= last > -1 and L.ee_kv_pages_bytes(n, 1000) >= now >= L.ee_kv_pages_bytes(n, 0) > 0
        last = now


# ---- beams ----------------------------------------------------------------------------------------------------------
def select(z=P, stride=100, dtype=B.EE_FP32, scores=FAR, fin=None, groups=2, beams=3, vocab=100, n=3, end=-1, tok=2 * FAR, par=3 * FAR, out=4 * FAR, fout=None,
           ws=P, size=1 << 30):
    return B.lib().ee_beam_select(z, stride, dtype, scores, fin, groups, beams, vocab, n, end, tok, par, out, fout, ws, size, None)


def test_selection_refuses():
    assert select(dtype=2) == INVALID and select(z=None) == INVALID and select(z=P + 2) == INVALID and select(z=P + 1, dtype=B.EE_BF16) == INVALID
    assert select(stride=99) == SHAPE and select(stride=1 << 61) == SHAPE
    for name in ("groups", "beams", "vocab", "n"):
        assert select(**{name: -1}) == INVALID
    assert select(beams=0) == INVALID and select(vocab=0) == INVALID and select(n=0) == INVALID
    assert select(beams=129) == UNSUPPORTED and select(n=129) == UNSUPPORTED and select(vocab=(1 << 24) + 1, stride=1 << 25) == UNSUPPORTED
    assert select(groups=65536, beams=1) == UNSUPPORTED
    assert select(vocab=1, beams=2, n=3) == SHAPE
    assert select(end=100) == INVALID and select(end=-2) == INVALID and select(fin=5 * FAR) == INVALID and "end_token" in B.ee_last_error()
    for name in ("scores", "tok", "par", "out"):
        assert select(**{name: None}) == INVALID and select(**{name: 9 * FAR + 2}) == INVALID
    assert select(fin=5 * FAR + 1, end=2) == INVALID and select(fout=5 * FAR + 2) == INVALID
    assert select(tok=FAR + 20) == INVALID and select(out=FAR) == INVALID and select(fin=5 * FAR, end=1, par=5 * FAR + 4) == INVALID
    assert select(par=2 * FAR + 8) == INVALID and select(fout=4 * FAR - 4) == INVALID and "each other" in B.ee_last_error()
    assert select(tok=P + 2392) == INVALID and select(scores=P + 64, out=P + 2396) == INVALID and "logits" in B.ee_last_error()
    assert select(ws=None) == WORKSPACE and select(ws=P + 16) == WORKSPACE and select(size=64) == WORKSPACE
    assert select(groups=0, z=None) == OK


def test_selection_workspaces_cover_smaller_calls():
    L = B.lib()
    assert L.ee_beam_select_bytes(1, 0, 10, 1) == 0 and L.ee_beam_select_bytes(-1, 1, 10, 1) == 0 and L.ee_beam_select_bytes(1, 1, 10, 11) == 0
    for vocab in (5, 3000, 4096, 4097, 32000, 150001):
        last = 0
        for n in range(1, 129):
            now = L.ee_beam_select_bytes(3, 64, vocab, n)
            assert now >= last
            last = now
        assert L.ee_beam_select_bytes(3, 64, vocab, 128) <= L.ee_beam_select_bytes(4, 64, vocab, 128) <= L.ee_beam_select_bytes(4, 65, vocab + 1, 128)


def reorder(x=P, xs=64, rows_in=4, parents=FAR, rows=8, row=64, out=2 * FAR, os=64):
    return B.lib().ee_reorder_rows(x, xs, rows_in, parents, rows, row, out, os, None)


def test_reorder_refuses():
    for name in ("rows_in", "rows", "row"):
        assert reorder(**{name: -1}) == INVALID
    assert reorder(x=None) == INVALID and reorder(out=None) == INVALID and reorder(parents=None) == INVALID and reorder(parents=FAR + 1) == INVALID
    assert reorder(xs=63) == SHAPE and reorder(os=60) == SHAPE and reorder(xs=1 << 62) == SHAPE
    assert reorder(row=1 << 41, xs=1 << 41, os=1 << 41) == UNSUPPORTED and reorder(rows=1 << 24) == UNSUPPORTED
    assert reorder(out=P + 255) == INVALID and reorder(out=P - 8 * 64 + 1) == INVALID and reorder(parents=2 * FAR + 4) == INVALID
    assert reorder(rows=0, x=None) == OK and reorder(row=0) == OK and reorder(rows_in=0) == OK


# ---- attention ------------------------------------------------------------------------------------------------------
def attend(d=desc(), c=B.ee_kv_cache(P, P, 10, 16), layer=1, heads=8, q=P, b=B.ee_batch(2, None, P, P, 4, 33, None), g=B.ee_prefix_groups(1, P, P, 2), out=Q,
           ws=None, size=0):
    return B.lib().ee_paged_attention_shared(ref(d), ref(c), layer, heads, q, ref(b), ref(g), out, ws, size, None)


def batch(rows=2, lens=P, tabs=P, max_blocks=4, max_context=33, row_table=None):
    return B.ee_batch(rows, None, lens, tabs, max_blocks, max_context, row_table)


def test_attention_refuses():
    assert attend(d=None) == INVALID and attend(c=None) == INVALID and attend(b=None) == INVALID and attend(g=None) == INVALID
    assert attend(c=B.ee_kv_cache(P + 8, P, 10, 16)) == INVALID and attend(c=B.ee_kv_cache(P, P + 4, 10, 16)) == INVALID
    assert attend(layer=0) == INVALID and attend(layer=3) == INVALID
    assert attend(heads=6) == SHAPE and attend(heads=0) == SHAPE and attend(heads=1 << 17) == UNSUPPORTED
    assert attend(q=None) == INVALID and attend(out=None) == INVALID and attend(q=P + 4) == INVALID and attend(out=Q + 8) == INVALID
    assert attend(out=P + 64) == INVALID and "overlap" in B.ee_last_error()
    for g in (B.ee_prefix_groups(-1, P, P, 2), B.ee_prefix_groups(1, None, P, 2), B.ee_prefix_groups(1, P, None, 2), B.ee_prefix_groups(1, P + 1, P, 2),
              B.ee_prefix_groups(1, P, P, -1)):
        assert attend(g=g) == INVALID
    assert attend(g=B.ee_prefix_groups(4097, P, P, 2)) == UNSUPPORTED
    assert attend(b=batch(rows=70000), heads=128, d=desc(d_model=64, n_heads=1), out=1 << 40) == UNSUPPORTED
    assert attend(b=batch(max_blocks=20000)) == UNSUPPORTED and attend(b=batch(max_context=65)) == SHAPE and attend(b=batch(lens=None)) == INVALID
    # a long context is divided, and says so without a workspace
    long = batch(rows=1, max_blocks=1000, max_context=16000)
    assert attend(b=long) == WORKSPACE and attend(b=long, ws=P + 64, size=1 << 30) == WORKSPACE and attend(b=long, ws=P, size=512) == WORKSPACE
    assert attend(b=batch(rows=0, lens=None, tabs=None)) == OK and attend(g=B.ee_prefix_groups(0, None, None, 0)) == OK


def test_attention_workspaces_cover_smaller_calls():
    """Sizes never shrink as rows, groups or contexts are added."""
    L = B.lib()
    size = L.ee_paged_attention_shared_bytes
    assert size(None, 8, 4, 1, 100) == 0 and size(ref(desc()), 6, 4, 1, 100) == 0 and size(ref(desc()), 8, 0, 1, 100) == 0
    assert size(ref(desc()), 8, 4, 0, 100) == 0 and size(ref(desc()), 8, 4, 1, 0) == 0 and size(ref(desc()), 8, 4, 1, 16384 * 16 + 1) == 0
    for dtype in (B.EE_BF16, B.EE_FP32):
        for kv, heads in ((4, 8), (1, 64), (32, 32), (8, 32), (1, 17), (5, 35)):
            d = desc(d_model=64 * kv, n_heads=kv, dtype=dtype)
            for along in (lambda x: size(ref(d), heads, x, 3, 20000), lambda x: size(ref(d), heads, 300, x, 5000), lambda x: size(ref(d), heads, 12, 2, 97 * x),
                          lambda x: size(ref(d), heads, x, x, 8000)):
                sizes = [along(x) for x in range(1, 400)]
                assert all(0 < x <= y for x, y in zip(sizes, sizes[1:]))
