"""Refusals of the 8-bit cache's and the rotary embedding's entry points, on the host (nothing is launched), and what their
workspace sizes promise."""
import ctypes as C

import pytest

from paper_2407_20272_amd import binding as B

P = 4096   # an aligned address nobody reads


def cache(**kw):
    d = dict(k_pool=P, v_pool=P, scales=P, n_layers=2, num_blocks=8, block_size=16, n_kv_heads=4, head_dim=64, format=B.EE_QUANT_INT8)
    d.update(kw)
    return B.ee_quant_cache(**d)


def batch(rows=2, lens=P, tables=P, max_blocks=4, max_context=33, row_table=None, tokens=None):
    return B.ee_batch(rows, tokens, lens, tables, max_blocks, max_context, row_table)


def ref(x):
    return C.byref(x) if x is not None else None


def append(c=cache(), layer=1, k=P, ks=256, v=P, vs=256, dtype=B.EE_FP32, b=batch()):
    return B.lib().ee_kv_quant_append(ref(c), layer, k, ks, v, vs, dtype, ref(b), None)


def read(c=cache(), layer=1, b=batch(), k=P, v=P, dtype=B.EE_FP32):
    return B.lib().ee_kv_quant_read(ref(c), layer, ref(b), k, v, dtype, None)


def attend(c=cache(), layer=1, heads=8, q=P, b=batch(), out=1 << 30, w_in=None, w_out=None, pitch=0, ws=None, size=0):
    return B.lib().ee_paged_attention_quant(ref(c), layer, heads, q, ref(b), out, w_in, w_out, pitch, ws, size, None)


def evict(c=cache(), layer=1, b=batch(), dst=None, dst_blocks=0, w=P, pitch=64, w_out=None, out_pitch=0, keep=20, recent=4, kept=P, lens=1 << 20,
          ws=P, size=1 << 30):
    return B.lib().ee_kv_quant_evict(ref(c), layer, ref(b), dst, dst_blocks, w, pitch, w_out, out_pitch, keep, recent, kept, lens, ws, size, None)


@pytest.mark.parametrize("call", [append, read, attend, evict])
def test_what_every_call_refuses(call):
    assert call(c=None) == B.EE_ERR_INVALID_ARG
    for name in ("k_pool", "v_pool", "scales"):
        assert call(c=cache(**{name: None})) == B.EE_ERR_INVALID_ARG
    assert call(c=cache(k_pool=P + 8)) == B.EE_ERR_INVALID_ARG and "16 bytes" in B.ee_last_error()
    assert call(c=cache(v_pool=P + 1)) == B.EE_ERR_INVALID_ARG
    assert call(c=cache(scales=P + 4)) == B.EE_ERR_INVALID_ARG
    assert call(c=cache(block_size=32)) == B.EE_ERR_UNSUPPORTED
    for name in ("n_layers", "num_blocks", "n_kv_heads"):
        assert call(c=cache(**{name: 0})) == B.EE_ERR_INVALID_ARG
    for dh in (0, 8, 72, 272):
        assert call(c=cache(head_dim=dh)) == B.EE_ERR_UNSUPPORTED and "head_dim" in B.ee_last_error()
    assert call(c=cache(n_kv_heads=5000)) == B.EE_ERR_UNSUPPORTED
    assert call(c=cache(format=2)) == B.EE_ERR_INVALID_ARG
    assert call(layer=0) == B.EE_ERR_INVALID_ARG and call(layer=3) == B.EE_ERR_INVALID_ARG
    assert call(b=None) == B.EE_ERR_INVALID_ARG
    assert call(b=batch(rows=-1)) == B.EE_ERR_INVALID_ARG
    assert call(b=batch(lens=None)) == B.EE_ERR_INVALID_ARG and call(b=batch(tables=None)) == B.EE_ERR_INVALID_ARG
    assert call(b=batch(max_blocks=0)) == B.EE_ERR_INVALID_ARG
    assert call(b=batch(max_blocks=20000)) == B.EE_ERR_UNSUPPORTED
    assert call(b=batch(max_context=65)) == B.EE_ERR_SHAPE and call(b=batch(max_context=0)) == B.EE_ERR_SHAPE
    assert call(b=batch(rows=0, lens=None, tables=None)) == B.EE_OK


def test_append_and_read_refuse():
    for call in (append, read):
        assert call(dtype=2) == B.EE_ERR_INVALID_ARG
        assert call(k=None) == B.EE_ERR_INVALID_ARG and call(v=None) == B.EE_ERR_INVALID_ARG
        assert call(k=P + 4) == B.EE_ERR_INVALID_ARG and call(dtype=B.EE_BF16, v=P + 2) == B.EE_ERR_INVALID_ARG
    assert append(ks=255) == B.EE_ERR_SHAPE and append(vs=254) == B.EE_ERR_SHAPE and append(ks=257) == B.EE_ERR_SHAPE
    assert append(ks=1 << 62) == B.EE_ERR_SHAPE


def test_attention_refuses():
    assert attend(heads=6) == B.EE_ERR_SHAPE and attend(heads=0) == B.EE_ERR_SHAPE
    assert attend(c=cache(n_kv_heads=1), heads=1025) == B.EE_ERR_UNSUPPORTED
    assert attend(q=None) == B.EE_ERR_INVALID_ARG and attend(out=None) == B.EE_ERR_INVALID_ARG and attend(q=P + 4) == B.EE_ERR_INVALID_ARG
    assert attend(q=P, out=P + 64) == B.EE_ERR_INVALID_ARG and "overlap" in B.ee_last_error()
    assert attend(w_in=P) == B.EE_ERR_INVALID_ARG
    assert attend(w_out=P, pitch=64, b=batch(row_table=P)) == B.EE_ERR_UNSUPPORTED
    assert attend(w_out=P, pitch=32) == B.EE_ERR_SHAPE
    assert attend(b=batch(rows=70000)) == B.EE_ERR_UNSUPPORTED
    assert attend(w_in=P, w_out=P + 512, pitch=64) == B.EE_ERR_INVALID_ARG and "overlap" in B.ee_last_error()
    assert attend(w_out=P, pitch=64) == B.EE_ERR_WORKSPACE
    assert attend(w_out=P, pitch=64, ws=P + 128, size=1 << 30) == B.EE_ERR_WORKSPACE and "aligned" in B.ee_last_error()
    assert attend(w_out=P, pitch=64, ws=P, size=64) == B.EE_ERR_WORKSPACE and "needed" in B.ee_last_error()
    # one sequence with a long context is split, and says so without a workspace
    assert attend(b=batch(rows=1, max_blocks=1000, max_context=16000)) == B.EE_ERR_WORKSPACE


def test_eviction_refuses():
    assert evict(keep=0) == B.EE_ERR_INVALID_ARG and evict(recent=-1) == B.EE_ERR_INVALID_ARG and evict(recent=21) == B.EE_ERR_INVALID_ARG
    assert evict(b=batch(row_table=P)) == B.EE_ERR_INVALID_ARG
    for name in ("w", "kept", "lens"):
        assert evict(**{name: None}) == B.EE_ERR_INVALID_ARG
    assert evict(pitch=32) == B.EE_ERR_SHAPE and evict(w_out=1 << 21, out_pitch=19) == B.EE_ERR_SHAPE
    assert evict(w_out=P, out_pitch=63) == B.EE_ERR_SHAPE
    assert evict(dst=P, dst_blocks=1) == B.EE_ERR_SHAPE and evict(dst=P, dst_blocks=-1) == B.EE_ERR_SHAPE
    assert evict(b=batch(rows=70000)) == B.EE_ERR_UNSUPPORTED
    assert evict(lens=P) == B.EE_ERR_INVALID_ARG and "out_lens" in B.ee_last_error()      # (context_lens are there)
    assert evict(lens=P + 4) == B.EE_ERR_INVALID_ARG
    assert evict(w_out=P + 256, out_pitch=64) == B.EE_ERR_INVALID_ARG and "overlap" in B.ee_last_error()
    assert evict(ws=None) == B.EE_ERR_WORKSPACE and evict(ws=P + 16) == B.EE_ERR_WORKSPACE and evict(size=100) == B.EE_ERR_WORKSPACE


def test_workspace_sizes_cover_smaller_calls():
    """A workspace for some sizes serves every call within them: sizes never shrink as rows, context or weights are added."""
    L = B.lib()
    for c, heads in ((cache(), 4), (cache(n_kv_heads=8, head_dim=128), 32), (cache(n_kv_heads=1, head_dim=256), 40)):
        for w in (0, 1):
            def need(rows, ctx):
                return L.ee_paged_attention_quant_bytes(C.byref(c), heads, rows, ctx, w)
            rows, contexts = [1, 2, 3, 7, 16, 33, 64, 200, 500], [1, 63, 64, 65, 257, 1000, 4096, 20000, 262144]
            table = [[need(r, x) for x in contexts] for r in rows]
            assert all(a <= b for line in table for a, b in zip(line, line[1:]))
            assert all(a <= b for up, down in zip(table, table[1:]) for a, b in zip(up, down))
            assert all(x % 256 == 0 for line in table for x in line)
            assert all(x > 0 for line in table for x in line)
    assert L.ee_paged_attention_quant_bytes(None, 8, 1, 64, 0) == 0
    assert L.ee_paged_attention_quant_bytes(C.byref(cache()), 7, 1, 64, 0) == 0 and "n_heads" in B.ee_last_error()
    assert L.ee_paged_attention_quant_bytes(C.byref(cache()), 8, 1, 1 << 20, 0) == 0
    a, b = L.ee_kv_quant_evict_bytes(C.byref(cache()), 4, 100), L.ee_kv_quant_evict_bytes(C.byref(cache()), 4, 1000)
    assert 4 * 4 * 7 * 2 * 16 * 64 <= a < b and L.ee_kv_quant_evict_bytes(C.byref(cache()), 0, 100) == 0


def desc(**kw):
    d = dict(head_dim=64, rotary_dim=64, layout=0, scaling=0, original_context=4096, theta=1e4, factor=2.0, turns_low=1.0, turns_high=4.0,
             amplitude=1.0)
    d.update(kw)
    return B.ee_rotary_desc(**d)


def rows(in_=P, out=1 << 20, in_stride=512, out_stride=512, n_heads=8):
    return B.ee_rotary_rows(in_, out, in_stride, out_stride, n_heads)


def rotate(d=desc(), freqs=P, positions=P, n=4, dtype=B.EE_FP32, q=rows(), k=None, transpose=0):
    return B.lib().ee_rotary(ref(d), freqs, positions, n, dtype, ref(q), ref(k), transpose, None)


@pytest.mark.parametrize("bad,code", [
    (dict(head_dim=1), B.EE_ERR_UNSUPPORTED), (dict(head_dim=2000), B.EE_ERR_UNSUPPORTED), (dict(rotary_dim=63), B.EE_ERR_SHAPE),
    (dict(rotary_dim=66), B.EE_ERR_SHAPE), (dict(rotary_dim=0), B.EE_ERR_SHAPE), (dict(layout=2), B.EE_ERR_INVALID_ARG),
    (dict(scaling=3), B.EE_ERR_INVALID_ARG), (dict(theta=0.0), B.EE_ERR_INVALID_ARG), (dict(theta=float("nan")), B.EE_ERR_INVALID_ARG),
    (dict(scaling=1, factor=0.0), B.EE_ERR_INVALID_ARG), (dict(scaling=2, original_context=0), B.EE_ERR_INVALID_ARG),
    (dict(scaling=2, turns_low=4.0), B.EE_ERR_INVALID_ARG), (dict(amplitude=float("inf")), B.EE_ERR_INVALID_ARG),
])
def test_rotary_descriptions_are_checked(bad, code):
    assert rotate(d=desc(**bad)) == code
    assert B.lib().ee_rotary_frequencies(C.byref(desc(**bad)), P, None) == code


def test_rotary_refuses():
    assert rotate(d=None) == B.EE_ERR_INVALID_ARG and rotate(q=None) == B.EE_ERR_INVALID_ARG
    assert rotate(freqs=None) == B.EE_ERR_INVALID_ARG and rotate(positions=None) == B.EE_ERR_INVALID_ARG and rotate(freqs=P + 4) == B.EE_ERR_INVALID_ARG
    assert rotate(dtype=2) == B.EE_ERR_INVALID_ARG and rotate(n=-1) == B.EE_ERR_INVALID_ARG and rotate(transpose=2) == B.EE_ERR_INVALID_ARG
    assert rotate(n=0, freqs=None, positions=None) == B.EE_OK
    assert rotate(q=rows(in_=None)) == B.EE_ERR_INVALID_ARG and rotate(q=rows(out=None)) == B.EE_ERR_INVALID_ARG
    assert rotate(q=rows(n_heads=0)) == B.EE_ERR_INVALID_ARG and rotate(q=rows(n_heads=9)) == B.EE_ERR_SHAPE
    assert rotate(q=rows(out_stride=511)) == B.EE_ERR_SHAPE and rotate(q=rows(in_stride=1 << 62)) == B.EE_ERR_SHAPE
    assert rotate(k=rows(in_=P + 2)) == B.EE_ERR_INVALID_ARG and "k" in B.ee_last_error()
    # results over other rows' inputs
    assert rotate(q=rows(in_=P, out=P + 4)) == B.EE_ERR_INVALID_ARG and "overlap" in B.ee_last_error()
    assert rotate(q=rows(in_=P, out=P + 2048)) == B.EE_ERR_INVALID_ARG
    assert rotate(q=rows(in_=P, out=P, in_stride=512, out_stride=600)) == B.EE_ERR_INVALID_ARG
    assert rotate(q=rows(in_=P, out=P + 2048, in_stride=512, out_stride=600)) == B.EE_ERR_INVALID_ARG
    assert rotate(q=rows(in_=P, out=P + 1024, in_stride=1024, out_stride=1024)) == B.EE_ERR_INVALID_ARG
    assert B.lib().ee_rotary_frequencies(None, P, None) == B.EE_ERR_INVALID_ARG
    assert B.lib().ee_rotary_frequencies(C.byref(desc()), None, None) == B.EE_ERR_INVALID_ARG


def test_rotary_refuses_results_over_the_other_side():
    far = 1 << 24

    def both(q_in, q_out, k_in, k_out, stride=1024, n=4, q_heads=8, k_heads=4):
        return rotate(n=n, q=rows(q_in, q_out, stride, stride, q_heads), k=rows(k_in, k_out, stride, stride, k_heads))
    for bad in (dict(q_in=P, q_out=far, k_in=far, k_out=2 * far), dict(q_in=P, q_out=far, k_in=2 * far, k_out=P),
                dict(q_in=P, q_out=far, k_in=2 * far, k_out=far), dict(q_in=P, q_out=far, k_in=far + 4 * 511, k_out=2 * far),
                dict(q_in=P, q_out=far, k_in=far - 4 * 255, k_out=2 * far), dict(q_in=P, q_out=far, k_in=far + 3 * 4096, k_out=2 * far),
                dict(q_in=P, q_out=P, k_in=P, k_out=P), dict(q_in=P, q_out=far, k_in=far, k_out=2 * far, n=1)):
        assert both(**bad) == B.EE_ERR_INVALID_ARG and "overlap" in B.ee_last_error(), bad
    # strides that differ: any shared range is refused
    assert rotate(q=rows(P, far, 512, 512, 8), k=rows(far + 4 * 512, 2 * far, 1024, 1024, 4)) == B.EE_ERR_INVALID_ARG


def test_eviction_refuses_more_than_a_context():
    assert evict(keep=262145, w_out=None) == B.EE_ERR_UNSUPPORTED and evict(keep=2**31 - 1) == B.EE_ERR_UNSUPPORTED


def test_names_of_the_binding():
    with pytest.raises(KeyError):
        B.make_rotary_desc(64, layout="quarter")
    with pytest.raises(KeyError):
        B.QuantKV(1, 1, 1, 16, format="int4", device="cpu")
