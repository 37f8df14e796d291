"""How many rows the 8-bit cache's calls take: what the header says is refused on the host, and the workspace sizes refuse what the calls refuse."""
import ctypes as C

import pytest

from paper_2407_20272_amd import binding as B
from test_quant_abi import P, attend, batch, cache


def need(c, heads, rows, context=33, weights=0):
    return B.lib().ee_paged_attention_quant_bytes(C.byref(c), heads, rows, context, weights)


@pytest.mark.parametrize("heads,kv,rows", [(32, 32, 65535), (128, 128, 65535), (64, 1, 16383), (17, 1, 32767)])
def test_single_rows(heads, kv, rows):
    """65535 tiles of up to 16 heads that share a K/V head."""
    c = cache(n_kv_heads=kv, head_dim=16)
    assert need(c, heads, rows, weights=1) > 0
    assert need(c, heads, rows + 1, weights=1) == 0 and "rows" in B.ee_last_error()
    assert attend(c=c, heads=heads, b=batch(rows=rows + 1), out=1 << 40) == B.EE_ERR_UNSUPPORTED and "rows" in B.ee_last_error()


@pytest.mark.parametrize("heads,kv,rows", [(32, 32, 65535 * 32), (128, 128, 65535 * 32), (64, 1, 32767), (24, 8, 65535 * 32 // 3)])
def test_rows_that_share_sequences(heads, kv, rows):
    """65535 tiles of 32 (row, head) pairs."""
    c = cache(n_kv_heads=kv, head_dim=16)
    assert need(c, heads, rows) > 0
    assert need(c, heads, rows + 1) == 0 and "rows" in B.ee_last_error()
    assert attend(c=c, heads=heads, b=batch(rows=rows + 1, row_table=P), out=1 << 40) == B.EE_ERR_UNSUPPORTED and "rows" in B.ee_last_error()


@pytest.mark.parametrize("dst", [None, P])
def test_eviction_of_many_blocks_and_heads(dst):
    from test_quant_abi import evict
    c, b = cache(n_kv_heads=4096, head_dim=16, num_blocks=1 << 14), batch(max_blocks=1 << 14, max_context=1 << 18)
    for keep in (1 << 17, 1 << 18):
        assert evict(c=c, b=b, keep=keep, pitch=1 << 18, dst=dst, dst_blocks=1 << 14, size=1 << 50) == B.EE_ERR_UNSUPPORTED
        assert B.lib().ee_kv_quant_evict_bytes(C.byref(c), 2, keep) == 0 and "blocks" in B.ee_last_error()
    assert B.lib().ee_kv_quant_evict_bytes(C.byref(c), 2, (1 << 17) - 16) > 0


def test_read_refuses_results_over_each_other():
    from test_quant_abi import read
    for k, v in ((P, P), (P, P + 8), (P + 2 * 256 * 4 - 8, P)):       # (2 rows of 4 heads of 64 channels)
        assert read(k=k, v=v) == B.EE_ERR_INVALID_ARG and "overlap" in B.ee_last_error()
