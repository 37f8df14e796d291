"""The 8-bit cache at the borders of what its calls take: the largest floats, rows of no sequence."""
import pytest
import torch

import quant_oracle as Q
import test_gpu_quant as T
from paper_2407_20272_amd import binding as B

pytestmark = pytest.mark.gpu
LARGEST = torch.finfo(torch.float32).max


@pytest.mark.parametrize("fmt", T.FORMATS)
@pytest.mark.parametrize("later", [False, True])
def test_the_largest_float(fmt, later):
    """It is cached as a float next to it, in a block of its own and where a block's scale grows to it, and stays one when it is moved."""
    tables, nb = T.tables_for([20], 1)
    kv = T.filled(1, nb, 1, 64, fmt, 1)
    x = torch.randn(20, 1, 64, generator=T.gen(1)) * 1e30
    x[3, 0, 5], x[3, 0, 6], x[17, 0, 63] = LARGEST, -LARGEST, -LARGEST
    calls = [list(range(3)), list(range(3, 20))] if later else [list(range(20))]
    for rows in calls:
        B.ee_kv_quant_append(kv, 1, x[rows].cuda(), -x[rows].cuda(), B.make_batch(None, T.i32(rows), T.i32(tables), 20, T.i32([0] * len(rows))))

    def check(places):
        k, v = torch.empty(20, 1, 64, device="cuda"), torch.empty(20, 1, 64, device="cuda")
        B.ee_kv_quant_read(kv, 1, B.make_batch(None, T.i32(range(20)), T.i32(tables if places is None else places), 20, T.i32([0] * 20)), k, v)
        for got, want in ((k, x), (v, -x)):
            got = got.cpu()
            assert bool(torch.isfinite(got).all())
            # half a step of the block's scale; 1e30 is far less than that
            step = LARGEST / 127 if fmt == "int8" else 2.0 ** 120 * 32
            assert bool(((got.double() - want.double()).abs() <= step * 0.51).all())
            assert abs(float(got[3, 0, 5]) / float(want[3, 0, 5]) - 1) < (2.0 ** -20 if fmt == "int8" else 2.0 ** -4)
    check(None)
    # all of it into other blocks, with one position more than stays
    free = [i for i in range(nb) if i not in tables.flatten().tolist()]
    dst = torch.tensor([free[:2]], dtype=torch.int32)
    kept, lens = torch.zeros(1, 1, 20, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ee_kv_quant_evict(kv, 1, B.make_batch(None, T.i32([20]), T.i32(tables), 20), torch.ones(1, 1, 20, device="cuda"), None, 20, 0, kept, lens, None, T.i32(dst))
    assert kept[0, 0].tolist() == list(range(20))
    check(dst)
