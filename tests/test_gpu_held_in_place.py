"""Writing rows into a held pool with the held values in the rows' own place."""
import numpy as np
import pytest
import torch

from held_reference import HeldBatch, write
from paper_2403_11805_b200 import binding as B
from test_gpu_held import SHAPES, desc_of, rows_for, same

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("name", SHAPES)
def test_held_values_in_the_rows_own_place(name, bits, dtype):
    """k_seen and v_seen are k and v.  Rows begin 16 bytes behind a multiple of 32, so that neighbouring heads and rows, which other
    warps read and write, lie in one sector of memory."""
    bt = HeldBatch([37, 16, 0, 1, 50, 33], bits=bits, dtype=dtype, seed=len(name), store=False, **SHAPES[name])
    k, v, first = rows_for(bt, [20, 16, 0, 1, 50, 2], before=2, behind=5)
    want, k_seen, v_seen = write(bt, 0, k, v, first.tolist(), dtype)
    row, n = bt.heads * bt.dim, len(k)
    buffer = torch.full((n * (2 * row + 8) + 16,), 7.0, dtype=dtype, device="cuda")
    kd, vd = (buffer.as_strided((n, bt.heads, bt.dim), (2 * row + 8, bt.dim, 1), 8 + i * row) for i in range(2))
    pool = torch.from_numpy(bt.pool.copy()).cuda()
    args = (bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len)
    nobody = torch.ones(n, dtype=torch.bool)
    nobody[int(first[0]):int(first[-1])] = False
    for _ in range(10):
        buffer.fill_(7.0)
        kd.copy_(k)
        vd.copy_(v)
        B.held_write(desc_of(bt), bits, 0, pool, kd, vd, *args, first_row=first.cuda(), k_seen=kd, v_seen=vd)
        assert np.array_equal(pool.cpu().numpy(), want)
        for got, seen, x in ((kd, k_seen, k), (vd, v_seen, v)):
            assert same(got[~nobody.cuda()], seen[~nobody]) and same(got[nobody.cuda()], x[nobody])
        rest = torch.ones(len(buffer), dtype=torch.bool, device="cuda")
        for i in range(2):
            rest.as_strided((n, row), (2 * row + 8, 1), 8 + i * row).fill_(False)
        assert (buffer[rest] == 7).all()
