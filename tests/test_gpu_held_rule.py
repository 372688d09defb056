"""The scale of a held group on the GPU, and how it stands to a swap record's."""
import numpy as np
import pytest
import torch

from gpu_helpers import gpu_compress
from held_reference import HeldBatch
from held_ties import TIES
from paper_2403_11805_b200 import binding as B
from paper_2403_11805_b200.synth import KVShape
from test_gpu_held import call_write, desc_of, rows_for

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def params_of(bt, pool, t):
    """Codes, scale and zero-point bits of token t of the only sequence: [2, heads, ...]."""
    row = int(bt.rows(0)[t])
    got = [bt.format.get(pool[0, :, row // 16], half, row % 16) for half in range(2)]
    return tuple(np.stack([x[i] for x in got]) for i in range(3))


def as_bits(x):
    return np.ascontiguousarray(x).view(np.uint16)


@pytest.mark.parametrize("bits,dtype", [(4, F16), (8, F16), (8, BF16)])
def test_scales_half_way_go_up(bits, dtype):
    """By write and by the append of attention."""
    ties = [x for x in TIES[bits] if dtype == F16 or torch.equal(torch.tensor(x[:2]).to(dtype).float(), torch.tensor(x[:2]))]
    assert ties
    bt = HeldBatch([len(ties)], bits=bits, dim=64, span=32, dtype=dtype, seed=1, store=False)
    k, v, first = rows_for(bt, [len(ties)])
    g = torch.Generator().manual_seed(2)
    for t, (hi, lo, _) in enumerate(ties):
        for x in (k, v):
            x[t] = (1.0 + 7.0 * torch.rand(bt.heads, 64, generator=g)).to(dtype)
            x[t, :, 5], x[t, :, 30], x[t, :, 40], x[t, :, 63] = hi, lo, lo, hi
    pool, _ = call_write(bt, k, v, first)
    for t, (_, lo, want) in enumerate(ties):
        _, scale, zero = params_of(bt, pool, t)
        assert (as_bits(scale) == want).all() and (zero == np.float16(lo)).all()
    # the last of them as the newest token
    held, out = torch.from_numpy(bt.pool.copy()).cuda(), torch.empty(1, bt.heads, 64, dtype=dtype, device="cuda")
    d = desc_of(bt)
    ws = torch.empty(B.held_workspace_bytes(d, bits, 1, bt.max_len), dtype=torch.uint8, device="cuda")
    B.held_attention(d, bits, 0, held, bt.q.contiguous().cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len, out, ws,
                     k_new=k[-1:].contiguous().cuda(), v_new=v[-1:].contiguous().cuda())
    for x, y in zip(params_of(bt, held.cpu().numpy(), len(ties) - 1), params_of(bt, pool, len(ties) - 1)):
        assert np.array_equal(as_bits(x) if x.dtype == np.float16 else x, as_bits(y) if y.dtype == np.float16 else y)


@pytest.mark.parametrize("values", ["any", "one sign", "one far channel"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim,span", [(64, 32), (128, 128)])
def test_what_is_held_beside_the_swap_record_of_the_same_values(dim, span, bits, values):
    """Zero-points are the record's; so is the scale, and with it every code, except where the quotient lies half-way: there the held
    scale is the next fp16 number above the record's."""
    tokens, heads = 2048, 4
    bt = HeldBatch([tokens], bits=bits, dim=dim, span=span, heads=heads, seed=3, store=False)
    k, v, first = rows_for(bt, [tokens])
    g = torch.Generator().manual_seed(4)
    for x in (k, v):
        x[:] = torch.randn(x.shape, generator=g).half()
        if values == "one sign":
            x[:] = x.abs()
        if values == "one far channel":
            x[..., 7::span] = (100.0 * x[..., 7::span].abs() + 8).half()
    pool, _ = call_write(bt, k, v, first, seen=False)

    sh = KVShape("one", n_layers=1, n_kv_heads=heads, n_q_heads=heads, head_dim=dim, n_tokens=tokens, chunk_len=16, group_size=span)
    kv = torch.stack([k, v])[None].transpose(2, 3).contiguous().cuda()        # [layer, K and V, head, token, channel]
    n = tokens // 16
    record, meta, _ = gpu_compress(sh, kv, list(range(n)), [bits] * n)
    groups, parts = dim // span, 0
    for c in range(n):
        mine = record[int(meta["offset"][c]):]
        params = mine[:2 * heads * 16 * groups * 4].view(np.uint16).reshape(2, heads, 16, groups, 2)
        body = mine[2 * heads * 16 * groups * 4:][:2 * heads * 16 * dim * bits // 8]
        codes = (body if bits == 8 else np.stack([body & 15, body >> 4], -1)).reshape(2, heads, 16, groups, span)
        for t in range(16):
            got, scale, zero = params_of(bt, pool, 16 * c + t)
            assert np.array_equal(as_bits(zero), params[:, :, t, :, 1])
            scale, old = as_bits(scale).astype(int), params[:, :, t, :, 0].astype(int)
            other = scale != old
            parts += int(other.sum())
            assert (scale[other] == old[other] + 1).all()
            assert np.array_equal(got.reshape(2, heads, groups, span)[~other], codes[:, :, t][~other])
            if other.any():
                x = torch.stack([k, v])[:, 16 * c + t].double().numpy().reshape(2, heads, groups, span)[other]
                quotient = (x.max(-1) - x.min(-1)) / (2 ** bits - 1)
                middle = sum(y[other].astype(np.uint16).view(np.float16).astype(np.float64) for y in (scale, old)) / 2
                assert (np.abs(quotient / middle - 1) <= 2.0 ** -22).all()       # four roundings to binary32 at most
    if values == "any":
        assert parts == 0                                     # (none among this many of values of both signs)
    if values == "one sign" and bits == 4:
        assert parts > 0
