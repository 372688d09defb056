"""Writing rows into a held pool (K and V at 8 or 4 bits) and reading them back, against plain forms: bit for bit."""
import math

import numpy as np
import pytest
import torch

from held_reference import HeldBatch, quantise, values, write
from paged_reference import bits as bits_of
from paper_2403_11805_b200 import binding as B

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
SHAPES = {
    "64": dict(dim=64), "64_span_32": dict(dim=64, span=32, heads=3), "96": dict(dim=96, span=32), "128": dict(dim=128), "128_span_64": dict(dim=128, span=64),
    "128_span_32": dict(dim=128, span=32), "256": dict(dim=256, heads=1), "256_span_128": dict(dim=256, span=128), "256_span_64": dict(dim=256, span=64),
}


def desc_of(bt):
    return B.make_desc(bt.layers, bt.heads, bt.heads * bt.group, bt.dim, bt.n_slots * bt.chunk, bt.chunk, bt.span)


def same(got, want):
    """Equal bits; a NaN equals any NaN."""
    got = got.cpu()
    return bool((torch.eq(bits_of(got), bits_of(want)) | (got.isnan() & want.isnan())).all())


def rows_for(bt, new, seed=0, before=0, behind=0):
    """Rows for the last new[b] tokens of every sequence, with nobody's rows around them."""
    first = torch.cumsum(torch.tensor([before] + new), 0).to(torch.int32)
    n = int(first[-1]) + behind
    g = torch.Generator().manual_seed(seed)
    kv = torch.randn(n, 2, bt.heads, bt.dim, generator=g, dtype=torch.float64) * torch.exp(torch.randn(1, 2, bt.heads, bt.dim, generator=g, dtype=torch.float64))
    kv = kv.to(bt.dtype)
    return kv[:, 0], kv[:, 1], first


def call_write(bt, k, v, first, layer=0, seen=True, lens=None, table=None, max_len=None, in_place=False):
    pool, kd, vd = torch.from_numpy(bt.pool.copy()).cuda(), k.cuda(), v.cuda()
    if in_place:
        seen_rows = [kd, vd]
    else:
        seen_rows = [torch.full(k.shape, 7.0, dtype=k.dtype, device="cuda") for _ in range(2)] if seen else [None, None]
    B.held_write(desc_of(bt), bt.bits, layer, pool, kd, vd, (bt.table if table is None else table).cuda(),
                 torch.tensor(bt.lens if lens is None else lens, dtype=torch.int32).cuda(), max_len or bt.max_len,
                 first_row=None if first is None else first.cuda(), k_seen=seen_rows[0], v_seen=seen_rows[1])
    torch.cuda.synchronize()
    return pool.cpu().numpy(), seen_rows


def call_read(bt, pool, first, rows, layer=0, dtype=None, lens=None, table=None):
    out = [torch.full((rows, bt.heads, bt.dim), 7.0, dtype=dtype or bt.dtype, device="cuda") for _ in range(2)]
    B.held_read(desc_of(bt), bt.bits, layer, torch.from_numpy(pool).cuda(), (bt.table if table is None else table).cuda(),
                torch.tensor(bt.lens if lens is None else lens, dtype=torch.int32).cuda(), bt.max_len, out[0], out[1],
                first_row=None if first is None else first.cuda())
    torch.cuda.synchronize()
    return out


def check(bt, new, layer=0, before=0, behind=0):
    k, v, first = rows_for(bt, new, before=before, behind=behind)
    want, k_seen, v_seen = write(bt, layer, k, v, first.tolist(), bt.dtype)
    got, seen = call_write(bt, k, v, first, layer)
    assert np.array_equal(got, want)
    assert same(seen[0], k_seen) and same(seen[1], v_seen)
    assert np.array_equal(call_write(bt, k, v, first, layer, seen=False)[0], want)
    back = call_read(bt, got, first, len(k), layer)
    assert same(back[0], k_seen) and same(back[1], v_seen)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("name", SHAPES)
def test_ragged_prompts(name, bits, dtype):
    bt = HeldBatch([37, 16, 0, 1, 50, 33], bits=bits, dtype=dtype, seed=len(name), store=False, **SHAPES[name])
    check(bt, [20, 16, 0, 1, 50, 2], before=2, behind=5)


@pytest.mark.parametrize("chunk", [16, 32, 48, 64])
def test_parts_of_tiles(chunk):
    """Every first and last place in a tile, and what lies around the new tokens stays."""
    lens = list(range(1, 40, 3)) + [64, 65, 100]
    bt = HeldBatch(lens, chunk=chunk, layers=2, seed=chunk, store=False)
    check(bt, [max(1, n // 2) for n in lens], layer=1)
    check(bt, [min(n, 1) for n in lens], layer=0, behind=1)
    check(bt, [0] * len(lens), behind=3)


@pytest.mark.parametrize("bits", [4, 8])
def test_a_row_per_sequence(bits):
    bt = HeldBatch([5, 0, 16, 17, 100, 1], bits=bits, dim=128, seed=3, store=False)
    k, v, _ = rows_for(bt, [1] * 6)
    want, k_seen, v_seen = write(bt, 0, k, v, None, bt.dtype)
    got, seen = call_write(bt, k, v, None)
    assert np.array_equal(got, want) and same(seen[0], k_seen) and same(seen[1], v_seen)
    back = call_read(bt, got, None, 6)
    assert same(back[0], k_seen) and same(back[1], v_seen) and (back[0][1] == 7).all()


def test_seen_rows_in_place():
    bt = HeldBatch([40, 23], dim=128, seed=4, store=False)
    k, v, first = rows_for(bt, [40, 11], behind=2)
    k, v = k.contiguous(), v.contiguous()
    want, k_seen, v_seen = write(bt, 0, k, v, first.tolist(), bt.dtype)
    got, seen = call_write(bt, k, v, first, in_place=True)
    assert np.array_equal(got, want)
    assert same(seen[0][:-2], k_seen[:-2]) and same(seen[1][:-2], v_seen[:-2]) and same(seen[0][-2:], k[-2:])


def test_many_sequences():
    lens = [(i * 7) % 41 for i in range(1500)]
    bt = HeldBatch(lens, dim=64, heads=1, seed=5, store=False)
    check(bt, [n - n // 3 for n in lens])
    many = HeldBatch([1] * 4096, dim=64, heads=1, seed=6, store=False)
    check(many, [1] * 4096)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bits", [4, 8])
def test_values_at_the_borders(bits, dtype):
    """Constant groups, zeros of both signs, the largest and smallest numbers, infinities and NaN."""
    bt = HeldBatch([16], bits=bits, dim=128, span=64, dtype=dtype, seed=7, store=False)
    k, v, first = rows_for(bt, [16])
    for x in (k, v):
        x[0] = 0.0
        x[1] = -0.0
        x[2] = 3.5
        x[3, 0, :64] = torch.tensor([-65504.0, 65504.0] * 32)
        x[4, 0, 5] = math.inf
        x[4, 1, 70] = -math.inf
        x[5, 0, 127] = math.nan
        x[6] = torch.arange(128) * 2.0 ** -24               # fp16's smallest steps: subnormal scales
        x[7] = torch.where(torch.arange(128) % 2 == 0, 0.0, -0.0)
        x[8] = torch.arange(128) * 2.0 ** -16
        x[9] = 1000.0 + torch.arange(128)
        x[10] = torch.arange(128) * 0.125
        if dtype == BF16:
            x[11] = 1e30
            x[12, 0, 3] = -1e30
            x[13, 0, 9] = 70000.0
            x[14] = 1e-30
    want, k_seen, v_seen = write(bt, 0, k, v, first.tolist(), dtype)
    got, seen = call_write(bt, k, v, first)
    assert np.array_equal(got, want)
    assert same(seen[0], k_seen) and same(seen[1], v_seen)
    assert k_seen[4, 0, :64].isnan().all() and k_seen[4, 0, 64:].isfinite().all() and k_seen[5, 0, 64:].isnan().all()


@pytest.mark.parametrize("bits", [4, 8])
def test_random_bit_patterns(bits):
    """Any 16 bits as input, infinities and NaN among them."""
    g = torch.Generator().manual_seed(8)
    for dtype in (F16, BF16):
        bt = HeldBatch([300], bits=bits, dim=64, span=32, dtype=dtype, seed=8, store=False)
        raw = torch.randint(-(1 << 15), 1 << 15, (300, 2, bt.heads, 64), generator=g).to(torch.int16).view(dtype)
        raw[:100] = raw[:100].nan_to_num(0, 1, -1)
        k, v, first = raw[:, 0], raw[:, 1], torch.tensor([0, 300], dtype=torch.int32)
        want, k_seen, v_seen = write(bt, 0, k, v, first.tolist(), dtype)
        got, seen = call_write(bt, k, v, first)
        assert np.array_equal(got, want)
        assert same(seen[0], k_seen) and same(seen[1], v_seen)


def test_the_rule_is_the_swap_records():
    """A chunk's codes and parameters are those of its record."""
    bt = HeldBatch([16], bits=4, dim=64, span=64, seed=9, heads=2)
    from gpu_helpers import gpu_compress
    from paper_2403_11805_b200.synth import KVShape
    sh = KVShape("one", n_layers=1, n_kv_heads=2, n_q_heads=2, head_dim=64, n_tokens=16, chunk_len=16, group_size=64)
    kv = bt.kv[:, :, :, bt.rows(0)].contiguous().cuda()
    for bits in (4, 8):
        record, _, _ = gpu_compress(sh, kv, [0], [bits])
        codes, scale, zero = quantise(kv.cpu(), bits, 64)
        params = record[:2 * 2 * 16 * 4].view(np.float16).reshape(1, 2, 2, 16, 1, 2)
        assert np.array_equal(params[..., 0], scale) and np.array_equal(params[..., 1], zero)
        body = record[2 * 2 * 16 * 4:][:codes.size * bits // 8]
        want = codes.reshape(-1) if bits == 8 else codes.reshape(-1)[0::2] | codes.reshape(-1)[1::2] << 4
        assert np.array_equal(body, want)


@pytest.mark.parametrize("bad", [1000, -3, 8])
def test_invalid_sequences_and_slots_are_not_stored_and_read_as_nan(bad):
    """A length out of range, or fewer tokens than rows; slots outside the pool."""
    bt = HeldBatch([30, 40, 50, 20], dim=64, seed=10, store=False)
    new = [10, 20, 40, 20]
    k, v, first = rows_for(bt, new, behind=1)
    lens, table = list(bt.lens), bt.table.clone()
    lens[1] = bad
    table[2, 1], table[2, 2] = bt.n_slots, -1                 # tokens 16 .. 47
    want, k_seen, v_seen = write(bt, 0, k, v, first.tolist(), F16)
    got, seen = call_write(bt, k, v, first, lens=lens, table=table)
    kept = bt.pool.copy()
    for b in (0, 2, 3):
        for t, row in enumerate(bt.rows(b).tolist()):
            if t >= bt.lens[b] - new[b] and not (b == 2 and 16 <= t < 48):
                for half in range(2):
                    tile, r, f = row // 16, row % 16, bt.format
                    for h in range(bt.heads):
                        f.put(kept[0, h, tile], half, r, *(x[0] for x in f.get(want[0, h, tile:tile + 1], half, r)))
    assert np.array_equal(got, kept)
    nan = torch.zeros(len(k), dtype=torch.bool)
    nan[10:30] = True                                         # sequence 1's rows
    nan[30 + 6:30 + 38] = True                                # sequence 2's tokens 16 .. 47 (its rows begin at token 10)
    back = call_read(bt, got, first, len(k), lens=lens, table=table)
    for x, y in ((seen[0], k_seen), (seen[1], v_seen), (back[0], k_seen), (back[1], v_seen)):
        x = x.cpu()
        assert x[nan].isnan().all() and same(x[~nan], y[~nan])


def test_rows_that_first_row_puts_outside_the_array_are_nobody_s():
    """first_row is device memory: whatever it holds, nothing outside the arrays is touched."""
    bt = HeldBatch([60, 60], dim=64, seed=11, store=False)
    k, v, _ = rows_for(bt, [10, 10])
    inside = torch.full((64, *k.shape[1:]), 7.0, dtype=F16, device="cuda")
    rows = slice(20, 40)
    for first in ([-5, 10, 30], [0, 40, 20], [15, 15, 1 << 30], [-(1 << 31), 0, (1 << 31) - 1]):
        pool = torch.from_numpy(bt.pool.copy()).cuda()
        buf = inside.clone()
        args = (bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len)
        first = torch.tensor(first, dtype=torch.int64).to(torch.int32).cuda()
        B.held_write(desc_of(bt), 4, 0, pool, k.cuda(), v.cuda(), *args, first_row=first, k_seen=buf[rows], v_seen=buf[rows].clone())
        B.held_read(desc_of(bt), 4, 0, pool, *args, buf[rows], buf[rows].clone(), first_row=first)
        torch.cuda.synchronize()
        assert (buf[:20] == 7).all() and (buf[40:] == 7).all()


def test_reading_the_first_tokens_and_another_type():
    bt = HeldBatch([77, 40], dim=128, span=32, seed=12)
    first, lens = torch.tensor([0, 30, 40], dtype=torch.int32), [30, 10]
    for dtype in (F16, BF16):
        got = call_read(bt, bt.pool, first, 40, dtype=dtype, lens=lens)
        for half in range(2):
            want = torch.cat([torch.stack([bt.row_values(bt.pool, 0, half, r, dtype) for r in bt.rows(b)[:lens[b]].tolist()]) for b in range(2)])
            assert same(got[half], want)


def test_strided_rows_and_another_stream():
    bt = HeldBatch([33, 20], dim=64, heads=4, seed=13, store=False)
    k, v, first = rows_for(bt, [33, 20])
    want, k_seen, v_seen = write(bt, 0, k, v, first.tolist(), F16)
    wide = torch.full((53, 3, 4, 64), 7.0, dtype=F16)
    wide[:, 0], wide[:, 2] = k, v
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        dev, seen, pool = wide.cuda(), torch.full((53, 5, 4, 64), 7.0, dtype=F16).cuda(), torch.from_numpy(bt.pool.copy()).cuda()
        B.held_write(desc_of(bt), 4, 0, pool, dev[:, 0], dev[:, 2], bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len,
                     first_row=first.cuda(), k_seen=seen[:, 1], v_seen=seen[:, 3])
    stream.synchronize()
    assert np.array_equal(pool.cpu().numpy(), want) and same(seen[:, 1], k_seen) and same(seen[:, 3], v_seen)
    assert (seen[:, [0, 2, 4]] == 7).all()


def test_captured_calls_follow_their_tables_and_lengths():
    bt = HeldBatch([64], dim=64, seed=14, store=False)
    k, v, _ = rows_for(bt, [1])
    pool, lens, table = torch.from_numpy(bt.pool.copy()).cuda(), torch.tensor([10], dtype=torch.int32).cuda(), bt.table.cuda()
    kd, vd, out = k.contiguous().cuda(), v.contiguous().cuda(), torch.zeros(2, 1, bt.heads, 64, dtype=F16, device="cuda")
    d = desc_of(bt)

    def both():
        B.held_write(d, 4, 0, pool, kd, vd, table, lens, 64)
        B.held_read(d, 4, 0, pool, table, lens, 64, out[0], out[1])

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for n in (11, 40, 64):
        lens.fill_(n)
        kd.copy_(k.cuda() * n)
        graph.replay()
        torch.cuda.synchronize()
        codes = quantise((k * n).to(F16), 4, 64)
        assert same(out[0], values(*codes, F16))


def test_beyond_32_bits():
    """A pool of more than 4 GiB: the last slots."""
    bt = HeldBatch([40], dim=256, span=256, bits=8, heads=2, seed=15, store=False)
    d = B.make_desc(2, 2, 2, 256, (1 << 18) * 16 + 48, 16, 256)
    assert B.held_bytes(d, 8) > 1 << 32
    pool = torch.zeros(B.held_bytes(d, 8), dtype=torch.uint8, device="cuda")
    slots = torch.tensor([[(1 << 18) + 2, 5, (1 << 18)]], dtype=torch.int32).cuda()
    k, v, first = rows_for(bt, [40])
    lens = torch.tensor([40], dtype=torch.int32).cuda()
    B.held_write(d, 8, 1, pool, k.cuda(), v.cuda(), slots, lens, 48, first_row=first.cuda())
    out = torch.zeros(2, 40, 2, 256, dtype=F16, device="cuda")
    B.held_read(d, 8, 1, pool, slots, lens, 48, out[0], out[1], first_row=first.cuda())
    for half, x in enumerate((k, v)):
        assert same(out[half], values(*quantise(x, 8, 256), F16))
    tile, tiles = 8704 * 2 - 8704 * 2 + B.held_bytes(B.make_desc(1, 1, 1, 256, 16, 16, 256), 8), (1 << 18) + 3
    assert int((pool.view(2, 2, tiles, tile) != 0).any(-1).sum()) == 6
