"""Attention of a new token over a held pool (K and V at 8 or 4 bits) against 64 bits."""
import math

import numpy as np
import pytest
import torch

from held_reference import HeldBatch, attend
from paged_reference import bits as bits_of
from paper_2403_11805_b200 import binding as B
from test_gpu_held import desc_of

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
RAGGED = [37, 16, 0, 1, 50, 33, 15, 17]
# more (sequence, KV head) items than a small call has, and more tokens than one
MANY_ITEMS, LONG = 1000, 9000


def workspace(d, bits, n, max_len, fill=0xff):
    return torch.full((B.held_workspace_bytes(d, bits, n, max_len),), fill, dtype=torch.uint8, device="cuda")


def call(bt, layer=0, window=0, append=False, scale=None, table=None, lens=None, pool=None):
    d, n = desc_of(bt), len(bt.lens)
    held, qkv = torch.from_numpy((bt.pool if pool is None else pool).copy()).cuda(), bt.qkv.cuda()
    hq = bt.heads * bt.group
    out = torch.full((n, hq, bt.dim), 9.0, dtype=bt.dtype, device="cuda")
    lse = torch.full((n, hq), 9.0, dtype=torch.float32, device="cuda")
    B.held_attention(d, bt.bits, layer, held, qkv[:, :hq], (bt.table if table is None else table).cuda(),
                     torch.tensor(bt.lens if lens is None else lens, dtype=torch.int32).cuda(), bt.max_len, out, workspace(d, bt.bits, n, bt.max_len),
                     k_new=qkv[:, hq:hq + bt.heads] if append else None, v_new=qkv[:, hq + bt.heads:] if append else None, window=window, scale=scale,
                     lse=lse)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), held.cpu().numpy()


def check(bt, **kw):
    want, wlse, wpool, (ot, lt) = attend(bt, **kw)
    out, lse, pool = call(bt, **kw)
    live = wlse > -math.inf
    assert torch.equal(lse == -math.inf, ~live)
    assert ((lse.double() - wlse)[live].abs() <= lt[live]).all()
    assert ((out.double() - want).abs() <= ot).all()
    assert np.array_equal(pool, wpool)


def padded(bt):
    """The batch between empty sequences, as many as make it a large one; and the place of its first sequence."""
    more = -(-MANY_ITEMS // bt.heads)
    front, n, g = more // 3, len(bt.lens), torch.Generator().manual_seed(99)

    def around(x, fill):
        rows = torch.full((more, *x.shape[1:]), fill, dtype=x.dtype)
        return torch.cat([rows[:front], x, rows[front:]])

    bt.lens = [0] * front + bt.lens + [0] * (more - front)
    bt.table = around(bt.table, -7)
    bt.qkv = around(bt.qkv, 0.0)
    bt.qkv[:front] = torch.randn(bt.qkv[:front].shape, generator=g).to(bt.dtype)
    bt.qkv[front + n:] = math.nan                             # nobody reads the rows of an empty sequence
    hq = bt.heads * bt.group
    bt.q, bt.k_new, bt.v_new = bt.qkv[:, :hq], bt.qkv[:, hq:hq + bt.heads], bt.qkv[:, hq + bt.heads:]
    return front


def batch(how="plain", **kw):
    """A batch in the forms that calls of different sizes may take: as it is, among many sequences, with a bound of a long one."""
    if how == "long_bound":
        kw["max_len"] = max(LONG, 2 * max(kw["lens"]))
    bt = HeldBatch(**kw)
    if how == "padded":
        padded(bt)
    return bt


SHAPES = {
    "64": dict(dim=64), "64_span_32_group_3": dict(dim=64, span=32, group=3), "96_group_5": dict(dim=96, span=32, group=5, heads=1),
    "128": dict(dim=128), "128_span_64_group_4": dict(dim=128, span=64, group=4), "128_span_32_group_8": dict(dim=128, span=32, group=8, heads=1),
    "256_group_2": dict(dim=256, group=2, heads=1), "256_span_128_group_8": dict(dim=256, span=128, group=8, heads=1),
    "256_span_64_group_16": dict(dim=256, span=64, group=16, heads=1), "64_group_17": dict(dim=64, group=17, heads=1),
    "128_group_12": dict(dim=128, group=12, heads=1), "64_group_40": dict(dim=64, group=40, heads=1),
}
HOW = ["plain", "padded", "long_bound"]


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("name", SHAPES)
def test_matches_64_bits(name, bits, how):
    bt = batch(how, lens=RAGGED, bits=bits, seed=len(name), dtype=BF16 if len(name) % 2 else F16, **SHAPES[name])
    check(bt)
    check(bt, append=True)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bits", [4, 8])
def test_long_sequences(bits, dtype):
    bt = HeldBatch([3000, 17, 2048, 999, 0, 4097], heads=2, group=4, dim=64, chunk=64, bits=bits, dtype=dtype, seed=1)
    check(bt, append=True)
    check(bt, window=1000)


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 64, 100, 500])
def test_lengths(length, how):
    check(batch(how, lens=[length], heads=3, dim=64, seed=length), append=True)


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("window", [1, 16, 23, 4096])
def test_window(window, how):
    bt = batch(how, lens=RAGGED + [200], seed=2, group=2, dim=128, chunk=32)
    check(bt, window=window)
    check(bt, window=window, append=True)


@pytest.mark.parametrize("how", HOW)
def test_layers_and_scale(how):
    bt = batch(how, lens=RAGGED, seed=3, layers=2)
    check(bt, layer=1, append=True)
    check(bt, layer=1, scale=-0.25)
    check(bt, scale=0.0)


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("gain", [40.0, 1e-3])
def test_steep_and_flat_weights(gain, how):
    """Keys of large size make one token take all the weight, of small size leave them even."""
    check(batch(how, lens=[300, 45, 7], gain=gain, seed=4, dim=128))


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scales_of_very_different_size(how, dtype):
    """Values of tokens whose ranges differ by factors of up to 2^20, growing and falling along the sequence."""
    bt = batch(how, lens=[400, 90, 33], seed=5, dim=64, dtype=dtype)
    for b in range(len(bt.lens)):
        rows = bt.rows(b).tolist()
        for t, row in enumerate(rows):
            factor = 2.0 ** ((t * 20 // len(rows)) - 10) if b % 2 else 2.0 ** (10 - t * 20 // len(rows))
            for h in range(bt.heads):
                bt.store(bt.pool, 0, h, 1, row, bt.kv[0, 1, h, row] * factor)
    check(bt)


@pytest.mark.parametrize("how", HOW)
def test_large_and_small_queries(how):
    """Query rows near the largest number of their type, and tiny ones."""
    for dtype, factors in ((F16, (1.0, 3000.0, 1e-6)), (BF16, (1.0, 1e6, 1e30, 1e-30))):
        bt = batch(how, lens=[60, 60, 60, 60], seed=6, dtype=dtype, dim=128)
        at = next(i for i, x in enumerate(bt.lens) if x)
        for i, f in enumerate(factors):
            bt.q[at + i] = (bt.q[at + i].double() * f).to(dtype)
        if dtype == BF16:                                     # keys small enough for logits that 32 bits hold
            for row in bt.rows(at + 2).tolist():
                for h in range(bt.heads):
                    bt.store(bt.pool, 0, h, 0, row, bt.kv[0, 0, h, row] * 0.0)
        check(bt)


@pytest.mark.parametrize("how", HOW)
def test_constant_groups(how):
    """Scales of 0: all of K, all of V, and single tokens."""
    bt = batch(how, lens=[40, 40, 40], seed=7, dim=64)
    at = next(i for i, x in enumerate(bt.lens) if x)
    for b, (half, every) in enumerate(((0, 1), (1, 1), (1, 3))):
        for t, row in enumerate(bt.rows(at + b).tolist()):
            if t % every == 0:
                for h in range(bt.heads):
                    bt.store(bt.pool, 0, h, half, row, torch.full((64,), 0.5 * (t % 5), dtype=F16))
    check(bt)


@pytest.mark.parametrize("how", HOW)
def test_nan_groups(how):
    """A NaN group of K makes its head's row NaN; one of V only its channels; neither before the window, behind the last token or in
    another sequence."""
    bt = batch(how, lens=[70, 70, 70, 70], seed=8, dim=128, span=64, group=2)
    at = next(i for i, x in enumerate(bt.lens) if x)
    nan = torch.full((64,), math.nan, dtype=F16)

    def spoil(b, t, head, half):
        row = int(bt.rows(at + b)[t])
        x = bt.kv[0, half, head, row].clone()
        x[64:] = nan
        bt.store(bt.pool, 0, head, half, row, x)

    spoil(0, 65, 0, 0)
    spoil(1, 65, 1, 1)
    spoil(2, 3, 0, 0)
    spoil(2, 4, 1, 1)
    clean = bt.pool
    out, lse, _ = call(bt, window=40)
    got, got_lse = out[at:at + 4], lse[at:at + 4]
    assert got[0, :2].isnan().all() and got_lse[0, :2].isnan().all() and got[0, 2:].isfinite().all()
    assert got[1, 2:, 64:].isnan().all() and got[1, 2:, :64].isfinite().all() and got_lse[1].isfinite().all() and got[1, :2].isfinite().all()
    assert got[2:].isfinite().all() and got_lse[2:].isfinite().all()
    assert clean is bt.pool


@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_queries_that_are_no_numbers(value, dtype, how):
    bt = batch(how, lens=[20, 20], seed=9, dtype=dtype, group=2)
    at = next(i for i, x in enumerate(bt.lens) if x)
    bt.q[at, 1, 7] = value
    out, lse, _ = call(bt)
    assert out[at, 1].isnan().all() and lse[at, 1].isnan()
    assert out[at, [0, 2, 3]].isfinite().all() and out[at + 1].isfinite().all() and lse[at, [0, 2, 3]].isfinite().all()


@pytest.mark.parametrize("how", HOW)
def test_a_newest_token_that_is_no_number(how):
    bt = batch(how, lens=[20, 33], seed=10)
    at = next(i for i, x in enumerate(bt.lens) if x)
    bt.k_new[at, 0, 3] = math.inf
    bt.v_new[at + 1, 1, 5] = math.nan
    _, _, want, _ = attend(bt, append=True)
    out, lse, pool = call(bt, append=True)
    assert np.array_equal(pool, want)
    assert out[at, 0].isnan().all() and out[at, 1].isfinite().all()
    assert out[at + 1, 1].isnan().all() and lse[at + 1].isfinite().all() and out[at + 1, 0].isfinite().all()


@pytest.mark.parametrize("bad_len", [100000, -3])
@pytest.mark.parametrize("how", HOW)
def test_invalid_lengths_and_slots_answer_nan_and_touch_nothing(bad_len, how):
    bt = batch(how, lens=[30, 40, 50, 60, 20], seed=12, group=2)
    at = next(i for i, x in enumerate(bt.lens) if x)
    want, wlse, wpool, (ot, lt) = attend(bt, append=True)
    lens, table = list(bt.lens), bt.table.clone()
    lens[at + 1] = bad_len
    table[at + 2, 1] = bt.n_slots                             # tokens 16 .. 31
    table[at + 3, 3] = -1                                     # the newest token's slot
    out, lse, pool = call(bt, append=True, lens=lens, table=table)
    for b in range(1, 4):
        assert out[at + b].isnan().all() and lse[at + b].isnan().all()
    for b in (0, 4):
        assert ((out[at + b].double() - want[at + b]).abs() <= ot[at + b]).all()
    same = bt.pool.copy()
    f = bt.format
    for b in (0, 2, 4):                                       # those whose newest token has a place
        row = int(bt.rows(at + b)[-1])
        for h in range(bt.heads):
            for half in range(2):
                f.put(same[0, h, row // 16], half, row % 16, *(x[0] for x in f.get(wpool[0, h, row // 16:row // 16 + 1], half, row % 16)))
    assert np.array_equal(pool, same)


def test_a_slot_outside_the_pool_before_the_window_is_not_looked_at():
    bt = HeldBatch([60], seed=13)
    want, _, _, (ot, _) = attend(bt, window=20)
    bt.table[0, 0] = -5
    out, lse, _ = call(bt, window=20)
    assert ((out.double() - want).abs() <= ot).all() and lse.isfinite().all()


@pytest.mark.parametrize("how", HOW)
def test_shared_prefix(how):
    bt = batch(lens=[48, 40], seed=14, group=2)
    bt.table[1, :2] = bt.table[0, :2]
    if how == "padded":
        padded(bt)
    check(bt, append=True)


def test_repeated_calls_give_the_same_bits():
    bt = HeldBatch([3000, 17, 0, 450] + [(i * 13) % 90 for i in range(300)], heads=2, group=4, dim=64, seed=2)
    small = HeldBatch([300, 20], heads=2, group=4, dim=64, seed=3)
    for b, window in ((bt, 0), (bt, 333), (small, 0)):
        first = call(b, append=True, window=window)
        for _ in range(3):
            again = call(b, append=True, window=window)
            assert torch.equal(bits_of(first[0]), bits_of(again[0])) and torch.equal(first[1], again[1]) and np.array_equal(first[2], again[2])


def test_the_largest_batch():
    bt = HeldBatch([i % 3 for i in range(4096)], heads=1, dim=64, seed=15)
    check(bt, append=True)


def test_beyond_32_bits():
    """A pool of more than 4 GiB: slots at its end."""
    small = HeldBatch([40], dim=256, bits=8, heads=2, seed=16)
    d = B.make_desc(2, 2, 2, 256, (1 << 18) * 16 + 48, 16, 256)
    tiles = (1 << 18) + 3
    pool = torch.zeros(2, 2, tiles, small.format.tile, dtype=torch.uint8, device="cuda")
    slots = [tiles - 1, 5, tiles - 3]
    for i, s in enumerate(slots):
        pool[1, :, s] = torch.from_numpy(small.pool[0, :, int(small.table[0, i])]).cuda()
    out = torch.zeros(1, 2, 256, dtype=F16, device="cuda")
    B.held_attention(d, 8, 1, pool, small.q.contiguous().cuda(), torch.tensor([slots], dtype=torch.int32).cuda(), torch.tensor([40], dtype=torch.int32).cuda(),
                     48, out, workspace(d, 8, 1, 48))
    want, _, _, (ot, _) = attend(small)
    assert ((out.cpu().double() - want).abs() <= ot).all()


def test_two_streams_with_workspaces_of_their_own():
    """Calls that overlap, each with its own workspace."""
    parts = [HeldBatch([3000 + 100 * i, 500], heads=2, group=2, dim=64, seed=20 + i) for i in range(2)]
    wants = [attend(bt) for bt in parts]
    streams, state = [torch.cuda.Stream() for _ in parts], []
    for bt in parts:
        d = desc_of(bt)
        state.append((d, torch.from_numpy(bt.pool).cuda(), bt.q.contiguous().cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(),
                      torch.empty(2, 4, 64, dtype=F16, device="cuda"), workspace(d, 4, 2, bt.max_len)))
    torch.cuda.synchronize()
    for _ in range(20):
        for bt, s, (d, held, q, table, lens, out, ws) in zip(parts, streams, state):
            with torch.cuda.stream(s):
                B.held_attention(d, 4, 0, held, q, table, lens, bt.max_len, out, ws)
    torch.cuda.synchronize()
    for (want, _, _, (ot, _)), s in zip(wants, state):
        assert ((s[5].cpu().double() - want).abs() <= ot).all()


@pytest.mark.parametrize("how", HOW)
def test_a_captured_step_follows_its_lengths(how):
    bt = batch(how, lens=[64, 40], seed=17)
    at = next(i for i, x in enumerate(bt.lens) if x)
    d, n = desc_of(bt), len(bt.lens)
    held, table, lens = torch.from_numpy(bt.pool.copy()).cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda()
    q, out, ws = bt.q.contiguous().cuda(), torch.zeros(n, bt.heads, bt.dim, dtype=F16, device="cuda"), workspace(d, 4, n, bt.max_len)
    step = lambda: B.held_attention(d, 4, 0, held, q, table, lens, bt.max_len, out, ws)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for length in (1, 17, 64):
        bt.lens[at] = length
        lens.copy_(torch.tensor(bt.lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want, _, _, (ot, _) = attend(bt)
        assert ((out.cpu().double() - want).abs() <= ot).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_a_prompt_then_tokens_then_reading_back(bits):
    """As a served batch uses the three calls: prompts are written, tokens attended to as they come, and the rows read back are what
    attention saw."""
    prompts, steps = [35, 20, 64], 20
    bt = HeldBatch([p + steps for p in prompts], bits=bits, heads=2, group=2, dim=64, span=32, seed=18, store=False)
    d, n, hq = desc_of(bt), 3, 4
    g = torch.Generator().manual_seed(19)
    rows = torch.randn(sum(prompts), 2, 2, 64, generator=g).half()
    first = torch.cumsum(torch.tensor([0] + prompts), 0).to(torch.int32)
    held, table = torch.from_numpy(bt.pool.copy()).cuda(), bt.table.cuda()
    lens = torch.tensor(prompts, dtype=torch.int32).cuda()
    B.held_write(d, bits, 0, held, rows[:, 0].cuda(), rows[:, 1].cuda(), table, lens, bt.max_len, first_row=first.cuda())
    ws, out = workspace(d, bits, n, bt.max_len), torch.empty(n, hq, 64, dtype=F16, device="cuda")
    stream = [torch.randn(n, hq + 4, 64, generator=g).half() for _ in range(steps)]
    for qkv in stream:
        lens += 1
        x = qkv.cuda()
        B.held_attention(d, bits, 0, held, x[:, :hq], table, lens, bt.max_len, out, ws, k_new=x[:, hq:hq + 2], v_new=x[:, hq + 2:])
    plain = HeldBatch([p + steps for p in prompts], bits=bits, heads=2, group=2, dim=64, span=32, seed=18, store=False)
    for b in range(n):
        for t, row in enumerate(plain.rows(b).tolist()):
            for half in range(2):
                for h in range(2):
                    x = rows[int(first[b]) + t, half, h] if t < prompts[b] else stream[t - prompts[b]][b, hq + 2 * half + h]
                    plain.store(plain.pool, 0, h, half, row, x)
    assert np.array_equal(held.cpu().numpy(), plain.pool)
    plain.q = stream[-1][:, :hq]
    want, _, _, (ot, _) = attend(plain)
    assert ((out.cpu().double() - want).abs() <= ot).all()
    total = sum(bt.lens)
    first = torch.cumsum(torch.tensor([0] + bt.lens), 0).to(torch.int32).cuda()
    back = torch.empty(2, total, 2, 64, dtype=F16, device="cuda")
    B.held_read(d, bits, 0, held, table, lens, bt.max_len, back[0], back[1], first_row=first)
    q = plain.q.double().reshape(n, 2, 2, 64)
    for b in range(n):
        k, v = back[:, int(first[b]):int(first[b + 1])].cpu().double()
        p = torch.softmax(torch.einsum("hgd,thd->hgt", q[b], k) / 8, -1)
        mine = torch.einsum("hgt,thd->hgd", p, v).reshape(hq, 64)
        # rows read back are rounded to fp16: keys by 2^-12 of their size, which moves a logit by at most that times |q| |k| / 8
        slack = 2.0 ** -12 * (q[b].abs().reshape(hq, 64).sum(1).max() * k.abs().max() / 4 * v.abs().max() + v.abs().max())
        assert ((out[b].cpu().double() - mine).abs() <= ot[b] + slack).all()


def test_poisoned_workspaces_and_pools_have_no_influence():
    """Whatever the workspace holds, and codes and parameters of rows that no token lies in."""
    bt = HeldBatch([30, 17, 5], seed=21, dim=128)
    first = call(bt)
    other = HeldBatch([30, 17, 5], seed=21, dim=128)
    keep = {(int(r) // 16, int(r) % 16) for b in range(3) for r in bt.rows(b)}
    f = bt.format
    for tile in range(other.pool.shape[2]):
        for t in range(16):
            if (tile, t) not in keep:
                for half in range(2):
                    other.pool[0, :, tile, f.param[half, t].reshape(-1)] = 0x7c                        # infinities near enough
    again = call(other)
    assert torch.equal(bits_of(first[0]), bits_of(again[0])) and torch.equal(first[1], again[1])
