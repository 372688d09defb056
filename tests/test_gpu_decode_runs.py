"""Attention of a new token where the batch's tiles are cut into runs (large batches, long contexts): decode_kernel without clusters, and
finish_kernel.  Small calls take the form with a cluster per item, so every batch here is either padded with empty sequences to more
items than that form takes, or has a length bound beyond it: the same shapes, masks and odd cases as in test_gpu_decode.py."""
import math

import pytest
import torch

from paper_2403_11805_b200 import binding as B
from paged_reference import Batch, attend, bits
from test_gpu_decode import RAGGED, SHAPES, call, check, desc_of, workspace

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
# more (sequence, KV head) items than clusters' CTAs get on the GPU in two rounds of three per SM
MANY_ITEMS = 1000
# more tokens than eight clustered CTAs take
LONG = 9000


def padded(bt):
    """The batch between empty sequences, as many as make it too many items for clusters; and the place of its first sequence."""
    more = -(-MANY_ITEMS // bt.heads)
    front, g, n = more // 3, torch.Generator().manual_seed(99), len(bt.lens)

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
    bt.mass = torch.cat([torch.full((bt.layers, front, *bt.mass.shape[2:]), 3.0), bt.mass,
                         torch.full((bt.layers, more - front, *bt.mass.shape[2:]), 4.0)], dim=1)
    return front


@pytest.mark.parametrize("how", ["padded", "long_bound"])
@pytest.mark.parametrize("name", SHAPES)
def test_matches_64_bits(name, how):
    kw = dict(SHAPES[name])
    if how == "long_bound":
        kw["max_len"] = max(LONG, 2 * max(kw["lens"]))
    bt = Batch(seed=len(name), **kw)
    if how == "padded":
        if len(bt.lens) > 3000:
            pytest.skip("as many sequences as a batch may have")
        padded(bt)
    check(bt)
    check(bt, append=True, mass="add")


MORE = {
    "bf16_144": dict(lens=RAGGED, dim=144, dtype=BF16, group=2), "bf16_192_group_9": dict(lens=[90, 17, 0, 300], dim=192, dtype=BF16, group=9, heads=1),
    "bf16_240_chunk_24": dict(lens=[90, 25, 49], dim=240, dtype=BF16, chunk=24), "bf16_80_chunk_7": dict(lens=RAGGED, dim=80, dtype=BF16, chunk=7, group=5),
    "256_chunk_5": dict(lens=[61, 5, 128], dim=256, chunk=5, group=16), "128_chunk_40_group_12": dict(lens=[200, 41], dim=128, chunk=40, group=12),
    "ragged_many": dict(lens=[(i * i * 7) % 211 for i in range(260)], heads=4, dim=96, group=3),
    "one_long_among_many": dict(lens=[3 if i != 77 else 4100 for i in range(300)], heads=4, dim=64, group=2),
}


@pytest.mark.parametrize("name", MORE)
def test_more_shapes(name):
    bt = Batch(seed=len(name), **MORE[name])
    if len(bt.lens) < 100:
        padded(bt)
    check(bt, append=True, mass="add")
    check(bt, mass="weights")
    check(bt)


WINDOWED = {
    "ragged": dict(lens=RAGGED), "ragged_bf16": dict(lens=RAGGED, dtype=BF16, dim=128, group=4), "chunk_5": dict(lens=[9, 53, 0, 81], chunk=5),
    "group_17": dict(lens=[50, 20], group=17, heads=1), "long": dict(lens=[5000], heads=4, dim=128), "mqa_256": dict(lens=[300, 7], heads=1, group=8, dim=256, dtype=BF16),
    "dim_80": dict(lens=[90, 0, 24, 23, 22], dim=80, group=5), "several_long": dict(lens=[3000, 17, 2048, 999, 0, 4097], heads=3, group=4, dim=64, chunk=64),
}


@pytest.mark.parametrize("window", [1, 16, 23, 1000, 4096])
@pytest.mark.parametrize("name", WINDOWED)
def test_window(name, window):
    bt = Batch(seed=3, **WINDOWED[name])
    padded(bt)
    check(bt, window=window, append=True, mass="add")
    check(bt, window=window, mass="weights")
    check(bt, window=window)


def test_in_place_weights_and_layers():
    bt = Batch(RAGGED, group=4, seed=11, layers=2)
    padded(bt)
    check(bt, mass="weights")
    check(bt, layer=1, mass="add", in_place=True, append=True)
    check(bt, layer=1, scale=-0.25)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_repeated_calls_give_the_same_bits(dtype):
    bt = Batch([3000, 17, 0, 450] + [(i * 13) % 90 for i in range(300)], heads=4, group=4, dim=128, seed=2, dtype=dtype)
    for window in (0, 333):
        first = call(bt, mass="add", append=True, window=window)
        for _ in range(3):
            again = call(bt, mass="add", append=True, window=window)
            assert all(torch.equal(bits(x), bits(y)) for x, y in zip(first, again))


def test_strided_pool():
    bt = Batch([70, 33, 0], heads=3, dim=96, layers=2, group=2, seed=9)
    padded(bt)
    T, d, n = bt.n_slots * bt.chunk, bt.dim, len(bt.lens)
    flat = torch.full((2, 3, 2, T * d + 40), 3.0, dtype=F16)                  # [layer][head][K, V][rows, padding]
    flat[..., :T * d] = bt.kv.permute(0, 2, 1, 3, 4).reshape(2, 3, 2, T * d)
    desc = desc_of(bt)
    desc.stride_s, desc.stride_h, desc.stride_l = T * d + 40, 2 * (T * d + 40), 6 * (T * d + 40)
    dev, out = flat.cuda(), torch.empty(n, 6, d, dtype=F16, device="cuda")
    B.decode_attention(desc, 1, dev, bt.q.contiguous().cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len, out,
                       workspace(desc, n, bt.max_len), k_new=bt.k_new.contiguous().cuda(), v_new=bt.v_new.contiguous().cuda())
    want, _, _, wkv, (ot, _, _) = attend(bt, 1, append=True)
    assert ((out.cpu().double() - want).abs() <= ot).all()
    got = dev.cpu()
    assert torch.equal(bits(got[..., :T * d].reshape(2, 3, 2, T, d).permute(0, 2, 1, 3, 4)), bits(wkv))
    assert (got[..., T * d:] == 3.0).all()


def test_shared_prefix():
    bt = Batch([48, 40], seed=8, group=2)
    bt.table[1, :2] = bt.table[0, :2]
    padded(bt)
    check(bt, append=True, mass="add")


@pytest.mark.parametrize("long", [40, 700])
def test_infinities_and_nan_in_seen_places(long):
    bt = Batch([long, long, long], seed=6)
    kv = bt.kv
    rows = [bt.rows(b) for b in range(3)]
    kv[0, 0, 0, rows[0][3]] = math.nan                        # head 0 of sequence 0: a NaN key
    kv[0, 1, 1, rows[1][long - 1], 5] = math.inf              # head 1 of sequence 1: one infinite value channel
    at = padded(bt)
    out, lse, mass, _ = call(bt, mass="weights")
    out, lse = out[at:at + 3], lse[at:at + 3]
    assert out[0, 0].isnan().all() and lse[0, 0].isnan()
    assert out[1, 1, 5] == math.inf and out[1, 1, :5].isfinite().all() and out[1, 1, 6:].isfinite().all()
    assert out[0, 1].isfinite().all() and out[1, 0].isfinite().all() and out[2].isfinite().all()
    assert mass[at, 0, :long].isnan().all() and mass[at, 1, :long].isfinite().all() and mass[at + 1:at + 3, :, :long].isfinite().all()


def test_junk_behind_the_last_token_and_before_the_window():
    """NaN keys and infinite values in every row that is not seen, of the sequence's own tokens too."""
    bt = Batch([90, 37, 1, 200], seed=7, group=3, dim=128)
    clean = bt.kv.clone()
    for b, n in enumerate(bt.lens):
        bt.kv[0, 0][:, bt.rows(b)[:max(0, n - 21)]] = math.nan
        bt.kv[0, 1][:, bt.rows(b)[:max(0, n - 21)]] = math.inf
    padded(bt)
    out, lse, mass, _ = call(bt, window=21, mass="weights")
    bt.kv = clean
    want, wlse, wmass, _, (ot, lt, mt) = attend(bt, window=21, mass_before=torch.full_like(bt.mass[0], 5.0))
    assert ((out.double() - want).abs() <= ot).all() and ((mass.double() - wmass).abs() <= mt).all()
    live = wlse > -math.inf
    assert ((lse.double() - wlse)[live].abs() <= lt[live]).all() and torch.equal(lse == -math.inf, ~live)


def test_rows_whose_logits_are_all_minus_infinity_are_empty():
    bt = Batch([20, 300], heads=1, seed=1)
    bt.q[:] = 1.0
    for b in range(2):
        bt.kv[0, 0, 0, bt.rows(b)] = -math.inf
    at = padded(bt)
    out, lse, mass, _ = call(bt, mass="add")
    assert (out[at:at + 2] == 0).all() and (lse == -math.inf).all()
    for b in range(2):
        assert torch.equal(mass[at + b, :, :bt.lens[at + b]], bt.mass[0][at + b, :, :bt.lens[at + b]])


@pytest.mark.parametrize("form", ["cluster", "whole_in_a_run", "over_runs", "cluster_of_parts"])
def test_rows_of_no_weight_are_zero_whatever_their_values(form):
    """All logits -inf: the row is 0 also where values are infinite or NaN."""
    length = {"cluster": 20, "whole_in_a_run": 20, "over_runs": 300, "cluster_of_parts": 100}[form]
    bt = Batch([length, length], heads=1, seed=1, group=3)
    bt.q[:] = 1.0
    bt.kv[0, 0, 0, bt.rows(0)] = -math.inf
    bt.kv[0, 1, 0, bt.rows(0)] = math.inf
    bt.kv[0, 1, 0, bt.rows(0)[5]] = math.nan
    at = 0 if form.startswith("cluster") else padded(bt)
    out, lse, mass, _ = call(bt, mass="add")
    assert (lse[at] == -math.inf).all() and torch.equal(mass[at, :, :length], bt.mass[0][at, :, :length])
    assert (out[at] == 0).all()
    assert out[at + 1].isfinite().all() and lse[at + 1].isfinite().all()


@pytest.mark.parametrize("bad_len", [1000, -3])
def test_invalid_lengths_and_slots_answer_nan_and_touch_nothing(bad_len):
    bt = Batch([30, 40, 50, 60, 20], seed=12, group=2)
    at = padded(bt)
    want, _, _, _, (ot, _, _) = attend(bt, append=True)
    ok = bt.kv.clone()
    ok_rows = {b: bt.rows(at + b)[-1] for b in (0, 4)}
    bt.table[at + 2, 1] = bt.n_slots                          # one behind the pool
    bt.table[at + 3, 3] = -1                                  # also the slot of the newest token
    d, kv, n = desc_of(bt), bt.kv.cuda(), len(bt.lens)
    lens = torch.tensor(bt.lens, dtype=torch.int32)
    lens[at + 1] = bad_len
    out, lse = torch.zeros(n, 4, 64, dtype=F16, device="cuda"), torch.zeros(n, 4, device="cuda")
    mass = torch.full((n, 2, 60), 5.0, device="cuda")
    B.decode_attention(d, 0, kv, bt.q.contiguous().cuda(), bt.table.cuda(), lens.cuda(), 60, out, workspace(d, n, 60, True),
                       k_new=bt.k_new.contiguous().cuda(), v_new=bt.v_new.contiguous().cuda(), lse=lse, mass_out=mass)
    out, lse, mass = out.cpu(), lse.cpu(), mass.cpu()
    for b in (1, 2, 3):
        assert out[at + b].isnan().all() and lse[at + b].isnan().all()
    for b in (0, 4):
        assert ((out[at + b].double() - want[at + b]).abs() <= ot[at + b]).all()
        assert mass[at + b, :, :bt.lens[at + b]].isfinite().all() and (mass[at + b, :, bt.lens[at + b]:] == 5.0).all()
    assert (mass[at + 1] == 5.0).all()                        # of an invalid length nothing is known
    for b, length in ((2, 50), (3, 60)):
        assert mass[at + b, :, :length].isnan().all() and (mass[at + b, :, length:] == 5.0).all()
    for b, row in ok_rows.items():
        ok[0, 0, :, row], ok[0, 1, :, row] = bt.k_new[at + b], bt.v_new[at + b]
    last = bt.table[at + 2, 50 // 16] * 16 + 49 % 16          # sequence 2's newest token has a slot
    ok[0, 0, :, last], ok[0, 1, :, last] = bt.k_new[at + 2], bt.v_new[at + 2]
    assert torch.equal(bits(kv.cpu()), bits(ok))


def test_far_slots():
    """Offsets past 2^31 elements and 2^32 bytes inside one slab."""
    heads, dim, chunk, n_slots = 1, 256, 16, 560000           # 8.96 million rows of 512 bytes: 4.6 GB for K, as much for V
    bt = Batch([50], heads=heads, group=4, dim=dim, chunk=chunk, seed=21, max_len=LONG)
    far = [n_slots - 1, 0, n_slots - 2, n_slots // 2 + 1]
    kv = torch.empty(1, 2, heads, n_slots * chunk, dim, dtype=F16, device="cuda")
    table = torch.full((1, -(-LONG // chunk)), -1, dtype=torch.int32)
    table[0, :4] = torch.tensor(far, dtype=torch.int32)
    for i, slot in enumerate(far):
        s = int(bt.table[0, i])
        kv[:, :, :, slot * chunk:(slot + 1) * chunk] = bt.kv[:, :, :, s * chunk:(s + 1) * chunk].cuda()
    d = B.make_desc(1, heads, 4, dim, n_slots * chunk, chunk, 16)
    out = torch.empty(1, 4, dim, dtype=F16, device="cuda")
    B.decode_attention(d, 0, kv, bt.q.contiguous().cuda(), table.cuda(), torch.tensor([50], dtype=torch.int32).cuda(), LONG, out,
                       workspace(d, 1, LONG), k_new=bt.k_new.contiguous().cuda(), v_new=bt.v_new.contiguous().cuda())
    want, _, _, _, (ot, _, _) = attend(bt, append=True)
    assert ((out.cpu().double() - want).abs() <= ot).all()
    row = far[49 // 16] * chunk + 49 % 16
    assert torch.equal(kv[0, 0, 0, row].cpu(), bt.k_new[0, 0]) and torch.equal(kv[0, 1, 0, row].cpu(), bt.v_new[0, 0])


def test_captured_and_replayed():
    """Two graphs share a workspace; lengths, queries and tables change between the replays, down to an empty batch."""
    bt = Batch([100, 20, 0, 700], group=4, seed=14, max_len=LONG, dim=128)
    d, n = desc_of(bt), 4
    bt.kv[bt.kv.isnan()] = 0.25
    kv, table, q = bt.kv.cuda(), bt.table.cuda(), bt.q.contiguous().cuda()
    lens = torch.tensor(bt.lens, dtype=torch.int32).cuda()
    ws = workspace(d, n, LONG, True)
    outs = [torch.zeros(n, 8, 128, dtype=F16, device="cuda") for _ in range(2)]
    mass = torch.zeros(n, 2, LONG, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.decode_attention(d, 0, kv, q, table, lens, LONG, outs[i], ws, mass_out=mass if i else None)
        graphs.append(g)
    own = bt.table.clone()
    for lens_now, swap in (([100, 20, 0, 700], False), ([37, 0, 0, 641], True), ([0, 0, 0, 0], False), ([99, 17, 0, 1], True), ([0, 1, 0, 700], False)):
        bt.lens = lens_now
        bt.table = own[[0, 1, 2, 3]].clone()
        if swap:                                              # other rows in the same places
            bt.table[3, :7], bt.table[0, :7] = own[0, :7], own[3, :7]
        table.copy_(bt.table)
        lens.copy_(torch.tensor(lens_now, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(sum(lens_now))).to(F16))
        bt.q = q.cpu()
        mass.fill_(5.0)
        for i, g in enumerate(graphs):
            outs[i].fill_(9.0)
            g.replay()
        torch.cuda.synchronize()
        want, _, wmass, _, (ot, _, mt) = attend(bt, mass_before=torch.full_like(bt.mass[0], 5.0))
        for o in outs:
            assert ((o.cpu().double() - want).abs() <= ot).all()
        assert torch.equal(outs[0], outs[1]) and ((mass.cpu().double() - wmass).abs() <= mt).all()


def test_two_streams_at_once():
    both = [Batch([900, 30, 0, 411] + [i % 50 for i in range(130)], heads=8, group=4, dim=128, seed=s) for s in (41, 42)]
    streams = [torch.cuda.Stream() for _ in both]
    n, jobs = len(both[0].lens), []
    for bt in both:
        d = desc_of(bt)
        jobs.append((d, bt.kv.cuda(), bt.q.contiguous().cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(),
                     [torch.empty(n, 32, 128, dtype=F16, device="cuda") for _ in range(10)], workspace(d, n, 900), bt.k_new.contiguous().cuda(),
                     bt.v_new.contiguous().cuda()))
    torch.cuda.synchronize()
    for i in range(10):
        for s, (d, kv, q, table, lens, outs, ws, k, v) in zip(streams, jobs):
            B.decode_attention(d, 0, kv, q, table, lens, 900, outs[i], ws, k_new=k, v_new=v, stream=s)
    torch.cuda.synchronize()
    for bt, job in zip(both, jobs):
        want, _, _, _, (ot, _, _) = attend(bt, append=True)
        for o in job[5]:
            assert torch.equal(o, job[5][0])
        assert ((job[5][0].cpu().double() - want).abs() <= ot).all()


def test_one_workspace_for_calls_of_different_shapes():
    """What an earlier call left in the workspace has no influence: other lengths, other groups, clusters and runs in turn."""
    a = Batch([400, 3, 0] + [i % 70 for i in range(260)], heads=4, group=2, dim=64, seed=1)
    b = Batch([60, 900], heads=1, group=7, dim=80, seed=2, max_len=LONG)
    c = Batch([90, 5], heads=2, group=4, dim=128, seed=3)
    size = max(B.decode_workspace_bytes(desc_of(x), len(x.lens), x.max_len, True) for x in (a, b, c))
    ws = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
    for x in (a, b, c, a, c, b, b, a):
        n, hq = len(x.lens), x.heads * x.group
        out, mass = torch.full((n, hq, x.dim), 7.0, dtype=F16, device="cuda"), torch.full((n, x.heads, x.max_len), 5.0, device="cuda")
        B.decode_attention(desc_of(x), 0, x.kv.cuda(), x.q.contiguous().cuda(), x.table.cuda(), torch.tensor(x.lens, dtype=torch.int32).cuda(), x.max_len,
                           out, ws, mass_out=mass)
        want, _, wmass, _, (ot, _, mt) = attend(x, mass_before=torch.full_like(x.mass[0], 5.0))
        assert ((out.cpu().double() - want).abs() <= ot).all() and ((mass.cpu().double() - wmass).abs() <= mt).all()
