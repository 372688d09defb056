"""Attention of a new token over the paged cache against its 64-bit form: lengths from none to long, head layouts, chunk
lengths that end inside a tile, windows, rows with junk behind the last token, the appended row, the accumulated weights."""
import math

import pytest
import torch

from paper_2403_11805_b200 import binding as B
from paged_reference import Batch, attend, bits

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def desc_of(bt, n_tokens=None):
    return B.make_desc(bt.layers, bt.heads, bt.heads * bt.group, bt.dim, bt.n_slots * bt.chunk if n_tokens is None else n_tokens, bt.chunk, 16)


def workspace(desc, n, max_len, mass=False):
    return torch.full((B.decode_workspace_bytes(desc, n, max_len, mass),), 0xA5, dtype=torch.uint8, device="cuda")


def call(bt, layer=0, window=0, append=False, mass=None, kv=None, in_place=False, scale=None):
    """-> (out, lse, mass_out, kv) on the host; mass: None, "weights" (no mass_in) or "add"."""
    d = desc_of(bt)
    n, hq = len(bt.lens), bt.heads * bt.group
    kv = bt.kv.cuda() if kv is None else kv
    qkv = bt.qkv.cuda()                                       # q, k and v: views of one tensor
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + bt.heads], qkv[:, hq + bt.heads:]
    out = torch.full((n, hq, bt.dim), 7.0, dtype=bt.dtype, device="cuda")
    lse = torch.full((n, hq), 7.0, device="cuda")
    mass_in = bt.mass[layer].cuda() if mass == "add" else None
    mass_out = None if mass is None else (mass_in if in_place else torch.full_like(bt.mass[layer], 5.0).cuda())
    B.decode_attention(d, layer, kv, q, bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len, out,
                       workspace(d, n, bt.max_len, mass is not None), k_new=k if append else None, v_new=v if append else None,
                       window=window, lse=lse, mass_in=mass_in, mass_out=mass_out, scale=scale)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), None if mass is None else mass_out.cpu(), kv.cpu()


def check(bt, layer=0, window=0, append=False, mass=None, in_place=False, scale=None):
    before = None if mass is None else (bt.mass[layer] if in_place else torch.full_like(bt.mass[layer], 5.0))
    out, lse, mass_out, kv = call(bt, layer, window, append, mass, in_place=in_place, scale=scale)
    want, wlse, wmass, wkv, (ot, lt, mt) = attend(bt, layer, window, append, bt.mass[layer] if mass == "add" else None, before, scale)
    assert torch.isfinite(out).all()
    assert ((out.double() - want).abs() <= ot).all(), float(((out.double() - want).abs() - ot).max())
    empty = wlse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and (out[empty] == 0).all()
    assert ((lse.double() - wlse)[~empty].abs() <= lt[~empty]).all(), float(((lse.double() - wlse)[~empty].abs() - lt[~empty]).max())
    if mass is not None:
        assert ((mass_out.double() - wmass).abs() <= mt).all(), float(((mass_out.double() - wmass).abs() - mt).max())
    assert torch.equal(bits(kv), bits(wkv))                   # the pool: the appended rows and nothing else
    return out, lse, mass_out


RAGGED = [37, 0, 1, 16, 15, 17, 64, 5, 200, 33]

SHAPES = {
    "one_token": dict(lens=[1]),
    "two_tokens": dict(lens=[2], dim=128),
    "tile": dict(lens=[16]), "tile_and_one": dict(lens=[17]),
    "ragged": dict(lens=RAGGED),
    "ragged_bf16": dict(lens=RAGGED, dtype=BF16, dim=128, group=4),
    "all_empty": dict(lens=[0, 0, 0], max_len=40),
    "mqa_256": dict(lens=[300, 7], heads=1, group=8, dim=256, dtype=BF16),
    "mqa_256_f16_long": dict(lens=[2049], heads=1, group=8, dim=256),
    "group_2": dict(lens=[100, 3], group=2), "group_3": dict(lens=[100, 31], group=3), "group_7": dict(lens=[90, 2], group=7, dim=80),
    "group_9": dict(lens=[70], group=9), "group_16": dict(lens=[130, 1], group=16, dim=64), "group_17": dict(lens=[50, 20], group=17, heads=1),
    "group_71": dict(lens=[45, 12], group=71, heads=1, dim=64, dtype=BF16),
    "dim_16": dict(lens=[40, 9], dim=16), "dim_32": dict(lens=[40, 9], dim=32, group=2), "dim_48": dict(lens=[41], dim=48),
    "dim_96": dict(lens=[77, 16], dim=96, group=4), "dim_112": dict(lens=[77], dim=112), "dim_144": dict(lens=[50], dim=144),
    "dim_192": dict(lens=[50, 18], dim=192, group=2, dtype=BF16), "dim_240": dict(lens=[33], dim=240, group=8),
    "chunk_1": dict(lens=[9, 20], chunk=1), "chunk_5": dict(lens=[9, 53, 0], chunk=5), "chunk_7": dict(lens=[70], chunk=7, dim=128),
    "chunk_8": dict(lens=[70, 3], chunk=8), "chunk_24": dict(lens=[100, 25], chunk=24, group=4), "chunk_32": dict(lens=[100, 31], chunk=32),
    "chunk_100": dict(lens=[250, 100, 101], chunk=100), "chunk_64": dict(lens=[64, 65, 63, 1000], chunk=64, heads=8, group=4, dim=128),
    "long": dict(lens=[5000], heads=4, dim=128), "long_one_head": dict(lens=[20011], heads=1, dim=64, group=4),
    "many_short": dict(lens=[(7 * i) % 23 for i in range(300)], heads=3),
    "loud": dict(lens=[500, 40], gain=12.0), "loud_bf16": dict(lens=[500, 40], gain=12.0, dtype=BF16, dim=128),
}


@pytest.mark.parametrize("name", SHAPES)
def test_matches_64_bits(name):
    bt = Batch(seed=len(name), **SHAPES[name])
    check(bt)
    check(bt, append=True, mass="add")


@pytest.mark.parametrize("name", ["ragged", "ragged_bf16", "chunk_5", "group_17", "long", "mqa_256", "dim_80w"])
@pytest.mark.parametrize("window", [1, 16, 23, 4096])
def test_window(name, window):
    bt = Batch(seed=3, **(SHAPES[name] if name in SHAPES else dict(lens=[90, 0, 24, 23, 22], dim=80, group=5)))
    check(bt, window=window, append=True, mass="add")
    check(bt, window=window, mass="weights")


def test_weights_without_an_accumulator_and_in_place():
    bt = Batch(RAGGED, group=4, seed=11)
    check(bt, mass="weights")
    check(bt, mass="add", in_place=True)


def test_layers_and_scale():
    bt = Batch([40, 18], layers=3, group=2, seed=5)
    for layer in range(3):
        check(bt, layer=layer, append=True)
    check(bt, layer=1, scale=0.5)
    check(bt, layer=1, scale=-0.25)
    check(bt, layer=2, scale=0.0)


def test_repeated_calls_give_the_same_bits():
    bt = Batch([3000, 17, 0, 450], heads=4, group=4, dim=128, seed=2)
    first = call(bt, mass="add")
    for _ in range(3):
        again = call(bt, mass="add")
        assert all(torch.equal(x, y) for x, y in zip(first[:3], again[:3]))


def test_strided_pool():
    """Heads and layers further apart than their rows, and K and V of a head next to each other."""
    bt = Batch([70, 33, 0], heads=3, dim=96, layers=2, group=2, seed=9)
    T, d = bt.n_slots * bt.chunk, bt.dim
    flat = torch.full((2, 3, 2, T * d + 40), 3.0, dtype=F16)                  # [layer][head][K, V][rows, padding]
    flat[..., :T * d] = bt.kv.permute(0, 2, 1, 3, 4).reshape(2, 3, 2, T * d)
    desc = desc_of(bt)
    desc.stride_s, desc.stride_h, desc.stride_l = T * d + 40, 2 * (T * d + 40), 6 * (T * d + 40)
    dev = flat.cuda()
    n, hq = 3, 6
    out, lse = torch.empty(n, hq, d, dtype=F16, device="cuda"), torch.empty(n, hq, device="cuda")
    lens = torch.tensor(bt.lens, dtype=torch.int32).cuda()
    B.decode_attention(desc, 1, dev, bt.q.contiguous().cuda(), bt.table.cuda(), lens, bt.max_len, out, workspace(desc, n, bt.max_len),
                       k_new=bt.k_new.contiguous().cuda(), v_new=bt.v_new.contiguous().cuda(), lse=lse)
    want, wlse, _, wkv, (ot, lt, _) = attend(bt, 1, append=True)
    assert ((out.cpu().double() - want).abs() <= ot).all()
    got = dev.cpu()
    assert torch.equal(bits(got[..., :T * d].reshape(2, 3, 2, T, d).permute(0, 2, 1, 3, 4)), bits(wkv))
    assert (got[..., T * d:] == 3.0).all()


def test_wide_table_and_stale_entries():
    """A table row longer than needed, its unused entries far outside the pool, and rows of a larger table."""
    bt = Batch([30, 64, 1], seed=4)
    wide = torch.full((3, 50), 0x7ffffff0, dtype=torch.int32)
    for b in range(3):
        k = -(-bt.lens[b] // bt.chunk)
        wide[b, :k] = bt.table[b, :k]
    want = call(bt)
    dev, d = wide.cuda(), desc_of(bt)
    for max_len in (64, 500):
        out = torch.empty(3, 2, 64, dtype=F16, device="cuda")
        B.decode_attention(d, 0, bt.kv.cuda(), bt.q.contiguous().cuda(), dev[:, :40] if max_len == 500 else dev,
                           torch.tensor(bt.lens, dtype=torch.int32).cuda(), max_len, out, workspace(d, 3, max_len))
        diff = (out.cpu().double() - want[0].double()).abs()
        assert (diff <= want[0].double().abs() * 2.0 ** -9 + 1e-3).all()


def test_shared_prefix():
    """Two sequences list the same slots for their first chunks."""
    bt = Batch([48, 40], seed=8, group=2)
    bt.table[1, :2] = bt.table[0, :2]
    check(bt, append=True, mass="add")


def test_infinities_and_nan_in_seen_places():
    bt = Batch([40, 40, 40], seed=6)
    kv = bt.kv
    rows = [bt.rows(b) for b in range(3)]
    kv[0, 0, 0, rows[0][3]] = math.nan                        # head 0 of sequence 0: a NaN key
    kv[0, 1, 1, rows[1][39], 5] = math.inf                    # head 1 of sequence 1: one infinite value channel
    out, lse, _, _ = call(bt)
    assert out[0, 0].isnan().all() and lse[0, 0].isnan()
    assert out[1, 1, 5] == math.inf and out[1, 1, :5].isfinite().all() and out[1, 1, 6:].isfinite().all()
    assert out[0, 1].isfinite().all() and out[1, 0].isfinite().all() and out[2].isfinite().all()


def test_a_row_whose_logits_are_all_minus_infinity_is_empty():
    bt = Batch([20], heads=1, seed=1, max_len=20)
    bt.q[:] = 1.0
    bt.kv[0, 0, 0, bt.rows(0)] = -math.inf
    out, lse, mass, _ = call(bt, mass="add")
    assert (out == 0).all() and (lse == -math.inf).all() and torch.equal(mass, bt.mass[0])


def test_invalid_lengths_and_slots_answer_nan_and_touch_nothing():
    bt = Batch([30, 40, 50, 60, 20], seed=12, group=2)
    want, wlse, _, _, (ot, lt, _) = attend(bt, append=True)
    ok = bt.kv.clone()
    ok_rows = {b: bt.rows(b)[-1] for b in (0, 4)}
    bt.table[2, 1] = bt.n_slots                               # one behind the pool
    bt.table[3, 3] = -1                                       # also the slot of the newest token
    d = desc_of(bt)
    kv = bt.kv.cuda()
    lens = torch.tensor([30, 1000, 50, 60, 20], dtype=torch.int32)
    for bad_len in (1000, -3):
        lens[1] = bad_len
        out, lse = torch.zeros(5, 4, 64, dtype=F16, device="cuda"), torch.zeros(5, 4, device="cuda")
        mass = torch.zeros(5, 2, 60, device="cuda")
        B.decode_attention(d, 0, kv, bt.q.contiguous().cuda(), bt.table.cuda(), lens.cuda(), 60, out, workspace(d, 5, 60, True),
                           k_new=bt.k_new.contiguous().cuda(), v_new=bt.v_new.contiguous().cuda(), lse=lse, mass_out=mass)
        out, lse = out.cpu(), lse.cpu()
        for b in (1, 2, 3):
            assert out[b].isnan().all() and lse[b].isnan().all()
        for b in (0, 4):
            assert ((out[b].double() - want[b]).abs() <= ot[b]).all()
    for b, row in ok_rows.items():
        ok[0, 0, :, row], ok[0, 1, :, row] = bt.k_new[b], bt.v_new[b]
    last = bt.table[2, 50 // 16] * 16 + 49 % 16               # sequence 2's newest token has a slot
    ok[0, 0, :, last], ok[0, 1, :, last] = bt.k_new[2], bt.v_new[2]
    assert torch.equal(bits(kv.cpu()), bits(ok))


def test_far_slots():
    """Offsets past 2^31 elements and 2^32 bytes inside one slab."""
    heads, dim, chunk, n_slots = 1, 256, 16, 560000           # 8.96 million rows of 512 bytes: 4.6 GB for K, as much for V
    bt = Batch([50], heads=heads, group=4, dim=dim, chunk=chunk, seed=21)
    far = [n_slots - 1, 0, n_slots - 2, n_slots // 2 + 1]
    kv = torch.empty(1, 2, heads, n_slots * chunk, dim, dtype=F16, device="cuda")
    table = torch.tensor([far], dtype=torch.int32)
    for i, slot in enumerate(far):
        s = int(bt.table[0, i])
        kv[:, :, :, slot * chunk:(slot + 1) * chunk] = bt.kv[:, :, :, s * chunk:(s + 1) * chunk].cuda()
    d = B.make_desc(1, heads, 4, dim, n_slots * chunk, chunk, 16)
    out = torch.empty(1, 4, dim, dtype=F16, device="cuda")
    B.decode_attention(d, 0, kv, bt.q.contiguous().cuda(), table.cuda(), torch.tensor([50], dtype=torch.int32).cuda(), 50, out,
                       workspace(d, 1, 50), k_new=bt.k_new.contiguous().cuda(), v_new=bt.v_new.contiguous().cuda())
    want, _, _, _, (ot, _, _) = attend(bt, append=True)
    assert ((out.cpu().double() - want).abs() <= ot).all()
    row = far[49 // 16] * chunk + 49 % 16
    assert torch.equal(kv[0, 0, 0, row].cpu(), bt.k_new[0, 0]) and torch.equal(kv[0, 1, 0, row].cpu(), bt.v_new[0, 0])


def test_captured_replayed_and_on_another_stream():
    """One captured call replayed while lengths, table and operands change; two graphs share the workspace."""
    bt = Batch([100, 20, 0], group=4, seed=14, max_len=128, dim=128)
    d = desc_of(bt)
    bt.kv[bt.kv.isnan()] = 0.25
    kv, table = bt.kv.cuda(), bt.table.cuda()
    q = bt.q.contiguous().cuda()
    lens = torch.tensor(bt.lens, dtype=torch.int32).cuda()
    ws = workspace(d, 3, 128, True)
    outs = [torch.zeros(3, 8, 128, dtype=F16, device="cuda") for _ in range(2)]
    mass = torch.zeros(3, 2, 128, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(s):
        B.decode_attention(d, 0, kv, q, table, lens, 128, outs[0], ws, mass_out=mass)
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                B.decode_attention(d, 0, kv, q, table, lens, 128, outs[i], ws, mass_out=mass if i else None)
            graphs.append(g)
    s.synchronize()
    for lens_now in ([100, 20, 0], [37, 0, 0], [99, 17, 0], [0, 1, 0]):
        bt.lens = lens_now
        lens.copy_(torch.tensor(lens_now, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(sum(lens_now))).to(F16))
        bt.q = q.cpu()
        for i, g in enumerate(graphs):
            outs[i].fill_(9.0)
            g.replay()
        torch.cuda.synchronize()
        want, _, _, _, (ot, _, _) = attend(bt)
        for o in outs:
            assert ((o.cpu().double() - want).abs() <= ot).all()
        assert torch.equal(outs[0], outs[1])


def test_largest_batch():
    """4096 sequences, most of them empty or a few tokens long."""
    bt = Batch([(i * 7919) % 5 if i % 3 else 0 for i in range(4095)] + [70], heads=1, dim=16, group=2, seed=17)
    check(bt, append=True, mass="add")


def test_two_streams_at_once():
    """Two batches in one pool, on two streams with a workspace each, many calls in flight."""
    both = [Batch([900, 30, 0, 411], heads=2, group=4, dim=128, seed=s) for s in (41, 42)]
    streams = [torch.cuda.Stream() for _ in both]
    jobs = []
    for bt in both:
        d = desc_of(bt)
        jobs.append((d, bt.kv.cuda(), bt.q.contiguous().cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(),
                     [torch.empty(4, 8, 128, dtype=F16, device="cuda") for _ in range(20)], workspace(d, 4, 900), bt.k_new.contiguous().cuda(),
                     bt.v_new.contiguous().cuda()))
    torch.cuda.synchronize()
    for i in range(20):
        for s, (d, kv, q, table, lens, outs, ws, k, v) in zip(streams, jobs):
            B.decode_attention(d, 0, kv, q, table, lens, 900, outs[i], ws, k_new=k, v_new=v, stream=s)
    torch.cuda.synchronize()
    for bt, job in zip(both, jobs):
        want, _, _, _, (ot, _, _) = attend(bt, append=True)
        for o in job[5]:
            assert torch.equal(o, job[5][0])
        assert ((job[5][0].cpu().double() - want).abs() <= ot).all()


def test_refusals():
    bt = Batch([20, 30], group=2, seed=1)
    d = desc_of(bt)
    kv, q, table, lens = bt.kv.cuda(), bt.q.contiguous().cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda()
    k = bt.k_new.contiguous().cuda()
    out, ws = torch.full_like(q, 5.0), workspace(d, 2, 30, True)
    mass = torch.zeros(2, 2, 30, device="cuda")

    def refused(status, **kw):
        args = dict(layer=0, kv=kv, q=q, chunk_table=table, lens=lens, max_len=30, out=out, workspace=ws)
        args.update(kw)
        with pytest.raises(B.LlmsError) as e:
            B.decode_attention(d, **args)
        assert e.value.status == status

    refused(B.ERR_INVALID_ARG, layer=1)
    refused(B.ERR_INVALID_ARG, layer=-1)
    refused(B.ERR_INVALID_ARG, max_len=33)                    # more than the table's two chunks hold
    refused(B.ERR_INVALID_ARG, max_len=0)
    refused(B.ERR_INVALID_ARG, window=-1)
    refused(B.ERR_INVALID_ARG, scale=math.inf)
    refused(B.ERR_INVALID_ARG, k_new=k)
    refused(B.ERR_INVALID_ARG, mass_in=mass)
    refused(B.ERR_INVALID_ARG, mass_out=mass[..., :29].contiguous())
    refused(B.ERR_INVALID_ARG, q=q.to(BF16))
    refused(B.ERR_INVALID_ARG, q=q.cpu())
    refused(B.ERR_INVALID_ARG, lens=lens.long())
    refused(B.ERR_INVALID_ARG, chunk_table=table.t())
    refused(B.ERR_INVALID_ARG, out=out[:1])
    refused(B.ERR_UNSUPPORTED, kv=kv.float())
    refused(B.ERR_MISALIGNED, workspace=ws[16:])
    refused(B.ERR_INVALID_ARG, workspace=ws[:0])              # an empty tensor has no address
    refused(B.ERR_BUF_TOO_SMALL, workspace=ws[:-1], mass_out=mass)
    torch.cuda.synchronize()
    assert (out == 5.0).all()
