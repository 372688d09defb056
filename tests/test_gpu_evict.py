"""Eviction by accumulated attention weight against its plain form, bit for bit, and the operators in a run together."""
import math

import pytest
import torch

from paper_2403_11805_b200 import binding as B
from paged_reference import Batch, attend, bits, evict
from test_gpu_decode import desc_of, workspace

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def call(bt, mass, budget, recent, dst_table=None, mass_out="other", kv=None):
    L, n, H, M = mass.shape
    dev_mass = mass.cuda()
    other = dev_mass if mass_out == "same" else torch.full_like(dev_mass, 5.0)
    kept = torch.full((L, n, H, budget), -9, dtype=torch.int32, device="cuda")
    new_lens = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    kv = bt.kv.cuda() if kv is None else kv
    B.evict_tokens(desc_of(bt), kv, dev_mass, bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len, budget, recent,
                   kept, new_lens, mass_out=None if mass_out == "same" else other, dst_table=None if dst_table is None else dst_table.cuda())
    torch.cuda.synchronize()
    return kept.cpu(), new_lens.cpu(), other.cpu(), kv.cpu()


def check(bt, mass, budget, recent, dst_table=None, mass_out="other"):
    got = call(bt, mass, budget, recent, dst_table, mass_out)
    before = mass if mass_out == "same" else torch.full_like(mass, 5.0)
    want = evict(bt, mass, budget, recent, dst_table, before)
    assert torch.equal(got[1], want[1])
    assert torch.equal(got[0], want[0])
    assert torch.equal(got[2].view(torch.int32), want[2].view(torch.int32))
    assert torch.equal(bits(got[3]), bits(want[3]))
    return got


def other_slots(bt, budget):
    """A table into slots that the batch's sequences do not list: the pool grows by them."""
    need = [-(-min(x, budget) // bt.chunk) for x in bt.lens]
    width = max(max(need), -(-min(budget, bt.max_len) // bt.chunk))
    first = bt.n_slots
    bt.n_slots += sum(need)
    extra = torch.zeros(*bt.kv.shape[:3], sum(need) * bt.chunk, bt.dim, dtype=bt.dtype)
    bt.kv = torch.cat([bt.kv, extra], dim=3)
    slots = list(range(first, bt.n_slots))
    dst = torch.full((len(bt.lens), width), -1, dtype=torch.int32)
    for b, k in enumerate(need):
        for i in range(k):
            dst[b, i] = slots.pop()
    return dst


SHAPES = {
    "one_token": (dict(lens=[1]), 1, 0),
    "keep_one": (dict(lens=[50, 3, 0, 1]), 1, 0), "keep_last": (dict(lens=[50, 3, 0, 1]), 1, 1),
    "ragged": (dict(lens=[37, 0, 1, 16, 15, 17, 64, 5, 200, 33]), 16, 4),
    "nothing_to_do": (dict(lens=[20, 7]), 64, 3), "exactly": (dict(lens=[64, 65]), 64, 8),
    "recent_only": (dict(lens=[100, 12]), 20, 20), "by_mass_only": (dict(lens=[100, 12]), 20, 0),
    "odd": (dict(lens=[2047], heads=1, dim=256, dtype=BF16, layers=3), 1001, 65),
    "layers_heads": (dict(lens=[90, 120], heads=5, dim=80, layers=4, chunk=32), 47, 13),
    "chunk_1": (dict(lens=[40, 9], chunk=1), 7, 2), "chunk_7": (dict(lens=[100, 33], chunk=7, dim=48), 31, 5),
    "dim_16": (dict(lens=[70], dim=16), 33, 1), "dim_112": (dict(lens=[70], dim=112, layers=2), 33, 1),
    "long": (dict(lens=[9001, 4096, 5], heads=2, dim=64), 3000, 100), "long_most": (dict(lens=[9001], heads=2, dim=64), 8999, 1),
    "longest": (dict(lens=[70000], heads=1, dim=16), 20000, 777),
    "long_among_many": (dict(lens=[20001, 17000] + [i % 5 for i in range(150)], heads=1, dim=16), 9000, 300),
}


@pytest.mark.parametrize("where", ["in_place", "other_slots"])
@pytest.mark.parametrize("name", SHAPES)
def test_matches_the_plain_form(name, where):
    kw, budget, recent = SHAPES[name]
    bt = Batch(seed=len(name), **kw)
    dst = other_slots(bt, budget) if where == "other_slots" else None
    check(bt, bt.mass, budget, recent, dst)
    check(bt, bt.mass, budget, recent, dst, mass_out="same")


# Calls of one kernel: few batches of rows; items enough for every SM; more items than run at once
ONE_KERNEL = {
    "one_batch": (dict(lens=[90, 33], heads=3, dim=256), 17, 2), "three_batches": (dict(lens=[190, 97, 0, 96]), 192 // 2, 5),
    "three_batches_512": (dict(lens=[1500, 385, 384, 383], dim=64), 384, 11), "four_batches": (dict(lens=[300, 200]), 193, 5),
    "many": (dict(lens=[i * 37 % 700 for i in range(120)], heads=2, dim=48), 400, 9),
    "many_512": (dict(lens=[1500] + [i * 41 % 300 for i in range(119)], heads=2, dim=80, dtype=BF16), 600, 0),
    "more_than_fit": (dict(lens=[1300, 0] + [i * 29 % 90 for i in range(98)], heads=7, dim=112), 1190, 30),
    "pairs": (dict(lens=[256, 255, 31, 32, 33, 0, 1, 2, 64], heads=3), 40, 7), "pairs_to_257": (dict(lens=[257, 256, 128]), 64, 0),
    "short_many": (dict(lens=[i % 64 for i in range(1, 101)], heads=7, dim=256), 9, 2),
    "pairs_many": (dict(lens=[i * 5 % 129 for i in range(100)], heads=7, dim=240, chunk=5), 70, 1),
    "little_kept": (dict(lens=[i * 53 % 601 for i in range(100)], heads=7, dim=80, dtype=BF16), 256, 200),
    "more_than_fit_layers": (dict(lens=[9, 800, 41, 300], heads=19, dim=256, layers=8), 500, 499),
}


@pytest.mark.parametrize("where", ["in_place", "other_slots"])
@pytest.mark.parametrize("name", ONE_KERNEL)
def test_selected_and_moved_by_one_kernel(name, where):
    kw, budget, recent = ONE_KERNEL[name]
    bt = Batch(seed=len(name), **kw)
    dst = other_slots(bt, budget) if where == "other_slots" else None
    check(bt, bt.mass, budget, recent, dst)
    check(bt, (bt.mass * 0.3).round(), budget, recent, dst, mass_out="same")


def test_invalid_lengths_and_slots_among_many():
    lens = [60 + i % 40 for i in range(150)]
    bt, clean = Batch(lens, heads=2, seed=9), Batch(lens, heads=2, seed=9)
    bt.table[2, 1] = bt.n_slots + 5
    given = list(lens)
    given[5], given[77] = 100, -3                 # above max_len, below zero
    d, kv = desc_of(bt), bt.kv.cuda()
    kept = torch.zeros(1, 150, 2, 40, dtype=torch.int32, device="cuda")
    new_lens = torch.zeros(150, dtype=torch.int32, device="cuda")
    B.evict_tokens(d, kv, bt.mass.cuda(), bt.table.cuda(), torch.tensor(given, dtype=torch.int32).cuda(), 99, 40, 3, kept, new_lens)
    assert new_lens.tolist() == [-1 if b in (5, 77) else 40 for b in range(150)] and (kept[:, [5, 77]] == -1).all()
    want, got = evict(clean, clean.mass, 40, 3), kv.cpu()
    for b in range(150):
        if b == 2:
            continue
        rows = clean.rows(b)
        assert torch.equal(bits(got[:, :, :, rows]), bits((bt.kv if b in (5, 77) else want[3])[:, :, :, rows])), b


@pytest.mark.parametrize("tokens", [327680, 327681, 393216, 500001])
def test_masses_up_to_and_beyond_a_cluster_s_shared_memory(tokens):
    bt = Batch([tokens, 3], heads=1, dim=16, seed=2)
    check(bt, bt.mass, 1000, 10)
    check(bt, bt.mass, tokens // 3, 10, mass_out="same")


@pytest.mark.parametrize("where", ["in_place", "other_slots"])
@pytest.mark.parametrize("lens", [[16500, 20000, 16384, 16385], [17001]], ids=["several_long", "one_long"])
def test_one_kernel_whose_masses_do_not_fit_shared_memory(lens, where):
    """More items than the GPU takes at once, and a length bound beyond what a CTA holds: masses are read again in every pass, and
    written over in place tile by tile."""
    bt = Batch(lens + [(i * 31) % 90 for i in range(100)], heads=7, dim=16, seed=len(lens))
    dst = other_slots(bt, 9000) if where == "other_slots" else None
    check(bt, bt.mass, 9000, 70, dst, mass_out="same")
    check(bt, (bt.mass * 0.3).round(), 9000, 70, dst, mass_out="same")
    check(bt, bt.mass, 9000, 70, dst)


VALUES = {
    "all_equal": lambda m: torch.full_like(m, 2.5), "all_zero": lambda m: torch.zeros_like(m),
    "few_values": lambda m: (m * 0.2).round(), "signed_zeros": lambda m: torch.where(m > 1, 0.0, -0.0),
    "nan": lambda m: torch.where(m > 0.5, math.nan, m), "all_nan": lambda m: torch.full_like(m, math.nan),
    "infinities": lambda m: torch.where(m > 5, math.inf, torch.where(m < 0.01, -math.inf, m)),
    "negative": lambda m: 3.0 - m, "lowest": lambda m: torch.where(m > 0.5, torch.finfo(torch.float32).min, m),
    "tiny": lambda m: m * 1e-41, "rising": lambda m: torch.arange(m.shape[-1]).float().expand(m.shape).contiguous(),
    "falling": lambda m: -torch.arange(m.shape[-1]).float().expand(m.shape).contiguous(),
    "close": lambda m: 1.0 + (m * 8).round() * 2.0 ** -23,
}


@pytest.mark.parametrize("name", VALUES)
def test_values(name):
    bt = Batch([300, 41, 0, 1100], layers=2, seed=3)
    mass = VALUES[name](bt.mass)
    for budget, recent in ((100, 10), (299, 0), (41, 41)):
        check(bt, mass, budget, recent)


@pytest.mark.parametrize("name", VALUES)
def test_values_of_few_tokens(name):
    bt = Batch([250, 41, 0, 97, 33], layers=2, seed=4)
    mass = VALUES[name](bt.mass)
    for budget, recent in ((100, 10), (32, 0), (41, 41), (249, 0), (1, 0)):
        check(bt, mass, budget, recent)
        check(bt, mass, budget, recent, mass_out="same")


def test_dst_table_may_be_the_table_itself():
    bt = Batch([90, 40], seed=5)
    a = call(bt, bt.mass, 33, 4)
    want = evict(bt, bt.mass, 33, 4, None, torch.full_like(bt.mass, 5.0))
    assert torch.equal(bits(a[3]), bits(want[3]))


def test_the_table_as_its_own_destination_is_in_place():
    bt = Batch([90, 40, 500], seed=5)
    dev, lens = bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda()
    kept, new_lens = torch.zeros(1, 3, 2, 33, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    kv = bt.kv.cuda()
    B.evict_tokens(desc_of(bt), kv, bt.mass.cuda(), dev, lens, 500, 33, 4, kept, new_lens, dst_table=dev)
    want = evict(bt, bt.mass, 33, 4)
    assert torch.equal(kept.cpu(), want[0]) and torch.equal(bits(kv.cpu()), bits(want[3]))


@pytest.mark.parametrize("lens", [[2000], [2000, 1500, 700]], ids=["one", "several"])
@pytest.mark.parametrize("view", ["whole", "first_chunks"])
def test_a_view_of_the_table_as_destination_is_in_place(view, lens):
    """16 batches of rows and a kernel of their own for moving: rows taken in another order than upwards would be overwritten."""
    bt = Batch(lens, heads=4, dim=128, seed=15)
    dev, n_lens = bt.table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    dst = dev if view == "whole" else dev[:, :-(-1000 // bt.chunk)]
    n = len(lens)
    kept, new_lens = torch.zeros(1, n, 4, 1000, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    kv, mass = bt.kv.cuda(), bt.mass.cuda()
    B.evict_tokens(desc_of(bt), kv, mass, dev, n_lens, 2000, 1000, 40, kept, new_lens, dst_table=dst)
    want = evict(bt, bt.mass, 1000, 40, None, bt.mass)
    assert torch.equal(kept.cpu(), want[0]) and torch.equal(new_lens.cpu(), want[1])
    assert torch.equal(mass.cpu(), want[2]) and torch.equal(bits(kv.cpu()), bits(want[3]))


def test_in_place_twice_and_repeatable():
    bt = Batch([3000, 777], heads=4, dim=128, seed=6, layers=2)
    first = call(bt, bt.mass, 1500, 64)
    for _ in range(3):
        again = call(bt, bt.mass, 1500, 64)
        assert all(torch.equal(x, y) for x, y in zip(first[:3], again[:3])) and torch.equal(bits(first[3]), bits(again[3]))
    small = Batch([3000, 777], heads=4, dim=128, seed=6, layers=2)
    small.kv, small.lens = first[3], first[1].tolist()
    check(small, first[2], 700, 10)


def test_invalid_lengths_and_slots_are_left_alone():
    bt = Batch([50, 60, 70], seed=7)
    bt.table[2, 1] = bt.n_slots + 5
    d = desc_of(bt)
    kv = bt.kv.cuda()
    kept = torch.zeros(1, 3, 2, 20, dtype=torch.int32, device="cuda")
    new_lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    mass, out = bt.mass.cuda(), torch.full_like(bt.mass, 5.0).cuda()
    B.evict_tokens(d, kv, mass, bt.table.cuda(), torch.tensor([50, 71, 70], dtype=torch.int32).cuda(), 70, 20, 3, kept, new_lens, mass_out=out)
    assert new_lens.tolist() == [20, -1, 20] and (kept[:, 1] == -1).all() and (out[:, 1] == 5.0).all()
    want = evict(Batch([50, 60, 70], seed=7), bt.mass, 20, 3)
    assert torch.equal(kept[:, 0].cpu(), want[0][:, 0]) and torch.equal(kept[:, 2].cpu(), want[0][:, 2])
    got = kv.cpu()
    rows = bt.rows(1, upto=60)
    assert torch.equal(bits(got[:, :, :, rows]), bits(bt.kv[:, :, :, rows]))
    rows = Batch([50, 60, 70], seed=7).rows(0)
    assert torch.equal(bits(got[:, :, :, rows]), bits(want[3][:, :, :, rows]))


def test_captured_and_replayed():
    bt = Batch([200, 90], seed=8, layers=2)
    d = desc_of(bt)
    dst = other_slots(bt, 64)
    d = desc_of(bt)
    kv, table, dst_dev, mass = bt.kv.cuda(), bt.table.cuda(), dst.cuda(), bt.mass.cuda()
    lens = torch.tensor(bt.lens, dtype=torch.int32).cuda()
    out = torch.full_like(mass, 5.0)
    kept, new_lens = torch.zeros(2, 2, 2, 64, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.evict_tokens(d, kv, mass, table, lens, 200, 64, 8, kept, new_lens, mass_out=out, dst_table=dst_dev)
    for now in ([200, 90], [64, 3], [130, 0]):
        bt.lens = now
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        bt.mass = torch.rand(bt.mass.shape, generator=torch.Generator().manual_seed(sum(now)))
        mass.copy_(bt.mass)
        out.fill_(5.0)
        bt.kv = kv.cpu()
        g.replay()
        torch.cuda.synchronize()
        want = evict(bt, bt.mass, 64, 8, dst, torch.full_like(bt.mass, 5.0))
        assert torch.equal(kept.cpu(), want[0]) and torch.equal(out.cpu(), want[2]) and torch.equal(bits(kv.cpu()), bits(want[3]))


def test_refusals():
    bt = Batch([20, 30], seed=1)
    d = desc_of(bt)
    kv, table, lens, mass = bt.kv.cuda(), bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.mass.cuda()
    kept, new_lens = torch.zeros(1, 2, 2, 8, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")

    def refused(status, **kw):
        args = dict(kv=kv, mass=mass, chunk_table=table, lens=lens, max_len=30, budget=8, recent=2, kept=kept, new_lens=new_lens)
        args.update(kw)
        with pytest.raises(B.LlmsError) as e:
            B.evict_tokens(d, **args)
        assert e.value.status == status

    refused(B.ERR_INVALID_ARG, budget=0, kept=kept[..., :0])
    refused(B.ERR_INVALID_ARG, recent=9)
    refused(B.ERR_INVALID_ARG, recent=-1)
    refused(B.ERR_INVALID_ARG, max_len=33)
    refused(B.ERR_INVALID_ARG, kept=kept[..., :7])
    refused(B.ERR_INVALID_ARG, new_lens=lens)
    refused(B.ERR_INVALID_ARG, kv=kv.float())
    refused(B.ERR_INVALID_ARG, mass=mass.double())
    refused(B.ERR_INVALID_ARG, mass=mass.cpu())
    refused(B.ERR_INVALID_ARG, mass_out=mass[..., :20])
    refused(B.ERR_INVALID_ARG, dst_table=table[:, :0])
    torch.cuda.synchronize()
    assert (kept == 0).all() and (new_lens == 0).all()


def test_generation_with_eviction_together():
    """Decode steps append tokens and gather weights in both layers; eviction shrinks every sequence; decoding goes on over
    what is left; each step against the 64-bit form on the state the device holds."""
    bt = Batch([60, 33, 0, 5], heads=2, group=4, dim=64, layers=2, seed=31, max_len=96)
    need = 96 // bt.chunk
    bt.table = torch.arange(4 * need, dtype=torch.int32).flip(0).reshape(4, need).contiguous()
    bt.n_slots = 4 * need
    g = torch.Generator().manual_seed(5)
    bt.kv = torch.randn(2, 2, 2, bt.n_slots * bt.chunk, 64, generator=g).half()
    d = desc_of(bt)
    kv, table = bt.kv.cuda(), bt.table.cuda()
    lens = torch.tensor(bt.lens, dtype=torch.int32).cuda()
    active = (lens > 0).int()
    mass = torch.zeros(2, 4, 2, 96, device="cuda")
    ws = workspace(d, 4, 96, True)
    kept, new_lens = torch.zeros(2, 4, 2, 40, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for step in range(14):
        lens += active
        bt.lens = lens.tolist()
        for layer in range(2):
            bt.qkv = torch.randn(4, 12, 64, generator=g).half()
            bt.q, bt.k_new, bt.v_new = bt.qkv[:, :8], bt.qkv[:, 8:10], bt.qkv[:, 10:]
            bt.kv, bt.mass = kv.cpu(), mass.cpu()
            dev = bt.qkv.cuda()
            out = torch.empty(4, 8, 64, dtype=torch.float16, device="cuda")
            B.decode_attention(d, layer, kv, dev[:, :8], table, lens, 96, out, ws, k_new=dev[:, 8:10], v_new=dev[:, 10:],
                               mass_in=mass[layer], mass_out=mass[layer])
            want, _, wmass, wkv, (ot, _, mt) = attend(bt, layer, append=True, mass_in=bt.mass[layer], mass_before=bt.mass[layer])
            assert ((out.cpu().double() - want).abs() <= ot).all()
            assert ((mass[layer].cpu().double() - wmass).abs() <= mt).all()
            assert torch.equal(bits(kv.cpu()), bits(wkv))
        if step in (5, 9):
            bt.kv, bt.mass = kv.cpu(), mass.cpu()
            B.evict_tokens(d, kv, mass, table, lens, 96, 40, 8, kept, new_lens)
            want = evict(bt, bt.mass, 40, 8, None, bt.mass)
            assert torch.equal(kept.cpu(), want[0]) and torch.equal(new_lens.cpu(), want[1])
            assert torch.equal(mass.cpu(), want[2]) and torch.equal(bits(kv.cpu()), bits(want[3]))
            lens.copy_(new_lens)
    assert lens.tolist() == [44, 44, 0, 19]
