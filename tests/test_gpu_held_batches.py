"""Attention over a held pool in the form that a call takes for large batches, against 64 bits: rings of two stages, as many warps as
an SM has room for, several rounds of runs.  A call takes it when n_seqs * KV heads * blocks of query rows * ceil(max_len / 32) is
above 32 for each of the warps that small batches get, of which there are at most eight per SM; the tests go by that bound."""
import math

import numpy as np
import pytest
import torch

import test_gpu_held_attention as A
from held_reference import Format, HeldBatch, attend, quantise
from paged_reference import bits as bits_of
from paper_2403_11805_b200 import binding as B

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def tiles_of_a_large_batch():
    return torch.cuda.get_device_properties(0).multi_processor_count * 8 * 32


def items(n, heads, group):
    return n * heads * -(-group // 16)


def large(how="large", **kw):
    """The batch between empty sequences, with a bound on the lengths that makes it a large one."""
    heads, group, lens = kw.get("heads", 2), kw.get("group", 1), kw["lens"]
    n = len(lens) + -(-A.MANY_ITEMS // heads)
    kw["max_len"] = max(max(lens), 32 * (tiles_of_a_large_batch() // items(n, heads, group) + 1))
    bt = HeldBatch(**kw)
    A.padded(bt)
    assert len(bt.lens) == n
    return bt


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("name", A.SHAPES)
def test_matches_64_bits(name, bits):
    bt = large(lens=A.RAGGED + [130, 257], bits=bits, seed=len(name), dtype=F16 if len(name) % 2 else BF16, **A.SHAPES[name])
    A.check(bt)
    A.check(bt, append=True)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 500])
def test_lengths(length):
    A.check(large(lens=[length], heads=3, dim=64, seed=length), append=True)


@pytest.mark.parametrize("bits,group", [(4, 1), (8, 4), (4, 9)])
def test_a_wide_window(bits, group):
    bt = large(lens=[2000, 1301, 1300, 1299, 37, 1], bits=bits, group=group, heads=1, dim=64, chunk=32, seed=40)
    assert items(len(bt.lens), 1, group) * (1300 // 32) > tiles_of_a_large_batch()
    A.check(bt, window=1300)
    A.check(bt, window=1300, append=True)


@pytest.mark.parametrize("window", [1, 40, 64])
def test_a_narrow_window(window):
    bt = HeldBatch([(i * 37) % 90 if i % 50 == 0 else 0 for i in range(4096)], heads=10, dim=64, seed=41)
    A.check(bt, window=window, append=True)


@pytest.mark.parametrize("test,args", [
    (A.test_layers_and_scale, ()), (A.test_steep_and_flat_weights, (40.0,)), (A.test_steep_and_flat_weights, (1e-3,)), (A.test_constant_groups, ()),
    (A.test_a_newest_token_that_is_no_number, ()), (A.test_large_and_small_queries, ()), (A.test_a_captured_step_follows_its_lengths, ()),
], ids=lambda x: getattr(x, "__name__", None) or "-".join(map(str, x)))
def test_what_smaller_batches_do(test, args, monkeypatch):
    monkeypatch.setattr(A, "batch", large)
    test(*args, "large")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_queries_that_are_no_numbers(value, dtype, monkeypatch):
    monkeypatch.setattr(A, "batch", large)
    A.test_queries_that_are_no_numbers(value, dtype, "large")


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scales_of_very_different_size(dtype, monkeypatch):
    monkeypatch.setattr(A, "batch", large)
    A.test_scales_of_very_different_size("large", dtype)


@pytest.mark.parametrize("bad_len", [100000, -3])
def test_invalid_lengths_and_slots(bad_len, monkeypatch):
    monkeypatch.setattr(A, "batch", large)
    A.test_invalid_lengths_and_slots_answer_nan_and_touch_nothing(bad_len, "large")


def test_nan_groups():
    """A NaN group of K makes its head's row NaN; one of V only its channels; neither that of another sequence."""
    bt = large(lens=[70, 70, 70], seed=8, dim=128, span=64, group=2)
    at = next(i for i, x in enumerate(bt.lens) if x)
    for half in range(2):
        row = int(bt.rows(at + half)[65])
        x = bt.kv[0, half, half, row].clone()
        x[64:] = math.nan
        bt.store(bt.pool, 0, half, half, row, x)
    out, lse, _ = A.call(bt)
    assert out[at, :2].isnan().all() and lse[at, :2].isnan().all() and out[at, 2:].isfinite().all() and lse[at, 2:].isfinite().all()
    assert out[at + 1, 2:, 64:].isnan().all() and out[at + 1, 2:, :64].isfinite().all() and out[at + 1, :2].isfinite().all() and lse[at + 1].isfinite().all()
    assert out[at + 2].isfinite().all() and lse[at + 2].isfinite().all()


def test_shared_prefix():
    bt = large(lens=[48, 40], seed=14, group=2)
    at = next(i for i, x in enumerate(bt.lens) if x)
    bt.table[at + 1, :2] = bt.table[at, :2]
    A.check(bt, append=True)


# ----------------------------------------------------------------------------- whole large batches: pool and formula on the GPU

class Large:
    """A pool of random codes, scales and zero-points, and a batch whose sequences lie in it in random order."""

    def __init__(self, lens, dim, bits, span, heads, group, dtype, chunk, seed, max_len=None):
        self.lens, self.dim, self.bits, self.span, self.heads, self.group, self.dtype, self.chunk = lens, dim, bits, span, heads, group, dtype, chunk
        self.max_len = max_len or max(lens)
        self.format = f = Format(dim, bits, span)
        g = torch.Generator(device="cuda").manual_seed(seed)
        need = [-(-x // chunk) for x in lens]
        slots = sum(need) + 2
        self.desc = B.make_desc(1, heads, heads * group, dim, slots * chunk, chunk, span)
        self.pool = torch.randint(0, 256, (heads, slots * chunk // 16, f.tile), dtype=torch.uint8, device="cuda", generator=g)
        scale, zero = (torch.randn(self.pool.shape[:2] + (f.params // 2,), device="cuda", generator=g) for _ in range(2))
        params = torch.stack([scale.abs() * 2 / (2 ** bits - 1), zero - 1], -1).half()
        self.pool[..., 2 * f.codes:] = params.reshape(heads, -1, f.params).view(torch.uint8)
        order = torch.randperm(slots, device="cuda", generator=g).to(torch.int32)
        self.table = torch.full((len(lens), -(-self.max_len // chunk)), -7, dtype=torch.int32, device="cuda")
        for b, n in enumerate(need):
            self.table[b, :n] = order[sum(need[:b]):sum(need[:b + 1])]
        self.qkv = torch.randn(len(lens), heads * (group + 2), dim, device="cuda", generator=g).to(dtype)
        hq = heads * group
        self.q, self.k_new, self.v_new = self.qkv[:, :hq], self.qkv[:, hq:hq + heads], self.qkv[:, hq + heads:]

    def newest(self, b):
        """The tile and the place in it of a sequence's newest token."""
        t = self.lens[b] - 1
        row = int(self.table[b, t // self.chunk]) * self.chunk + t % self.chunk
        return row // 16, row % 16

    def with_newest(self):
        """The pool with the new tokens' rows in it."""
        pool = self.pool.clone()
        k, v = quantise(self.k_new.cpu(), self.bits, self.span), quantise(self.v_new.cpu(), self.bits, self.span)
        for b, n in enumerate(self.lens):
            if n:
                tile, place = self.newest(b)
                mine = pool[:, tile].cpu().numpy()
                for h in range(self.heads):
                    for half, x in enumerate((k, v)):
                        self.format.put(mine[h], half, place, *(p[b, h] for p in x))
                pool[:, tile] = torch.from_numpy(mine).cuda()
        return pool

    def parts(self, pool, b, first):
        """(codes * scale, zero-point) of K and of V of tokens first .. of a sequence: [heads, tokens, dim] in 64 bits; V's scales."""
        n, f = self.lens[b], self.format
        t = torch.arange(first // 16 * 16, n, 16, device="cuda")
        tiles = pool[:, self.table[b, t // self.chunk].long() * (self.chunk // 16) + t % self.chunk // 16]
        cut = slice(first % 16, first % 16 + n - first)
        got = []
        for half in range(2):
            at, shift = (torch.from_numpy(x[half]).cuda() for x in (f.byte, f.shift))
            codes = ((tiles[..., at] >> shift.to(torch.uint8)) & (2 ** self.bits - 1)).flatten(1, 2)[:, cut].double()
            p = tiles[..., 2 * f.codes + half * f.params:][..., :f.params].contiguous().view(torch.float16).double()
            p = p.reshape(self.heads, -1, f.groups, 2)[:, cut]
            scale, zero = (p[..., i].repeat_interleave(self.span, -1) for i in range(2))
            got.append((codes * scale, zero))
        return got, p[..., 0]

    def attend(self, pool, b, window):
        """(out, lse, their tolerances) of a sequence, by held_reference's formulas and bounds."""
        n, G = self.lens[b], self.group
        first = max(0, n - window) if window else 0
        ((kc, kz), (vc, vz)), v_scale = self.parts(pool, b, first)
        q, scale, half_step, groups = self.q[b].double().reshape(self.heads, G, self.dim), self.dim ** -0.5, torch.finfo(self.dtype).eps / 2, self.dim // self.span
        s = q @ (kc + kz).mT * scale
        es = (q.abs() @ (kc.abs() + kz.abs()).mT).amax(2, keepdim=True) * scale * (self.dim + groups + 4) * 2.0 ** -23
        es = es + s.abs().amax(2, keepdim=True) * 2.0 ** -21 + 2.0 ** -20 + (n - first) * 2.0 ** -24
        p = torch.softmax(s, 2)
        out, lse = p @ (vc + vz), torch.logsumexp(s, 2)
        lost = p.amax(2, keepdim=True) * v_scale.amax((1, 2))[:, None, None] * (n - first) * (2 ** self.bits - 1) * 2.0 ** -29
        tol = out.abs() * half_step + (2 * es + 2.0 ** -19) * (p @ (vc.abs() + vz.abs())) + 2.0 ** -25 + lost
        return out.flatten(0, 1), lse.flatten(), tol.flatten(0, 1), (es[..., 0] + lse.abs() * 2.0 ** -23).flatten()

    def check(self, window=0, append=False):
        n, hq = len(self.lens), self.heads * self.group
        seen = min(self.max_len, window) if window else self.max_len
        assert items(n, self.heads, self.group) * (seen // 32) > tiles_of_a_large_batch()
        held, want_pool = self.pool.clone(), self.with_newest() if append else self.pool
        out, lse = torch.full((n, hq, self.dim), 9.0, dtype=self.dtype, device="cuda"), torch.full((n, hq), 9.0, device="cuda")
        B.held_attention(self.desc, self.bits, 0, held, self.q, self.table, torch.tensor(self.lens, dtype=torch.int32).cuda(), self.max_len, out,
                         A.workspace(self.desc, self.bits, n, self.max_len), k_new=self.k_new if append else None, v_new=self.v_new if append else None,
                         window=window, lse=lse)
        torch.cuda.synchronize()
        assert torch.equal(held, want_pool)
        for b, length in enumerate(self.lens):
            if length == 0:
                assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
                continue
            want, want_lse, tol, lse_tol = self.attend(want_pool, b, window)
            assert ((out[b].double() - want).abs() <= tol).all(), b
            assert ((lse[b].double() - want_lse).abs() <= lse_tol).all(), b


POOLS = [(64, 4, 64), (64, 8, 32), (96, 4, 32), (96, 8, 32), (128, 4, 128), (128, 4, 32), (128, 8, 64), (256, 4, 256), (256, 4, 64), (256, 8, 128)]


@pytest.mark.parametrize("group", [1, 3, 8, 16])
@pytest.mark.parametrize("dim,bits,span", POOLS)
def test_long_runs(dim, bits, span, group):
    """Two long sequences: a run has some ten to sixty tiles, a ring is gone round many times."""
    bt = Large([170017, 161000], dim, bits, span, heads=4, group=group, dtype=BF16 if (dim + group) % 3 == 0 else F16, chunk=64 if bits == 4 else 16, seed=dim + group)
    bt.check(append=group != 3)


@pytest.mark.parametrize("bound", [9000, 18000])
@pytest.mark.parametrize("group", [1, 4, 8, 40])
@pytest.mark.parametrize("dim,bits,span", POOLS[::3])
def test_several_rounds_of_runs(dim, bits, span, group, bound):
    """Ragged sequences far below the bound on their lengths: more runs than warps, that begin and end anywhere in an item."""
    lens = [(i * 977) % 4001 for i in range(70)] + [0, 1, 16, 33]
    bt = Large(lens, dim, bits, span, heads=4, group=group, dtype=F16 if bits == 4 else BF16, chunk=48, seed=bits + group, max_len=bound)
    bt.check(append=True)


@pytest.mark.parametrize("dim,bits,span", POOLS[1::4])
def test_windows_of_long_sequences(dim, bits, span):
    lens = [(i * 977) % 9001 for i in range(60)]
    Large(lens, dim, bits, span, heads=8, group=2, dtype=F16, chunk=32, seed=5, max_len=9000).check(window=4097, append=True)


# ----------------------------------------------------------------------------- what must have no influence

JUNK = {"infinite": 0x7c00, "negative infinite": 0xfc00, "largest": 0x7bff, "most negative": 0xfbff, "not a number": 0x7e00}


@pytest.mark.parametrize("how", A.HOW + ["large"])
@pytest.mark.parametrize("append", [False, True])
def test_workspaces_and_rows_without_tokens_have_no_influence(how, append):
    """Results are the same bits whatever the workspace holds and whatever codes and parameters lie in rows that no token lies in."""
    make = large if how == "large" else A.batch
    shape = dict(lens=[30, 17, 5, 64, 100], dim=128, span=64, group=2)
    bt = make(how, seed=21, **shape)
    d, n, hq, f = A.desc_of(bt), len(bt.lens), bt.heads * bt.group, bt.format
    taken = np.zeros((bt.pool.shape[2], 16), dtype=bool)
    for b in range(n):
        rows = bt.rows(b).numpy()
        taken[rows // 16, rows % 16] = True
    g = np.random.default_rng(22)

    def pool_with(junk):
        pool = bt.pool.copy()
        noise = g.integers(0, 256, pool.shape, dtype=np.uint8)
        word = np.array([junk], dtype="<u2").view(np.uint8)
        for tile, t in zip(*np.nonzero(~taken)):
            for half in range(2):
                pool[0, :, tile, f.byte[half, t]] = noise[0, :, tile, f.byte[half, t]]
                pool[0, :, tile, f.param[half, t].reshape(-1)] = np.tile(word, 2 * f.groups)[:, None]
        return pool

    def run(pool, fill):
        held, qkv = torch.from_numpy(pool.copy()).cuda(), bt.qkv.cuda()
        out, lse = torch.full((n, hq, bt.dim), 9.0, dtype=bt.dtype, device="cuda"), torch.full((n, hq), 9.0, device="cuda")
        B.held_attention(d, bt.bits, 0, held, qkv[:, :hq], bt.table.cuda(), torch.tensor(bt.lens, dtype=torch.int32).cuda(), bt.max_len, out,
                         A.workspace(d, bt.bits, n, bt.max_len, fill), k_new=qkv[:, hq:hq + bt.heads] if append else None,
                         v_new=qkv[:, hq + bt.heads:] if append else None, lse=lse)
        torch.cuda.synchronize()
        return bits_of(out.cpu()), lse.cpu(), held.cpu().numpy()

    want, want_lse, want_pool, (tol, lse_tol) = attend(bt, append=append)
    first = run(bt.pool, 0xff)
    assert ((first[0].view(bt.dtype).double() - want).abs() <= tol).all() and np.array_equal(first[2], want_pool)
    newest = np.array([int(bt.rows(b)[-1]) for b in range(n) if bt.lens[b]])
    for fill, junk in zip((0x00, 0x3f, 0x7f, 0xff, 0x80), JUNK.values()):
        pool = pool_with(junk)
        out, lse, after = run(pool, fill)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
        if append:                                            # the new tokens' places are taken; all else stays as it was
            for row in newest:
                for half in range(2):
                    for at in (f.byte[half, row % 16], f.param[half, row % 16].reshape(-1)):
                        assert np.array_equal(after[0, :, row // 16][:, at], want_pool[0, :, row // 16][:, at])
                        pool[0, :, row // 16, at] = after[0, :, row // 16, at]
        assert np.array_equal(after, pool)


@pytest.mark.parametrize("how", A.HOW + ["large"])
def test_without_a_new_token_the_pool_stays_as_it_is(how):
    """Also where groups are NaN, lengths invalid and slots outside the pool."""
    bt = (large if how == "large" else A.batch)(how, lens=[70, 70, 70], seed=8, dim=128, span=64, group=2)
    at = next(i for i, x in enumerate(bt.lens) if x)
    x = bt.kv[0, 0, 0, int(bt.rows(at)[65])].clone()
    x[64:] = math.nan
    bt.store(bt.pool, 0, 0, 0, int(bt.rows(at)[65]), x)
    lens, table = list(bt.lens), bt.table.clone()
    lens[at + 1], table[at + 2, 1] = -3, bt.n_slots
    _, _, after = A.call(bt, lens=lens, table=table)
    assert np.array_equal(after, bt.pool)
