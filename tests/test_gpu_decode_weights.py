"""How exactly the weights enter the product with V: as a pair of 16-bit values, so that an output is as exact as its own type is.

Every query row has one channel that is not zero, so a logit is one product, exact but for its scaling: with |v| <= 3 (v: the logit in units
of log2) the scaled logit and its distance from the reference are off by 3 * 2^-22 in all, which makes a weight off by less than 2^-20, the
exponential's 2^-22 included.  The pair of parts: the first is cut off (to 11 bits in fp16, 8 in bf16) at a value up to 2^-12 (2^-9) below the
weight, the second is rounded: off by less than (2^-10 + 2^-12) * 2^-11 < 2^-20 (fp16), (2^-7 + 2^-9) * 2^-9 < 2^-15.6 (bf16) of the
weight.  The sums over 64 tokens in binary32: 8 multiplications of tiles and their joins, off by at most 2^-22 of the terms' absolute
sum each, 2^-18 in all.  Together less than 2^-17 (fp16) and 2^-15 (bf16) of sum p |V|, and half a step of the output."""
import pytest
import torch

from paged_reference import Batch, attend
from test_gpu_decode import call
from test_gpu_decode_runs import LONG, padded

F16, BF16 = torch.float16, torch.bfloat16
OFF = {F16: 2.0 ** -17, BF16: 2.0 ** -15}


def first_part(p, dtype):
    """What is left of weights (float64, largest 1) when the second part is dropped."""
    bits = {F16: 11, BF16: 8}[dtype]
    m, e = torch.frexp(p * (1 - 2.0 ** -(bits + 1)))
    return torch.ldexp(torch.floor(torch.ldexp(m, torch.tensor(bits))), e - bits)


def weights(bt, b=0):
    s = bt.q[b].double() @ bt.kv[0, 0, 0, bt.rows(b)].double().T * bt.scale
    return torch.exp(s - s.amax(1, keepdim=True))             # [query heads, tokens]


def batch(dtype, group, max_len=None):
    """One KV head, 64 tokens; the values of channel c are large where a weight of query head c % group loses most with its second
    part and negative where it loses least, and cancel: the output is near 0, the loss is not."""
    bt = Batch([64], heads=1, group=group, dim=64, dtype=dtype, seed=group, max_len=max_len)
    rows = bt.rows(0)
    k = torch.zeros(64, 64, dtype=torch.float64)
    k[:, 0] = torch.linspace(-2, 2, 64, dtype=torch.float64)[torch.randperm(64, generator=torch.Generator().manual_seed(5))]
    bt.kv[0, 0, 0, rows] = k.to(dtype)
    bt.qkv[:, :group] = 0
    bt.qkv[0, :group, 0] = torch.linspace(4, 7, group).to(dtype)
    p = weights(bt)
    lost = (p - first_part(p, dtype)) / p
    v = lost - (lost * p).sum(1, keepdim=True) / p.sum(1, keepdim=True)
    v = v / v.abs().amax(1, keepdim=True)
    bt.kv[0, 1, 0, rows] = v[torch.arange(64) % group].T.to(dtype)
    return bt


def bound(bt, want, first=0):
    p = weights(bt)
    p = p / p.sum(1, keepdim=True)
    return want[first].abs() * torch.finfo(bt.dtype).eps / 2 + OFF[bt.dtype] * (p @ bt.kv[0, 1, 0, bt.rows(0)].double().abs()) + 2.0 ** -25


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("group", [1, 4, 8, 16])
def test_the_cases_tell_one_part_from_two(dtype, group):
    """On the CPU: the outputs with the first parts alone lie outside the bound."""
    bt = batch(dtype, group)
    want = attend(bt)[0]
    p = weights(bt)
    half = (first_part(p, dtype) @ bt.kv[0, 1, 0, bt.rows(0)].double()) / p.sum(1, keepdim=True)
    over = (half - want[0]).abs() / bound(bt, want)
    mine = torch.arange(64)[None, :] % group == torch.arange(group)[:, None]  # channels made for the query head
    assert (over[mine] > 2).all(), float(over[mine].min())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("group", [1, 2, 4, 5, 8, 11, 16])
@pytest.mark.parametrize("form", ["cluster", "padded", "long_bound"])
def test_two_parts(dtype, group, form):
    bt = batch(dtype, group, LONG if form == "long_bound" else None)
    want = attend(bt)[0]
    limit = bound(bt, want)
    at = padded(bt) if form == "padded" else 0
    out = call(bt)[0][at].double()
    assert ((out - want[0]).abs() <= limit).all(), float(((out - want[0]).abs() / limit).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("gap", [12, 18, 22, 26])
def test_small_weights_beside_one_large(dtype, gap):
    """A token with a value of 0 takes nearly all the weight; the others have 2^-gap of it each.  In fp16 a weight is off by up to
    2^-31 of the largest one besides: all others together by 4000 times that, times their values."""
    n = 4001
    bt = Batch([n], heads=1, group=4, dim=64, dtype=dtype, seed=1)
    rows = bt.rows(0)
    bt.kv[0, 0, 0, rows] = 0
    bt.kv[0, 0, 0, rows[7], 0] = 1.0
    bt.qkv[:, :4] = 0
    q = gap * 0.6931471805599453 / bt.scale                   # a logit of gap * ln 2, as near as the type can hold it
    bt.qkv[0, :4, 0] = q
    bt.kv[0, 1, 0, rows] = (1.0 + torch.rand(n, 64, generator=torch.Generator().manual_seed(2))).to(dtype)
    bt.kv[0, 1, 0, rows[7]] = 0
    out = call(bt)[0][0].double()
    want = attend(bt)[0][0]
    # the logits are exact products here too; |v| up to 26 makes a weight off by 26 * 4 * 2^-24 + 2^-22 < 2^-17; 4001 tokens are 251 tiles,
    # whose sums of terms of one sign lose up to 251 * 2 * 2^-23 < 2^-14 where every addition truncates
    p = weights(bt)
    total = p.sum(1, keepdim=True)
    small = 2.0 ** -31 * bt.kv[0, 1, 0, rows].double().abs().sum(0) / total if dtype == F16 else 0.0
    limit = want.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -13.5 + OFF[dtype]) + small + 2.0 ** -25
    assert ((out - want).abs() <= limit).all(), float(((out - want).abs() / limit).max())
