"""The paged-cache calls' argument checks: all on the host, before anything is launched.  No GPU needed."""
import ctypes as C

import pytest

from paper_2403_11805_b200 import binding as B

A = 1 << 20                                                   # an aligned address that is never read


def pool(**kw):
    args = dict(n_layers=2, n_kv_heads=4, n_q_heads=8, head_dim=64, n_tokens=160, chunk_len=16, group_size=16)
    args.update(kw)
    return B.make_desc(**args)


DECODE = dict(dtype=0, layer=0, kv=A, q=A, q_stride=512, k_new=None, v_new=None, new_stride=0, chunk_table=A, table_stride=5, lens=A,
              n_seqs=3, max_len=80, window=0, scale=0.125, out=A, lse=None, mass_in=None, mass_out=None, mass_stride=0, workspace=A,
              workspace_bytes=1 << 40, stream=None)
EVICT = dict(kv=A, mass=A, mass_stride=80, chunk_table=A, table_stride=5, lens=A, n_seqs=3, max_len=80, budget=20, recent=4, dst_table=None,
             dst_stride=0, mass_out=A, kept=A, new_lens=2 * A, stream=None)


def decode(desc=None, **kw):
    desc = pool() if desc is None else desc
    assert set(kw) <= set(DECODE)
    return B.lib().llms_decode_attention(C.addressof(desc), *{**DECODE, **kw}.values())


def evict(desc=None, **kw):
    desc = pool() if desc is None else desc
    assert set(kw) <= set(EVICT)
    return B.lib().llms_evict_tokens(C.addressof(desc), *{**EVICT, **kw}.values())


INVALID, MISALIGNED, SMALL, UNSUPPORTED = B.ERR_INVALID_ARG, B.ERR_MISALIGNED, B.ERR_BUF_TOO_SMALL, B.ERR_UNSUPPORTED


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(dtype=2)), (INVALID, dict(dtype=-1)), (INVALID, dict(layer=2)), (INVALID, dict(layer=-1)), (INVALID, dict(window=-1)),
    (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))), (INVALID, dict(kv=None)), (INVALID, dict(q=None)),
    (INVALID, dict(chunk_table=None)), (INVALID, dict(lens=None)), (INVALID, dict(out=None)), (INVALID, dict(workspace=None)),
    (INVALID, dict(k_new=A, new_stride=256)), (INVALID, dict(v_new=A, new_stride=256)), (INVALID, dict(k_new=A, v_new=A, new_stride=248)),
    (INVALID, dict(mass_in=A)), (INVALID, dict(mass_out=A, mass_stride=79)), (INVALID, dict(table_stride=4)), (INVALID, dict(table_stride=0)),
    (INVALID, dict(q_stride=504)), (INVALID, dict(n_seqs=-1)), (INVALID, dict(max_len=0)), (INVALID, dict(max_len=81)),
    (MISALIGNED, dict(kv=A + 8)), (MISALIGNED, dict(q=A + 2)), (MISALIGNED, dict(out=A + 4)), (MISALIGNED, dict(q_stride=516)),
    (MISALIGNED, dict(workspace=A + 128)), (MISALIGNED, dict(k_new=A + 8, v_new=A, new_stride=256)), (MISALIGNED, dict(lens=A + 2)),
    (MISALIGNED, dict(k_new=A, v_new=A, new_stride=260)), (MISALIGNED, dict(chunk_table=A + 1)), (MISALIGNED, dict(mass_out=A + 1, mass_stride=80)),
    (SMALL, dict(workspace_bytes=0)), (SMALL, dict(workspace_bytes=1, mass_out=A, mass_stride=80)), (UNSUPPORTED, dict(n_seqs=4097)),
    (UNSUPPORTED, dict(max_len=0x7fffffff, table_stride=0x7fffffff, n_seqs=4096)),
], ids=str)
def test_decode_refusals(status, kw):
    assert decode(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (MISALIGNED, dict(head_dim=40, group_size=8)), (UNSUPPORTED, dict(head_dim=272)), (INVALID, dict(n_q_heads=6)), (INVALID, dict(chunk_len=0)),
], ids=str)
def test_descriptor_refusals(status, kw):
    assert decode(pool(**kw)) == status
    assert evict(pool(**kw)) == status
    nb = C.c_uint64()
    desc = pool(**kw)
    assert B.lib().llms_decode_workspace_bytes(C.addressof(desc), 3, 80, 0, C.addressof(nb)) == status


def test_strides_must_keep_slabs_aligned():
    d = pool()
    d.stride_h += 4
    assert decode(d) == evict(d) == MISALIGNED


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(budget=0, recent=0)), (INVALID, dict(recent=21)), (INVALID, dict(recent=-1)), (INVALID, dict(kv=None)), (INVALID, dict(mass=None)),
    (INVALID, dict(mass_out=None)), (INVALID, dict(kept=None)), (INVALID, dict(new_lens=None)), (INVALID, dict(new_lens=A)), (INVALID, dict(lens=None)),
    (INVALID, dict(chunk_table=None)), (INVALID, dict(table_stride=4)), (INVALID, dict(mass_stride=79)), (INVALID, dict(max_len=0)),
    (INVALID, dict(n_seqs=-1)), (INVALID, dict(dst_table=A, dst_stride=1)), (INVALID, dict(dst_table=A, dst_stride=0)),
    (MISALIGNED, dict(kv=A + 8)), (MISALIGNED, dict(mass=A + 2)), (MISALIGNED, dict(kept=A + 2)), (MISALIGNED, dict(dst_table=A + 1, dst_stride=2)),
    (UNSUPPORTED, dict(n_seqs=4097)),
], ids=str)
def test_evict_refusals(status, kw):
    assert evict(**kw) == status


def test_a_table_as_its_own_destination_keeps_its_stride():
    """With several sequences another stride would make rows of one the places of another."""
    assert evict(dst_table=A, table_stride=8, dst_stride=5) == INVALID
    assert evict(dst_table=A, table_stride=5, dst_stride=8) == INVALID


@pytest.fixture
def on_the_host(monkeypatch):
    """The binding's checks over tensors in host memory; the C calls are only noted."""
    import torch
    called = []
    fake = type("Lib", (), {name: staticmethod(lambda *a, name=name: called.append(name) or 0) for name in ("llms_decode_attention", "llms_evict_tokens")})
    fake.llms_strerror = B.lib().llms_strerror
    B._CACHE_TYPES.update({torch.float16: B.DTYPE_F16, torch.bfloat16: B.DTYPE_BF16})
    monkeypatch.setattr(B, "_torch", torch)
    monkeypatch.setattr(B, "_current", lambda stream: (-1, 0))               # where host tensors say they are
    monkeypatch.setattr(B, "_lib", fake)
    return called


def binding_calls():
    import torch
    kv, i32 = torch.zeros(2, 2, 4, 160, 64, dtype=torch.float16), dict(dtype=torch.int32)
    table, lens = torch.zeros(3, 5, **i32), torch.zeros(3, **i32)
    q, out, mass = torch.zeros(3, 8, 64, dtype=torch.float16), torch.zeros(3, 8, 64, dtype=torch.float16), torch.zeros(2, 3, 4, 80)
    return (lambda **kw: B.decode_attention(pool(), **{**dict(layer=0, kv=kv, q=q, chunk_table=table, lens=lens, max_len=80, out=out,
                                                              workspace=torch.zeros(1 << 20, dtype=torch.uint8)), **kw}),
            lambda **kw: B.evict_tokens(pool(), **{**dict(kv=kv, mass=mass, chunk_table=table, lens=lens, max_len=80, budget=20, recent=4,
                                                          kept=torch.zeros(2, 3, 4, 20, **i32), new_lens=torch.zeros(3, **i32)), **kw}))


@pytest.mark.parametrize("which,kw", [
    (0, dict(window=1 << 32)), (0, dict(window=(1 << 32) + 16)), (0, dict(window=1 << 31)), (0, dict(layer=1 << 32)), (0, dict(layer=-(1 << 32))),
    (1, dict(recent=1 << 32)), (1, dict(recent=-(1 << 32) + 2)),
], ids=str)
def test_numbers_beyond_the_c_call_s_are_refused(which, kw, on_the_host):
    """They would reach the call cut off to 32 bits, as other numbers."""
    calls = binding_calls()
    for call in calls:
        call()
    assert on_the_host == ["llms_decode_attention", "llms_evict_tokens"]
    with pytest.raises(B.LlmsError) as e:
        calls[which](**kw)
    assert e.value.status == INVALID and len(on_the_host) == 2


def test_a_workspace_without_the_bytes_that_its_size_says_is_refused(on_the_host):
    """A view's nbytes counts its elements, wherever they lie."""
    import torch
    decode_call, _ = binding_calls()
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 21, dtype=torch.uint8)[::2]):
        with pytest.raises(B.LlmsError) as e:
            decode_call(workspace=ws)
        assert e.value.status == INVALID
    assert on_the_host == []
    decode_call(workspace=torch.zeros(256, 4096, dtype=torch.uint8))
    assert on_the_host == ["llms_decode_attention"]


def test_an_empty_batch_does_nothing():
    assert decode(n_seqs=0, q=None, out=None) == B.OK
    assert evict(n_seqs=0, kept=None) == B.OK


def test_workspace_size_grows_with_the_batch():
    d = pool()
    sizes = [B.decode_workspace_bytes(d, n, length, mass) for n, length, mass in ((0, 1, False), (1, 80, False), (64, 80, False), (64, 80, True))]
    assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
    with pytest.raises(B.LlmsError):
        B.decode_workspace_bytes(d, 1, 0)
    assert B.lib().llms_decode_workspace_bytes(C.addressof(d), 1, 80, 0, None) == INVALID
