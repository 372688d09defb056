"""The held-pool calls' argument checks: all on the host, before anything is launched.  No GPU needed."""
import ctypes as C

import pytest

from paper_2403_11805_b200 import binding as B

A = 1 << 20                                                   # an aligned address that is never read


def pool(**kw):
    args = dict(n_layers=2, n_kv_heads=4, n_q_heads=8, head_dim=64, n_tokens=160, chunk_len=16, group_size=64)
    args.update(kw)
    return B.make_desc(**args)


WRITE = dict(bits=4, dtype=0, layer=0, held=A, held_size=1 << 40, k=A, v=A, row_stride=256, n_rows=7, first_row=A, chunk_table=A, table_stride=5, lens=A, n_seqs=3,
             max_len=80, k_seen=None, v_seen=None, seen_stride=0, stream=None)
READ = dict(bits=4, dtype=0, layer=0, held=A, held_size=1 << 40, chunk_table=A, table_stride=5, lens=A, n_seqs=3, max_len=80, first_row=A, n_rows=7, k_out=A, v_out=A,
            out_stride=256, stream=None)
ATTEND = dict(bits=4, dtype=0, layer=0, held=A, held_size=1 << 40, q=A, q_stride=512, k_new=None, v_new=None, new_stride=0, chunk_table=A, table_stride=5, lens=A,
              n_seqs=3, max_len=80, window=0, scale=0.125, out=A, lse=None, workspace=A, workspace_bytes=1 << 40, stream=None)


def caller(name, defaults):
    def call(desc=None, **kw):
        desc = pool() if desc is None else desc
        assert set(kw) <= set(defaults)
        return getattr(B.lib(), name)(C.addressof(desc), *{**defaults, **kw}.values())
    return call


write, read, attend = caller("llms_held_write", WRITE), caller("llms_held_read", READ), caller("llms_held_attention", ATTEND)
INVALID, MISALIGNED, SMALL, UNSUPPORTED, BAD_BITS = B.ERR_INVALID_ARG, B.ERR_MISALIGNED, B.ERR_BUF_TOO_SMALL, B.ERR_UNSUPPORTED, B.ERR_BAD_BITS

COMMON = [
    (INVALID, dict(dtype=2)), (INVALID, dict(dtype=-1)), (INVALID, dict(layer=2)), (INVALID, dict(layer=-1)), (INVALID, dict(held=None)),
    (INVALID, dict(chunk_table=None)), (INVALID, dict(lens=None)), (INVALID, dict(table_stride=4)), (INVALID, dict(table_stride=0)),
    (INVALID, dict(n_seqs=-1)), (INVALID, dict(max_len=0)), (INVALID, dict(max_len=81)), (MISALIGNED, dict(held=A + 8)),
    (MISALIGNED, dict(chunk_table=A + 2)), (MISALIGNED, dict(lens=A + 1)), (UNSUPPORTED, dict(n_seqs=4097)), (UNSUPPORTED, dict(bits=2)),
    (UNSUPPORTED, dict(bits=1)), (BAD_BITS, dict(bits=3)), (BAD_BITS, dict(bits=0)), (BAD_BITS, dict(bits=16)), (SMALL, dict(held_size=0)), (SMALL, dict(held_size=2 * 4 * 10 * 1152 - 1)),
]


@pytest.mark.parametrize("status,kw", COMMON, ids=str)
@pytest.mark.parametrize("call", [write, read, attend], ids=["write", "read", "attend"])
def test_what_all_calls_refuse(call, status, kw):
    assert call(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(k=None)), (INVALID, dict(v=None)), (INVALID, dict(row_stride=248)), (INVALID, dict(n_rows=-1)), (INVALID, dict(first_row=None)),
    (INVALID, dict(k_seen=A)), (INVALID, dict(v_seen=A, seen_stride=256)), (INVALID, dict(k_seen=A, v_seen=A, seen_stride=248)),
    (MISALIGNED, dict(k=A + 8)), (MISALIGNED, dict(v=A + 2)), (MISALIGNED, dict(row_stride=260)), (MISALIGNED, dict(first_row=A + 2)),
    (MISALIGNED, dict(k_seen=A + 8, v_seen=A, seen_stride=256)), (MISALIGNED, dict(k_seen=A, v_seen=A, seen_stride=260)),
], ids=str)
def test_write_refusals(status, kw):
    assert write(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(k_out=None)), (INVALID, dict(v_out=None)), (INVALID, dict(out_stride=248)), (INVALID, dict(n_rows=-1)), (INVALID, dict(first_row=None)),
    (MISALIGNED, dict(k_out=A + 8)), (MISALIGNED, dict(v_out=A + 2)), (MISALIGNED, dict(out_stride=260)), (MISALIGNED, dict(first_row=A + 1)),
], ids=str)
def test_read_refusals(status, kw):
    assert read(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(window=-1)), (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))), (INVALID, dict(q=None)), (INVALID, dict(out=None)),
    (INVALID, dict(workspace=None)), (INVALID, dict(q_stride=504)), (INVALID, dict(k_new=A, new_stride=256)), (INVALID, dict(v_new=A, new_stride=256)),
    (INVALID, dict(k_new=A, v_new=A, new_stride=248)), (MISALIGNED, dict(q=A + 2)), (MISALIGNED, dict(out=A + 4)), (MISALIGNED, dict(q_stride=516)),
    (MISALIGNED, dict(workspace=A + 128)), (MISALIGNED, dict(k_new=A + 8, v_new=A, new_stride=256)), (MISALIGNED, dict(k_new=A, v_new=A, new_stride=260)),
    (MISALIGNED, dict(lse=A + 2)), (SMALL, dict(workspace_bytes=0)), (UNSUPPORTED, dict(max_len=0x7fffffff, table_stride=0x7fffffff, n_seqs=4096)),
], ids=str)
def test_attention_refusals(status, kw):
    assert attend(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (MISALIGNED, dict(head_dim=40, group_size=8)), (UNSUPPORTED, dict(head_dim=80, group_size=16)), (UNSUPPORTED, dict(head_dim=192)),
    (UNSUPPORTED, dict(head_dim=512)), (INVALID, dict(n_q_heads=6)), (INVALID, dict(chunk_len=0)), (UNSUPPORTED, dict(chunk_len=8)),
    (UNSUPPORTED, dict(chunk_len=24)), (UNSUPPORTED, dict(group_size=16)), (UNSUPPORTED, dict(head_dim=96, group_size=96)),
    (UNSUPPORTED, dict(head_dim=256, group_size=32)), (INVALID, dict(group_size=128)), (UNSUPPORTED, dict(quant_mode=1)),
], ids=str)
def test_descriptor_refusals(status, kw):
    desc, nb = pool(**kw), C.c_uint64()
    assert write(desc) == read(desc) == attend(desc) == status
    assert B.lib().llms_held_bytes(C.addressof(desc), 4, C.addressof(nb)) == status
    assert B.lib().llms_held_workspace_bytes(C.addressof(desc), 4, 3, 80, C.addressof(nb)) == status


@pytest.mark.parametrize("dim,span,bits,tile", [(64, 64, 4, 1152), (64, 32, 8, 2304), (96, 32, 4, 1920), (128, 128, 4, 2176), (128, 32, 8, 4608), (256, 128, 4, 4352),
                                                (256, 64, 8, 8704)])
def test_pool_size(dim, span, bits, tile):
    """Tiles of 16 tokens: 2 x 16 x (dim x bits / 8 + 4 x groups) bytes."""
    assert tile == 32 * (dim * bits // 8 + 4 * dim // span)
    assert B.held_bytes(pool(head_dim=dim, group_size=span, n_tokens=170), bits) == 2 * 4 * 10 * tile
    with pytest.raises(B.LlmsError):
        B.held_bytes(pool(), 2)
    assert B.lib().llms_held_bytes(C.addressof(pool()), 4, None) == INVALID


def test_an_empty_batch_does_nothing():
    assert write(n_seqs=0, k=None) == read(n_seqs=0, k_out=None) == attend(n_seqs=0, q=None) == B.OK
    assert write(n_rows=0, k=None) == read(n_rows=0, k_out=None) == B.OK


def test_the_workspace_grows_with_the_batch():
    sizes = [B.held_workspace_bytes(pool(), 4, n, length) for n, length in ((0, 1), (1, 80), (64, 80))]
    assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)


@pytest.fixture
def on_the_host(monkeypatch):
    """The binding's checks over tensors in host memory; the C calls are only noted."""
    import torch
    called, names = [], ("llms_held_write", "llms_held_read", "llms_held_attention")
    fake = type("Lib", (), {name: staticmethod(lambda *a, name=name: called.append(name) or 0) for name in names})
    fake.llms_strerror = B.lib().llms_strerror
    B._CACHE_TYPES.update({torch.float16: B.DTYPE_F16, torch.bfloat16: B.DTYPE_BF16})
    monkeypatch.setattr(B, "_torch", torch)
    monkeypatch.setattr(B, "_current", lambda stream: (-1, 0))               # where host tensors say they are
    monkeypatch.setattr(B, "_lib", fake)
    return called


def binding_calls():
    import torch
    i32, f16 = dict(dtype=torch.int32), dict(dtype=torch.float16)
    held, table, lens = torch.zeros(2, 4, 10, 1152, dtype=torch.uint8), torch.zeros(3, 5, **i32), torch.zeros(3, **i32)
    k, v, first = torch.zeros(7, 4, 64, **f16), torch.zeros(7, 4, 64, **f16), torch.zeros(4, **i32)
    batch = dict(bits=4, layer=0, held=held, chunk_table=table, lens=lens, max_len=80)
    return (lambda **kw: B.held_write(pool(), **{**batch, **dict(k=k, v=v, first_row=first), **kw}),
            lambda **kw: B.held_read(pool(), **{**batch, **dict(k_out=k, v_out=v, first_row=first), **kw}),
            lambda **kw: B.held_attention(pool(), **{**batch, **dict(q=torch.zeros(3, 8, 64, **f16), out=torch.zeros(3, 8, 64, **f16),
                                                                     workspace=torch.zeros(1 << 20, dtype=torch.uint8)), **kw}))


def test_the_binding_s_checks(on_the_host):
    import torch
    f16 = dict(dtype=torch.float16)
    calls = binding_calls()
    for call in calls:
        call()
    assert len(on_the_host) == 3
    rows = lambda n, **kw: torch.zeros(n, 4, 64, **{**f16, **kw})  # noqa: E731
    for which, wrong in [
        (0, dict(k=rows(6))), (0, dict(k=rows(7, dtype=torch.float32))), (0, dict(v=rows(7, dtype=torch.bfloat16))), (0, dict(first_row=None)),
        (0, dict(first_row=torch.zeros(3, dtype=torch.int32))), (0, dict(first_row=torch.zeros(4, dtype=torch.int64))), (0, dict(k_seen=rows(7))),
        (0, dict(k_seen=rows(6), v_seen=rows(6))), (0, dict(k=torch.zeros(7, 64, 4, **f16).transpose(1, 2))), (0, dict(v=torch.zeros(7, 2, 4, 64, **f16)[:, 0])),
        (1, dict(k_out=rows(6))), (1, dict(v_out=rows(7, dtype=torch.float32))), (1, dict(first_row=None)), (1, dict(k_out=rows(8)[:, :3])),
        (2, dict(q=torch.zeros(3, 8, 32, **f16))), (2, dict(out=torch.zeros(3, 8, 64))), (2, dict(k_new=rows(3))), (2, dict(k_new=rows(2), v_new=rows(2))),
        (2, dict(lse=torch.zeros(3, 4))), (2, dict(window=1 << 32)), (2, dict(workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 20))),
    ] + [(i, w) for i in range(3) for w in (
        dict(held=torch.zeros(2, 4, 10, 2304, dtype=torch.uint8)[..., ::2]),
        dict(chunk_table=torch.zeros(3, 4, dtype=torch.int32)), dict(chunk_table=torch.zeros(2, 5, dtype=torch.int32)),
        dict(lens=torch.zeros(3, dtype=torch.int64)), dict(lens=torch.zeros(3, 1, dtype=torch.int32)), dict(layer=1 << 32), dict(bits=(1 << 32) + 4))]:
        with pytest.raises(B.LlmsError):
            calls[which](**wrong)
    assert len(on_the_host) == 3
    qkv = torch.zeros(3, 16, 64, **f16)
    calls[2](q=qkv[:, :8], k_new=qkv[:, 8:12], v_new=qkv[:, 12:])
    calls[0](k=torch.zeros(7, 2, 4, 64, **f16)[:, 0], v=torch.zeros(7, 2, 4, 64, **f16)[:, 1], k_seen=rows(7), v_seen=rows(7))
    calls[0](k=rows(3), v=rows(3), first_row=None)
    assert len(on_the_host) == 6
