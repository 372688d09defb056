"""Contexts of the multi-app pool served token by token: decode, shrink, growth into new chunks, and Reclaim / Load of what is left."""
import numpy as np
import pytest
import torch

import oracle
from paper_2403_11805_b200 import synth
from paper_2403_11805_b200.multiapp import MultiApp
from gpu_helpers import bits_view, odesc
from paged_reference import Batch, attend, bits, evict

pytestmark = pytest.mark.gpu


def batch_of(s, sh, app):
    """The served batch as the reference sees it."""
    bt = Batch([1] * len(s.ctxs), heads=sh.n_kv_heads, group=sh.n_q_heads // sh.n_kv_heads, dim=sh.head_dim, chunk=sh.chunk_len,
               layers=sh.n_layers, max_len=s.capacity, junk=0.0)
    bt.lens, bt.table, bt.n_slots, bt.kv, bt.mass = s.lengths.tolist(), s.table.cpu(), app.n_slots, app.pool.cpu(), s.mass.cpu()
    assert s.lens.tolist() == bt.lens and np.array_equal(bt.table.numpy(), s.host_table)
    return bt


def consistent(app):
    res = app.slot >= 0
    assert np.array_equal(res, app.table["resident"] != 0)
    assert sorted(app.slot[res].tolist() + app.free) == list(range(app.n_slots))
    live = np.concatenate([app.rows(c) for c in range(app.n_ctx)])
    assert set(np.flatnonzero(res)) <= set(live.tolist())


@pytest.mark.parametrize("aot", [False, True], ids=["reclaim", "aot"])
def test_decode_shrink_and_swap(aot):
    sh = synth.KVShape("apps", 2, 2, 8, 64, 128, 16, 64, window=4, seed=5, n_contexts=6)      # 8 chunks per context
    app = MultiApp(sh, n_slots=19, seed=2, log_ops=True, aot=aot)
    app.build()
    g = torch.Generator().manual_seed(1)
    state = {}

    def serve(s):
        n = len(s.ctxs)

        def token():
            s.advance()
            for layer in range(sh.n_layers):
                bt = batch_of(s, sh, app)
                bt.qkv = torch.randn(n, sh.n_q_heads + 2 * sh.n_kv_heads, sh.head_dim, generator=g).half()
                q, k, v = bt.qkv.split([sh.n_q_heads, sh.n_kv_heads, sh.n_kv_heads], dim=1)
                bt.q, bt.k_new, bt.v_new = q, k, v
                dev = bt.qkv.cuda().split([sh.n_q_heads, sh.n_kv_heads, sh.n_kv_heads], dim=1)
                out = s.decode(layer, *dev)
                want, _, wmass, wkv, (ot, _, mt) = attend(bt, layer, append=True, mass_in=bt.mass[layer], mass_before=bt.mass[layer])
                assert ((out.cpu().double() - want).abs() <= ot).all()
                assert ((s.mass[layer].cpu().double() - wmass).abs() <= mt).all()
                assert torch.equal(bits(app.pool.cpu()), bits(wkv))

        if (s.lengths == s.capacity).any():
            with pytest.raises(RuntimeError):
                s.advance()
            s.shrink(100, 100)                                # nothing accumulated yet: the last 100 tokens
        for _ in range(5):
            token()
        bt = batch_of(s, sh, app)
        kept = s.shrink(70, 9)
        want = evict(bt, bt.mass, 70, 9, None, bt.mass)
        assert torch.equal(kept.cpu(), want[0]) and torch.equal(s.mass.cpu(), want[2]) and torch.equal(bits(app.pool.cpu()), bits(want[3]))
        assert s.lens.tolist() == [70] * n
        consistent(app)
        for _ in range(12):                                   # 70 -> 82 tokens: into a sixth chunk
            token()
        assert s.lens.tolist() == [82] * n
        for i, c in enumerate(s.ctxs):
            assert (s.host_table[i] >= 0).sum() == 6
        state["served"] = {c: app.pool.cpu()[..., bt_rows, :] for c, bt_rows in zip(s.ctxs, [batch_of(s, sh, app).rows(i, upto=96) for i in range(n)])}

    first = app.step(k=2, serve=serve)
    consistent(app)
    assert [app.lengths[c] for c in first] == [82, 82]
    saved = dict(state["served"])
    back = set()
    for _ in range(12):                                       # others push them out; they come back as their records say
        consistent(app)
        before = len(app.ops)
        for c in app.step(k=1):
            loaded = {row for op, row, _ in app.ops[before:] if op == "load"}
            if c in saved and c not in back:
                back.add(c)
                got = app.context_kv(c).cpu()
                one = odesc(sh.with_(n_tokens=sh.chunk_len))
                for i in range(6):
                    chunk = np.ascontiguousarray(bits_view(saved[c])[..., i * 16:(i + 1) * 16, :])
                    if c * app.cpc + i not in loaded:         # stayed in its slot
                        assert np.array_equal(bits_view(got[..., i * 16:(i + 1) * 16, :]), chunk), (c, i)
                        continue
                    buf, meta = oracle.compress_chunks(one, chunk, [0], [int(app.table["bits"][c * app.cpc + i])])
                    out = np.zeros_like(chunk)
                    oracle.decompress_chunks(one, buf, meta, out)
                    assert np.array_equal(bits_view(got[..., i * 16:(i + 1) * 16, :]), out), (c, i)
    app.finish()
    consistent(app)
    assert back, "no served context came back within the steps"


def test_serving_keeps_to_its_capacity():
    sh = synth.KVShape("apps", 1, 2, 2, 64, 64, 16, 64, window=4, seed=1, n_contexts=4)
    app = MultiApp(sh, n_slots=8, seed=3)
    app.build()

    def serve(s):
        with pytest.raises(RuntimeError):
            s.advance()
        assert s.lengths.tolist() == [64, 64] and s.lens.tolist() == [64, 64]
        s.shrink(64, 4)                                       # nothing to drop
        assert s.lens.tolist() == [64, 64] and (s.host_table >= 0).all()
        s.shrink(1, 1)
        assert s.lens.tolist() == [1, 1] and (s.host_table >= 0).sum() == 2

    served = app.step(k=2, serve=serve)
    consistent(app)
    assert [app.lengths[c] for c in served] == [1, 1]
    for _ in range(4):
        app.step(k=2)
        consistent(app)


@pytest.mark.parametrize("aot", [False, True], ids=["reclaim", "aot"])
def test_a_serve_that_raises_leaves_the_pool_in_order(aot):
    sh = synth.KVShape("apps", 1, 2, 2, 64, 64, 16, 64, window=4, seed=1, n_contexts=4)
    app = MultiApp(sh, n_slots=8, seed=3, aot=aot)
    app.build()
    served = []

    def serve(s):
        served.extend(s.ctxs)
        s.shrink(20, 4)
        s.advance()
        raise KeyError("the model's own")

    with pytest.raises(KeyError):
        app.step(k=2, serve=serve)
    consistent(app)
    assert len(served) == 2 and [app.lengths[c] for c in served] == [21, 21] and not app.table["locked"].any()
    for _ in range(4):
        app.step(k=2)
        consistent(app)
    app.finish()


def test_more_reclaims_in_a_step_than_the_pool_has_workspaces():
    """A context grows by 90 chunks in one call while the pool is full of modified ones: each growth reclaims a chunk of others, and
    every record that left has its own checksum and comes back."""
    sh = synth.KVShape("apps", 1, 1, 1, 64, 100 * 16, 16, 64, window=4, seed=4, n_contexts=4)         # 100 chunks per context
    app = MultiApp(sh, n_slots=200, seed=2)
    app.build()
    chosen = []
    app.draw_contexts = lambda k: list(chosen)

    def step(c, serve=None):
        chosen[:] = [c]
        app.step(k=1, serve=serve)
        consistent(app)

    step(2, lambda s: s.shrink(16, 1))
    step(3)
    step(1)
    full = app.pool.cpu()
    slots = {r: int(app.slot[r]) for r in np.flatnonzero(app.slot >= 0)}
    app.clean[list(slots)] = False
    one = odesc(sh.with_(n_tokens=16))

    def grow(s):
        for _ in range(90 * 16):
            s.advance()

    before = app._ws_next
    step(2, grow)
    assert app._ws_next - before > 64
    gone = [r for r in slots if app.slot[r] < 0]
    assert len(gone) >= 80
    records = {}
    for r in gone:
        chunk = np.ascontiguousarray(bits_view(full[..., slots[r] * 16:(slots[r] + 1) * 16, :]))
        buf, meta = oracle.compress_chunks(one, chunk, [0], [int(app.table["bits"][r])])
        assert app.checksum[r] == meta[0]["checksum"], r
        out = np.zeros_like(chunk)
        oracle.decompress_chunks(one, buf, meta, out)
        records[r] = out
    for c in (1, 3):
        step(c)
        for i, r in enumerate(app.rows(c)):
            if r in records:
                assert np.array_equal(bits_view(app.context_kv(c))[..., i * 16:(i + 1) * 16, :], records[r])


def reference_step(bt, sh, qkv, layer):
    """The reference batch with a token's rows, and what the layer's decode call has to give."""
    bt.qkv = qkv
    bt.q, bt.k_new, bt.v_new = qkv.split([sh.n_q_heads, sh.n_kv_heads, sh.n_kv_heads], dim=1)
    return attend(bt, layer, append=True, mass_in=bt.mass[layer], mass_before=bt.mass[layer])


def pool_of_modified_chunks(n_slots=40):
    """Contexts of 16 chunks, n_slots of them full of modified ones, context 2 down to a chunk."""
    sh = synth.KVShape("apps", 1, 2, 8, 64, 256, 16, 64, window=4, seed=6, n_contexts=5)
    app = MultiApp(sh, n_slots=n_slots, seed=2)
    app.build()
    chosen = []
    app.draw_contexts = lambda k: list(chosen)

    def step(c, serve=None):
        chosen[:] = [c]
        app.step(k=1, serve=serve)
        consistent(app)

    for c in (2, 3, 4):
        step(c, (lambda s: s.shrink(16, 1)) if c == 2 else None)
    app.clean[:] = False
    return sh, app, step


def test_serving_on_a_stream_of_its_own():
    """The callback's stream is late by a delay in front of every token, and every growth reclaims a chunk of others: what leaves
    is what lay in the slots, and attention sees the rows that were stored."""
    sh, app, step = pool_of_modified_chunks()
    side = torch.cuda.Stream()
    g = torch.Generator().manual_seed(3)
    left = {}

    def serve(s):
        with torch.cuda.stream(side):
            for _ in range(7 * 16):
                grows = s.lengths[0] % 16 == 0
                if grows:
                    side.synchronize()
                    torch.cuda.synchronize()
                    before, slots = app.pool.cpu(), {int(r): int(app.slot[r]) for r in np.flatnonzero(app.slot >= 0)}
                torch.cuda._sleep(200000)
                s.advance()
                if grows:
                    for r, slot in slots.items():
                        if app.slot[r] < 0:
                            left[r] = before[..., slot * 16:(slot + 1) * 16, :]
                torch.cuda._sleep(200000)
                qkv = torch.randn(1, 12, 64, generator=g).half()
                dev = qkv.cuda(non_blocking=True).split([8, 2, 2], dim=1)
                if grows:                                     # with a reference: everything in between has been waited for then
                    side.synchronize()
                    bt = batch_of(s, sh, app)
                    want, _, wmass, wkv, (ot, _, mt) = reference_step(bt, sh, qkv, 0)
                out = s.decode(0, *dev)
                if grows:
                    assert ((out.cpu().double() - want).abs() <= ot).all()
                    assert ((s.mass[0].cpu().double() - wmass).abs() <= mt).all()
                    assert torch.equal(bits(app.pool.cpu()), bits(wkv))

    step(2, serve)
    app.finish()
    assert len(left) >= 4
    one = odesc(sh.with_(n_tokens=16))
    arena = app.arena.numpy()
    for r, chunk in left.items():
        buf, meta = oracle.compress_chunks(one, np.ascontiguousarray(bits_view(chunk)), [0], [int(app.table["bits"][r])])
        off = int(app.arena_off[r])
        assert app.checksum[r] == meta[0]["checksum"] and np.array_equal(arena[off:off + buf.size], buf), r
    for c in (3, 4):
        step(c)


def test_a_captured_decode_replayed_between_growth_and_shrinking():
    sh, app, step = pool_of_modified_chunks()
    g = torch.Generator().manual_seed(4)

    def serve(s):
        qkv = torch.zeros(1, 12, 64, dtype=torch.float16, device="cuda")
        q, k, v = qkv.split([8, 2, 2], dim=1)
        out = torch.zeros(1, 8, 64, dtype=torch.float16, device="cuda")
        s.advance()
        s.decode(0, q, k, v, out)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            s.decode(0, q, k, v, out)
        with torch.cuda.stream(side):
            for i in range(60):
                s.advance()
                if i == 40:
                    s.shrink(24, 4)
                    s.advance()
                token = torch.randn(1, 12, 64, generator=g).half()
                qkv.copy_(token)
                side.synchronize()
                bt = batch_of(s, sh, app)
                want, _, wmass, wkv, (ot, _, mt) = reference_step(bt, sh, token, 0)
                graph.replay()
                assert ((out.cpu().double() - want).abs() <= ot).all()
                assert ((s.mass[0].cpu().double() - wmass).abs() <= mt).all()
                assert torch.equal(bits(app.pool.cpu()), bits(wkv))

    step(2, serve)
    assert app.lengths[2] == 24 + 20
