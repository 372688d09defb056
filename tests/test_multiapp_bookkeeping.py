"""The multi-app pool's bookkeeping without a GPU: the module itself, over a device that is imitated on the host.

Work that the module queues runs when the host waits for it and not before, in the order in which it was queued, as on a device
that is always behind: meta arrays and workspaces hold results only then.  A chunk's content is one number, which is its record
and its checksum too."""
import contextlib
import types

import numpy as np
import pytest
import torch

from paper_2403_11805_b200 import binding as B, multiapp, serving, synth


class Device:
    """Slots, the swap buffers' and the arena's records by position, and the work queued for them."""

    def __init__(self):
        self.queue, self.slots, self.staged, self.arena, self.corrupt, self.fresh = [], {}, {}, {}, {}, 1000
        self.waits = 0
        self.main = Stream(0, self)
        self.current, self.log = self.main, []               # the current stream; (what, on which stream) in the order of the calls

    @contextlib.contextmanager
    def stream(self, s):
        self.current, before = s, self.current
        yield
        self.current = before

    def wait(self, *_):
        self.waits += 1
        for work in self.queue:
            work()
        self.queue = []

    def new_content(self):
        self.fresh += 1
        return self.fresh

    # ---- the binding's calls
    def compress_chunks(self, desc, kv, ids, bits, out, meta, ws, **_):
        ids = [int(i) for i in ids]
        self.log.append(("compress", self.current.cuda_stream))

        def work():
            for i, slot in enumerate(ids):
                meta["checksum"][i] = self.slots[slot]
            self.staged[out.data_ptr()] = [self.slots[slot] for slot in ids]
            self.corrupt[ws.data_ptr()] = 0                  # a call's workspace begins as zeros
        self.queue.append(work)

    def swap_out(self, buf, meta, arena, host_offsets, n, **_):
        where = [int(x) for x in host_offsets]
        self.queue.append(lambda: self.arena.update(zip(where, self.staged[buf.data_ptr()])))

    def swap_in(self, arena, meta, buf, host_offsets, **_):
        where = [int(x) for x in host_offsets]
        self.queue.append(lambda: self.staged.update({buf.data_ptr(): [self.arena[x] for x in where]}))

    def decompress_chunks(self, desc, buf, meta, ids, kv, ws):
        slots, sums = [int(x) for x in meta["chunk_id"]], [int(x) for x in meta["checksum"]]   # read when the call is made

        def work():
            got = self.staged[buf.data_ptr()]
            self.corrupt[ws.data_ptr()] = sum(a != b for a, b in zip(got, sums))
            self.slots.update(zip(slots, got))
        self.queue.append(work)

    def codec_corrupt_count(self, ws):
        self.wait()
        return self.corrupt[ws.data_ptr()]

    def evict_tokens(self, desc, kv, mass, table, lens, max_len, budget, recent, kept, new_lens, **_):
        new_lens.copy_(lens.clamp(max=budget))


class Event:
    def __init__(self, device):
        self.synchronize = device.wait

    def record(self, *_):
        pass

    def elapsed_time(self, other):
        return 0.0


class Stream:
    def __init__(self, address=0, device=None):
        self.cuda_stream, self.device = address, device

    def wait_event(self, *_):
        pass

    def wait_stream(self, other):
        self.device.log.append(("wait", self.cuda_stream, other.cuda_stream))


@pytest.fixture
def device(monkeypatch):
    dev = Device()

    def made(name):
        def make(*shape, device=None, **kw):
            return getattr(torch, name)(*shape, **kw)
        return make

    cuda = types.SimpleNamespace(synchronize=dev.wait, current_stream=lambda *_: dev.current, stream=dev.stream, Stream=Stream,
                                 Event=lambda **_: Event(dev))
    fake = types.SimpleNamespace(cuda=cuda, **{n: made(n) for n in ("zeros", "empty", "full")},
                                 **{n: getattr(torch, n) for n in ("from_numpy", "empty_like", "cat", "uint8", "int32", "float16", "float32")})
    monkeypatch.setattr(multiapp, "torch", fake)
    monkeypatch.setattr(serving, "torch", fake)
    monkeypatch.setattr(torch.Tensor, "cuda", lambda self, *_, **__: self.clone())
    monkeypatch.setattr(torch.Tensor, "pin_memory", lambda self, *_, **__: self)
    for name in ("compress_chunks", "swap_out", "swap_in", "decompress_chunks", "codec_corrupt_count", "evict_tokens"):
        monkeypatch.setattr(B, name, getattr(dev, name))
    monkeypatch.setattr(B, "new_event", lambda *_: Event(dev))
    monkeypatch.setattr(B, "current_stream", lambda: dev.current.cuda_stream)
    return dev


CHUNKS = 100


def pool(device, n_contexts=4, aot=False):
    """Contexts of 100 chunks of 16 tokens with room for two of them; every record in the arena, the first two contexts resident
    and modified since."""
    sh = synth.KVShape("apps", 1, 1, 1, 16, CHUNKS * 16, 16, 16, window=4, seed=1, n_contexts=n_contexts)
    app = multiapp.MultiApp(sh, n_slots=2 * CHUNKS, seed=1, aot=aot)
    app._alloc_buffers()
    for c in range(n_contexts):
        bits, _ = B.assign_bits(np.arange(CHUNKS, dtype=np.float32), app.frac)
        app._place_in_arena(c, bits)
    for row in range(n_contexts * CHUNKS):
        app.checksum[row] = device.arena[int(app.arena_off[row])] = device.new_content()
    for c in range(2):
        app._load(np.arange(c * CHUNKS, (c + 1) * CHUNKS))
    app._end_of_step()
    modify(device, app, range(2 * CHUNKS))
    app.chosen = []
    app.draw_contexts = lambda k: app.chosen
    return app


def modify(device, app, rows):
    """The chunks in these rows get other content, behind everything that is queued."""
    slots = [int(app.slot[r]) for r in rows]
    device.queue.append(lambda: device.slots.update((s, device.new_content()) for s in slots))
    app.clean[rows] = False


def step(app, ctxs, serve=None):
    app.chosen = list(ctxs)
    return app.step(k=len(ctxs), serve=serve)


def grow(device, app, chunks):
    """A serve callback: every context of the batch grows by so many chunks."""
    def serve(s):
        for _ in range(chunks):
            for _ in range(16):
                s.advance()
            for i, c in enumerate(s.ctxs):
                modify(device, app, [c * CHUNKS + (int(s.lengths[i]) - 1) // 16])
    return serve


def crowded(device):
    """Context 2 is down to one chunk and out; the pool is full of modified chunks of contexts 1 and 3, and their content by row."""
    app = pool(device)
    step(app, [2], lambda s: s.shrink(16, 1))
    step(app, [3])
    step(app, [1])
    if app.slot[2 * CHUNKS] >= 0:
        app._evict([2 * CHUNKS])
    rows = np.flatnonzero(app.slot >= 0)
    modify(device, app, rows)
    app._end_of_step()
    return app, {int(r): device.slots[int(app.slot[r])] for r in rows}


def test_more_reclaims_in_a_step_than_the_ring_has_entries(device):
    app, was = crowded(device)
    before = app._ws_next
    step(app, [2], grow(device, app, 95))
    assert app._ws_next - before > len(app.ws) + 20
    gone = [r for r in was if app.slot[r] < 0]
    assert len(gone) >= 90
    wrong = [r for r in gone if app.checksum[r] != was[r]]
    assert not wrong, f"{len(wrong)} of {len(gone)} records have another record's checksum"
    assert all(device.arena[int(app.arena_off[r])] == was[r] for r in gone)
    step(app, [1])                                           # and they are read back
    step(app, [3])
    back = [r for r in gone if app.slot[r] >= 0]
    assert back and all(device.slots[int(app.slot[r])] == was[r] for r in back)


def test_a_corrupt_record_is_reported_however_much_follows_in_its_step(device):
    app, _ = crowded(device)
    device.arena[int(app.arena_off[2 * CHUNKS])] += 1
    with pytest.raises(RuntimeError, match="checksum"):
        step(app, [2], grow(device, app, 95))
    step(app, [1])                                           # reported once


def test_a_step_of_few_reclaims_waits_at_its_end_only(device):
    app, _ = crowded(device)
    waits, inside = device.waits, []
    step(app, [2], lambda s: (grow(device, app, 40)(s), inside.append(device.waits - waits)))
    assert inside == [0]


def test_a_callback_on_a_stream_of_its_own(device):
    """What growth and shrinking queue goes to the pool's stream, behind the caller's work and before its next."""
    app, _ = crowded(device)
    side = Stream(7, device)

    def serve(s):
        device.log.clear()
        with device.stream(side):
            grow(device, app, 3)(s)
            grown = list(device.log)
            device.log.clear()
            s.shrink(16, 1)
        assert [e for e in grown if e[0] == "compress"] == [("compress", 0)] * 3
        for i, e in enumerate(grown):
            if e[0] == "compress":
                assert grown[i - 1] == ("wait", 0, 7) and grown[i + 1] == ("wait", 7, 0)
        assert device.log == [("wait", 0, 7), ("wait", 7, 0)]

    step(app, [2], serve)
    device.log.clear()
    step(app, [1], lambda s: s.shrink(1600, 1))              # on the pool's own stream nothing has to be ordered
    assert not [e for e in device.log if e[0] == "wait"]


def test_a_batch_is_not_used_behind_its_step(device):
    app, _ = crowded(device)
    kept = []
    step(app, [2], kept.append)
    lengths, slots = list(app.lengths), app.slot.copy()
    s = kept[0]
    for use in (s.advance, lambda: s.decode(0, None, None, None), lambda: s.shrink(1, 1)):
        with pytest.raises(RuntimeError, match="has ended"):
            use()
    assert app.lengths == lengths and np.array_equal(app.slot, slots)


def test_contexts_whose_last_chunk_is_not_whole(device):
    """The pool holds whole chunks; the tokens behind the last one take no part, and no rows of the next context."""
    sh = synth.KVShape("apps", 1, 1, 1, 16, 5 * 16 + 7, 16, 16, window=4, seed=1, n_contexts=4)
    app = multiapp.MultiApp(sh, n_slots=10, seed=1)
    app._alloc_buffers()
    for c in range(4):
        bits, _ = B.assign_bits(np.arange(5, dtype=np.float32), app.frac)
        app._place_in_arena(c, bits)
    for row in range(20):
        app.checksum[row] = device.arena[int(app.arena_off[row])] = device.new_content()
    for c in (2, 3, 0, 1):
        assert app.rows(c).tolist() == list(range(5 * c, 5 * c + 5))
        lengths = []
        app.draw_contexts = lambda k, c=c: [c]
        app.step(k=1, serve=lambda s: lengths.extend(s.lengths))
        assert lengths == [80] and app.table["resident"][5 * c:5 * c + 5].all() and app.table["resident"].sum() <= 10
        assert set(np.flatnonzero(app.table["last_access_step"] == app.step_no)) == set(range(5 * c, 5 * c + 5))


def test_a_step_with_every_context_resident_serves_none(device):
    """Shrunk contexts all fit: nothing is drawn, and that is an empty step, not an error."""
    app = pool(device)
    for c in range(4):
        step(app, [c], lambda s: s.shrink(20, 1))
    del app.draw_contexts
    for c in (0, 1):                                          # whatever is out comes in
        app.step(k=4)
    assert all(app.table["resident"][app.rows(c)].all() for c in range(4))
    served, before = [], (app.slot.copy(), list(app.free), app.table.copy())
    assert app.step(k=2, serve=served.append) == [] and not served
    assert np.array_equal(app.slot, before[0]) and app.free == before[1] and np.array_equal(app.table, before[2])


def test_an_empty_step_settles_what_the_last_one_left(device):
    app = pool(device, aot=True)
    for c in range(4):
        step(app, [c], lambda s: s.shrink(20, 1))
    del app.draw_contexts
    app.step(k=4)
    app.step(k=4)
    assert device.queue == [] and not app._pending
    assert all(app.checksum[r] == device.slots[int(app.slot[r])] for c in range(4) for r in app.rows(c) if app.slot[r] >= 0)


@pytest.mark.parametrize("aot", [False, True], ids=["reclaim", "aot"])
@pytest.mark.parametrize("seed", range(6))
def test_random_steps_keep_every_chunk(device, seed, aot):
    """Contexts are served, grown, shrunk, and their callbacks raise, in a pool that holds a third of them: every chunk is in its
    slot or, with its checksum, in the arena."""
    rng = np.random.RandomState(seed)
    cpc, n_ctx = 7, 9
    sh = synth.KVShape("apps", 1, 1, 1, 16, cpc * 16, 16, 16, window=4, seed=1, n_contexts=n_ctx)
    app = multiapp.MultiApp(sh, n_slots=3 * cpc, seed=seed, aot=aot)
    app._alloc_buffers()
    for c in range(n_ctx):
        bits, _ = B.assign_bits(np.arange(cpc, dtype=np.float32), app.frac)
        app._place_in_arena(c, bits)
    truth = {}
    for row in range(n_ctx * cpc):
        truth[row] = app.checksum[row] = device.arena[int(app.arena_off[row])] = device.new_content()

    def change(row):
        slot, truth[row] = int(app.slot[row]), device.new_content()
        device.queue.append(lambda value=truth[row]: device.slots.update({slot: value}))

    def serve(s):
        held = {r: (int(app.slot[r]), truth[r]) for c in s.ctxs for r in app.rows(c)}
        device.wait()
        assert all(device.slots[slot] == value for slot, value in held.values())
        for _ in range(rng.randint(0, 60)):
            if rng.rand() < 0.15:
                s.shrink(int(rng.randint(1, cpc * 16)), 1)
                for i, c in enumerate(s.ctxs):
                    for r in range(c * cpc, c * cpc + -(-int(s.lengths[i]) // 16)):
                        change(r)
            elif (s.lengths < s.capacity).all():
                s.advance()
                for i, c in enumerate(s.ctxs):
                    change(c * cpc + (int(s.lengths[i]) - 1) // 16)
        if rng.rand() < 0.2:
            raise KeyError("the model's own")

    for _ in range(60):
        try:
            app.step(k=int(rng.randint(1, 4)), serve=serve if rng.rand() < 0.8 else None)
        except KeyError:
            pass
        if rng.rand() < 0.3:
            app.finish()
        device.wait()
        app._collect_checksums()
        live = np.concatenate([app.rows(c) for c in range(n_ctx)])
        res = np.flatnonzero(app.slot >= 0)
        assert set(res) <= set(live) and not app.table["locked"].any() and np.array_equal(app.slot >= 0, app.table["resident"] != 0)
        assert sorted([int(x) for x in app.slot[res]] + app.free) == list(range(app.n_slots))
        for r in live:
            if app.slot[r] >= 0:
                assert device.slots[int(app.slot[r])] == truth[r]
            if app.slot[r] < 0 or app.clean[r]:
                assert device.arena[int(app.arena_off[r])] == truth[r] == app.checksum[r]
