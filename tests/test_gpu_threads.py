"""Calls from host threads of their own, one after another and several at once."""
import threading

import pytest
import torch

import oracle
from paper_2403_11805_b200 import binding as B, synth
from gpu_helpers import bits_view, odesc
from paged_reference import Batch, attend, bits, evict
from test_gpu_decode import desc_of, workspace

pytestmark = pytest.mark.gpu


def in_a_new_thread(call):
    raised = []

    def work():
        try:
            call()
        except Exception as e:
            raised.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    if raised:
        raise raised[0]


def test_a_thread_whose_first_use_of_the_device_is_a_decode_call():
    bt = Batch([100, 7], group=2, dim=64, seed=1)
    d, kv, q, table = desc_of(bt), bt.kv.cuda(), bt.q.contiguous().cuda(), bt.table.cuda()
    lens, out, ws = torch.tensor(bt.lens, dtype=torch.int32).cuda(), torch.zeros(2, 4, 64, dtype=torch.float16).cuda(), workspace(d, 2, 100)
    torch.cuda.synchronize()
    in_a_new_thread(lambda: B.decode_attention(d, 0, kv, q, table, lens, 100, out, ws))
    want, _, _, _, (ot, _, _) = attend(bt)
    assert ((out.cpu().double() - want).abs() <= ot).all()


def test_a_thread_whose_first_use_of_the_device_is_a_score_call():
    sh = synth.KVShape("score", 1, 1, 8, 64, 256, 32, 64, window=8, seed=3)   # 64 query rows per KV head: the tcgen05 kernel
    kv, q = synth.kv_tensor(sh, device="cuda"), synth.q_window(sh, 8, device="cuda")
    d = B.desc_of(sh)
    scores, ws = torch.zeros(sh.n_chunks, device="cuda"), torch.empty(B.tolerance_workspace_bytes(d, 8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    in_a_new_thread(lambda: B.chunk_tolerance(d, kv, q, 8, scores, ws))
    want = oracle.chunk_tolerance(odesc(sh), bits_view(kv), bits_view(q), 8)
    assert (abs(scores.cpu().numpy() - want) / want).max() < 1e-4


# Several threads at once, each with a stream, tensors and a workspace of its own.  The sizes are such that neighbouring threads'
# calls launch the same kernels with different amounts of shared memory.

def run_together(jobs, calls):
    """Each job `calls` times in a thread of its own; what a thread raised is raised here."""
    raised, start = [], threading.Barrier(len(jobs))

    def work(job):
        try:
            start.wait()
            for _ in range(calls):
                job()
        except Exception as e:
            raised.append(e)

    threads = [threading.Thread(target=work, args=(job,)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    if raised:
        raise raised[0]


@pytest.mark.parametrize("max_len", [300, 5000], ids=["cluster_per_item", "runs"])
def test_decode_from_several_threads(max_len):
    checks, jobs = [], []
    for i, group in enumerate((1, 4, 2, 3)):
        bt = Batch([300, 7], heads=2, group=group, dim=128, seed=i, max_len=max_len)
        d, n, stream = desc_of(bt), 2, torch.cuda.Stream()
        kv, q, table = bt.kv.cuda(), bt.q.contiguous().cuda(), bt.table.cuda()
        lens, out, ws = torch.tensor(bt.lens, dtype=torch.int32).cuda(), torch.zeros(n, 2 * group, 128, dtype=torch.float16).cuda(), workspace(d, n, max_len)
        jobs.append(lambda d=d, kv=kv, q=q, table=table, lens=lens, out=out, ws=ws, s=stream:
                    B.decode_attention(d, 0, kv, q, table, lens, max_len, out, ws, stream=s))
        checks.append((bt, out))
    torch.cuda.synchronize()
    run_together(jobs, 8000)
    for bt, out in checks:
        want, _, _, _, (ot, _, _) = attend(bt)
        assert ((out.cpu().double() - want).abs() <= ot).all()


def test_evict_from_several_threads():
    checks, jobs = [], []
    for i, tokens in enumerate((40000, 4100, 17000, 6000)):
        bt = Batch([tokens], heads=1, dim=16, seed=i)
        d, stream = desc_of(bt), torch.cuda.Stream()
        kv, table, mass = bt.kv.cuda(), bt.table.cuda(), bt.mass.cuda()
        lens, out = torch.tensor(bt.lens, dtype=torch.int32).cuda(), torch.full_like(mass, 5.0)
        kept, new_lens = torch.zeros(1, 1, 1, tokens, dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
        # nothing is dropped: the calls repeat themselves
        jobs.append(lambda d=d, kv=kv, mass=mass, table=table, lens=lens, out=out, kept=kept, new=new_lens, n=tokens, s=stream:
                    B.evict_tokens(d, kv, mass, table, lens, n, n, 5, kept, new, mass_out=out, stream=s))
        checks.append((bt, out, kept, kv))
    torch.cuda.synchronize()
    run_together(jobs, 2000)
    for bt, out, kept, kv in checks:
        want = evict(bt, bt.mass, bt.lens[0], 5, None, torch.full_like(bt.mass, 5.0))
        assert torch.equal(kept.cpu(), want[0]) and torch.equal(out.cpu(), want[2]) and torch.equal(bits(kv.cpu()), bits(want[3]))
