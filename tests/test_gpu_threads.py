"""Calls from host threads of their own."""
import threading

import pytest
import torch

import oracle
from paper_2403_11805_b200 import binding as B, synth
from gpu_helpers import bits_view, odesc
from paged_reference import Batch, attend
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
