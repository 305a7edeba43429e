"""A call of the binding gives up the interpreter's lock while it is in the library, so that one that waits there (the stream's queue is full) does not stop other Python threads."""
import sys
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def calls(gpu):
    from paper_2603_19133_amd import binding as ps
    from paper_2603_19133_amd import training
    V = 100
    z, grad, table = torch.randn((4, V), device=gpu), torch.randn((4, V), device=gpu), torch.randn((9, V), device=gpu)
    tok = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device=gpu)
    into, sums = torch.empty_like(z), torch.empty_like(table)
    rec = ps.compress(z, V, 1.0, 5)
    leaf, rows = z.clone().requires_grad_(), table.clone().requires_grad_()
    return {"compress": lambda: ps.compress(z, V, 1.0, 5, out=rec),
            "adjust": lambda: ps.adjust(z, V, presence=1.0, out=into),
            "adjust_grad": lambda: ps.adjust_grad(grad, z, V, repetition=2.0, out=into),
            "embed": lambda: ps.embed(table, tok, out=into),
            "embed_grad": lambda: ps.embed_grad(grad, tok, 9, out=sums),
            "clip_grad": lambda: ps.clip_grad([grad], 1e9),
            "training.adjust": lambda: training.adjust(leaf, V, presence=1.0),
            "training.embed": lambda: training.embed(rows, tok),
            "training.distill_loss": lambda: training.distill_loss(leaf, rec, V, 1.0)}


@pytest.mark.parametrize("name", ["compress", "adjust", "adjust_grad", "embed", "embed_grad", "clip_grad", "training.adjust", "training.embed", "training.distill_loss"])
def test_another_thread_goes_on(gpu, calls, name):
    print(f"[case] threads {name}", flush=True)
    call, gate, passed = calls[name], threading.Lock(), []
    for _ in range(3):
        call()
    torch.cuda.synchronize()
    gate.acquire()
    other = threading.Thread(target=lambda: (gate.acquire(), passed.append(True)))
    before = sys.getswitchinterval()
    try:
        other.start()
        sys.setswitchinterval(1000.0)                    # (from here on the lock changes hands only where a call gives it up)
        gate.release()
        kept = []                                        # (torch gives the lock up where it frees a tensor)
        while not passed and len(kept) < 5000:           # (the other thread has to wake up in the meantime)
            kept.append(call())
        went_on = bool(passed)
    finally:
        sys.setswitchinterval(before)
        other.join()
    torch.cuda.synchronize()
    assert went_on
