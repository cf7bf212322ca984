"""GPU: the operators over sequences where calls meet: several host threads, rows and states at the edge of what counts, waits that run out."""
import threading

import pytest
import torch

from paper_1606_03401_b200 import binding as B
from tests.test_gpu_sequence_ops import Distill

pytestmark = pytest.mark.gpu


def _together(calls):
    """Each call by a host thread of its own, on a stream of its own; what a thread raises is raised here."""
    raised = []
    start = threading.Barrier(len(calls))

    def run(call):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(60)
                call()
                torch.cuda.synchronize()
        except Exception as e:  # noqa: BLE001  (handed on)
            raised.append(e)

    threads = [threading.Thread(target=run, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if raised:
        raise raised[0]


@pytest.mark.parametrize("dtype,sizes", [("bf16", (32000, 20000, 5000)), ("fp32", (16000, 9000, 70000)), ("bf16", (2040, 1800, 1600))])
def test_distill_calls_of_host_threads_whose_rows_differ_in_length(dtype, sizes):
    """Kernels that take all these lengths with shared memory of another size for each: a call of one thread must not find the limit
    that another thread's call has just set for shorter rows."""
    problems = [Distill(dtype, 2, V, 9, seed=V).upload() for V in sizes]

    def outputs(p):
        return p.loss, p.row_loss, p.DX

    for p in problems:
        p.both()
    torch.cuda.synchronize()
    want = [[v.clone() for v in outputs(p)] for p in problems]

    def repeat(p):
        # (the C interface: what happens between its calls should be as little as possible)
        stream = torch.cuda.current_stream().cuda_stream
        a = [x.data_ptr() for x in (p.X, *p.dev, p.dloss)]
        o = [x.data_ptr() for x in outputs(p)]
        for _ in range(3000):
            st = B.lib.mebptt_distill_loss_grad(B.C.addressof(p.desc), *a, stream, *o)
            assert st == B.MEBPTT_OK, st

    _together([lambda p=p: repeat(p) for p in problems])
    for p, w in zip(problems, want):
        assert all(torch.equal(x, y) for x, y in zip(outputs(p), w))
