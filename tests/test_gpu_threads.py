"""GPU: steps of several host threads, whose kernels take shared memory of different sizes."""
import threading

import pytest
import torch

from paper_1606_03401_b200 import synth
from tests.util import assert_bit_identical

pytestmark = pytest.mark.gpu


def test_float32_runs_of_host_threads_whose_layers_differ_in_width():
    """A step sets its kernels' limit of shared memory before it launches them: not below what another thread's step needs."""
    from paper_1606_03401_b200 import binding as B
    from paper_1606_03401_b200 import harness
    problems = []
    for H in (320, 1024):
        cfg = synth.with_overrides(synth.CONFIGS["c1"], dtype="tf32", input=64, hidden=H, batch=32, t=24, readout=32)
        dp = harness.DeviceProblem(cfg)
        plan = dp.plan("msm", 8)
        assert B.mebptt_test_route(dp.desc, plan)["route"] == "runs_f32"
        problems.append((dp, plan, dp.run(plan)))
    raised, start = [], threading.Barrier(len(problems))

    def repeat(dp, plan):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(60)
                for _ in range(100):
                    dp.enqueue(plan)
                torch.cuda.synchronize()
        except Exception as e:  # noqa: BLE001  (handed on)
            raised.append(e)

    threads = [threading.Thread(target=repeat, args=p[:2]) for p in problems]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not raised, raised
    for dp, plan, clean in problems:
        last = {k: (v.cpu().numpy().copy() if v is not None else None) for k, v in dp.out.items()}
        last["loss"] = float(last["loss"][0])
        assert last["counters"][3] == 0
        assert_bit_identical(last, clean)
        assert_bit_identical(dp.run(plan), clean)
