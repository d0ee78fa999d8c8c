"""A call of hybrid linear attention can be captured though it is the first of its kernels in the process (run by itself, this file is that)."""
import pytest
import torch

from hla_testlib import Sample, check, run
from hta_testlib import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,full", (((4, 2, 32), True), ((4, 1, 64), False), ((16, 2, 128), True), ((8, 2, 128), False)))
def test_first_call_in_a_capture(heads, full):
    say(f"  hla capture {heads} full={full}")
    s = Sample([120, 65], [3, 40], *heads, full, seed=1, state=True)
    b = s.batch()
    b.prepare_backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(s, b)
    for _ in range(3):
        for t in got.values():
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(got, s)
        run(s, b)
