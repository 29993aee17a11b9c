"""A first call makes its workspace while a capture is under way elsewhere, in every mode of capturing."""
import pytest
import torch

from tests import test_gpu_decode as bf
from tests.test_gpu_decode import binding, clean  # noqa: F401 (binding is a fixture)
from tests.test_gpu_q4 import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["global", "thread_local", "relaxed"])
def test_workspaces_are_made_whatever_the_mode_of_another_streams_capture(binding, mode):  # noqa: F811
    """First calls, the call that makes the workspace ahead, and the results of both: on a stream that is not being captured."""
    a, b = Step(73, 4, 2, 64, 16, [(100, 2)], "chain"), bf.Step(74, 4, 2, 64, 16, [(100, 2)], "chain")
    c, d, e = (binding.Context() for _ in range(3))
    x = torch.zeros(4, device="cuda")
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode=mode):
        x.add_(1)
        with torch.cuda.stream(other):
            a.call(c)
            b.call(d)
            e.reserve_decode()
        x.add_(1)
    g.replay()
    torch.cuda.synchronize()
    assert x.tolist() == [2.0] * 4
    for ctx, step in ((c, a), (d, b)):
        clean(ctx)
        step.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode=mode):                         # and into a capture of its own
        a.call(e)
    a.blank()
    g.replay()
    clean(e)
    a.check()
