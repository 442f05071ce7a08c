"""The velocity that apply_muon makes at its first use is not made inside a graph, whose every replay would clear it."""
import pytest

from tests.test_gpu_learner_updates import learner

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", [0, 1])
def test_a_first_update_cannot_be_captured_and_a_second_keeps_its_velocity(mode):
    import torch
    one, *_ = learner(mode, 93)
    two, *_ = learner(mode, 93)
    try:
        for lrn in (one, two):
            lrn.calgrad()
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="captured"):
            with torch.cuda.graph(graph, stream=side):
                two.apply_muon(0.02, 0.1, momentum=0.9)
        assert two.velocity is None
        torch.cuda.synchronize()
        # without momentum there is none to make
        still = torch.cuda.CUDAGraph()
        with torch.cuda.graph(still, stream=side):
            two.apply_muon(0.0, 0.0, momentum=0.0)
        still.replay()
        for lrn in (one, two):
            lrn.apply_muon(0.02, 0.1, momentum=0.9)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            two.calgrad()
            two.apply_muon(0.02, 0.1, momentum=0.9)
        for _ in range(3):
            graph.replay()
            one.calgrad()
            one.apply_muon(0.02, 0.1, momentum=0.9)
            torch.cuda.synchronize()
            assert torch.equal(one.theta, two.theta) and torch.equal(one.velocity, two.velocity)
    finally:
        one.close()
        two.close()
