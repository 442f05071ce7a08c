"""The orthogonalised update of the adapters that a batch has, on every path of the launches: those that ids holds take the step that all would take, bit by bit, the
others stay."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", [0, 1])
# in one workgroup; beyond its LDS; few tiles of S; parts of the contraction; 128 x 128; 256 x 128 tiles
@pytest.mark.parametrize("count,rows,cols", [(100, 16, 1024), (7, 256, 16), (1, 1, 1), (24, 64, 1024), (9, 128, 2048), (3, 700, 130), (2, 90, 4100), (40, 512, 520), (44, 700, 1100)])
def test_those_of_the_batch_alone(count, rows, cols, mode):
    from paper_1904_04956_amd import binding as bl
    g = torch.Generator(device="cuda:0").manual_seed(rows + cols)
    shape = (count, rows, cols)
    normal = lambda s: s * torch.randn(shape, device="cuda:0", generator=g)  # noqa: E731
    theta, grad, velocity = normal(0.1), normal(1e-3), normal(4e-3)
    n = bl.muon_orthogonalize_scratch_bytes(*shape, mode)
    scratch = torch.full((n + 4096,), 0x7F, dtype=torch.uint8, device="cuda:0")
    all_theta, all_v, all_shadow = theta.clone(), velocity.clone(), theta.bfloat16()
    bl.muon_matrices_step(all_theta, all_shadow, grad, all_v, *shape, mode, 0.02, 0.9, 0.1, 1, scratch, n)
    rng = np.random.default_rng(count)
    for ids in (rng.integers(-1, max(1, count // 2), 1 + 3 * count), [count - 1], [-1, count, 2 ** 31 - 1, -2 ** 31], np.arange(count)[::-1], np.concatenate([np.full(3000, -1), [0]])):
        ids = torch.from_numpy(np.asarray(ids, dtype=np.int32)).to("cuda:0")
        here = torch.zeros(count, dtype=torch.bool, device="cuda:0")
        here[ids[(ids >= 0) & (ids < count)].long()] = True
        scratch.fill_(0x7F)
        new, v, shadow = theta.clone(), velocity.clone(), theta.bfloat16()
        bl.muon_adapters_step(new, shadow, grad, v, ids, ids.numel(), *shape, mode, 0.02, 0.9, 0.1, 1, scratch, n)
        assert bool((scratch[n:] == 0x7F).all())
        for got, start, want in ((new, theta, all_theta), (v, velocity, all_v), (shadow, theta.bfloat16(), all_shadow)):
            assert torch.equal(got[here], want[here]) and torch.equal(got[~here], start[~here])


def test_a_captured_step_goes_by_the_ids_of_its_replay():
    from paper_1904_04956_amd import binding as bl
    shape = (6, 16, 200)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    theta, grad, velocity = (torch.randn(shape, device="cuda:0", generator=g) for _ in range(3))
    eager = [theta.clone(), velocity.clone()]
    ids = torch.zeros(9, dtype=torch.int32, device="cuda:0")
    n = bl.muon_orthogonalize_scratch_bytes(*shape, 0)
    scratch = [torch.empty(n, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    step = lambda t, v, s: bl.muon_adapters_step(t, None, grad, v, ids, 9, *shape, 0, 0.02, 0.9, 0.0, 0, s, n)  # noqa: E731
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step(theta, velocity, scratch[0])
    for k in range(4):
        ids.copy_(torch.from_numpy(np.random.default_rng(k).integers(-1, 6, 9).astype(np.int32)))
        graph.replay()
        step(*eager, scratch[1])
        torch.cuda.synchronize()
        assert torch.equal(theta, eager[0]) and torch.equal(velocity, eager[1])
