"""The orthogonalised update on the GPU against the float64 oracle.

Tolerances (2-norm of the difference over 2-norm of the result, a matrix at a time).  A step rounds three operands (X, S, B), each by at most half
a step e of what it is held in: 2^-12 in mode 1 (halves), 2^-22 in mode 0 (pairs of halves).  The polynomial's slope where singular values end up is at most 1.6 in
size and B's coefficients below 5, so that a rounding arrives with a factor of 4 on average over the steps; fifteen of them, independent: 4 sqrt(15) e < 16 e.
Sums are in float: sqrt(n) 2^-24 of a product of norm one, below 16 * 2^-22 for the sizes here.  X in bf16 adds 2^-9 of each element (and at most half a step:
2^-8 of the largest below it)."""
import numpy as np
import pytest

from oracle import blstm_oracle as orc
from oracle import muon

pytestmark = pytest.mark.gpu
E = {0: 16 * 2.0 ** -22, 1: 16 * 2.0 ** -12}
BF16 = 2.0 ** -8


def gradient(rng, count, rows, cols):
    """A few directions that are common, and noise; rows of unequal size."""
    some = rng.normal(size=(count, rows, 4)) @ rng.normal(size=(count, 4, cols))
    return (1e-3 * np.exp(0.5 * rng.normal(size=(count, rows, 1))) * (some + rng.normal(size=(count, rows, cols)))).astype(np.float32)


def off(got, want):
    return np.linalg.norm(np.asarray(got, dtype=np.float64) - want) / max(np.linalg.norm(want), 1e-30)


def guarded(n):
    """n bytes of scratch filled with NaN patterns, and the 4096 behind them."""
    import torch
    t = torch.full((n + 4096,), 0x7F, dtype=torch.uint8, device="cuda:0")
    return t, lambda: bool((t[n:] == 0x7F).all())


SHAPES = [(1, 1, 1), (1, 1, 37), (1, 37, 1), (3, 5, 9), (2, 64, 64), (2, 65, 63), (5, 16, 1024), (4, 256, 16), (1, 129, 513), (2, 700, 130), (1, 130, 4100), (1, 5000, 200),
          (3, 602, 1204), (300, 7, 24), (20, 512, 260), (36, 512, 1024)]


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("count,rows,cols", SHAPES)
def test_orthogonalize(mode, count, rows, cols):
    import torch
    from paper_1904_04956_amd import binding as bl
    G = gradient(np.random.default_rng(rows * 7 + cols), count, rows, cols)
    X = torch.full((count, rows, cols), 7.0, dtype=torch.bfloat16 if mode else torch.float32, device="cuda:0")
    n = bl.muon_orthogonalize_scratch_bytes(count, rows, cols, mode)
    scratch, kept = guarded(n)
    g = torch.from_numpy(G).to("cuda:0")
    bl.muon_orthogonalize(g, X, count, rows, cols, mode, scratch, n)
    got = X.float().cpu().numpy()
    assert kept() and np.array_equal(g.cpu().numpy(), G)
    for k in range(min(count, 8)):
        want = muon.orthogonalize(G[k])
        assert off(got[k], want) < E[mode] + (BF16 if mode else 0), k
    first = X.clone()
    bl.muon_orthogonalize(g, X, count, rows, cols, mode, scratch, n)
    assert torch.equal(first, X)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("R,C", [(40, 70), (130, 200), (90, 700)], ids=["in one workgroup", "both halves", "long rows"])
def test_gradients_of_any_size_zero_matrices_and_what_is_no_number(mode, R, C):
    import torch
    from paper_1904_04956_amd import binding as bl
    rng = np.random.default_rng(5)
    G = gradient(rng, 8, R, C)
    G[1] *= 1e-30                               # squares that float does not hold
    G[2] *= 1e30
    G[3] = 0
    G[4, 3, 5] = np.nan
    G[5, R - 1, C - 1] = np.inf
    G[6, :, 3:] = 0                             # rank three
    G[7, 1:] = 0                                # one row
    X = torch.empty((8, R, C), dtype=torch.bfloat16 if mode else torch.float32, device="cuda:0")
    n = bl.muon_orthogonalize_scratch_bytes(8, R, C, mode)
    bl.muon_orthogonalize(torch.from_numpy(G).to("cuda:0"), X, 8, R, C, mode, torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda:0"))
    got = X.float().cpu().numpy()
    assert np.all(got[3] == 0) and np.isnan(got[4]).all() and np.isnan(got[5]).all()
    for k in (0, 1, 2, 6, 7):
        assert off(got[k], muon.orthogonalize(G[k].astype(np.float64))) < E[mode] + (BF16 if mode else 0), k


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("momentum,nesterov", [(0.95, True), (0.9, False), (0.0, False)])
def test_matrices_step(mode, momentum, nesterov):
    import torch
    from paper_1904_04956_amd import binding as bl
    rng = np.random.default_rng(6)
    shape = (3, 75, 33)
    theta, g, v = rng.uniform(-0.1, 0.1, shape).astype(np.float32), gradient(rng, *shape), 4 * gradient(rng, *shape)
    want, want_v = muon.matrices_step(theta.astype(np.float64), g.astype(np.float64), v.astype(np.float64), 0.02, momentum, 0.1, nesterov)
    t, gd, vd = (torch.from_numpy(x).to("cuda:0") for x in (theta.copy(), g, v.copy()))
    shadow = torch.empty(shape, dtype=torch.bfloat16, device="cuda:0") if mode else None
    n = bl.muon_orthogonalize_scratch_bytes(*shape, mode)
    scratch, kept = guarded(n)
    bl.muon_matrices_step(t, shadow, gd, vd if momentum else None, *shape, mode, 0.02, momentum, 0.1, bl.MUON_NESTEROV if nesterov else 0, scratch, n)
    assert kept()
    # theta = (1 - lr wd) theta - lr sqrt(75/33) O: three roundings in float beside O's error
    step = 0.02 * np.sqrt(75 / 33) * np.linalg.norm(muon.orthogonalize((g + momentum * want_v if nesterov else want_v)[0].astype(np.float64)))
    for k in range(3):
        assert np.linalg.norm(t[k].cpu().numpy() - want[k]) < step * E[mode] * 1.5 + 3 * 2.0 ** -24 * np.linalg.norm(want[k])
    assert np.abs(vd.cpu().numpy() - (want_v if momentum else v)).max() <= 2.0 ** -23 * np.abs(want_v).max()
    if mode:
        assert torch.equal(shadow, t.to(torch.bfloat16))


MODELS = [dict(D=40, H=32, L=1, P=0, V=100), dict(D=5, H=3, L=3, P=7, V=11), dict(D=260, H=301, L=2, P=67, V=301), dict(D=64, H=128, L=2, P=256, V=3000),
          dict(D=1, H=1, L=1, P=0, V=1), dict(D=260, H=512, L=2, P=256, V=500)]


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("flags", [0, 7])
@pytest.mark.parametrize("dims", MODELS, ids=lambda d: f"H{d['H']}")
def test_model_step(mode, flags, dims):
    import torch
    from paper_1904_04956_amd import binding as bl
    dm = orc.Dims(T=1, B=1, **dims)
    n, rng = orc.param_count(dm), np.random.default_rng(dims["H"])
    layout = orc.layout(dm)
    theta = rng.uniform(-0.1, 0.1, n).astype(np.float32)
    g, v = np.empty(n, np.float32), np.empty(n, np.float32)
    for _, at, shape in layout:
        size, two = int(np.prod(shape)), (shape if len(shape) == 2 else (shape[0], 1))
        g[at:at + size], v[at:at + size] = gradient(rng, 1, *two).reshape(-1), 4 * gradient(rng, 1, *two).reshape(-1)
    want, want_v = muon.step(layout, *(x.astype(np.float64) for x in (theta, g, v)), 0.02, 0.1, 0.9, 0.1, bool(flags & 1), bool(flags & 2), bool(flags & 4))
    ctx = bl.blstm_create(1, 1, dims["D"], dims["H"], dims["L"], dims["P"], dims["V"], mode)
    try:
        t, gd, vd = (torch.from_numpy(x.copy()).to("cuda:0") for x in (theta, g, v))
        shadow = torch.empty(n, dtype=torch.bfloat16, device="cuda:0") if mode else None
        nbytes = bl.muon_scratch_bytes(ctx, flags)
        scratch, kept = guarded(nbytes)
        bl.muon_step(ctx, t, shadow, gd, vd, 0.02, 0.1, 0.9, 0.1, flags, scratch, nbytes)
        assert kept() and np.array_equal(gd.cpu().numpy(), g)
    finally:
        bl.blstm_destroy(ctx)
    got = t.cpu().numpy()
    ortho = {at: (R, C) for at, R, C in muon.matrices(layout, bool(flags & 2), bool(flags & 4))}
    rest = np.ones(n, bool)
    for at, (R, C) in ortho.items():
        part = slice(at, at + R * C)
        rest[part] = False
        step = 0.02 * np.sqrt(max(1.0, R / C)) * np.sqrt(min(R, C)) * 1.2          # no singular value exceeds 1.2
        assert np.linalg.norm(got[part] - want[part]) < step * E[mode] + 3 * 2.0 ** -24 * np.linalg.norm(want[part]), (at, R, C)
    assert np.abs(got[rest] - want[rest]).max() <= 2.0 ** -22 * max(1e-3, np.abs(want[rest]).max()) if rest.any() else True
    assert np.abs(vd.cpu().numpy() - want_v).max() <= 2.0 ** -23 * np.abs(want_v).max()
    if mode:
        assert torch.equal(shadow, t.to(torch.bfloat16))


def test_replayed_steps_are_the_eager_ones():
    import torch
    from paper_1904_04956_amd import binding as bl
    rng = np.random.default_rng(9)
    shape = (4, 200, 96)
    start = [torch.from_numpy(x).to("cuda:0") for x in (rng.uniform(-0.1, 0.1, shape).astype(np.float32), gradient(rng, *shape), gradient(rng, *shape))]
    n = bl.muon_orthogonalize_scratch_bytes(*shape, 1)
    call = lambda t, g, v, s: bl.muon_matrices_step(t, None, g, v, *shape, 1, 0.02, 0.9, 0.0, 1, s, n)  # noqa: E731
    eager, held = [x.clone() for x in start], [x.clone() for x in start]
    own, other = (torch.empty(n, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(*held, other)
    for _ in range(4):
        graph.replay()
        call(*eager, own)
        own.fill_(255)
        torch.cuda.synchronize()
        assert torch.equal(held[0], eager[0]) and torch.equal(held[2], eager[2])
        held[1].mul_(0.5)
        eager[1].mul_(0.5)


def test_steps_on_two_streams_at_once():
    import torch
    from paper_1904_04956_amd import binding as bl
    rng = np.random.default_rng(10)
    shape = (2, 300, 256)
    G = torch.from_numpy(gradient(rng, *shape)).to("cuda:0")
    n = bl.muon_orthogonalize_scratch_bytes(*shape, 1)
    want = torch.empty(shape, dtype=torch.bfloat16, device="cuda:0")
    bl.muon_orthogonalize(G, want, *shape, 1, torch.empty(n, dtype=torch.uint8, device="cuda:0"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = [(torch.empty_like(want), torch.empty(n, dtype=torch.uint8, device="cuda:0")) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (X, scratch) in zip(streams, work):
            bl.muon_orthogonalize(G, X, *shape, 1, scratch, None, s)
    torch.cuda.synchronize()
    assert all(torch.equal(X, want) for X, _ in work)
