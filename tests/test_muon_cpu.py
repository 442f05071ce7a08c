"""The orthogonalised update without a GPU: the float64 oracle against singular values, the calls' refusals, their scratch, what they launch."""
import numpy as np
import pytest

from oracle import blstm_oracle as orc
from oracle import muon
from paper_1904_04956_amd import binding as bl
from tests.test_dispatch_cpu import recorder  # noqa: F401


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (6, 6), (1, 7), (7, 1)])
def test_the_oracle_maps_singular_values_and_keeps_the_vectors(shape):
    G = np.random.default_rng(1).normal(size=shape)
    u, s, vt = np.linalg.svd(G, full_matrices=False)
    s = s / np.sqrt((s * s).sum())
    for _ in range(muon.STEPS):
        s = muon.A * s + muon.B * s ** 3 + muon.C * s ** 5
    assert np.abs(muon.orthogonalize(G) - (u * s) @ vt).max() < 1e-12
    assert s.max() < 1.21 and (min(shape) == 1 or s.min() > 0.3)


def test_the_oracle_of_scales_signs_and_zero():
    G = np.random.default_rng(2).normal(size=(4, 6))
    O = muon.orthogonalize(G)
    assert np.abs(muon.orthogonalize(1e-6 * G) - O).max() < 1e-12 and np.abs(muon.orthogonalize(-G) + O).max() < 1e-12
    assert np.abs(muon.orthogonalize(G.T) - O.T).max() < 1e-14
    assert np.all(muon.orthogonalize(np.zeros((3, 2))) == 0)


def test_the_model_step_is_the_matrices_steps_and_momentum():
    dm = orc.Dims(T=2, B=2, D=5, H=4, L=2, P=3, V=7)
    r = np.random.default_rng(3)
    n = orc.param_count(dm)
    theta, g, v = (r.normal(size=n) for _ in range(3))
    new, w = muon.step(orc.layout(dm), theta, g, v, 0.02, 0.1, 0.9, 0.1, True, False, False)
    assert np.array_equal(w, 0.9 * v + g)
    names = {name: (at, shape) for name, at, shape in orc.layout(dm)}
    for name in ("Wx0.0", "Uh1.1", "Wp"):
        at, (R, C) = names[name]
        part = slice(at, at + R * C)
        one, _ = muon.matrices_step(*(x[part].reshape(1, R, C) for x in (theta, g, v)), 0.02, 0.9, 0.1, True)
        assert np.abs(new[part].reshape(1, R, C) - one).max() < 1e-15
    for name in ("b0.1", "bp", "Ws", "bs"):
        at, shape = names[name]
        part = slice(at, at + int(np.prod(shape)))
        assert np.abs(new[part] - (theta[part] - 0.1 * (g[part] + 0.9 * w[part]))).max() < 1e-15


# ---- refusals --------------------------------------------------------------------------------------------------------

@pytest.fixture
def ctx():
    c = bl.blstm_create(2, 2, 5, 4, 2, 3, 7, 1)
    yield c
    bl.blstm_destroy(c)


def model(ctx, **change):
    a = dict(theta=4096, shadow=4096, grad=4096, velocity=4096, lr=0.02, lr_rest=0.1, momentum=0.9, decay=0.1, flags=7, scratch=4096,
             nbytes=bl.muon_scratch_bytes(ctx, 7) if ctx else 1 << 20)
    a.update(change)
    return bl.muon_step(ctx, a["theta"], a["shadow"], a["grad"], a["velocity"], a["lr"], a["lr_rest"], a["momentum"], a["decay"], a["flags"], a["scratch"],
                        a["nbytes"], 0)


def batch(_, **change):
    a = dict(theta=4096, shadow=4096, grad=4096, velocity=4096, count=2, rows=5, cols=7, mode=1, lr=0.02, momentum=0.9, decay=0.1, flags=1, scratch=4096,
             nbytes=bl.muon_orthogonalize_scratch_bytes(2, 5, 7, 1))
    a.update(change)
    return bl.muon_matrices_step(a["theta"], a["shadow"], a["grad"], a["velocity"], a["count"], a["rows"], a["cols"], a["mode"], a["lr"], a["momentum"],
                                 a["decay"], a["flags"], a["scratch"], a["nbytes"], 0)


@pytest.mark.parametrize("change,code", [
    (dict(theta=None), -1), (dict(grad=None), -1), (dict(scratch=None), -1), (dict(velocity=None), -1),
    (dict(momentum=1.0), -2), (dict(momentum=-0.1), -2), (dict(momentum=float("nan")), -2), (dict(decay=-1e-3), -2), (dict(decay=float("nan")), -2),
    (dict(flags=8), -2), (dict(theta=4100), -4), (dict(shadow=4098), -4), (dict(grad=4104), -4), (dict(velocity=4100), -4), (dict(scratch=4104), -4),
    (dict(nbytes=100), -3)])
@pytest.mark.parametrize("call", [model, batch])
def test_calls_refuse(ctx, call, change, code):
    with pytest.raises(bl.BlstmError) as e:
        call(ctx, **change)
    assert e.value.code == code


def test_models_and_matrices_are_refused(ctx):
    with pytest.raises(bl.BlstmError) as e:
        model(None)
    assert e.value.code == -1
    for change in (dict(count=0), dict(rows=0), dict(cols=-1), dict(mode=2), dict(count=1 << 20, rows=1 << 12, cols=1 << 12), dict(flags=2)):
        with pytest.raises(bl.BlstmError) as e:
            batch(None, **change)
        assert e.value.code == -2
    for sizes in ((0, 1, 1, 0), (1, 1, 0, 0), (1, 1, 1, 3), (1, 1 << 24, 1, 1), (1 << 30, 1 << 6, 1 << 6, 1)):
        with pytest.raises(bl.BlstmError):
            bl.muon_orthogonalize_scratch_bytes(*sizes)
    # a workgroup of 1024 threads a matrix, and fewer than 2^32 threads a launch
    assert bl.muon_orthogonalize_scratch_bytes((1 << 22) - 1, 1, 1, 1) > 0
    with pytest.raises(bl.BlstmError):
        bl.muon_orthogonalize_scratch_bytes(1 << 22, 1, 1, 1)
    with pytest.raises(bl.BlstmError):
        bl.muon_scratch_bytes(ctx, 8)
    ok = bl.muon_orthogonalize_scratch_bytes(1, 3, 4, 0)
    for G, X, scratch, n, code in ((None, 16, 16, ok, -1), (16, None, 16, ok, -1), (16, 16, None, ok, -1), (20, 16, 16, ok, -4), (16, 20, 16, ok, -4),
                                   (16, 16, 24, ok, -4), (16, 16, 16, ok - 1, -3)):
        with pytest.raises(bl.BlstmError) as e:
            bl.muon_orthogonalize(G, X, 1, 3, 4, 0, scratch, n, 0)
        assert e.value.code == code


# ---- launches ----------------------------------------------------------------------------------------------------------

def test_a_failed_launch_is_reported(recorder):  # noqa: F811
    got = recorder("""
        out = []
        c = bl.blstm_create(2, 2, 5, 4, 2, 3, 7, 1)
        n = bl.muon_scratch_bytes(c, 0)
        step = lambda: bl.muon_step(c, P, P, P, P, 0.02, 0.1, 0.9, 0.1, 0, P, n, 0)
        for part in (b"", b"muon"):
            rec.recorder_fail(part)
            try:
                step()
                out.append(0)
            except bl.BlstmError as e:
                out.append(e.code)
    """)
    assert got == [0, -5]


def test_no_launch_is_larger_than_its_work(recorder):  # noqa: F811
    got = recorder("""
        out = []
        for dims in ((260, 512, 4, 256, 32000, 1), (260, 301, 2, 67, 3001, 1), (40, 32, 1, 0, 100, 0), (1, 1, 1, 0, 1, 1)):
            c = bl.blstm_create(1, 1, *dims[:4], dims[4], dims[5])
            for flags in (0, 7):
                names = launches(lambda: bl.muon_step(c, P, P, P, P, 0.02, 0.1, 0.9, 0.1, flags, P, bl.muon_scratch_bytes(c, flags), 0))
                out.append([len(names), min(rec.recorder_grid(i, 0) for i in range(rec.recorder_count()))])
    """)
    assert all(count <= 24 and least >= 1 for count, least in got)
