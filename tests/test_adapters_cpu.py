"""Low-rank adapters without a GPU: the float64 oracle against finite differences, the calls' refusals, their scratch, what they launch."""
import numpy as np
import pytest

from oracle import adapters
from paper_1904_04956_amd import binding as bl
from tests.test_dispatch_cpu import recorder  # noqa: F401


def draw(seed, T=3, B=5, K=4, N=3, r=2, count=3):
    g = np.random.default_rng(seed)
    W, b, A, Bm, x = g.normal(size=(N, K)), g.normal(size=N), g.normal(size=(count, r, K)), g.normal(size=(count, N, r)), g.normal(size=(T, B, K))
    return W, b, A, Bm, np.array([1, -1, 2, 1, 0][:B]), x, g.normal(size=(T, B, N))


def test_gradients_are_the_differences():
    W, b, A, Bm, ids, x, dy = draw(1)
    f = lambda W, b, A, Bm, x: (adapters.forward(W, b, A, Bm, ids, x, 0.7)[0] * dy).sum()  # noqa: E731
    dx, dA, dB, dW, db = adapters.backward(W, A, Bm, ids, x, adapters.forward(W, b, A, Bm, ids, x, 0.7)[1], dy, 0.7)
    args = [W, b, A, Bm, x]
    for k, got in ((0, dW), (1, db), (2, dA), (3, dB), (4, dx)):
        for i in np.ndindex(args[k].shape):
            up, down = [v.copy() for v in args], [v.copy() for v in args]
            up[k][i] += 1e-5
            down[k][i] -= 1e-5
            assert abs((f(*up) - f(*down)) / 2e-5 - got[i]) < 1e-8


def test_a_batch_is_its_sequences_one_by_one():
    W, b, A, Bm, ids, x, _ = draw(2)
    y, t = adapters.forward(W, b, A, Bm, ids, x, 1.3)
    for s, a in enumerate(ids):
        full = W + (1.3 * Bm[a] @ A[a] if a >= 0 else 0)
        assert np.abs(y[:, s] - (x[:, s] @ full.T + b)).max() < 1e-12
    assert np.all(t[:, 1] == 0)
    assert np.isnan(adapters.forward(W, b, A, Bm, np.array([3, -2, 0, 0, 0]), x, 1.0)[0][:, :2]).all()


# ---- refusals --------------------------------------------------------------------------------------------------------

def config(**change):
    a = dict(T=3, B=5, K=16, N=8, rank=2, count=4, mode=1, scale=1.0)
    a.update(change)
    return bl.adapter_config(*a.values())


def forward(cfg=config(), **change):
    a = dict(W=4096, b=4096, A=4096, Bm=4096, ids=4096, x=4096, y=4096, t=4096, scratch=4096, nbytes=1 << 30)
    a.update(change)
    return bl.adapter_forward(cfg, *a.values(), 0)


def backward(cfg=config(), **change):
    a = dict(W=4096, A=4096, Bm=4096, ids=4096, x=4096, t=4096, dy=4096, dx=4096, dA=4096, dB=4096, dW=4096, db=4096, scratch=4096, nbytes=1 << 30)
    a.update(change)
    return bl.adapter_backward(cfg, *a.values(), 0)


@pytest.mark.parametrize("call,change,code", [
    *[(forward, {k: None}, -1) for k in ("W", "A", "Bm", "ids", "x", "y", "scratch")],
    *[(backward, {k: None}, -1) for k in ("W", "A", "Bm", "ids", "x", "t", "dy", "dA", "dB", "scratch", "dW")],
    *[(forward, {k: 4097}, -4) for k in ("W", "b", "A", "Bm", "x", "y")], *[(forward, {k: 4098}, -4) for k in ("ids", "t")],
    *[(backward, {k: 4097}, -4) for k in ("W", "A", "Bm", "x", "dy", "dx")], *[(backward, {k: 4098}, -4) for k in ("ids", "t", "dA", "dB", "dW", "db")],
    (forward, dict(scratch=4104), -4), (backward, dict(scratch=4104), -4), (forward, dict(nbytes=8), -3), (backward, dict(nbytes=8), -3)])
def test_calls_refuse(call, change, code):
    with pytest.raises(bl.BlstmError) as e:
        call(**change)
    assert e.value.code == code


def test_float_tensors_are_aligned_to_their_elements():
    with pytest.raises(bl.BlstmError) as e:
        forward(config(mode=0), W=4098)
    assert e.value.code == -4


@pytest.mark.parametrize("change", [dict(T=0), dict(B=0), dict(K=0), dict(N=-1), dict(rank=0), dict(rank=129), dict(count=0), dict(count=4097), dict(mode=2),
                                    dict(T=1 << 16, B=1 << 15), dict(T=1 << 15, B=1 << 15, K=1 << 14), dict(count=4096, K=1 << 30)])
def test_sizes_are_refused(change):
    for which in (bl.ADAPTER_FORWARD, bl.ADAPTER_BACKWARD):
        with pytest.raises(bl.BlstmError) as e:
            bl.adapter_scratch_bytes(config(**change), which)
        assert e.value.code == -2
    for call in (forward, backward):
        with pytest.raises(bl.BlstmError) as e:
            call(config(**change))
        assert e.value.code == -2


@pytest.mark.parametrize("which,change", [(bl.ADAPTER_FORWARD, dict(T=(1 << 30) + 1, B=1, K=1, N=1)), (bl.ADAPTER_FORWARD, dict(T=1, B=2048, count=2048, N=1 << 22)),
                                          (bl.ADAPTER_FORWARD, dict(T=1 << 20, B=256, N=16384)), (bl.ADAPTER_BACKWARD, dict(T=1 << 20, B=256, K=16384)),
                                          (bl.ADAPTER_BACKWARD, dict(count=4096, rank=128, N=32768)), (bl.ADAPTER_BACKWARD, dict(K=1 << 18, N=1 << 18))])
def test_launches_beyond_a_grid_are_refused(which, change):
    with pytest.raises(bl.BlstmError) as e:
        bl.adapter_scratch_bytes(config(**change), which)
    assert e.value.code == -2
    with pytest.raises(bl.BlstmError) as e:
        (forward if which == bl.ADAPTER_FORWARD else backward)(config(**change))
    assert e.value.code == -2


def test_no_config_and_no_such_call():
    for call in (lambda: bl.adapter_scratch_bytes(None, 0), lambda: bl.adapter_scratch_bytes(config(), 2), lambda: forward(None), lambda: backward(None)):
        with pytest.raises(bl.BlstmError):
            call()


# ---- launches ----------------------------------------------------------------------------------------------------------

def test_launches_and_failures(recorder):  # noqa: F811
    got = recorder("""
        out = []
        c = bl.adapter_config(21, 32, 64, 24, 8, 5, 1, 1.0)
        n = [bl.adapter_scratch_bytes(c, k) for k in (0, 1)]
        fwd = lambda: bl.adapter_forward(c, P, P, P, P, P, P, P, P, P, n[0], 0)
        bwd = lambda dW: bl.adapter_backward(c, P, P, P, P, P, P, P, P, P, P, dW, dW, P, n[1], 0)
        for call in (fwd, lambda: bwd(P), lambda: bwd(None)):
            out.append([x for x in launches(call) if "adapt" not in x])
        # batches of few sequences find their tiles, others have a plan made first
        many, large = bl.adapter_config(1, 300, 64, 24, 8, 5, 1, 1.0), bl.adapter_config(100, 32, 64, 240, 8, 5, 1, 1.0)
        out.append([len(launches(fwd)), len(launches(lambda: bl.adapter_forward(many, P, P, P, P, P, P, P, P, P, 1 << 30, 0)))])
        for part, call in ((b"adapt_plan", lambda: bl.adapter_forward(many, P, P, P, P, P, P, P, P, P, 1 << 30, 0)), (b"adapt_rows", fwd),
                           (b"adapt_tile", lambda: bl.adapter_forward(large, P, P, P, P, P, P, P, P, P, 1 << 30, 0)),
                           (b"adapt_transpose", lambda: bwd(P)), (b"adapt_grad", lambda: bwd(P))):
            rec.recorder_fail(part)
            try:
                call()
                out.append(0)
            except bl.BlstmError as e:
                out.append(e.code)
    """)
    assert got[0] == [] and got[2] == [] and len(got[1]) >= 1            # the shared projection's gradient is an ordinary product
    assert got[3] == [1, 2]
    assert got[4:] == [-5, -5, -5, -5, -5]
