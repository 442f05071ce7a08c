"""Adapters: infinite inputs and factors are what the definition makes of them on every path."""
import numpy as np
import pytest
import torch

from oracle import adapters
from tests.test_gpu_adapters import run_backward, run_forward, tensors, wide

pytestmark = pytest.mark.gpu
# few rows, tiles of 64 rows and of 128 (T B, K and N as in the cases of test_gpu_adapters), ranks of one and several steps
SHAPES = [(1, 4, 32, 16, 3, 2), (21, 60, 602, 467, 5, 7), (21, 80, 640, 328, 32, 3), (70, 30, 96, 300, 64, 2), (130, 130, 40, 72, 20, 3), (20, 90, 129, 327, 128, 3)]


def same_kind(got, want, what):
    got = got.double().cpu().numpy()
    for of in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(of(got), of(want)), (what, of.__name__)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("where", ["x", "A", "Bm"])
def test_infinities(where, shape, mode):
    # all weights positive (or of one sign), so that the definition has infinities and no NaN among them
    T, B, K, N, rank, count = shape
    ids = np.arange(B) % (count + 1) - 1
    s = tensors(11, *shape, mode, ids)
    for k in ("W", "b", "A", "Bm", "x", "dy"):
        s[k] = s[k].abs() + 0.01
    s["Bm"][:, 1::2] *= -1                       # y falls to minus infinity in every other column
    s["W"][1::2] *= -1
    if where == "x":
        s["x"][T // 2, 1:3, K - 1] = float("inf")
    elif where == "A":
        s["A"][count - 1, rank - 1, K // 2] = float("inf")
    else:
        s["Bm"][count - 1, :3, rank - 1] *= float("inf")
    w = wide(s)
    y, t = run_forward(s, (*shape, mode))
    want_y, want_t = adapters.forward(w["W"], w["b"], w["A"], w["Bm"], w["ids"], w["x"], 1.5)
    assert np.isinf(want_y).any() and not np.isnan(want_y).any()
    same_kind(t, want_t, "t")
    same_kind(y, want_y, "y")


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("where", ["t", "Bm", "x", "dy"])
def test_infinities_in_the_gradients(where, shape, mode):
    T, B, K, N, rank, count = shape
    ids = np.arange(B) % (count + 1) - 1         # (sequence 1 has adapter 0)
    s = tensors(12, *shape, mode, ids)
    for k in ("W", "A", "Bm", "x", "dy"):
        s[k] = s[k].abs() + 0.01
    t = torch.rand((T, B, rank), device="cuda:0") + 0.1
    t[:, s["ids"] < 0] = 0
    if where == "t":
        t[T // 2, 1, rank - 1] = float("inf")
    elif where == "Bm":
        s["Bm"][count - 1, N - 1, 0] = float("inf")
    else:
        s[where][T // 2, 1, 0] = float("inf")
    w = wide(s)
    got = run_backward(s, (*shape, mode), t, 1.5)
    with np.errstate(invalid="ignore"):      # (numpy looks at padding lanes too)
        want = dict(zip(("dx", "dA", "dB", "dW", "db"), adapters.backward(w["W"], w["A"], w["Bm"], w["ids"], w["x"], t.double().cpu().numpy(), w["dy"], 1.5)))
    touched = dict(t=["dB"], Bm=["dx", "dA"], x=["dA", "dW"], dy=["dx", "dA", "dB", "dW", "db"])[where]
    assert all(np.isinf(want[k]).any() == (k in touched) and not np.isnan(want[k]).any() for k in want)
    for k in want:
        same_kind(got[k], want[k], k)


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_neighbours_of_an_infinity_keep_their_bits(shape, mode):
    # sequences of the same adapter, in the same tiles, and the same adapter's other columns
    T, B, K, N, rank, count = shape
    s = tensors(13, *shape, mode, np.zeros(B))
    y, t = run_forward(s, (*shape, mode))
    clean = run_backward(s, (*shape, mode), t, 1.5)
    others = [b for b in range(B) if b != 1]
    before = {k: s[k].clone() for k in ("x", "dy")}
    s["x"][T // 2, 1, K // 2] = float("inf")
    y2, t2 = run_forward(s, (*shape, mode))
    assert torch.equal(y[:, others], y2[:, others]) and torch.equal(t[:, others], t2[:, others]) and not torch.isfinite(y2[T // 2, 1]).any()
    frames = [i for i in range(T) if i != T // 2]
    assert torch.equal(y[frames, 1], y2[frames, 1])
    got = run_backward(s, (*shape, mode), t, 1.5)                # x's infinity is in one column of dA and of dW
    columns = [k for k in range(K) if k != K // 2]
    assert torch.equal(got["dx"], clean["dx"]) and torch.equal(got["dB"], clean["dB"])
    assert torch.equal(got["dA"][0][:, columns], clean["dA"][0][:, columns]) and not torch.isfinite(got["dA"][0][:, K // 2]).any()
    s["x"].copy_(before["x"])
    infinite = t.clone()
    infinite[T // 2, 1, rank - 1] = float("inf")                 # t's in one column of dB
    got = run_backward(s, (*shape, mode), infinite, 1.5)
    columns = list(range(rank - 1))
    assert torch.equal(got["dA"], clean["dA"]) and torch.equal(got["dx"], clean["dx"])
    assert torch.equal(got["dB"][0][:, columns], clean["dB"][0][:, columns]) and not torch.isfinite(got["dB"][0][:, rank - 1]).any()
