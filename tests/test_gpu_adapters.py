"""Low-rank adapters on the GPU against the float64 oracle, element by element.

Bounds: a sum of n products in float is off by at most (n + 1) 2^-24 of the sum of their sizes, which the oracle gives on absolute values.  Mode 1: t (and q)
enter the product for y (dx) as two bf16 numbers, 2^-16 of them, and y and dx leave rounded, 2^-8 of the value; for dA and dB they are three, 2^-24."""
import numpy as np
import pytest

from oracle import adapters

pytestmark = pytest.mark.gpu
F, TWO, BF16 = 2.0 ** -24, 2.0 ** -16, 2.0 ** -8
DEV = "cuda:0"


def tensors(seed, T, B, K, N, rank, count, mode, ids=None):
    import torch
    kind = torch.bfloat16 if mode else torch.float32
    r = np.random.default_rng(seed)
    real = dict(W=r.uniform(-0.1, 0.1, (N, K)), b=r.uniform(-0.1, 0.1, N), A=r.normal(size=(count, rank, K)) / np.sqrt(K), Bm=0.1 * r.normal(size=(count, N, rank)),
                x=np.tanh(r.normal(size=(T, B, K))), dy=1e-3 * r.normal(size=(T, B, N)))
    out = {k: torch.from_numpy(v.astype(np.float32)).to(kind).to(DEV) for k, v in real.items()}
    if ids is None:
        ids = r.integers(-1, count, B)
    out["ids"] = torch.from_numpy(np.asarray(ids, dtype=np.int32)).to(DEV)
    return out


def wide(s):
    return {k: v.double().cpu().numpy() if v.is_floating_point() else v.cpu().numpy() for k, v in s.items()}


def guarded(n):
    import torch
    t = torch.full((n + 4096,), 0x7F, dtype=torch.uint8, device=DEV)
    return t, lambda: bool((t[n:] == 0x7F).all())


def run_forward(s, shape, scale=1.5, bias=True, t=True, stream=None, scratch=None):
    import torch
    from paper_1904_04956_amd import binding as bl
    T, B, K, N, rank, count, mode = shape
    cfg = bl.adapter_config(*shape, scale)
    n = bl.adapter_scratch_bytes(cfg, bl.ADAPTER_FORWARD)
    own, kept = (scratch, lambda: True) if scratch is not None else guarded(n)
    y = torch.full((T, B, N), 7.0, dtype=s["x"].dtype, device=DEV)
    low = torch.full((T, B, rank), 7.0, device=DEV) if t else None
    bl.adapter_forward(cfg, s["W"], s["b"] if bias else None, s["A"], s["Bm"], s["ids"], s["x"], y, low, own, n, stream)
    assert kept()
    return y, low


def run_backward(s, shape, t, scale=1.5, dx=True, shared=True):
    import torch
    from paper_1904_04956_amd import binding as bl
    T, B, K, N, rank, count, mode = shape
    cfg = bl.adapter_config(*shape, scale)
    n = bl.adapter_scratch_bytes(cfg, bl.ADAPTER_BACKWARD)
    scratch, kept = guarded(n)
    real = lambda *d: torch.full(d, 7.0, device=DEV)  # noqa: E731
    out = dict(dx=torch.full((T, B, K), 7.0, dtype=s["x"].dtype, device=DEV) if dx else None, dA=real(count, rank, K), dB=real(count, N, rank),
               dW=real(N, K) if shared else None, db=real(N) if shared else None)
    bl.adapter_backward(cfg, s["W"], s["A"], s["Bm"], s["ids"], s["x"], t, s["dy"], *out.values(), scratch, n)
    assert kept()
    return out


def inside(got, want, bound, what):
    got = got.double().cpu().numpy()
    same = np.isnan(want)
    assert np.array_equal(np.isnan(got), same), what
    off = np.abs(np.where(same, 0, got - want)) - np.where(same, 0, bound)
    assert off.max() <= 0, (what, off.max(), np.unravel_index(off.argmax(), off.shape))


def check(seed, shape, scale=1.5, ids=None, bias=True, dx=True, shared=True):
    T, B, K, N, rank, count, mode = shape
    s = tensors(seed, *shape, ids)
    w = wide(s)
    a = {k: np.abs(v) if k != "ids" else v for k, v in w.items()}
    y, t = run_forward(s, shape, scale, bias)
    want_y, want_t = adapters.forward(w["W"], w["b"] if bias else None, w["A"], w["Bm"], w["ids"], w["x"], scale)
    size_y, size_t = adapters.forward(a["W"], a["b"] if bias else None, a["A"], a["Bm"], a["ids"], a["x"], abs(scale))
    low = abs(scale) * adapters.forward(0 * a["W"], None, a["A"], a["Bm"], a["ids"], a["x"], 1.0)[0]
    inside(t, want_t, (K + 1) * F * size_t, "t")
    inside(y, want_y, (K + rank + 6) * F * size_y + (TWO * low + BF16 * np.abs(want_y) * 1.01 if mode else 0), "y")
    # the backward pass is given its own t, held in float
    got = run_backward(s, shape, t, scale, dx, shared)
    given = t.double().cpu().numpy()
    want = dict(zip(("dx", "dA", "dB", "dW", "db"), adapters.backward(w["W"], w["A"], w["Bm"], w["ids"], w["x"], np.nan_to_num(given), w["dy"], scale)))
    size = dict(zip(("dx", "dA", "dB", "dW", "db"), adapters.backward(a["W"], a["A"], a["Bm"], a["ids"], a["x"], np.abs(np.nan_to_num(given)), a["dy"], abs(scale))))
    M = T * B
    if dx:
        low = adapters.backward(0 * a["W"], a["A"], a["Bm"], a["ids"], a["x"], size_t, a["dy"], abs(scale))[0]
        inside(got["dx"], want["dx"], (N + rank + 6) * F * size["dx"] + (TWO * low + BF16 * np.abs(want["dx"]) * 1.01 if mode else 0), "dx")
    inside(got["dA"], want["dA"], (N + M + 6) * F * size["dA"], "dA")
    inside(got["dB"], want["dB"], (M + 6) * F * size["dB"], "dB")
    if shared:
        inside(got["dW"], want["dW"], (M + 2) * F * size["dW"], "dW")
        inside(got["db"], want["db"], (M + 2) * F * size["db"], "db")
    # the same inputs give the same bits
    y2, t2 = run_forward(s, shape, scale, bias)
    again = run_backward(s, shape, t, scale, dx, shared)
    for p, q in [(y, y2), (t, t2)] + [(got[k], again[k]) for k in got if got[k] is not None]:
        assert np.array_equal(p.float().cpu().numpy(), q.float().cpu().numpy(), equal_nan=True)


SHAPES = [(1, 1, 1, 1, 1, 1), (1, 1, 1024, 256, 16, 4), (1, 64, 1024, 256, 16, 64), (1, 3, 40, 130, 3, 2), (5, 1, 64, 64, 8, 1), (21, 30, 602, 67, 5, 7), (21, 40, 640, 128, 32, 3),
          (4, 17, 72, 300, 33, 9), (2, 9, 129, 127, 128, 3), (70, 3, 96, 40, 64, 2), (300, 2, 50, 24, 17, 5), (1, 2500, 24, 16, 4, 2500), (3, 1100, 16, 8, 2, 700), (21, 256, 256, 128, 16, 100),
          # tiles of 64 rows, and of 128
          (21, 60, 602, 467, 5, 7), (21, 80, 640, 328, 32, 3), (40, 40, 72, 500, 33, 9), (40, 40, 500, 72, 33, 9), (70, 30, 96, 300, 64, 2), (70, 30, 300, 96, 64, 2),
          (20, 90, 129, 327, 128, 3), (20, 90, 327, 129, 128, 3), (300, 8, 50, 424, 17, 5), (130, 130, 40, 72, 20, 3), (130, 130, 37, 43, 5, 2)]


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_passes(shape, mode):
    check(sum(shape), (*shape, mode))


@pytest.mark.parametrize("mode", [0, 1])
def test_who_has_which_adapter(mode):
    shape = (7, 12, 48, 40, 6, 5, mode)
    for k, ids in enumerate(([-1] * 12, [4] * 12, [0, 1, 2, 3, 4, -1] * 2, [3, 3, 3, -1, -1, 0, 0, 0, 0, 3, 3, 4], [5, -2, 2 ** 31 - 1, -2 ** 31, 0, 1, -1, 2, 5, 0, 4, 3])):
        check(100 + k, shape, ids=ids)


@pytest.mark.parametrize("mode", [0, 1])
def test_what_is_left_out(mode):
    shape = (5, 6, 64, 32, 8, 3, mode)
    check(1, shape, bias=False)
    check(2, shape, dx=False)
    check(3, shape, shared=False)
    check(4, shape, scale=0.0)
    check(5, shape, scale=-2.25)
    s = tensors(6, *shape)
    assert np.array_equal(run_forward(s, shape, t=False)[0].float().cpu(), run_forward(s, shape)[0].float().cpu())


@pytest.mark.parametrize("mode", [0, 1])
def test_tensors_anywhere_in_a_flat_vector(mode):
    # an element behind a whole word: the same results
    import torch
    shape = (3, 10, 64, 24, 8, 4, mode)
    s = tensors(7, *shape)
    y, t = run_forward(s, shape)
    moved = dict(s)
    for k in ("W", "b", "A", "Bm", "x", "dy"):
        flat = torch.empty(s[k].numel() + 1, dtype=s[k].dtype, device=DEV)
        moved[k] = flat[1:].view(s[k].shape)
        moved[k].copy_(s[k])
    y2, t2 = run_forward(moved, shape)
    assert torch.equal(y, y2) and torch.equal(t, t2)
    a, b = run_backward(s, shape, t), run_backward(moved, shape, t)
    for k in ("dx", "dA", "dB"):
        assert torch.equal(a[k], b[k]), k
    assert float((a["dW"] - b["dW"]).abs().max()) <= 2 * 32 * F * 30 * 5e-3


def test_what_one_sequence_or_adapter_holds_stays_with_it():
    import torch
    shape = (4, 6, 32, 16, 4, 3, 1)
    s = tensors(8, *shape, ids=[0, 1, 2, 0, -1, 1])
    y, t = run_forward(s, shape)
    g = run_backward(s, shape, t, shared=False)
    s["x"][:, 2], s["A"][2, 1, 3], s["Bm"][2, 0] = float("inf"), float("nan"), float("inf")
    y2, t2 = run_forward(s, shape)
    g2 = run_backward(s, shape, t2, shared=False)
    others = [0, 1, 3, 4, 5]
    for p, q in ((y[:, others], y2[:, others]), (t[:, others], t2[:, others]), (g["dx"][:, others], g2["dx"][:, others]), (g["dA"][:2], g2["dA"][:2]), (g["dB"][:2], g2["dB"][:2])):
        assert torch.equal(p, q)
    assert torch.isnan(y2[:, 2].float()).any()


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("mode", [0, 1])
def test_an_infinite_input_without_adapter(T, mode):
    # y is what the shared projection alone makes of it, t is zero
    import torch
    shape = (T, 4, 32, 16, 3, 2, mode)
    s = tensors(10, *shape, ids=[0, -1, 1, -1])
    s["x"][:, 1, 5] = float("inf")
    y, t = run_forward(s, shape)
    assert torch.equal(t[:, 1], torch.zeros_like(t[:, 1])) and torch.equal(t[:, 3], torch.zeros_like(t[:, 3]))
    assert torch.equal(y[:, 1].float(), (s["W"][:, 5].float() * float("inf")).expand(T, 16))


def test_replays_and_streams():
    import torch
    shape = (21, 40, 64, 48, 8, 6, 1)
    s = tensors(9, *shape)
    y, t = run_forward(s, shape)
    held = {k: v.clone() for k, v in s.items()}
    from paper_1904_04956_amd import binding as bl
    cfg = bl.adapter_config(*shape, 1.5)
    n = [bl.adapter_scratch_bytes(cfg, k) for k in (0, 1)]
    real = lambda *d: torch.zeros(d, device=DEV)  # noqa: E731
    out = dict(y=torch.zeros_like(y), t=torch.zeros_like(t), dx=torch.zeros_like(s["x"]), dA=real(6, 8, 64), dB=real(6, 48, 8), dW=real(48, 64), db=real(48))
    scratch = [torch.empty(k, dtype=torch.uint8, device=DEV) for k in n]

    def both(stream=None):
        bl.adapter_forward(cfg, held["W"], held["b"], held["A"], held["Bm"], held["ids"], held["x"], out["y"], out["t"], scratch[0], None, stream)
        bl.adapter_backward(cfg, held["W"], held["A"], held["Bm"], held["ids"], held["x"], out["t"], held["dy"], out["dx"], out["dA"], out["dB"], out["dW"], out["db"], scratch[1], None, stream)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        both()
    for k in range(3):
        # other members in every replay: the plan is made on the device
        ids = np.random.default_rng(k).integers(-1, 6, 40)
        held["ids"].copy_(torch.from_numpy(ids.astype(np.int32)))
        s["ids"] = held["ids"].clone()
        for v in scratch:
            v.fill_(255)
        graph.replay()
        y, t = run_forward(s, shape)
        want = dict(run_backward(s, shape, t), y=y, t=t)
        torch.cuda.synchronize()
        assert all(torch.equal(out[name], want[name]) for name in out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ys = []
    for _ in range(5):
        for st in streams:
            with torch.cuda.stream(st):
                ys.append(run_forward(s, shape, stream=st)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(v, y) for v in ys)
