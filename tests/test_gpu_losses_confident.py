"""The softmax layer's losses where the model is good: frames whose label has nearly all of the probability, a student that is close to its
teacher.  dE/du is then a small difference of large probabilities, and the tolerances are relative to dE/du itself.

Weights and activations are whole multiples of powers of two whose products and sums are exact in float, so that logits have no error
in any order of their sums.  What is left, with U = 2^-24 and x the distance of a logit from its row's largest (over the temperature):
- a probability is right to (V + 2 x + 64) U of itself: its sum of V terms, its exponent's rounding, some exponentials and products; a
  teacher's to (K + 2 x + 64) U.  Both enter dE/du as differences ("parts": the sum of the absolute values).
- dE/du then enters the product for dz as one bf16 number (2^-8 of itself) and those for W_s and b_s as two (2^-16); in float it is one.
- sums of n products: n U of the sum of their absolute values; the result's own rounding (bf16 2^-8).
"""
import numpy as np
import pytest

from oracle import softmax_losses as sl
from tests.test_gpu_losses import Layer, U, layer_id

pytestmark = pytest.mark.gpu


def exact_layer(T, B, V, Z, mode, seed, **more):
    """Logits of standard deviation 6 or so, exact in float.  Every class of the upper half has a rival in the lower half, with the same weights and a bias that is
    less by 3 to 10: of a frame that is sure of its class, the rival is often the next best, and far in front of it.  Frames lean towards a class each by up to 36."""
    layer = Layer(T, B, V, Z, mode, seed, **more)
    t, rng = layer.torch, layer.rng
    f = 2.0 ** round(np.log2(6 / (0.15 * np.sqrt(Z))))
    W = np.clip(np.round(rng.normal(size=(V, Z)) * 2.4), -15, 15) / 16 * f
    b = np.clip(np.round(rng.normal(size=V) * 2.4), -15, 15) / 16
    half = V // 2
    W[:half] = W[half:2 * half]
    b[:half] = b[half:2 * half] - rng.integers(12, 41, half) / 4
    heard = W[rng.integers(half, 2 * half, layer.M)]
    z = rng.normal(size=(layer.M, Z)) + rng.uniform(0, 36, (layer.M, 1)) * heard / (heard ** 2).sum(axis=1, keepdims=True)
    z = np.clip(np.round(z * 4), -15, 15) / 4
    layer.theta[layer.at_w:layer.at_w + V * Z] = t.from_numpy(W.reshape(-1)).to(layer.kind)
    layer.theta[layer.at_b:layer.at_b + V] = t.from_numpy(b).to(layer.kind)
    layer.z = t.from_numpy(z).to(layer.kind)
    assert np.array_equal(layer.W, W) and np.array_equal(layer.z.double().numpy(), z) and np.array_equal(layer.b, b)
    return layer


def best_labels(layer, u):
    """The largest class of most frames, any class of some, none of others."""
    lab = u.argmax(axis=1).astype(np.int32)
    some = layer.rng.random(layer.M) < 0.1
    lab[some] = layer.rng.integers(0, layer.V, some.sum())
    lab[layer.rng.random(layer.M) < 0.1] = sl.NO_LABEL
    return lab


def check(layer, got, ref, du, parts, live):
    """parts: sum of the absolute values of what dE/du is the difference of, each times its own error in U."""
    dz, dW, db = ref
    z = np.where(live[:, None], layer.z.double().numpy(), 0.0)
    one, two, own = (2.0 ** -8, 2.0 ** -16, 2.0 ** -8) if layer.mode == 1 else (U, U, U)
    rows = (3 if layer.mode == 1 else 1) * layer.M
    a, e, tiny = np.abs(du), parts * U, 1e-37
    worst = {}
    bound = (one * a + e) @ np.abs(layer.W) + ((a + e) @ np.abs(layer.W)) * layer.V * U
    bound += own * (np.abs(dz) + bound) + tiny
    worst["dz"] = np.max(np.abs(got["dz"] - dz) / bound)
    bound = (two * a + e).T @ np.abs(z) + ((a + e).T @ np.abs(z)) * rows * U + U * np.abs(dW) + tiny
    worst["dW"] = np.max(np.abs(got["dW"] - dW) / bound)
    bound = (two * a + e).sum(axis=0) + (a + e).sum(axis=0) * rows * U + U * np.abs(db) + tiny
    worst["db"] = np.max(np.abs(got["db"] - db) / bound)
    assert all(v <= 1 for v in worst.values()), worst


SHAPES = [(3, 43, 600, 64), (2, 129, 1501, 256), (5, 26, 333, 250), (2, 70, 600, 264), (2, 70, 900, 640)]


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("shape", SHAPES, ids=layer_id)
def test_policy_loss_of_sure_frames(shape, mode):
    layer = exact_layer(*shape, mode, 41, loss_scale=0.125)
    try:
        z = layer.z.double().numpy()
        u = z @ layer.W.T + layer.b
        lab = best_labels(layer, u)
        live = lab != sl.NO_LABEL
        A = layer.rng.normal(size=layer.M).astype(np.float32)
        lp = sl.logprob(layer.W, layer.b, z, lab)
        p = np.exp(lp[live])
        assert all(((p > lo) & (p < hi)).sum() >= 3 for lo, hi in ((0.9, 0.99), (0.99, 0.999), (0.999, 0.99999)))
        want = sl.policy(layer.W, layer.b, z, lab, A, None, None, float(layer.s), 0.2, 0.2, 0.0)
        got = layer.policy(lab, A, None, None, 0.2, 0.2, 0.0)
        hot = np.zeros_like(u)
        hot[np.flatnonzero(live), lab[live]] = 1.0
        g = (-float(layer.s) * A.astype(np.float64) * live)[:, None]
        prob = np.exp(sl._log_softmax(u))
        du = g * (hot - prob)
        units = layer.V + 64 + 2 * (u.max(axis=1, keepdims=True) - u)
        # (z of up to 256, bf16: the label's class stays out of the sum, 1 - p is right to its own rounding)
        parts = units * (np.abs(du) if mode == 1 and layer.Z <= 256 else np.abs(g) * (hot + prob))
        check(layer, got, want[2:], du, parts, live)
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("shape", SHAPES, ids=layer_id)
@pytest.mark.parametrize("tau,hard", [(1.0, 0.5), (2.0, 0.5), (2.0, 0.0), (1.0, 0.0), (3.0, 0.25)])
def test_a_student_close_to_its_teacher(shape, tau, hard, mode):
    layer = exact_layer(*shape, mode, 42, loss_scale=0.125)
    try:
        K, soft, s = 16, 0.75, float(layer.s)
        z = layer.z.double().numpy()
        u = z @ layer.W.T + layer.b
        lab = best_labels(layer, u)
        given = lab if hard else np.full_like(lab, sl.NO_LABEL)
        top = np.argsort(-u, axis=1, kind="stable")[:, :K]
        classes = np.take_along_axis(top, layer.rng.permuted(np.tile(np.arange(K), (layer.M, 1)), axis=1), axis=1).astype(np.int32)
        values = (np.take_along_axis(u, classes.astype(np.int64), axis=1) + 0.02 * layer.rng.normal(size=(layer.M, K))).astype(np.float32)
        classes[layer.rng.random(layer.M) < 0.1] = sl.NO_LABEL
        q, some = sl.teacher_distribution(values, classes, layer.V, tau)
        live = (given != sl.NO_LABEL) | some
        want = sl.distill(layer.W, layer.b, z, given, values, classes, s, tau, hard, soft)
        got = layer.distill(lab if hard else None, values, classes, tau, hard, soft)
        labelled = given != sl.NO_LABEL
        hot = np.zeros_like(u)
        hot[np.flatnonzero(labelled), given[labelled]] = 1.0
        ph, pt = np.exp(sl._log_softmax(u)) * labelled[:, None], np.exp(sl._log_softmax(u / tau)) * some[:, None]
        du = s * (hard * (ph - hot) + soft * tau * (pt - q))
        x = u.max(axis=1, keepdims=True) - u
        parts = s * ((layer.V + 64 + 2 * x) * (hard * (ph + hot) + soft * tau * pt) + (K + 64 + 2 * x / tau) * soft * tau * q)
        check(layer, got, want[1:], du, parts, live)
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 264])
@pytest.mark.parametrize("tau,hard", [(0.01, 0.0), (2.0 ** -13, 0.0), (0.01, 0.5)])
def test_small_temperatures_and_logits_far_below_zero(tau, hard, Z, mode):
    # 2000 below zero and, over a temperature of 0.01 or 2^-13, 2e5 or 2e7: the temperature does not move where a class counts as ruled out
    layer = exact_layer(2, 35, 300, Z, mode, 43, loss_scale=0.125)
    try:
        K, soft, s = 16, 0.75, float(layer.s)
        low = 2048.0
        layer.theta[layer.at_b:layer.at_b + layer.V] = -low
        z = layer.z.double().numpy()
        u = z @ layer.W.T + layer.b
        lab = best_labels(layer, u)
        given = lab if hard else np.full_like(lab, sl.NO_LABEL)
        classes = np.argsort(-u, axis=1, kind="stable")[:, :K].astype(np.int32)
        # (the teacher's are not far below zero, and a few of them count)
        values = (tau * layer.rng.normal(size=(layer.M, K))).astype(np.float32)
        classes[layer.rng.random(layer.M) < 0.1] = sl.NO_LABEL
        q, some = sl.teacher_distribution(values, classes, layer.V, tau)
        live = (given != sl.NO_LABEL) | some
        want = sl.distill(layer.W, layer.b, z, given, values, classes, s, tau, hard, soft)
        got = layer.distill(lab if hard else None, values, classes, tau, hard, soft)
        labelled = given != sl.NO_LABEL
        hot = np.zeros_like(u)
        hot[np.flatnonzero(labelled), given[labelled]] = 1.0
        ph, pt = np.exp(sl._log_softmax(u)) * labelled[:, None], np.exp(sl._log_softmax(u / tau)) * some[:, None]
        du = s * (hard * (ph - hot) + soft * tau * (pt - q))
        x = u.max(axis=1, keepdims=True) - u
        parts = s * ((layer.V + 64 + 2 * x) * hard * (ph + hot) + (layer.V + 64 + 2 * x / tau) * soft * tau * pt + (K + 64) * soft * tau * q)
        check(layer, got, want[1:], du, parts, live)
        assert np.isfinite(got["loss"])
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 250, 256, 264, 640])
@pytest.mark.parametrize("kind", ["policy", "tau 1", "tau 2", "teacher 1", "teacher 2"])
def test_the_classes_of_a_frame_see_the_logits_that_its_sum_has_seen(kind, Z, mode):
    # dE/du of a frame adds up to nothing, as its probabilities and the teacher's add up to one.  Every logit is 32768 and some, whose roundings (2^-9, and others in another order of
    # the product's sum) are thousands of times what the sums of V terms may leave: so whatever makes the probabilities has to have the logits of the sum, bit by bit.
    # One frame: db_s is its dE/du, in float.
    layer = Layer(1, 1, 600, Z, mode, 44, scale=4 / np.sqrt(Z), loss_scale=1.0)
    try:
        W = layer.theta[layer.at_w:layer.at_w + 600 * Z].view(600, Z)
        W[:, 5], layer.z[0, 5] = 256.0, 128.0
        u = layer.z.double().numpy() @ layer.W.T + layer.b
        lab = u.argmax(axis=1).astype(np.int32)
        if kind == "policy":
            du = layer.policy(lab, np.ones(1, dtype=np.float32), None, None, 0.2, 0.2, 0.0)["db"]
        else:
            classes = np.argsort(-u, axis=1, kind="stable")[:, :16].astype(np.int32)
            values = np.take_along_axis(u, classes.astype(np.int64), axis=1).astype(np.float32)
            tau, hard = float(kind[-1]), 0.0 if kind.startswith("teacher") else 0.5
            du = layer.distill(lab if hard else None, values, classes, tau, hard, 0.5)["db"]
        assert np.abs(du).sum() > 0.1
        # (a probability is right to V + 64 roundings of itself at most; the parts of dE/du are up to 1 and 2 in sum)
        assert abs(du.sum()) <= 4 * (600 + 64) * U, du.sum()
    finally:
        layer.close()
