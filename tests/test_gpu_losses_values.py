"""The softmax layer's losses at the ends of what their inputs may hold: terms that are switched off, probabilities of nothing, values that are
no numbers, logits far from zero."""
import numpy as np
import pytest

from oracle import softmax_losses as sl
from tests.test_gpu_losses import Layer, U
from tests.test_gpu_losses_confident import best_labels, exact_layer

pytestmark = pytest.mark.gpu
KEYS = ("loss", "dz", "dW", "db")


def same(x, y, keys=KEYS):
    return all(np.array_equal(x[k], y[k]) for k in keys)


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 264])
def test_a_kl_weight_of_zero_is_no_term(Z, mode):
    # whatever the reference's log-probabilities are: exp(ref - lp) may be infinite, and they may be no numbers
    layer = Layer(2, 20, 90, Z, mode, 51)
    try:
        lab = layer.labels("whole")
        lp = layer.logprob(lab).astype(np.float32)
        A = layer.rng.normal(size=layer.M).astype(np.float32)
        ref = lp.copy()
        ref[3], ref[7], ref[11], ref[12] = lp[3] + 200, np.inf, np.nan, -np.inf
        got, want = layer.policy(lab, A, lp, ref, 0.2, 0.2, 0.0), layer.policy(lab, A, lp, None, 0.2, 0.2, 0.0)
        assert np.isfinite(want["loss"]) and same(got, want, KEYS + ("logp",))
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 264])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("ruled_out", [-float("inf"), None])
def test_a_teachers_class_without_probability_is_as_if_it_were_not_there(tau, ruled_out, Z, mode):
    # a class that the teacher and the student rule out: 0 (log 0 - (-inf)) is nothing, and the lowest value over 0.5 is -inf
    layer = Layer(2, 20, 90, Z, mode, 52)
    try:
        lab = layer.labels("whole")
        lab = np.where(lab < 10, lab + 10, lab).astype(np.int32)
        layer.theta[layer.at_b:layer.at_b + 10] = layer.torch.finfo(layer.kind).min if ruled_out is None else ruled_out
        values, classes = layer.lists(6, "whole")
        classes = classes % 80 + 10                       # (a class may be there twice)
        classes[:, 2], classes[:, 5] = 3, 4
        values[:, 2], values[:, 5] = np.finfo(np.float32).min, -1e30
        less = classes.copy()
        less[:, [2, 5]] = sl.NO_LABEL
        for hard in (0.0, 0.5):
            got, want = layer.distill(lab, values, classes, tau, hard, 0.5), layer.distill(lab, values, less, tau, hard, 0.5)
            assert np.isfinite(want["loss"]) and same(got, want), (got["loss"], want["loss"])
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 264])
@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_a_teachers_value_that_is_no_number_is_not_used_and_its_frames_loss_is_nan(value, Z, mode):
    layer = Layer(2, 20, 90, Z, mode, 53)
    try:
        lab = layer.labels("whole")
        values, classes = layer.lists(6, "whole")
        values[4, 1] = value
        values[9, :] = value                              # nothing else in the list
        classes[15, 3], values[15, 3] = sl.NO_LABEL, value   # (not used in any case)
        less = classes.copy()
        less[4, 1] = less[9, :] = sl.NO_LABEL
        for tau, hard in ((1.0, 0.5), (2.0, 0.5), (2.0, 0.0)):
            got, want = layer.distill(lab, values, classes, tau, hard, 0.5), layer.distill(lab, values, less, tau, hard, 0.5)
            assert np.isnan(got["loss"]) and np.isfinite(want["loss"]) and same(got, want, KEYS[1:])
        less[15, 3] = classes[15, 3] = sl.NO_LABEL
        got = layer.distill(lab, values, less, 2.0, 0.5, 0.5)
        assert np.isfinite(got["loss"])
    finally:
        layer.close()
