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


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 264])
@pytest.mark.parametrize("tau,hard", [(1.0, 0.5), (2.0, 0.5), (2.0, 0.0), (0.25, 0.5)])
def test_an_offset_of_all_logits_is_none_of_the_losses(tau, hard, Z, mode):
    # Logits exact in float, all of them 32768 lower, the teacher's 4096 higher.  What is left of a frame's terms are sums of V and K terms, some logarithms and products, and
    # the roundings of distances from the largest logit (x, over the temperature) and of log q.
    layer = exact_layer(2, 35, 300, Z, mode, 54, loss_scale=0.125)
    try:
        K, soft, s = 16, 0.75, float(layer.s)
        layer.theta[layer.at_b:layer.at_b + layer.V] = -32768.0
        z = layer.z.double().numpy()
        u = z @ layer.W.T + layer.b
        lab = best_labels(layer, u)
        given = lab if hard else np.full_like(lab, sl.NO_LABEL)
        classes = np.argsort(-u, axis=1, kind="stable")[:, :K].astype(np.int32)
        values = (np.round(16 * (np.take_along_axis(u, classes.astype(np.int64), axis=1) + 0.5 * layer.rng.normal(size=(layer.M, K)))) / 16 + 32768 + 4096).astype(np.float32)
        classes[layer.rng.random(layer.M) < 0.1] = sl.NO_LABEL
        some, labelled = (classes >= 0).any(axis=1), given != sl.NO_LABEL
        want = sl.distill(layer.W, layer.b, z, given, values, classes, s, tau, hard, soft)
        got = layer.distill(lab if hard else None, values, classes, tau, hard, soft)
        top = u.max(axis=1)
        xk = np.where(some, top - np.take_along_axis(u, np.maximum(classes, 0), axis=1).min(axis=1), 0) / tau
        xy = np.where(labelled, top - u[np.arange(layer.M), np.maximum(given, 0)], 0)
        vk = np.where(some, values.max(axis=1) - values.min(axis=1), 0).astype(np.float64) / tau
        log_v = np.log(layer.V)
        each = hard * labelled * (layer.V + 64 + 8 * (xy + log_v)) + soft * tau * tau * some * (layer.V + K + 64 + 8 * (xk + vk + log_v))
        size = hard * labelled * (xy + log_v) + soft * tau * tau * some * (xk + vk + log_v)
        assert abs(got["loss"] - want[0]) <= s * U * (each.sum() + layer.M * size.sum()), (got["loss"] - want[0]) / (s * U * (each.sum() + layer.M * size.sum()))
        lp = sl.logprob(layer.W, layer.b, z, lab)
        assert np.all(np.abs(layer.logprob(lab) - lp) <= U * (layer.V + 64 + 8 * (np.abs(lp) + log_v)))
    finally:
        layer.close()


def test_threads_that_share_a_context():
    # each with a stream, scratch and outputs of its own; the calls of one thread are the others' in another order
    import threading
    import torch
    layer = Layer(4, 60, 700, 96, 1, 55)
    bl = layer.bl
    try:
        lab, A = layer.labels("ragged"), layer.rng.normal(size=layer.M).astype(np.float32)
        values, classes = layer.lists(7, "ragged")
        theta, z, dlab, dA, dv, dc = (layer.dev(t) for t in (layer.theta, layer.z, lab, A, values, classes))

        def made():
            return [layer.outputs() for _ in range(2)], [layer.scratch(bl.SOFTMAX_POLICY), layer.scratch(bl.SOFTMAX_DISTILL, 7), layer.scratch(bl.SOFTMAX_LOGPROB)], torch.zeros(layer.M, device="cuda")

        def calls(held, order, stream):
            (p, d), (s1, s2, s3), logp = held
            for k in order:
                if k == 0:
                    bl.softmax_policy_fwd_bwd(layer.ctx, theta, z, dlab, dA, None, None, 0.2, 0.2, 0.0, p["loss"], None, p["dz"], p["grad"], s1, None, stream)
                elif k == 1:
                    bl.softmax_distill_fwd_bwd(layer.ctx, theta, z, dlab, dv, dc, 7, 2.0, 0.5, 0.5, d["loss"], d["dz"], d["grad"], s2, None, stream)
                else:
                    bl.softmax_logprob(layer.ctx, theta, z, dlab, logp, s3, None, stream)

        want = made()
        calls(want, (0, 1, 2), torch.cuda.current_stream())
        sets, streams = [made() for _ in range(4)], [torch.cuda.Stream() for _ in range(4)]
        torch.cuda.synchronize()
        failed = []

        def work(k):
            try:
                for _ in range(5):
                    calls(sets[k], [(k + j) % 3 for j in range(3)], streams[k])
            except Exception as e:
                failed.append(e)

        threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert not failed
        for outs, _, logp in sets:
            for got, ref in zip(outs, want[0]):
                for key in ("loss", "dz", "grad"):
                    assert torch.equal(got[key], ref[key]), key
            assert torch.equal(logp, want[2])
    finally:
        layer.close()
