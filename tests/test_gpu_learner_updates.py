"""The learner's orthogonalised update and its adapters: gradients against the oracle on weights with the adapters multiplied out, and several steps as they
would be used.  Budgets of gradients are the framework's (max|gpu - ref| / max|ref| of a tensor: 1e-4 in float, 2e-2 in bf16)."""
import numpy as np
import pytest

from oracle import blstm_oracle as orc
from oracle import muon

pytestmark = pytest.mark.gpu
BUDGET = {0: 1e-4, 1: 2e-2}
DIMS = dict(T=5, B=9, D=12, H=16, L=2, P=24, V=50)
IDS = [0, 1, -1, 2, 0, 1, 1, -1, 2]


def learner(mode, seed, momentum=0.0, options={}, **dims):
    from paper_1904_04956_amd import inputs
    from paper_1904_04956_amd.harness import Learner
    d = dict(DIMS, **dims)
    lrn = Learner(mode=mode, momentum=momentum, **d, **options)
    theta = inputs.make_theta(lrn.n, seed, bf16=mode == 1)
    x, labels = inputs.make_batch(d["T"], d["B"], d["D"], d["V"], seed, bf16=mode == 1)
    lrn.set_theta(theta)
    lrn.set_batch(x, labels)
    return lrn, d, theta, x, labels


def adapted(mode, seed, count=3, rank=4, scale=1.5, ids=IDS, **dims):
    import torch
    from paper_1904_04956_amd.inputs import round_to_bf16
    lrn, d, theta, x, labels = learner(mode, seed, **dims)
    a = lrn.attach_adapters(count, rank, scale)
    r = np.random.default_rng(seed + 1)
    A, Bm = (0.3 * r.normal(size=tuple(t.shape)).astype(np.float32) for t in (a.A, a.Bm))
    if mode == 1:
        A, Bm = round_to_bf16(A), round_to_bf16(Bm)
    a.A.copy_(torch.from_numpy(A))
    a.Bm.copy_(torch.from_numpy(Bm))
    a.refresh()
    a.ids.copy_(torch.tensor(ids, dtype=torch.int32))
    return lrn, a, d, theta.astype(np.float64), x, labels, A.astype(np.float64), Bm.astype(np.float64)


def oracle_gradients(d, theta, x, labels, A, Bm, ids, scale):
    """Sequences of one adapter see W_p + scale B_a A_a; whole-batch loss scale."""
    dm = orc.Dims(**d)
    at = {n: (o, s) for n, o, s in orc.layout(dm)}
    o, shape = at["Wp"]
    part = slice(o, o + int(np.prod(shape)))
    loss, grad, dA, dB = 0.0, np.zeros(theta.size), np.zeros(A.shape), np.zeros(Bm.shape)
    for a in sorted(set(ids)):
        seqs = [s for s, i in enumerate(ids) if i == a]
        th = theta.copy()
        if a >= 0:
            th[part] += scale * (Bm[a] @ A[a]).reshape(-1)
        one = orc.Dims(**dict(d, B=len(seqs), loss_scale=1.0 / (d["T"] * d["B"])))
        l, g = orc.loss_and_grad(one, th, x[:, seqs], labels[:, seqs])
        loss, grad = loss + l, grad + g
        if a >= 0:
            dW = g[part].reshape(shape)
            dA[a], dB[a] = scale * Bm[a].T @ dW, scale * dW @ A[a].T
    return loss, grad, dA, dB


def near(got, want, mode, what):
    got = got.detach().float().cpu().numpy().reshape(want.shape)
    assert np.abs(got - want).max() <= BUDGET[mode] * np.abs(want).max(), what


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dims", [dict(), dict(H=13, P=11, D=7)], ids=["whole words", "padded widths"])
def test_adapted_gradients(mode, dims):
    lrn, a, d, theta, x, labels, A, Bm = adapted(mode, 81, **dims)
    try:
        lrn.calgrad_adapted()
        loss, grad, dA, dB = oracle_gradients(d, theta, x, labels, A, Bm, IDS, 1.5)
        assert abs(lrn.loss_value() - loss) <= BUDGET[mode] * abs(loss)
        near(a.dA, dA, mode, "dA")
        near(a.dB, dB, mode, "dB")
        for name, o, shape in orc.layout(orc.Dims(**d)):
            size = int(np.prod(shape))
            near(lrn.grad[o:o + size], grad[o:o + size].reshape(shape), mode, name)
        # the adapters alone: the same gradients of theirs, nothing of the model's but the softmax layer's
        first = a.dA.clone(), a.dB.clone()
        lrn.grad.fill_(7.0)
        lrn.calgrad_adapted(shared=False)
        assert np.array_equal(first[0].cpu(), a.dA.cpu()) and np.array_equal(first[1].cpu(), a.dB.cpu())
        o = {n: o for n, o, _ in orc.layout(orc.Dims(**d))}["Ws"]
        assert float((lrn.grad[:o] - 7.0).abs().max()) == 0.0
    finally:
        lrn.close()


@pytest.mark.parametrize("mode", [0, 1])
def test_sequences_without_adapter_are_the_model_itself(mode):
    lrn, a, d, theta, x, labels, A, Bm = adapted(mode, 82, ids=[-1] * 9)
    try:
        lrn.calgrad_adapted()
        got, loss = lrn.grad.clone(), lrn.loss_value()
        lrn.calgrad()
        assert abs(loss - lrn.loss_value()) <= BUDGET[mode] * abs(loss)
        for _, o, shape in orc.layout(orc.Dims(**d)):
            size = int(np.prod(shape))
            near(got[o:o + size], lrn.grad[o:o + size].double().cpu().numpy(), mode, o)
        assert float(a.dA.abs().max()) == 0.0 and float(a.dB.abs().max()) == 0.0
    finally:
        lrn.close()


@pytest.mark.parametrize("mode", [0, 1])
def test_steps_as_they_are_used(mode):
    # gradients with adapters, the orthogonalised update of the model and of the factors: each update is the oracle's of the gradient that was there
    lrn, a, d, *_ = adapted(mode, 83)
    try:
        layout, E = orc.layout(orc.Dims(**d)), 16 * 2.0 ** -22         # (few columns: products of both halves in either mode)
        v, vA, vB = np.zeros(lrn.n), np.zeros(tuple(a.A.shape)), np.zeros(tuple(a.Bm.shape))
        for k in range(3):
            lrn.calgrad_adapted()
            wide = lambda t: t.double().cpu().numpy()  # noqa: E731
            before, g, A, Bm, dA, dB = (wide(t) for t in (lrn.theta, lrn.grad, a.A, a.Bm, a.dA, a.dB))
            gates = bool(k & 1)
            lrn.apply_muon(0.02, 0.1, momentum=0.9, weight_decay=0.01, gates=gates, softmax=gates)
            lrn.apply_adapters(0.02, momentum=0.9)
            want, v = muon.step(layout, before, g, v, 0.02, 0.1, 0.9, 0.01, True, gates, gates)
            want_A, vA = muon.matrices_step(A, dA, vA, 0.02, 0.9, 0.0, True)
            want_B, vB = muon.matrices_step(Bm, dB, vB, 0.02, 0.9, 0.0, True)
            for got, ref, rms in ((lrn.theta, want, 0.02), (a.A, want_A, 0.02), (a.Bm, want_B, 0.02)):
                assert np.linalg.norm(wide(got) - ref) <= 1.2 * rms * E * np.sqrt(ref.size) + 4 * 2.0 ** -24 * np.linalg.norm(ref)
            v, vA, vB = wide(lrn.velocity), wide(a.vA), wide(a.vB)
            if mode == 1:
                assert np.array_equal(lrn.shadow.float().cpu(), lrn.theta.bfloat16().float().cpu()) and np.array_equal(a.A_bf16.float().cpu(), a.A.bfloat16().float().cpu())
    finally:
        lrn.close()


def test_a_captured_step_is_the_eager_one():
    import torch
    one, a, *_ = adapted(1, 84)
    two, b, *_ = adapted(1, 84)
    try:
        def step(lrn, stream=None):
            lrn.calgrad_adapted(stream=stream)
            lrn.apply_muon(0.02, 0.1, stream=stream)
            lrn.apply_adapters(0.02, stream=stream)
        for lrn in (one, two):
            step(lrn)                                                   # (makes scratch and velocities)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            step(two)
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            two.check_status()
            step(one)
            torch.cuda.synchronize()
            assert torch.equal(one.theta, two.theta) and torch.equal(a.A, b.A) and torch.equal(a.Bm, b.Bm) and torch.equal(one.loss, two.loss)
    finally:
        one.close()
        two.close()


def test_adapters_attached_anew():
    # other sizes need other scratch
    import torch
    lrn, a, *_ = adapted(1, 86, count=2, rank=2, ids=[0, 1, -1, 1, 0, 1, 1, -1, 0])
    try:
        lrn.calgrad_adapted()
        b = lrn.attach_adapters(300, 40)
        b.A.normal_()
        b.Bm.normal_()
        b.refresh()
        b.ids.copy_(torch.arange(9, dtype=torch.int32) * 30)
        lrn.calgrad_adapted()
        torch.cuda.synchronize()
        used = torch.zeros(300, dtype=torch.bool, device="cuda:0")
        used[b.ids.long()] = True
        assert bool((b.dA[used].abs().amax((1, 2)) > 0).all()) and float(b.dA[~used].abs().max()) == 0.0 and bool(torch.isfinite(b.dB).all())
    finally:
        lrn.close()


def test_the_stack_has_the_learners_options():
    # without kept copies, weights may be written without a word
    import torch
    one, a, *_ = adapted(1, 87, options=dict(keep_weight_copies=False), H=13, D=7)
    two, b, *_ = adapted(1, 88, H=13, D=7)
    try:
        one.calgrad_adapted()
        for to, of in ((one.theta, two.theta), (one.shadow, two.shadow), (one.x, two.x), (one.labels, two.labels), (a.A, b.A), (a.Bm, b.Bm), (a.A_bf16, b.A_bf16), (a.Bm_bf16, b.Bm_bf16)):
            to.copy_(of)
        one.calgrad_adapted()
        two.calgrad_adapted()
        torch.cuda.synchronize()
        assert torch.equal(one.grad, two.grad) and torch.equal(a.dA, b.dA) and torch.equal(one.loss, two.loss)
    finally:
        one.close()
        two.close()


def test_the_stacks_status_is_the_learners(monkeypatch):
    from paper_1904_04956_amd import binding as bl
    lrn, a, *_ = adapted(1, 89)
    try:
        asked, real = [], bl.blstm_device_status
        monkeypatch.setattr(bl, "blstm_device_status", lambda ctx, stream=None: (asked.append(ctx), real(ctx, stream)))
        lrn.check_status()
        assert asked == [lrn.ctx, a.stack]
    finally:
        lrn.close()


def test_adapters_that_are_not_there():
    from paper_1904_04956_amd import binding as bl
    lrn, *_ = learner(1, 90)
    try:
        calls = (lrn.forward_adapted, lrn.calgrad_adapted, lambda: lrn.apply_adapters(0.1))
        for attempt in range(2):
            for call in calls:
                with pytest.raises(ValueError):
                    call()
            if attempt == 0:                                            # refused adapters leave none, and a learner that works
                lrn.attach_adapters(2, 4)
                with pytest.raises(bl.BlstmError):
                    lrn.attach_adapters(2, 129)
        lrn.calgrad()
        lrn.apply(0.1)
        lrn.check_status()
    finally:
        lrn.close()


def test_a_model_without_bottleneck_has_no_place_for_adapters():
    lrn, *_ = learner(0, 85, P=0)
    try:
        with pytest.raises(ValueError):
            lrn.attach_adapters(2, 4)
    finally:
        lrn.close()
