"""A learner with adapters attached: what its plain calls do, and whose adapters an update moves."""
import numpy as np
import pytest

from tests.test_gpu_learner_updates import adapted, learner

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("dims", [dict(), dict(H=13, P=11, D=7)], ids=["whole words", "padded widths"])
def test_plain_calls_leave_the_softmax_layers_gradient_to_the_backward_pass_as_before(mode, dims):
    import torch
    from paper_1904_04956_amd import binding as bl
    plain, *_ = learner(mode, 91, **dims)
    other, *_ = adapted(mode, 91, **dims)
    try:
        other.calgrad_adapted()
        for lrn in (plain, other):
            lrn.forward()
            lrn.grad.fill_(7.0)
            bl.softmax_xent_fwd_bwd(lrn.ctx, lrn.theta_fwd, lrn.z, lrn.labels, lrn.loss, lrn.dz, lrn.grad)
        assert torch.equal(plain.grad, other.grad)
        for lrn in (plain, other):
            lrn.calgrad()
        assert torch.equal(plain.grad, other.grad) and torch.equal(plain.loss, other.loss)
        # and the adapted pass, which leaves nothing, whatever the plain one did
        other.forward()
        bl.softmax_xent_fwd_bwd(other.ctx, other.theta_fwd, other.z, other.labels, other.loss, other.dz, other.grad)
        other.calgrad_adapted()
        first = other.grad.clone()
        other.grad.fill_(7.0)
        other.calgrad_adapted()
        assert torch.equal(first, other.grad)
    finally:
        plain.close()
        other.close()


@pytest.mark.parametrize("mode", [0, 1])
def test_speakers_who_were_not_in_the_batch_stay_as_they_are(mode):
    import torch
    from oracle import muon
    lrn, a, *_ = adapted(mode, 92, count=5, ids=[0, 1, -1, 2, 0, 1, 4, 4, 2])
    wide = lambda t: t.double().cpu().numpy()  # noqa: E731
    try:
        E = 16 * 2.0 ** -22
        vA, vB = wide(a.vA), wide(a.vB)
        for k, ids in enumerate(([0, 1, -1, 2, 0, 1, 4, 4, 2], [4, 4, -1, -1, 0, 0, 0, 7, -5], [-1] * 9, [3] * 9)):
            a.ids.copy_(torch.tensor(ids, dtype=torch.int32))
            lrn.calgrad_adapted()
            a.ids.fill_(1)                                               # (the next batch's may be there already)
            before = [t.clone() for t in (a.A, a.Bm, a.vA, a.vB)] + [t.clone() for t in (a.A_bf16, a.Bm_bf16) if t is not None]
            A, Bm, dA, dB = (wide(t) for t in (a.A, a.Bm, a.dA, a.dB))
            lrn.apply_adapters(0.02, momentum=0.9, weight_decay=0.1)
            after = [a.A, a.Bm, a.vA, a.vB] + [t for t in (a.A_bf16, a.Bm_bf16) if t is not None]
            there = sorted({i for i in ids if 0 <= i < 5})
            absent = [i for i in range(5) if i not in there]
            for p, q in zip(before, after):
                assert torch.equal(p[absent], q[absent]), k
            if there and k != 1:                                         # (an invalid id makes the loss and everything after it NaN)
                for got, theta, g, v in ((a.A, A, dA, vA), (a.Bm, Bm, dB, vB)):
                    want, _ = muon.matrices_step(theta[there], g[there], v[there], 0.02, 0.9, 0.1, True)
                    assert np.linalg.norm(wide(got)[there] - want) <= 1.2 * 0.02 * E * np.sqrt(want.size) * max(1, np.sqrt(max(want.shape[1:]) / min(want.shape[1:]))) + 4 * 2.0 ** -24 * np.linalg.norm(want)
            if k == 1:
                for t in (a.A, a.Bm, a.vA, a.vB):
                    t[there] = 0.01 * torch.randn_like(t[there])
                a.refresh()
            vA, vB = wide(a.vA), wide(a.vB)
    finally:
        lrn.close()
