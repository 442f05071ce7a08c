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
