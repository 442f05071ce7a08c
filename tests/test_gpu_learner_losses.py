"""The learner's calls of the softmax layer beyond cross-entropy: their arguments, their scratch, other weights than its own."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DIMS = dict(T=4, B=10, D=12, H=16, L=1, P=24, V=150)


def learner(seed, **dims):
    from paper_1904_04956_amd.harness import Learner
    d = dict(DIMS, **dims)
    lrn = Learner(mode=1, **d)
    rng = np.random.default_rng(seed)
    lrn.set_theta(rng.uniform(-0.1, 0.1, lrn.n).astype(np.float32))
    lrn.set_batch(rng.standard_normal((d["T"], d["B"], d["D"])).astype(np.float32), rng.integers(0, d["V"], (d["T"], d["B"])).astype(np.int32))
    return lrn


def test_lists_of_every_length_share_their_scratch():
    from paper_1904_04956_amd import binding as bl
    lrn = learner(61)
    try:
        values, classes = lrn.top_logits(150)
        at = lrn.loss_scratch(bl.SOFTMAX_TOPK, 150).data_ptr()
        for K in (1, 7, 64):
            v, c = lrn.top_logits(K)
            assert np.array_equal(v.cpu(), values[..., :K].cpu()) and np.array_equal(c.cpu(), classes[..., :K].cpu())
            assert lrn.loss_scratch(bl.SOFTMAX_TOPK, K).data_ptr() == at
        with pytest.raises(bl.BlstmError):
            lrn.top_logits(151)
        # a distillation's grows with its lists
        assert lrn.loss_scratch(bl.SOFTMAX_DISTILL, 100).numel() > lrn.loss_scratch(bl.SOFTMAX_DISTILL, 1).numel()
    finally:
        lrn.close()
