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


@pytest.mark.parametrize("dims", [dict(), dict(T=21, B=40, D=40, H=301, L=2, P=67)], ids=["whole words", "padded widths"])
def test_given_weights_are_read_anew_in_every_call(dims):
    # weights that are made for one call often lie where those of an earlier call lay: the copies that a pass keeps go by that address
    import torch
    lrn, other = learner(62, **dims), learner(63, **dims)
    try:
        own_lp, own_top = lrn.log_probs(), lrn.top_logits(5)
        other.x.copy_(lrn.x), other.labels.copy_(lrn.labels)
        want = {"own": (own_lp, own_top), "other": (other.log_probs(), other.top_logits(5))}
        assert not torch.equal(want["other"][0], own_lp)
        buffer = torch.empty_like(lrn.theta_fwd)
        for name, src in (("own", lrn), ("other", other), ("own", lrn)):
            buffer.copy_(src.theta_fwd)
            assert torch.equal(lrn.log_probs(weights=buffer), want[name][0])
        for name, src in (("other", other), ("own", lrn)):
            buffer.copy_(src.theta_fwd)
            values, classes = lrn.top_logits(5, weights=buffer)
            assert torch.equal(values, want[name][1][0]) and torch.equal(classes, want[name][1][1])
        assert torch.equal(lrn.log_probs(), own_lp)
    finally:
        lrn.close()
        other.close()


def test_arguments_of_another_kind_are_refused():
    import torch
    lrn = learner(64)
    try:
        T, B, V = DIMS["T"], DIMS["B"], DIMS["V"]
        values, classes = lrn.top_logits(5)
        lp = lrn.log_probs()
        whole = torch.zeros((T, B, 10), device="cuda")
        for bad in (dict(values=values.double()), dict(classes=classes.long()), dict(classes=classes[:, :4].contiguous()), dict(values=values[..., :3].contiguous()), dict(values=whole[..., ::2]),
                    dict(values=values.cpu()), dict(classes=classes.transpose(0, 1).contiguous()), dict(values=values.cpu().numpy())):
            with pytest.raises((TypeError, ValueError)):
                lrn.calgrad_distill(**dict(dict(values=values, classes=classes), **bad))
        for bad in (dict(advantage=lp[:-1].contiguous()), dict(advantage=lp.double()), dict(old_logp=lp.t()), dict(ref_logp=lp.half()), dict(logp=torch.empty((T, B - 1), device="cuda")),
                    dict(advantage=lp.cpu())):
            with pytest.raises((TypeError, ValueError)):
                lrn.calgrad_policy(**dict(dict(advantage=lp), **bad))
        for bad in (dict(labels=lrn.labels.long()), dict(labels=lrn.labels[:2]), dict(weights=lrn.theta), dict(weights=lrn.theta_fwd[:-1])):
            with pytest.raises((TypeError, ValueError)):
                lrn.log_probs(**bad)
        with pytest.raises((TypeError, ValueError)):
            lrn.top_logits(5, weights=lrn.theta)
        # and what a program gives as it should is taken
        lrn.calgrad_distill(values, classes, temperature=2.0)
        grad = lrn.grad.clone()
        lrn.calgrad_distill(values.view(T * B, 5), classes.view(T * B, 5), temperature=2.0)
        assert torch.equal(lrn.grad, grad)
        lrn.calgrad_policy(lp, lp.view(-1), lp, logp=torch.empty_like(lp))
        assert np.isfinite(lrn.loss_value())
    finally:
        lrn.close()
