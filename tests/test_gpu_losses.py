"""The softmax layer beyond cross-entropy on the GPU, through the C-ABI, against the float64 oracle.

Tolerances are element by element, from the number formats alone.  With u the unit roundoff of float (2^-24) and Z terms a logit,
a logit is off by at most eu = (Z + 2) u (|z| |W|^T + |b|); a probability by a factor exp(2 eu) and a few roundings of exponentials whose
arguments are as large as the logits.  dE/du enters the product for dz as one bf16 (2^-8) and those for W_s and b_s as two
(2^-16), or as a float; then come as many roundings as there are terms, and that of the result's own type.
"""
import numpy as np
import pytest

from oracle import softmax_losses as sl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class Layer:
    """A softmax layer of M = T B frames with its arrays, host copies beside them."""

    def __init__(self, T, B, V, Z, mode, seed, scale=1.0, loss_scale=0.0, **dims):
        import torch
        from paper_1904_04956_amd import binding as bl
        self.bl, self.torch, self.mode = bl, torch, mode
        # (z is the bottleneck's output, or 2H wide without one)
        d = dict(D=8, H=8, L=1, P=Z)
        d.update(dims)
        self.ctx = bl.blstm_create(T, B, d["D"], d["H"], d["L"], d["P"], V, mode, loss_scale)
        self.M, self.V, self.Z, self.s = T * B, V, Z, np.float32(loss_scale if loss_scale > 0 else 1.0 / (T * B))
        self.kind = torch.bfloat16 if mode == 1 else torch.float32
        g = torch.Generator().manual_seed(seed)
        self.n = bl.blstm_param_count(self.ctx)
        self.at_w, self.at_b = bl.blstm_param_offset(self.ctx, 0, 0, bl.BLSTM_WS)[0], bl.blstm_param_offset(self.ctx, 0, 0, bl.BLSTM_BS)[0]
        self.theta = (scale * 0.3 * torch.randn(self.n, generator=g)).to(self.kind)
        self.z = torch.randn(self.M, Z, generator=g).to(self.kind)
        self.rng = np.random.default_rng(seed)

    def close(self):
        self.bl.blstm_destroy(self.ctx)

    W = property(lambda self: self.theta[self.at_w:self.at_w + self.V * self.Z].double().numpy().reshape(self.V, self.Z))
    b = property(lambda self: self.theta[self.at_b:self.at_b + self.V].double().numpy())

    def labels(self, kind):
        lab = self.rng.integers(0, self.V, self.M).astype(np.int32)
        if kind == "ragged":
            lab[self.rng.random(self.M) < 0.4] = sl.NO_LABEL
            lab[0] = sl.NO_LABEL
        if kind == "none":
            lab[:] = sl.NO_LABEL
        return lab

    def lists(self, K, kind):
        values = (2 * self.rng.normal(size=(self.M, K))).astype(np.float32)
        classes = np.stack([self.rng.permutation(self.V)[:K] for _ in range(self.M)]).astype(np.int32)
        if kind == "ragged":
            classes[self.rng.random((self.M, K)) < 0.3] = sl.NO_LABEL
            classes[self.rng.random(self.M) < 0.3] = sl.NO_LABEL
            values[self.rng.random((self.M, K)) < 0.2] = -np.inf
            if K > 2:
                classes[:, 2] = classes[:, 0]          # twice in a list
        if kind == "none":
            classes[:] = sl.NO_LABEL
        return values, classes

    def dev(self, a):
        return None if a is None else (a if hasattr(a, "cuda") else self.torch.from_numpy(np.ascontiguousarray(a))).cuda()

    def scratch(self, call, K=0):
        # garbage: nothing in it may matter
        return self.torch.full((self.bl.softmax_scratch_bytes(self.ctx, call, K),), 0xFF, dtype=self.torch.uint8, device="cuda")

    def outputs(self):
        t = self.torch
        return dict(loss=t.full((1,), -1.0, device="cuda"), dz=t.full((self.M, self.Z), -1.0, dtype=self.kind, device="cuda"), grad=t.full((self.n,), -1.0, device="cuda"),
                    logp=t.full((self.M,), -1.0, device="cuda"))

    def logprob(self, lab):
        o = self.outputs()
        self.bl.softmax_logprob(self.ctx, self.dev(self.theta), self.dev(self.z), self.dev(lab), o["logp"], self.scratch(self.bl.SOFTMAX_LOGPROB))
        return o["logp"].double().cpu().numpy()

    def distill(self, lab, values, classes, tau, hard, soft, o=None):
        o = o or self.outputs()
        K = classes.shape[1]
        self.bl.softmax_distill_fwd_bwd(self.ctx, self.dev(self.theta), self.dev(self.z), self.dev(lab), self.dev(values), self.dev(classes), K, tau, hard, soft,
                                        o["loss"], o["dz"], o["grad"], self.scratch(self.bl.SOFTMAX_DISTILL, K))
        return self.taken(o)

    def policy(self, lab, A, old, ref, low, high, kl):
        o = self.outputs()
        self.bl.softmax_policy_fwd_bwd(self.ctx, self.dev(self.theta), self.dev(self.z), self.dev(lab), self.dev(A), self.dev(old), self.dev(ref), low, high, kl,
                                       o["loss"], o["logp"], o["dz"], o["grad"], self.scratch(self.bl.SOFTMAX_POLICY))
        return self.taken(o)

    def taken(self, o):
        g = o["grad"].double().cpu().numpy()
        assert np.all(g[:self.at_w] == -1)             # nothing but the two slices
        return dict(loss=float(o["loss"]), dz=o["dz"].double().cpu().numpy(), dW=g[self.at_w:self.at_w + self.V * self.Z].reshape(self.V, self.Z),
                    db=g[self.at_b:self.at_b + self.V], logp=o["logp"].double().cpu().numpy())

    # ---- bounds -------------------------------------------------------------------------------
    def errors(self, live, sharpest=1.0):
        """Largest error of a logit, and of a probability in relation to it, over the frames that count."""
        if not live.any():
            return 0.0, 0.0
        z = np.abs(self.z.double().numpy()[live])
        b = np.where(np.isfinite(self.b), self.b, 0.0)
        size = (z @ np.abs(self.W).T + np.abs(b)).max()
        eu = (self.Z + 2) * U * size
        return eu, 4 * sharpest * eu + 16 * U + 8 * U * sharpest * size + self.V * U

    def check_gradients(self, got, ref, du, live, rel, extra=0.0):
        """du: the reference's dE/du, of which every element is right to `rel` of itself and `extra`."""
        dz, dW, db = ref
        z = np.where(live[:, None], self.z.double().numpy(), 0.0)
        a = np.abs(du) * (1 + rel) + extra * live[:, None]
        one, two = (2.0 ** -8, 2.0 ** -16) if self.mode == 1 else (U, U)
        rows = 2 * self.M if self.mode == 1 else self.M
        off = lambda r: np.abs(du) * r + extra * live[:, None]  # noqa: E731
        tiny = 1e-37                                     # (results below the normal range may flush)
        bound = off(rel + one) @ np.abs(self.W) + (a @ np.abs(self.W)) * self.V * U
        own = (2.0 ** -8 if self.mode == 1 else U) * (np.abs(dz) + bound)
        assert np.all(np.abs(got["dz"] - dz) <= bound + own + tiny), np.max(np.abs(got["dz"] - dz) / (bound + own + tiny))
        bound = off(rel + two).T @ np.abs(z) + (a.T @ np.abs(z)) * rows * U
        assert np.all(np.abs(got["dW"] - dW) <= bound + U * np.abs(dW) + tiny), np.max(np.abs(got["dW"] - dW) / (bound + U * np.abs(dW) + tiny))
        bound = off(rel + two).sum(axis=0) + a.sum(axis=0) * rows * U
        assert np.all(np.abs(got["db"] - db) <= bound + U * np.abs(db) + tiny), np.max(np.abs(got["db"] - db) / (bound + U * np.abs(db) + tiny))
        assert np.all(got["dz"][~live] == 0)


def du_of(layer, labels, g=None, q=None, some=None, tau=1.0, hard=0.0, soft=0.0):
    """dE/du of the oracle's formula, and its parts' absolute values (their errors do not cancel)."""
    live = labels != sl.NO_LABEL
    counts = live if some is None else live | some
    _, u, lp = sl._rows(layer.W, layer.b, layer.z.double().numpy(), counts)
    hot = np.zeros_like(u)
    hot[np.flatnonzero(live), labels[live]] = 1.0
    if g is not None:
        return layer.s * np.abs(g)[:, None] * (hot + np.exp(lp)) * live[:, None]
    lpt = sl._log_softmax(u / tau)
    return layer.s * (hard * (np.exp(lp) * live[:, None] + hot) + soft * tau * (np.exp(lpt) * some[:, None] + q))


SHAPES = [                                               # T, B, V, Z
    (1, 1, 1, 8), (1, 1, 7, 16), (1, 3, 64, 8), (2, 2, 65, 33), (1, 1, 1000, 256), (3, 43, 129, 67), (5, 26, 300, 256), (2, 64, 128, 64),
    (3, 43, 1001, 250), (7, 37, 515, 264), (1, 129, 257, 320), (4, 65, 260, 640), (2, 150, 3001, 128),
]


def layer_id(v):
    return "x".join(map(str, v)) if isinstance(v, tuple) else str(v)


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("shape", SHAPES, ids=layer_id)
@pytest.mark.parametrize("mask", ["whole", "ragged", "none"])
def test_log_probabilities(shape, mode, mask):
    T, B, V, Z = shape
    layer = Layer(T, B, V, Z, mode, 11)
    try:
        lab = layer.labels(mask)
        ref = sl.logprob(layer.W, layer.b, layer.z.double().numpy(), lab)
        got = layer.logprob(lab)
        eu, _ = layer.errors(lab != sl.NO_LABEL)
        size = np.abs(layer.z.double().numpy() @ layer.W.T + layer.b).max()
        assert np.all(np.abs(got - ref) <= 2 * eu + 8 * U * (np.abs(ref) + size + 1) + V * U), np.abs(got - ref).max()
        assert np.all(got[lab == sl.NO_LABEL] == 0)
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("shape", SHAPES, ids=layer_id)
@pytest.mark.parametrize("mask,tau,hard", [("whole", 2.0, 0.5), ("ragged", 0.5, 0.25), ("ragged", 1.0, 0.5), ("whole", 3.0, 0.0), ("ragged", 1.0, 0.0), ("none", 2.0, 0.5)])
def test_distillation(shape, mode, mask, tau, hard):
    T, B, V, Z = shape
    layer = Layer(T, B, V, Z, mode, 12, loss_scale=0.125)
    try:
        K = min(V, 1 if T * B == 1 else 9)
        lab = layer.labels(mask)
        values, classes = layer.lists(K, mask)
        given = lab if hard else np.full_like(lab, sl.NO_LABEL)
        q, some = sl.teacher_distribution(values, classes, V, tau)
        ref = sl.distill(layer.W, layer.b, layer.z.double().numpy(), given, values, classes, float(layer.s), tau, hard, 0.75)
        got = layer.distill(lab if hard else None, values, classes, tau, hard, 0.75)
        live = (given != sl.NO_LABEL) | some
        eu, rel = layer.errors(live, max(1.0, 1 / tau))
        du = du_of(layer, given, None, q, some, tau, hard, 0.75)
        layer.check_gradients(got, ref[1:], du, live, rel + K * U + 64 * U * (1 + 8 / tau))
        # every term of a frame's loss is right to the logits' errors and a few roundings of the largest
        size = np.abs(np.where(live[:, None], layer.z.double().numpy(), 0) @ layer.W.T + layer.b).max() * max(1, 1 / tau) + np.log(V) + 10 / tau
        each = 2 * eu * max(1, 1 / tau) + (16 + K) * U * size + V * U
        assert abs(got["loss"] - ref[0]) <= layer.s * (hard * each + 0.75 * tau * tau * each) * live.sum() + layer.M * U * layer.s * live.sum() * size * (hard + tau * tau)
        if not live.any():
            assert got["loss"] == 0 and not got["dW"].any() and not got["db"].any() and not got["dz"].any()
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("shape", SHAPES, ids=layer_id)
@pytest.mark.parametrize("mask,old,ref", [("whole", True, True), ("ragged", True, True), ("ragged", False, True), ("whole", True, False), ("ragged", False, False), ("none", True, True)])
def test_policy(shape, mode, mask, old, ref):
    T, B, V, Z = shape
    layer = Layer(T, B, V, Z, mode, 13)
    try:
        lab = layer.labels(mask)
        live = lab != sl.NO_LABEL
        low, high, kl = np.float32(0.25), np.float32(0.375), np.float32(0.125)
        z = layer.z.double().numpy()
        lp = sl.logprob(layer.W, layer.b, z, lab)
        eu, rel = layer.errors(live)
        size = np.abs(np.where(live[:, None], z, 0) @ layer.W.T + layer.b).max()
        elp = 2 * eu + 8 * U * (np.abs(lp).max() + size + 1) + V * U
        d = 0.3 * layer.rng.normal(size=layer.M)
        for edge in (-np.log(1 - low), -np.log(1 + high)):       # where a rounding would decide whether a frame counts
            d = np.where(np.abs(d - edge) < 4 * elp + 1e-5, d + 8 * elp + 1e-4, d)
        o = (lp + d).astype(np.float32) if old else None
        r = (lp + 0.3 * layer.rng.normal(size=layer.M)).astype(np.float32) if ref else None
        A = layer.rng.normal(size=layer.M).astype(np.float32)
        A[layer.rng.random(layer.M) < 0.1] = 0.0
        want = sl.policy(layer.W, layer.b, z, lab, A, o, r, float(layer.s), low, high, kl)
        got = layer.policy(lab, A, o, r, low, high, kl)
        assert np.all(np.abs(got["logp"] - want[1]) <= elp)
        assert np.all(got["logp"][~live] == 0)
        ratio = np.exp(lp - o) if old else np.ones(layer.M)
        off = np.exp(r - lp) if ref else np.zeros(layer.M)
        slope = np.abs(A) * ratio + kl * (1 + off)       # each part of g is right to elp and a few roundings of itself
        du = du_of(layer, lab, slope)
        layer.check_gradients(got, want[2:], du, live, rel + 2 * elp + 32 * U)
        each = (np.abs(A) * ratio + kl * (off + 2 + np.abs(lp)))[live].sum() * (2 * elp + (32 + layer.M) * U)
        assert abs(got["loss"] - want[0]) <= layer.s * each + 1e-37
    finally:
        layer.close()


def grid_layer(T, B, V, Z, mode, seed):
    """Weights and activations whose products and sums are exact in float: equal logits are equal in any order of the sum."""
    layer = Layer(T, B, V, Z, mode, seed)
    t = layer.torch
    layer.theta = ((layer.theta.float() * 8).round().clamp(-15, 15) / 16).to(layer.kind)
    layer.z = ((layer.z.float() * 4).round().clamp(-15, 15) / 4).to(layer.kind)
    return layer


def run_topk(layer, K):
    t = layer.torch
    values, classes = t.full((layer.M, K), -1.0, device="cuda"), t.full((layer.M, K), -7, dtype=t.int32, device="cuda")
    layer.bl.softmax_topk(layer.ctx, layer.dev(layer.theta), layer.dev(layer.z), K, values, classes, layer.scratch(layer.bl.SOFTMAX_TOPK, K))
    return values.double().cpu().numpy(), classes.cpu().numpy()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("shape,K", [((1, 1, 1, 8), 1), ((1, 1, 7, 16), 7), ((1, 3, 64, 8), 64), ((2, 2, 65, 33), 5), ((1, 1, 1000, 256), 256), ((3, 43, 129, 67), 129),
                                     ((5, 26, 300, 256), 1), ((3, 43, 1001, 250), 64), ((7, 37, 515, 264), 100), ((4, 65, 260, 640), 33), ((2, 150, 3001, 128), 20),
                                     ((21, 80, 9001, 64), 65)], ids=layer_id)
def test_the_largest_logits(shape, K, mode):
    layer = grid_layer(*shape, mode, 14)
    try:
        u = layer.z.double().numpy() @ layer.W.T + layer.b
        values, classes = run_topk(layer, K)
        order = np.argsort(-u, axis=1, kind="stable")[:, :K]
        assert np.array_equal(classes, order)
        assert np.array_equal(values, np.take_along_axis(u, order, axis=1))
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
def test_the_largest_of_equal_and_odd_logits(mode):
    # all weights zero: the logits are the bias, the same in every frame
    V = 700
    layer = grid_layer(2, 70, V, 64, mode, 15)
    try:
        layer.theta[:] = 0
        b = layer.theta[layer.at_b:]
        for fill in ("equal", "half", "nan", "inf", "zeros", "lowest"):
            b[:] = 0.5
            if fill == "half":
                b[::2] = 0.25
            if fill == "nan":
                b[: V - 5] = float("nan")
            if fill == "inf":
                b[:] = -float("inf")
                b[600] = float("inf")
                b[3] = 1.0
            if fill == "zeros":
                b[:] = 0.0
                b[1::2] = -0.0
            if fill == "lowest":
                b[:] = layer.torch.finfo(layer.kind).min
                b[77] = 0.0
            want, order = sl.topk(layer.b[None, :], 40)
            values, classes = run_topk(layer, 40)
            assert np.array_equal(classes, np.repeat(order, layer.M, 0)), fill
            assert np.array_equal(values, np.repeat(want, layer.M, 0), equal_nan=True), fill
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("lowest", [-float("inf"), None])
def test_classes_that_are_ruled_out(mode, lowest):
    # a bias of -inf or of the type's lowest value, whole strips of classes and the last ones among them
    layer = Layer(3, 41, 333, 64, mode, 16)
    try:
        low = layer.torch.finfo(layer.kind).min if lowest is None else lowest
        out = np.zeros(333, dtype=bool)
        out[64:192] = out[256:333] = out[3] = True
        b = layer.theta[layer.at_b:layer.at_b + 333]
        b[layer.torch.from_numpy(out)] = low
        lab = layer.labels("ragged")
        allowed = np.flatnonzero(~out)
        lab = np.where(lab == sl.NO_LABEL, lab, allowed[lab % len(allowed)]).astype(np.int32)
        live = lab != sl.NO_LABEL
        A = layer.rng.normal(size=layer.M).astype(np.float32)
        with np.errstate(all="ignore"):
            z = layer.z.double().numpy()
            want = sl.policy(layer.W, np.where(out, -1e30, layer.b), z, lab, A, None, None, float(layer.s), 0.2, 0.2, 0.0)
        got = layer.policy(lab, A, None, None, 0.2, 0.2, 0.0)
        keep = layer.theta.clone()
        b[layer.torch.from_numpy(out)] = 0               # (for the bounds' sizes)
        eu, rel = layer.errors(live)
        layer.theta = keep
        hot = np.zeros((layer.M, 333))
        hot[np.flatnonzero(live), lab[live]] = 1
        du = layer.s * np.abs(A)[:, None] * (hot + np.exp(sl._log_softmax(np.where(live[:, None], z, 0) @ layer.W.T + np.where(out, -1e30, layer.b)))) * live[:, None]
        layer.check_gradients(got, want[2:], du, live, rel + 64 * U)
        assert not got["db"][out].any() and not got["dW"][out].any()
        assert np.isfinite(got["loss"]) and np.all(np.isfinite(got["logp"]))
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 67])
def test_padding_may_hold_nan_and_infinities(mode, Z):
    layer = Layer(4, 33, 200, Z, mode, 17)
    try:
        lab = layer.labels("ragged")
        values, classes = layer.lists(6, "whole")
        classes[lab == sl.NO_LABEL] = sl.NO_LABEL
        A, old, ref = (layer.rng.normal(size=layer.M).astype(np.float32) for _ in range(3))
        old -= 5
        ref -= 5
        first = layer.logprob(lab), layer.distill(lab, values, classes, 2.0, 0.5, 0.5), layer.policy(lab, A, old, ref, 0.2, 0.2, 0.1)
        out = lab == sl.NO_LABEL
        for k, x in enumerate((np.nan, np.inf, -np.inf)):
            layer.z[np.flatnonzero(out)[k::3]] = x
            values[np.flatnonzero(out)[k::3]] = x
            for a in (A, old, ref):
                a[np.flatnonzero(out)[k::3]] = x
        second = layer.logprob(lab), layer.distill(lab, values, classes, 2.0, 0.5, 0.5), layer.policy(lab, A, old, ref, 0.2, 0.2, 0.1)
        assert np.array_equal(first[0], second[0])
        for x, y in zip(first[1:], second[1:]):
            for k in ("loss", "dz", "dW", "db"):
                assert np.array_equal(x[k], y[k]), k
            assert np.isfinite(x["loss"])
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
def test_a_class_that_does_not_exist_makes_its_frames_terms_nan_and_nothing_else(mode):
    layer = Layer(3, 21, 90, 32, mode, 18)
    try:
        lab = layer.labels("whole")
        values, classes = layer.lists(5, "whole")
        A = np.ones(layer.M, dtype=np.float32)
        without, bad = lab.copy(), lab.copy()
        without[[2, 40]] = sl.NO_LABEL
        bad[2], bad[40] = 90, -5
        lp, ref = layer.logprob(bad), layer.logprob(without)
        assert np.all(np.isnan(lp[[2, 40]])) and np.array_equal(np.delete(lp, [2, 40]), np.delete(ref, [2, 40]))
        x, y = layer.policy(bad, A, None, None, 0.2, 0.2, 0.0), layer.policy(without, A, None, None, 0.2, 0.2, 0.0)
        assert np.isnan(x["loss"]) and all(np.array_equal(x[k], y[k]) for k in ("dz", "dW", "db"))
        x, y = layer.distill(bad, values, classes, 2.0, 0.5, 0.5), layer.distill(without, values, classes, 2.0, 0.5, 0.5)
        assert np.isnan(x["loss"]) and all(np.array_equal(x[k], y[k]) for k in ("dz", "dW", "db"))
        worse, less = classes.copy(), classes.copy()
        worse[7, 1], less[7, 1] = 1 << 30, sl.NO_LABEL
        worse[9, :], less[9, :] = -2, sl.NO_LABEL
        x, y = layer.distill(lab, values, worse, 2.0, 0.5, 0.5), layer.distill(lab, values, less, 2.0, 0.5, 0.5)
        assert np.isnan(x["loss"]) and all(np.array_equal(x[k], y[k]) for k in ("dz", "dW", "db"))
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
def test_ratios_and_advantages_at_their_ends(mode):
    # a ratio of zero and of infinity, an advantage of zero with either: the clip decides, and 0 times infinity is nothing
    layer = Layer(1, 8, 50, 16, mode, 19)
    try:
        lab = layer.labels("whole")
        lp = layer.logprob(lab).astype(np.float32)
        old = lp + np.array([200, -200, 200, -200, 200, -200, 0, 0], dtype=np.float32)
        A = np.array([1, 1, -1, -1e-3, 0, 0, 1, -1], dtype=np.float32)
        A[3] = 0                                         # (an infinite ratio with a negative advantage is an infinite loss)
        got = layer.policy(lab, A, old, None, 0.25, 0.25, 0.0)
        # frame 0: r = 0, inner 0 < 0.75; 1: inf, clipped to 1.25; 2: r = 0: clipped to -0.75; 6, 7: about 1
        want = -(0 + 1.25 - 0.75 + 0 + 0 + 0 + 1 - 1) / 8
        assert abs(got["loss"] - want) < 1e-5
        assert not got["dz"][:6].any() and got["dz"][6:].any(axis=1).all() and np.all(np.isfinite(got["dz"]))
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
def test_large_logits(mode):
    # logits of some hundreds: exponentials of anything but differences would overflow
    layer = Layer(2, 40, 400, 64, mode, 20, scale=40.0)
    try:
        lab = layer.labels("whole")
        z = layer.z.double().numpy()
        ref = sl.logprob(layer.W, layer.b, z, lab)
        eu, _ = layer.errors(np.ones(layer.M, dtype=bool))
        size = np.abs(z @ layer.W.T + layer.b).max()
        assert size > 150
        assert np.all(np.abs(layer.logprob(lab) - ref) <= 2 * eu + 8 * U * (np.abs(ref) + size + 1) + 400 * U)
        values, classes = layer.lists(7, "whole")
        got = layer.distill(lab, 100 * values, classes, 0.25, 0.5, 0.5)
        assert all(np.all(np.isfinite(v)) for v in got.values())
    finally:
        layer.close()


def test_a_captured_call_replays_on_new_inputs_and_beside_eager_ones():
    import torch
    layer = Layer(5, 30, 300, 256, 1, 21)
    bl = layer.bl
    try:
        lab = layer.labels("ragged")
        values, classes = layer.lists(9, "ragged")
        A = layer.rng.normal(size=layer.M).astype(np.float32)
        theta, z, dlab, dA = layer.dev(layer.theta), layer.dev(layer.z).clone(), layer.dev(lab), layer.dev(A)
        dv, dc = layer.dev(values), layer.dev(classes)

        def calls(o, p, s1, s2):
            bl.softmax_policy_fwd_bwd(layer.ctx, theta, z, dlab, dA, None, None, 0.2, 0.2, 0.0, o["loss"], o["logp"], o["dz"], o["grad"], s1)
            bl.softmax_distill_fwd_bwd(layer.ctx, theta, z, dlab, dv, dc, 9, 2.0, 0.5, 0.5, p["loss"], p["dz"], p["grad"], s2)

        side = torch.cuda.Stream()
        s = layer.scratch(bl.SOFTMAX_POLICY), layer.scratch(bl.SOFTMAX_DISTILL, 9)
        o, p = layer.outputs(), layer.outputs()
        eager = layer.outputs(), layer.outputs()
        es = layer.scratch(bl.SOFTMAX_POLICY), layer.scratch(bl.SOFTMAX_DISTILL, 9)
        with torch.cuda.stream(side):
            calls(o, p, *s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls(o, p, *s)
        for k in range(4):
            z.copy_(torch.randn(z.shape, generator=torch.Generator().manual_seed(k)))
            for x in s:
                x.fill_(0xFF)
            graph.replay()
            calls(*eager, *es)                           # (scratch of its own)
            torch.cuda.synchronize()
            for x, y in zip((o, p), eager):
                for key in ("loss", "dz", "grad"):
                    assert torch.equal(x[key], y[key]), (k, key)
    finally:
        layer.close()


def test_two_streams_with_scratch_of_their_own_and_the_same_bits():
    import torch
    layer = Layer(9, 40, 1500, 128, 1, 22)
    bl = layer.bl
    try:
        lab, A = layer.labels("ragged"), layer.rng.normal(size=layer.M).astype(np.float32)
        theta, z, dlab, dA = layer.dev(layer.theta), layer.dev(layer.z), layer.dev(lab), layer.dev(A)
        out = []
        streams = [torch.cuda.Stream() for _ in range(2)]
        sets = [(layer.outputs(), layer.scratch(bl.SOFTMAX_POLICY)) for _ in range(6)]
        torch.cuda.synchronize()
        for k, (o, s) in enumerate(sets):
            bl.softmax_policy_fwd_bwd(layer.ctx, theta, z, dlab, dA, None, None, 0.2, 0.2, 0.0, o["loss"], o["logp"], o["dz"], o["grad"], s, None, streams[k % 2])
        torch.cuda.synchronize()
        for o, _ in sets[1:]:
            for key in ("loss", "logp", "dz", "grad"):
                assert torch.equal(o[key], sets[0][0][key]), key
    finally:
        layer.close()


@pytest.mark.parametrize("dims,mode", [(dict(T=6, B=20, D=12, H=16, L=2, P=24, V=150), 1), (dict(T=6, B=20, D=12, H=16, L=1, P=0, V=150), 0),
                                       (dict(T=21, B=40, D=40, H=301, L=1, P=67, V=2000), 1)])
def test_a_teacher_a_student_and_a_policy_step(dims, mode):
    # what a program does with them: a teacher annotates a batch, a student learns from it, then a policy step follows on the
    # student's own log-probabilities.  The gradients of the whole model are the xent path's where both say the same.
    import torch
    from paper_1904_04956_amd import binding as bl
    from paper_1904_04956_amd.harness import Learner
    teacher, student = Learner(mode=mode, **dims), Learner(mode=mode, **dims)
    try:
        rng = np.random.default_rng(23)
        V = dims["V"]
        x = rng.standard_normal((dims["T"], dims["B"], dims["D"])).astype(np.float32)
        labels = rng.integers(0, V, (dims["T"], dims["B"])).astype(np.int32)
        for lrn, seed in ((teacher, 1), (student, 2)):
            lrn.set_theta(np.random.default_rng(seed).uniform(-0.1, 0.1, lrn.n).astype(np.float32))
            lrn.set_batch(x, labels)
        values, classes = teacher.top_logits(8)
        student.calgrad_distill(values, classes, temperature=2.0, hard_weight=0.5)
        first = student.loss_value()
        student.apply(0.1)
        assert np.isfinite(first) and torch.isfinite(student.grad).all()
        # a list of the label alone, at temperature 1, is cross-entropy; so is the policy loss with an advantage of one
        student.calgrad()
        loss, grad = student.loss_value(), student.grad.clone()
        big = float(grad.abs().max())
        only = student.labels[..., None].contiguous()
        student.calgrad_distill(torch.zeros_like(only, dtype=torch.float32), only, temperature=1.0, hard_weight=0.0, soft_weight=1.0)
        tol = 2e-2 if mode == 1 else 1e-4                # (of the xent path, as everywhere in these tests)
        assert abs(student.loss_value() - loss) <= tol * loss
        assert float((student.grad - grad).abs().max()) <= tol * big
        lp = student.log_probs()
        assert abs(float(-lp.mean()) - loss) <= tol * loss
        got = torch.empty_like(lp)
        student.calgrad_policy(torch.ones_like(lp), old_logp=lp, ref_logp=lp, kl_weight=0.1, logp=got)
        # (the two calls sum in orders of their own: each is within the bound of test_log_probabilities of the exact value)
        off, n = bl.blstm_param_offset(student.ctx, 0, 0, bl.BLSTM_WS)
        z, W, b = student.z.double().view(-1, student.zdim), student.theta_fwd[off:off + n].double().view(V, -1), student.theta_fwd[off + n:off + n + V].double()
        eu = (student.zdim + 2) * U * float((z.abs() @ W.abs().t() + b.abs()).max())
        size = float((z @ W.t() + b).abs().max())
        assert float((got - lp).abs().max()) <= 2 * (2 * eu + 8 * U * (float(lp.abs().max()) + size + 1) + V * U)
        assert float((student.grad - grad).abs().max()) <= tol * big
        student.apply(0.1)
        assert float(-student.log_probs().mean()) < loss
    finally:
        teacher.close()
        student.close()


@pytest.mark.parametrize("shape", [(2, 4150, 140, 40), (1, 8200, 70, 264), (1, 90, 40000, 24)], ids=layer_id)
@pytest.mark.parametrize("mode", [1, 0])
def test_many_frames_and_many_classes(shape, mode):
    # more than 8192 frames, classes in parts of the rows, float rows that no workgroup holds in registers
    test_policy(shape, mode, "ragged", True, True)
    test_distillation(shape, mode, "ragged", 2.0, 0.5)
    test_distillation(shape, mode, "ragged", 2.0, 0.0)
    test_log_probabilities(shape, mode, "ragged")


@pytest.mark.parametrize("shape,K,tau,hard", [((2, 70, 200, 96), 150, 2.0, 0.5), ((2, 70, 200, 96), 150, 2.0, 0.0), ((1, 130, 300, 256), 256, 1.0, 0.5), ((2, 70, 260, 264), 129, 3.0, 0.25),
                                              ((1, 70, 140000, 16), 40, 2.0, 0.5), ((3, 1400, 150, 32), 100, 2.0, 0.0)], ids=layer_id)
@pytest.mark.parametrize("mode", [1, 0])
def test_long_lists(shape, K, tau, hard, mode):
    # several thousand entries in a block of 64 frames and 128 classes, or more blocks than threads that count them
    T, B, V, Z = shape
    layer = Layer(T, B, V, Z, mode, 31, loss_scale=0.125)
    try:
        lab = layer.labels("ragged")
        values, classes = layer.lists(K, "ragged")
        classes[5, :] = classes[5, 0] if classes[5, 0] >= 0 else 7      # one class all along a list
        given = lab if hard else np.full_like(lab, sl.NO_LABEL)
        q, some = sl.teacher_distribution(values, classes, V, tau)
        ref = sl.distill(layer.W, layer.b, layer.z.double().numpy(), given, values, classes, float(layer.s), tau, hard, 0.75)
        got = layer.distill(lab if hard else None, values, classes, tau, hard, 0.75)
        live = (given != sl.NO_LABEL) | some
        _, rel = layer.errors(live, max(1.0, 1 / tau))
        du = du_of(layer, given, None, q, some, tau, hard, 0.75)
        layer.check_gradients(got, ref[1:], du, live, rel + K * U + 64 * U * (1 + 8 / tau))
        again = layer.distill(lab if hard else None, values, classes, tau, hard, 0.75)
        for key in ("loss", "dz", "dW", "db"):
            assert np.array_equal(got[key], again[key]), key
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("T,B,V,Z,K", [(1, 67, 140000, 16, 256), (1, 4600, 60000, 16, 20), (1, 2, 70001, 264, 3)])
def test_the_largest_of_very_many(T, B, V, Z, K, mode):
    # more strips than a wavefront chooses from, and more logits than are held at a time
    import torch
    layer = grid_layer(T, B, V, Z, mode, 32)
    try:
        values, classes = run_topk(layer, K)
        W = layer.theta[layer.at_w:layer.at_w + V * Z].view(V, Z).float().cuda()
        b = layer.theta[layer.at_b:layer.at_b + V].float().cuda()
        for m0 in range(0, layer.M, 512):
            u = layer.z[m0:m0 + 512].float().cuda() @ W.t() + b             # (exact, as every product and sum)
            # equal values by falling order of V - class: whole numbers of 1/64
            key = (u * 64).round().long() * (1 << 22) + ((1 << 22) - 1 - torch.arange(V, device="cuda"))
            at = (1 << 22) - 1 - (torch.topk(key, K, dim=1).values & ((1 << 22) - 1))
            assert np.array_equal(classes[m0:m0 + 512], at.cpu().numpy())
            assert np.array_equal(values[m0:m0 + 512], u.gather(1, at).double().cpu().numpy())
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z", [64, 67, 320])
def test_calls_without_gradients_in_a_replayed_graph_and_on_a_stream(mode, Z):
    import torch
    layer = grid_layer(3, 50, 900, Z, mode, 33)
    bl = layer.bl
    try:
        theta, z, lab = layer.dev(layer.theta), layer.dev(layer.z).clone(), layer.dev(layer.labels("ragged"))
        side = torch.cuda.Stream()

        def made():
            return dict(logp=torch.zeros(layer.M, device="cuda"), values=torch.zeros(layer.M, 11, device="cuda"), classes=torch.zeros(layer.M, 11, dtype=torch.int32, device="cuda"),
                        s1=layer.scratch(bl.SOFTMAX_LOGPROB), s2=layer.scratch(bl.SOFTMAX_TOPK, 11))

        def calls(o, stream=None):
            bl.softmax_logprob(layer.ctx, theta, z, lab, o["logp"], o["s1"], None, stream)
            bl.softmax_topk(layer.ctx, theta, z, 11, o["values"], o["classes"], o["s2"], None, stream)

        held, eager = made(), made()
        torch.cuda.synchronize()
        calls(held, side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls(held)
        for k in range(4):
            z.copy_(layer.z[torch.randperm(layer.M, generator=torch.Generator().manual_seed(k))])
            for key in ("s1", "s2"):
                held[key].fill_(0xFF)
            graph.replay()
            calls(eager)
            torch.cuda.synchronize()
            for key in ("logp", "values", "classes"):
                assert torch.equal(held[key], eager[key]), (k, key)
    finally:
        layer.close()


@pytest.mark.parametrize("mode", [1, 0])
@pytest.mark.parametrize("Z,dims", [(64, dict(D=7, H=3)), (0, dict(D=5, H=4)), (5, dict(D=3, H=5)), (0, dict(D=3, H=133))], ids=str)
def test_other_widths_of_the_model(mode, Z, dims):
    # cells and bottlenecks of odd widths in front of W_s, z as wide as the cells of both directions
    layer = Layer(2, 33, 150, Z or 2 * dims["H"], mode, 34, **dims, **({} if Z else dict(P=0)))
    try:
        lab = layer.labels("ragged")
        live = lab != sl.NO_LABEL
        A = layer.rng.normal(size=layer.M).astype(np.float32)
        want = sl.policy(layer.W, layer.b, layer.z.double().numpy(), lab, A, None, None, float(layer.s), 0.2, 0.2, 0.0)
        got = layer.policy(lab, A, None, None, 0.2, 0.2, 0.0)
        eu, rel = layer.errors(live)
        layer.check_gradients(got, want[2:], du_of(layer, lab, np.abs(A)), live, rel + 32 * U)
    finally:
        layer.close()


def test_a_learner_on_streams_and_in_a_graph_keeps_its_scratch():
    import torch
    from paper_1904_04956_amd import binding as bl
    from paper_1904_04956_amd.harness import Learner
    lrn = Learner(T=4, B=10, D=12, H=16, L=1, P=24, V=150, mode=1)
    try:
        rng = np.random.default_rng(35)
        lrn.set_theta(rng.uniform(-0.1, 0.1, lrn.n).astype(np.float32))
        lrn.set_batch(rng.standard_normal((4, 10, 12)).astype(np.float32), rng.integers(0, 150, (4, 10)).astype(np.int32))
        lp, (values, classes) = lrn.log_probs(), lrn.top_logits(5)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for stream in (side, side.cuda_stream):
            got, (v, c) = lrn.log_probs(stream=stream), lrn.top_logits(5, stream=stream)
            side.synchronize()
            assert torch.equal(got, lp) and torch.equal(v, values) and torch.equal(c, classes)
        adv = torch.ones_like(lp)
        lrn.calgrad_policy(adv, stream=side)
        side.synchronize()
        grad = lrn.grad.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            lrn.calgrad_policy(adv)
        at = lrn.loss_scratch(bl.SOFTMAX_POLICY).data_ptr()
        for k in range(3):
            lrn.calgrad_distill(values, classes, temperature=2.0)        # (other scratch, larger)
            lrn.top_logits(100 + k)
            torch.cuda.synchronize()
            lrn.grad.fill_(-1.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(lrn.grad, grad) and lrn.loss_scratch(bl.SOFTMAX_POLICY).data_ptr() == at
    finally:
        lrn.close()
