"""Device-memory plumbing around the C-ABI calls: one learner's buffers and step order.

PyTorch allocates the buffers and provides the stream; every computation is a call
into the library through `binding`.  Used by the GPU tests, the smoke check and the
benchmark.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as bl
from . import inputs


def checked(name, tensor, dtype, shape, device):
    """`tensor`, if it is what a call reads or writes: the library sees an address and nothing else."""
    if not isinstance(tensor, torch.Tensor):
        raise TypeError(f"{name} must be a tensor, not {type(tensor).__name__}")
    if tensor.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {tensor.dtype}")
    if tuple(tensor.shape) != tuple(shape) or not tensor.is_contiguous():
        raise ValueError(f"{name} must be {tuple(shape)} and contiguous, not {tuple(tensor.shape)} with strides {tensor.stride()}")
    if tensor.device != device:
        raise ValueError(f"{name} must be on {device}, not on {tensor.device}")
    return tensor


class Learner:
    """Buffers of one learner: master weights, bf16 shadow, gradient, batch, workspace."""

    def __init__(self, T, B, D, H, L, P, V, mode, loss_scale=0.0, device="cuda:0", momentum=0.0, recurrent_path=0, recurrent_sync=None, keep_weight_copies=True,
                 defer_softmax_wgrad=True):
        if not torch.cuda.is_available():
            raise RuntimeError("a GPU is required: the HIP path has no CPU fallback")
        self.dims = dict(T=T, B=B, D=D, H=H, L=L, P=P, V=V)
        self.mode = mode
        self.device = torch.device(device)
        self.ctx = bl.blstm_create(T, B, D, H, L, P, V, mode, loss_scale)
        # the copies the passes derive from the weights are kept across steps: every method below that changes the
        # weights reports it (weights_changed)
        self.options = {bl.BLSTM_OPT_KEEP_WEIGHT_COPIES: int(bool(keep_weight_copies))}
        if recurrent_path:
            self.options[bl.BLSTM_OPT_RECURRENT_PATH] = recurrent_path
        if recurrent_sync is not None:
            self.options[bl.BLSTM_OPT_RECURRENT_SYNC] = recurrent_sync
        for option, value in self.options.items():
            bl.blstm_set_option(self.ctx, option, value)
        # calgrad() always runs softmax_xent_fwd_bwd and blstm_backward back to back on the same gradient vector, so the
        # softmax layer's weight gradient may join the backward pass's grouped launch
        bl.blstm_set_option(self.ctx, bl.BLSTM_OPT_DEFER_SOFTMAX_WGRAD, int(bool(defer_softmax_wgrad)))
        self.defer_softmax_wgrad = bool(defer_softmax_wgrad)
        self.n = bl.blstm_param_count(self.ctx)
        self.zdim = P if P > 0 else 2 * H
        self.act_dtype = torch.bfloat16 if mode == 1 else torch.float32
        dev = self.device
        self.workspace = torch.empty(bl.blstm_workspace_bytes(self.ctx), dtype=torch.uint8, device=dev)
        bl.blstm_bind(self.ctx, self.workspace)
        self.theta = torch.zeros(self.n, dtype=torch.float32, device=dev)
        self.shadow = torch.zeros(self.n, dtype=torch.bfloat16, device=dev) if mode == 1 else None
        self.grad = torch.zeros(self.n, dtype=torch.float32, device=dev)
        self.velocity = torch.zeros(self.n, dtype=torch.float32, device=dev) if momentum != 0.0 else None
        self.momentum = momentum
        self.x = torch.zeros((T, B, D), dtype=self.act_dtype, device=dev)
        self.labels = torch.zeros((T, B), dtype=torch.int32, device=dev)
        self.z = torch.zeros((T, B, self.zdim), dtype=self.act_dtype, device=dev)
        self.dz = torch.zeros((T, B, self.zdim), dtype=self.act_dtype, device=dev)
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        self.scratch = {}         # of the calls that take scratch, each made when it is first used
        self.adapters = None      # attach_adapters()
        self.held = None          # HYBRID only: the pulled weights the next gradient is taken on

    def close(self):
        if self.ctx is not None:
            bl.blstm_destroy(self.ctx)
            self.ctx = None
        if getattr(self, "adapters", None) is not None:
            self.adapters.close()
            self.adapters = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- data in ---------------------------------------------------------------------
    def set_theta(self, theta_f32: np.ndarray):
        assert theta_f32.dtype == np.float32 and theta_f32.size == self.n
        self.theta.copy_(torch.from_numpy(theta_f32))
        if self.shadow is not None:
            bl.blstm_shadow_refresh(self.theta, self.shadow, self.n)
        self.weights_changed()

    def weights_changed(self):
        """To be called after anything has written the weights (or the held copy) outside this class."""
        bl.blstm_weights_changed(self.ctx)
        if self.adapters is not None:
            bl.blstm_weights_changed(self.adapters.stack)

    def set_batch(self, x_f32: np.ndarray, labels_i32: np.ndarray):
        self.x.copy_(torch.from_numpy(x_f32).to(self.act_dtype))
        self.labels.copy_(torch.from_numpy(labels_i32.astype(np.int32)))

    @property
    def theta_fwd(self):
        """The weights as the forward and backward passes read them."""
        return self.shadow if self.mode == 1 else self.theta

    # ---- the step ----------------------------------------------------------------------
    def forward(self, stream=None):
        bl.blstm_forward(self.ctx, self.theta_fwd, self.x, self.z, stream)

    def calgrad(self, stream=None, weights=None):
        """g = calGrad(W): forward, softmax cross-entropy, backward (on `weights` if given, in the
        storage type of the mode, else on the learner's own)."""
        th = self.theta_fwd if weights is None else weights
        bl.blstm_forward(self.ctx, th, self.x, self.z, stream)
        bl.softmax_xent_fwd_bwd(self.ctx, th, self.z, self.labels, self.loss, self.dz, self.grad, stream)
        bl.blstm_backward(self.ctx, th, self.x, self.dz, self.grad, stream)

    # ---- the softmax layer beyond cross-entropy ------------------------------------------
    # (tensors of frames are [T][B] or [T B], float32, labels and classes int32, all contiguous and on the learner's device: else TypeError or ValueError)
    def _frames(self, name, tensor, dtype=torch.float32, width=()):
        T, B = self.labels.shape
        flat = isinstance(tensor, torch.Tensor) and tensor.shape[:1] == (T * B,) and tensor.dim() == 1 + len(width)
        return checked(name, tensor, dtype, (T * B, *width) if flat else (T, B, *width), self.x.device)

    def loss_scratch(self, call, K=0, stream=None):
        """Scratch of one of the softmax layer's calls (binding.SOFTMAX_*), kept for the next time: a captured graph holds its address."""
        # (only a distillation's size depends on K)
        n, key = bl.softmax_scratch_bytes(self.ctx, call, K), (call, K if call == bl.SOFTMAX_DISTILL else 0)
        if key not in self.scratch:
            self.scratch[key] = self._empty((n,), torch.uint8, stream)
        return self.scratch[key]

    def _empty(self, shape, dtype, stream):
        """Memory for a call on `stream` (the allocator hands out what other work on the stream that it belongs to may still be writing)."""
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=self.device)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _forward_on(self, weights, stream):
        """A forward pass on `weights` if given, else on the learner's own; returns which."""
        if weights is None:
            self.forward(stream)
            return self.theta_fwd
        checked("weights", weights, self.act_dtype, (self.n,), self.x.device)
        # the copies that passes keep go by address, and another call's weights may have lain at this one
        self.weights_changed()
        bl.blstm_forward(self.ctx, weights, self.x, self.z, stream)
        return weights

    def log_probs(self, labels=None, weights=None, stream=None):
        """log p[label] [T][B] of the batch (of `labels` if given, else its own): a forward pass (without adapters), then the softmax layer."""
        labels = self.labels if labels is None else self._frames("labels", labels, torch.int32)
        th = self._forward_on(weights, stream)
        out = self._empty(self.labels.shape, torch.float32, stream)
        bl.softmax_logprob(self.ctx, th, self.z, labels, out, self.loss_scratch(bl.SOFTMAX_LOGPROB, 0, stream), None, stream)
        return out

    def top_logits(self, K, weights=None, stream=None):
        """Values and classes [T][B][K] of the batch's K largest logits (without adapters): what a student's calgrad_distill takes."""
        th = self._forward_on(weights, stream)
        shape = (*self.labels.shape, K)
        values, classes = self._empty(shape, torch.float32, stream), self._empty(shape, torch.int32, stream)
        bl.softmax_topk(self.ctx, th, self.z, K, values, classes, self.loss_scratch(bl.SOFTMAX_TOPK, K, stream), None, stream)
        return values, classes

    def calgrad_distill(self, values, classes, temperature=1.0, hard_weight=0.5, soft_weight=0.5, stream=None):
        """calgrad() with the loss against a teacher's lists [T][B][K] (and, with a hard_weight, the batch's labels)."""
        K = classes.shape[-1] if isinstance(classes, torch.Tensor) and classes.dim() > 0 else 0
        self._frames("classes", classes, torch.int32, (K,))
        self._frames("values", values, torch.float32, (K,))
        bl.blstm_forward(self.ctx, self.theta_fwd, self.x, self.z, stream)
        bl.softmax_distill_fwd_bwd(self.ctx, self.theta_fwd, self.z, self.labels if hard_weight != 0 else None, values, classes, K, temperature, hard_weight,
                                   soft_weight, self.loss, self.dz, self.grad, self.loss_scratch(bl.SOFTMAX_DISTILL, K, stream), None, stream)
        bl.blstm_backward(self.ctx, self.theta_fwd, self.x, self.dz, self.grad, stream)

    def calgrad_policy(self, advantage, old_logp=None, ref_logp=None, clip_low=0.2, clip_high=0.2, kl_weight=0.0, logp=None, stream=None):
        """calgrad() with the clipped policy loss on the batch's labels, which were sampled."""
        self._frames("advantage", advantage)
        for name, t in (("old_logp", old_logp), ("ref_logp", ref_logp), ("logp", logp)):
            if t is not None:
                self._frames(name, t)
        bl.blstm_forward(self.ctx, self.theta_fwd, self.x, self.z, stream)
        bl.softmax_policy_fwd_bwd(self.ctx, self.theta_fwd, self.z, self.labels, advantage, old_logp, ref_logp, clip_low, clip_high, kl_weight, self.loss, logp,
                                  self.dz, self.grad, self.loss_scratch(bl.SOFTMAX_POLICY, 0, stream), None, stream)
        bl.blstm_backward(self.ctx, self.theta_fwd, self.x, self.dz, self.grad, stream)

    def apply(self, lr, stream=None):
        """W' = apply(W, g)."""
        bl.sgd_step(self.theta, self.shadow, self.grad, self.n, lr, self.momentum, self.velocity, stream)
        self.weights_changed()

    def apply_muon(self, lr, lr_rest, momentum=0.95, weight_decay=0.0, nesterov=True, gates=False, softmax=False, full=False, stream=None):
        """W' = apply(W, g) with the matrices' updates orthogonalised (binding.muon_step): the LSTM's and the bottleneck's at lr, with `softmax` the softmax
        layer's too; the rest at lr_rest.  `gates`: each gate's block is a matrix of its own.  `full`: mode 1 is as exact as mode 0.  The velocity is the learner's (made of zeros at first
        use, which a graph cannot hold)."""
        if momentum != 0.0 and self.velocity is None:
            self.velocity = self._zeros((self.n,), torch.float32, stream)
        flags = (bl.MUON_NESTEROV if nesterov else 0) | (bl.MUON_GATES if gates else 0) | (bl.MUON_SOFTMAX if softmax else 0) | (bl.MUON_FULL if full else 0)
        bl.muon_step(self.ctx, self.theta, self.shadow, self.grad, self.velocity, lr, lr_rest, momentum, weight_decay, flags,
                     self._kept(("muon", flags), lambda: bl.muon_scratch_bytes(self.ctx, flags), stream), None, stream)
        self.weights_changed()

    def _kept(self, key, nbytes, stream):
        """Scratch of a call, kept for the next time: a captured graph holds its address."""
        if key not in self.scratch:
            self.scratch[key] = self._empty((nbytes(),), torch.uint8, stream)
        return self.scratch[key]

    def _zeros(self, shape, dtype, stream):
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=self.device)
        with torch.cuda.stream(stream):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("zeros made while a graph is captured would be made again by every replay: call once before")
            return torch.zeros(shape, dtype=dtype, device=self.device)

    # ---- low-rank adapters beside the bottleneck's projection ------------------------------
    def attach_adapters(self, count, rank, scale=1.0):
        """`count` adapters of `rank` beside the bottleneck (binding.adapter_forward, W = W_p), each sequence's by adapters.ids [B] (BLSTM_NO_ADAPTER at first).
        Their factors are adapters.A [count][rank][2H] and .Bm [count][P][rank], float, zero at first (write one of the two: both gradients are zero where both factors are); after writing
        them call adapters.refresh().  They take part in forward_adapted and calgrad_adapted; all other passes of the learner are the model's without them."""
        if self.dims["P"] == 0:
            raise ValueError("adapters stand beside the bottleneck's projection, and this model has none")
        if self.adapters is not None:
            self.adapters.close()
            self.adapters = None
        self.adapters = Adapters(self, count, rank, scale)
        return self.adapters

    def _attached(self):
        if self.adapters is None:
            raise ValueError("no adapters are attached")
        return self.adapters

    def forward_adapted(self, stream=None):
        """z of the batch with each sequence's adapter."""
        a = self._attached()
        bl.blstm_forward(a.stack, self.theta_fwd, self.x, a.h, stream)
        bl.adapter_forward(a.cfg, a.W, a.b, a.A_fwd, a.Bm_fwd, a.ids, a.h, self.z, a.t, a.scratch(bl.ADAPTER_FORWARD, self, stream), None, stream)

    def calgrad_adapted(self, shared=True, stream=None):
        """calgrad() with the adapters: their gradients in adapters.dA and .dB and, with `shared`, the model's in grad (without: the softmax layer's alone; elsewhere grad is
        what it was, and not for an apply())."""
        a = self._attached()
        a.take_ids(stream)
        self.forward_adapted(stream)
        # the backward pass runs on the stack's own context, so nothing of the softmax layer's gradient may be left to this one's
        bl.blstm_set_option(self.ctx, bl.BLSTM_OPT_DEFER_SOFTMAX_WGRAD, 0)
        try:
            bl.softmax_xent_fwd_bwd(self.ctx, self.theta_fwd, self.z, self.labels, self.loss, self.dz, self.grad, stream)
        finally:
            bl.blstm_set_option(self.ctx, bl.BLSTM_OPT_DEFER_SOFTMAX_WGRAD, int(self.defer_softmax_wgrad))
        bl.adapter_backward(a.cfg, a.W, a.A_fwd, a.Bm_fwd, a.ids, a.h, a.t, self.dz, a.dh if shared else None, a.dA, a.dB, a.dW if shared else None,
                            a.db if shared else None, a.scratch(bl.ADAPTER_BACKWARD, self, stream), None, stream)
        if shared:
            bl.blstm_backward(a.stack, self.theta_fwd, self.x, a.dh, self.grad, stream)

    def apply_adapters(self, lr, momentum=0.95, weight_decay=0.0, nesterov=True, stream=None):
        """The orthogonalised update of both factors of the adapters that the batch of the last calgrad_adapted had (binding.muon_adapters_step)."""
        a = self._attached()
        for name, theta, shadow, grad, velocity in (("A", a.A, a.A_bf16, a.dA, a.vA), ("B", a.Bm, a.Bm_bf16, a.dB, a.vB)):
            sizes = (*theta.shape, self.mode)
            bl.muon_adapters_step(theta, shadow, grad, velocity, a.ids_taken, a.ids_taken.numel(), *sizes, lr, momentum, weight_decay, bl.MUON_NESTEROV if nesterov else 0,
                                  self._kept(("muon", name, sizes), lambda: bl.muon_orthogonalize_scratch_bytes(*sizes), stream), None, stream)

    def hold(self):
        """Keeps a copy of the weights as forward/backward read them now (a device-to-device copy on
        torch's current stream): what pull_weights() returned, for the next iteration's gradient."""
        if self.held is None:
            self.held = torch.empty_like(self.theta_fwd)
        self.held.copy_(self.theta_fwd)
        self.weights_changed()

    def train_step(self, lr, stream=None):
        self.calgrad(stream)
        self.apply(lr, stream)

    def check_status(self, stream=None):
        """Synchronises and raises if a persistent kernel abandoned a wait."""
        bl.blstm_device_status(self.ctx, stream)
        if self.adapters is not None:
            bl.blstm_device_status(self.adapters.stack, stream)

    # ---- data out --------------------------------------------------------------------
    def loss_value(self) -> float:
        return float(self.loss.cpu()[0])

    def grad_numpy(self) -> np.ndarray:
        return self.grad.cpu().numpy()

    def theta_numpy(self) -> np.ndarray:
        return self.theta.cpu().numpy()

    def z_numpy(self) -> np.ndarray:
        return self.z.float().cpu().numpy()


class Adapters:
    """Buffers of a learner's adapters, and a context of the LSTM stack alone: its z is what the bottleneck's projection reads, and its parameters are the
    beginning of the model's vector."""

    def __init__(self, learner, count, rank, scale):
        d, dev, kind = learner.dims, learner.device, learner.act_dtype
        T, B, K, N = d["T"], d["B"], 2 * d["H"], d["P"]
        self.cfg = bl.adapter_config(T, B, K, N, rank, count, learner.mode, scale)
        bl.adapter_scratch_bytes(self.cfg, bl.ADAPTER_BACKWARD)          # refuses what the calls would
        self.stack = bl.blstm_create(T, B, d["D"], d["H"], d["L"], 0, 1, learner.mode)
        for option, value in learner.options.items():
            bl.blstm_set_option(self.stack, option, value)
        self.workspace = torch.empty(bl.blstm_workspace_bytes(self.stack), dtype=torch.uint8, device=dev)
        bl.blstm_bind(self.stack, self.workspace)
        real = lambda *shape: torch.zeros(shape, dtype=torch.float32, device=dev)  # noqa: E731
        self.A, self.Bm, self.dA, self.dB, self.vA, self.vB = (real(count, *s) for s in 3 * ((rank, K), (N, rank)))
        self.A_bf16, self.Bm_bf16 = (torch.zeros_like(t, dtype=torch.bfloat16) if learner.mode == 1 else None for t in (self.A, self.Bm))
        self.ids, self.ids_taken = (torch.full((B,), bl.BLSTM_NO_ADAPTER, dtype=torch.int32, device=dev) for _ in range(2))
        self.h, self.dh = (torch.zeros((T, B, K), dtype=kind, device=dev) for _ in range(2))
        self.t = real(T, B, rank)
        part = lambda flat, which: flat[slice(*(lambda o, n: (o, o + n))(*bl.blstm_param_offset(learner.ctx, 0, 0, which)))]  # noqa: E731
        self.W, self.b = part(learner.theta_fwd, bl.BLSTM_WP), part(learner.theta_fwd, bl.BLSTM_BP)
        self.dW, self.db = part(learner.grad, bl.BLSTM_WP), part(learner.grad, bl.BLSTM_BP)

    @property
    def A_fwd(self):
        return self.A if self.A_bf16 is None else self.A_bf16

    @property
    def Bm_fwd(self):
        return self.Bm if self.Bm_bf16 is None else self.Bm_bf16

    def scratch(self, call, learner, stream):
        return learner._kept(("adapt", call, self.cfg.rank, self.cfg.count), lambda: bl.adapter_scratch_bytes(self.cfg, call), stream)

    def take_ids(self, stream=None):
        """Keeps whose gradients dA and dB are: ids may be the next batch's when the update comes."""
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=self.ids.device)
        with torch.cuda.stream(stream):
            torch.add(self.ids, 0, out=self.ids_taken)               # (a kernel: a captured copy would be a node of another kind)

    def refresh(self, stream=None):
        """After writing A or Bm: their bf16 copies anew."""
        for master, copy in ((self.A, self.A_bf16), (self.Bm, self.Bm_bf16)):
            if copy is not None:
                bl.blstm_shadow_refresh(master, copy, master.numel(), stream)

    def close(self):
        if self.stack is not None:
            bl.blstm_destroy(self.stack)
            self.stack = None


def learner_for(workload: inputs.Workload, B=None, device="cuda:0", momentum=0.0) -> Learner:
    d = workload.dims()
    if B is not None:
        d["B"] = B
    return Learner(mode=workload.mode, device=device, momentum=momentum, **d)


def mix(learners, partner, stream=None):
    """One ADPSGD averaging step over the learners' weights (and their bf16 shadows)."""
    masters = [l.theta for l in learners]
    shadows = [l.shadow for l in learners] if learners[0].shadow is not None else None
    bl.adpsgd_mix(masters, shadows, learners[0].n, len(learners), partner, stream)
    for l in learners:
        l.weights_changed()


# ---- the strategies of section 3.2 as orders of the library's calls, R learners in one GPU's memory ----

def adpsgd_step(learners, lr, partner, fused=False, stream=None):
    """Eq. 4 in the synchronous order: g_i = calGrad(W_i), W_i' = apply(W_i, g_i), then the pairs average.
    With fused=True each pair's update and average are one pass over the weights (sgd_mix_pair)."""
    for l in learners:
        l.calgrad(stream)
    if not fused:
        for l in learners:
            l.apply(lr, stream)
        mix(learners, partner, stream)
        return
    for i, j in enumerate(partner):
        a = learners[i]
        if j == i:
            a.apply(lr, stream)
        elif j > i:
            b = learners[j]
            bl.sgd_mix_pair(a.theta, b.theta, a.shadow, b.shadow, a.grad, b.grad, a.n, lr, a.momentum,
                            a.velocity, b.velocity, stream)
            a.weights_changed(); b.weights_changed()


def stale_adpsgd_step(learners, lr, partner, stream=None):
    """The integration order of Fig. 3b: the gradient is computed on the learner's own weights, the
    weights are then replaced by the pair's average (pull) and the gradient is applied to that."""
    for l in learners:
        l.calgrad(stream)
    mix(learners, partner, stream)
    for l in learners:
        l.apply(lr, stream)


def sync_step(learners, lr, stream=None):
    """SYNC of Fig. 3a: every learner applies its own gradient, then all take the mean of the results."""
    for l in learners:
        l.calgrad(stream)
        l.apply(lr, stream)
    masters = [l.theta for l in learners]
    shadows = [l.shadow for l in learners] if learners[0].shadow is not None else None
    bl.sync_average(masters, shadows, learners[0].n, len(learners), stream)
    for l in learners:
        l.weights_changed()


def hybrid_step(learners, lr):
    """HYBRID of Fig. 3c with its push as an average over all learners (section 3.2): the gradient is taken
    on the weights pulled in the iteration before (the common initial weights at first), the pull is the
    mean of what every learner pushed at the end of that iteration (sync_average over the masters), and the
    gradient is applied to the pulled weights.  Runs on the default stream (the held copy is a torch copy)."""
    for l in learners:
        l.calgrad(weights=l.held)
    masters = [l.theta for l in learners]
    shadows = [l.shadow for l in learners] if learners[0].shadow is not None else None
    bl.sync_average(masters, shadows, learners[0].n, len(learners))
    for l in learners:
        l.weights_changed()
        l.hold()
        l.apply(lr)
