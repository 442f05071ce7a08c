"""The softmax layer's operators beyond cross-entropy, timed and compared with their plain forms.

A case is a dict of plain values:

  call      "logprob"  log p[label] of every frame (scoring; what the policy loss keeps of the weights that sampled, and of the reference's)
            "topk"     the K largest logits of every frame with their classes (what a teacher hands to its student)
            "distill"  the loss against a teacher's top K logits at a temperature, and against labels, with its gradients
            "policy"   the clipped policy loss with a KL term to a reference, with its gradients
  T, B, H, P, V  frames, sequences, cells per direction, bottleneck (0: none, z is 2H wide), classes
  mode      0 = fp32, 1 = bf16 storage with fp32 accumulation
  K         entries a frame ("topk", "distill")
  hard      weight of the labels' cross-entropy ("distill"; 0: no labels are given)
  padded    sequences end early: frames behind a sequence's end have label -1, or no teacher entry
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TEMPERATURE, SOFT = 2.0, 0.5
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.25, 0.05


def _case(name, call, B, T=21, H=512, P=256, V=32000, mode=1, **more):
    return dict(name=name, call=call, T=T, B=B, H=H, P=P, V=V, mode=mode, **more)


def listed():
    return [
        # one frame of one stream, scored as it arrives: the smallest call, nothing but latency and one reading of the weights
        _case("logprob-frame", "logprob", 1, T=1),
        # a training batch scored with the paper-shaped softmax layer: old and reference log-probabilities
        _case("logprob-b256", "logprob", 256),
        # a model without bottleneck: z of 640, few thousand classes, every size ragged
        _case("logprob-odd640", "logprob", 50, H=320, P=0, V=3001, padded=True),
        # a teacher's top 20 for a few utterances
        _case("topk-b16", "topk", 16, K=20),
        # ... and its top 64 for a whole batch, as a corpus is annotated
        _case("topk-b256", "topk", 256, K=64),
        # a student's step on few sequences, unlabelled speech: the teacher's list alone
        _case("distill-b8", "distill", 8, K=16, hard=0.0, padded=True),
        # the paper-shaped batch: labels and the teacher's top 64
        _case("distill-b256", "distill", 256, K=64, hard=0.5, padded=False),
        # full precision, ragged in every size
        _case("distill-odd-fp32", "distill", 30, H=62, P=67, V=9001, mode=0, K=33, hard=0.5, padded=True),
        # a policy step on few sampled alignments
        _case("policy-b16", "policy", 16, padded=False),
        # the short last batch of an epoch, sequences of unequal length
        _case("policy-b173", "policy", 173, padded=True),
        # the large-batch regime
        _case("policy-b2048", "policy", 2048, padded=True),
        # the paper-shaped layer at full precision
        _case("policy-b64-fp32", "policy", 64, mode=0, padded=False),
    ]


def _width(case):
    return case["P"] if case["P"] > 0 else 2 * case["H"]


def _frames(case):
    return case["T"] * case["B"]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Flops of a case, an fp32 one weighed by the ratio of the two matrix rates."""
    return work(case)["flops"] * (16 if case["mode"] == 0 else 1)


def draw(rng):
    biggest = max(_cost(c) for c in listed())
    while True:
        call = rng.choice(["logprob", "topk", "distill", "distill", "policy", "policy"])
        c = dict(call=call, T=rng.choice([21, 21, 1, rng.randint(2, 40)]), B=_log(rng, 1, 2048), H=rng.choice([512, 320, rng.randint(32, 800)]),
                 P=rng.choice([256, 256, 0, rng.randint(33, 512)]), V=rng.choice([32000, _log(rng, 100, 32000)]), mode=rng.choice([1, 1, 1, 0]))
        if call in ("topk", "distill"):
            c["K"] = _log(rng, 1, min(128, c["V"]))
        if call == "distill":
            c["hard"] = rng.choice([0.0, 0.5])
        if call != "topk":
            c["padded"] = rng.choice([False, True])
        if _cost(c) <= biggest:
            return c


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def prepare(case, seed):
    g = _generator(seed)
    M, V, Z, K = _frames(case), case["V"], _width(case), case.get("K", 0)
    kind = torch.bfloat16 if case["mode"] == 1 else torch.float32
    uniform = lambda *shape: torch.empty(shape, device=DEVICE).uniform_(-0.1, 0.1, generator=g)  # noqa: E731
    normal = lambda *shape: torch.randn(shape, device=DEVICE, generator=g)  # noqa: E731
    W, b, z = uniform(V, Z), uniform(V), normal(M, Z)
    if case["call"] == "topk":
        # Which class comes first has to follow from the inputs and not from the order of a sum: weights on a grid of 1/512 and
        # activations on one of 1/16 (a model kept in 8 bits) make every partial sum exact in 32 bits.  Equal logits then happen.
        W, b, z = (W * 512).round() / 512, (b * 512).round() / 512, (z * 16).round().clamp(-63, 63) / 16
    W, b, z = W.to(kind), b.to(kind), z.to(kind)
    s = dict(case=case, W=W, b=b, z=z, scale=1.0 / M)
    labels = torch.randint(0, V, (M,), device=DEVICE, generator=g, dtype=torch.int32)
    if case.get("padded"):
        # time-major frames; a few sequences are empty, the first is whole
        length = torch.randint(0, case["T"] + 1, (case["B"],), device=DEVICE, generator=g)
        length[0] = case["T"]
        live = (torch.arange(case["T"], device=DEVICE)[:, None] < length[None, :]).reshape(M)
    else:
        live = torch.ones(M, dtype=torch.bool, device=DEVICE)
    if case["call"] == "distill":
        # the teacher: other weights, its K largest logits; a list ends where the teacher thought the rest not worth keeping
        u = z.float() @ (W.float() + 0.3 * uniform(V, Z)).t() + b.float()
        top, index = torch.topk(u, K, dim=1)
        del u
        used = torch.randint((K + 1) // 2, K + 1, (M, 1), device=DEVICE, generator=g)
        keep = (torch.arange(K, device=DEVICE)[None, :] < used) & live[:, None]
        s.update(values=torch.where(keep, top, torch.zeros_like(top)), indices=torch.where(keep, index, -torch.ones_like(index)).to(torch.int32))
        s["labels"] = torch.where(live, labels, -torch.ones_like(labels)) if case["hard"] else None
    elif case["call"] != "topk":
        s["labels"] = torch.where(live, labels, -torch.ones_like(labels))
    if case["call"] == "policy":
        # Log-probabilities of the same labels under the weights that sampled them and under the reference's: a little off the
        # present ones.  No ratio lies within 1e-3 of where the clip begins (a rounding would decide whether the frame counts).
        lp = _label_logp(_logits(s), s["labels"])
        d = 0.25 * normal(M)
        for edge in (-math.log(1 - CLIP_LOW), -math.log(1 + CLIP_HIGH)):
            d = torch.where((d - edge).abs() < 2e-3, d + 0.01, d)
        s.update(old=torch.where(live, lp + d, torch.zeros_like(lp)), ref=torch.where(live, lp + 0.3 * normal(M), torch.zeros_like(lp)))
        # what a sampled alignment scored above the running mean, which lags behind
        s["advantage"] = torch.where(live, 0.3 + normal(M), torch.zeros_like(lp))
    if own:
        s.update(_handle(case, s))
    return s


def _handle(case, s):
    """What a program keeps for the framework's calls: a context, the flat weights, scratch and outputs."""
    from paper_1904_04956_amd import binding as bl
    M, V, Z, K = _frames(case), case["V"], _width(case), case.get("K", 0)
    ctx = bl.blstm_create(case["T"], case["B"], 260, case["H"], 1, case["P"], V, case["mode"])
    n = bl.blstm_param_count(ctx)
    at_w, at_b = bl.blstm_param_offset(ctx, 0, 0, bl.BLSTM_WS)[0], bl.blstm_param_offset(ctx, 0, 0, bl.BLSTM_BS)[0]
    theta = torch.zeros(n, dtype=s["W"].dtype, device=DEVICE)
    theta[at_w:at_w + V * Z] = s["W"].reshape(-1)
    theta[at_b:at_b + V] = s["b"]
    call = {"logprob": bl.SOFTMAX_LOGPROB, "topk": bl.SOFTMAX_TOPK, "distill": bl.SOFTMAX_DISTILL, "policy": bl.SOFTMAX_POLICY}[case["call"]]
    h = dict(bl=bl, ctx=ctx, theta=theta, at_w=at_w, at_b=at_b, scratch=torch.empty(bl.softmax_scratch_bytes(ctx, call, K), dtype=torch.uint8, device=DEVICE))
    real = lambda *shape: torch.empty(shape, device=DEVICE)  # noqa: E731
    if case["call"] in ("logprob", "policy"):
        h["logp"] = real(M)
    if case["call"] == "topk":
        h.update(top=real(M, K), index=torch.empty((M, K), dtype=torch.int32, device=DEVICE))
    if case["call"] in ("distill", "policy"):
        h.update(loss=real(1), dz=torch.empty_like(s["z"]), grad=torch.zeros(n, device=DEVICE))
    h["closed"] = _Closed(bl, ctx)
    return h


class _Closed:
    """Destroys the context with the state."""

    def __init__(self, bl, ctx):
        self.bl, self.ctx = bl, ctx

    def __del__(self):
        self.bl.blstm_destroy(self.ctx)


def run(s):
    call = s["case"]["call"]
    if own:
        return _run_own(s, call)
    return {"logprob": _logprob, "topk": _topk, "distill": _distill, "policy": _policy}[call](s)


def _run_own(s, call):
    bl, c, V, Z = s["bl"], s["case"], s["case"]["V"], _width(s["case"])
    if call == "logprob":
        bl.softmax_logprob(s["ctx"], s["theta"], s["z"], s["labels"], s["logp"], s["scratch"])
        return {"logp": s["logp"]}
    if call == "topk":
        bl.softmax_topk(s["ctx"], s["theta"], s["z"], c["K"], s["top"], s["index"], s["scratch"])
        return {"values": s["top"], "indices": s["index"]}
    out = {}
    if call == "distill":
        bl.softmax_distill_fwd_bwd(s["ctx"], s["theta"], s["z"], s["labels"], s["values"], s["indices"], c["K"], TEMPERATURE, c["hard"], SOFT,
                                   s["loss"], s["dz"], s["grad"], s["scratch"])
    else:
        bl.softmax_policy_fwd_bwd(s["ctx"], s["theta"], s["z"], s["labels"], s["advantage"], s["old"], s["ref"], CLIP_LOW, CLIP_HIGH, KL,
                                  s["loss"], s["logp"], s["dz"], s["grad"], s["scratch"])
        out["logp"] = s["logp"]
    out.update(loss=s["loss"], dz=s["dz"], dW=s["grad"][s["at_w"]:s["at_w"] + V * Z].view(V, Z), db=s["grad"][s["at_b"]:s["at_b"] + V])
    return out


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _logits(s):
    return s["z"].float() @ s["W"].float().t() + s["b"].float()


def _softmax(u):
    """exp(u - max) of every row, their sums and the maxima."""
    top = u.amax(1, keepdim=True)
    e = torch.exp(u - top)
    return e, e.sum(1, keepdim=True), top


def _at(u, labels):
    return u.gather(1, labels.clamp(min=0).long()[:, None])[:, 0]


def _label_logp(u, labels):
    _, total, top = _softmax(u)
    return torch.where(labels >= 0, _at(u, labels) - top[:, 0] - torch.log(total[:, 0]), torch.zeros_like(total[:, 0]))


def _logprob(s):
    return {"logp": _label_logp(_logits(s), s["labels"])}


def _topk(s):
    u = _logits(s)
    # one whole number for a logit and its class: larger for the larger logit, and among equal ones for the lower class
    bits = (u + 0.0).view(torch.int32).long()
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
    key = order * (1 << 24) + ((1 << 24) - 1 - torch.arange(u.shape[1], device=u.device))
    key = torch.topk(key, s["case"]["K"], dim=1).values
    index = (1 << 24) - 1 - (key & ((1 << 24) - 1))
    return {"values": u.gather(1, index), "indices": index.to(torch.int32)}


def _gradients(s, du):
    W, z = s["W"].float(), s["z"].float()
    return {"dz": (du @ W).to(s["z"].dtype), "dW": du.t() @ z, "db": du.sum(0)}


def _distill(s):
    c, labels, scale, tau = s["case"], s["labels"], s["scale"], TEMPERATURE
    u = _logits(s)
    used = s["indices"] >= 0
    index = s["indices"].clamp(min=0).long()
    some = used.any(1, keepdim=True)
    t = torch.where(used, s["values"] / tau, torch.full_like(s["values"], -math.inf))
    e = torch.where(used, torch.exp(t - torch.where(some, t.amax(1, keepdim=True), torch.zeros_like(t[:, :1]))), torch.zeros_like(t))
    q = e / torch.where(some, e.sum(1, keepdim=True), torch.ones_like(t[:, :1]))
    es, total, top = _softmax(u / tau)
    log_p = u.gather(1, index) / tau - top - torch.log(total)
    log_q = torch.log(torch.where(used & (q > 0), q, torch.ones_like(q)))
    loss = SOFT * tau * tau * torch.where(used, q * (log_q - log_p), torch.zeros_like(q)).sum(1)
    weight = scale * SOFT * tau
    du = torch.where(some, es * (weight / total), torch.zeros_like(es))
    du.scatter_add_(1, index, -weight * q)
    if c["hard"]:
        eh, total, top = _softmax(u)
        labelled = labels >= 0
        loss = loss + c["hard"] * torch.where(labelled, top[:, 0] + torch.log(total[:, 0]) - _at(u, labels), torch.zeros_like(loss))
        du += torch.where(labelled[:, None], eh * (scale * c["hard"] / total), torch.zeros_like(eh))
        du.scatter_add_(1, labels.clamp(min=0).long()[:, None], torch.where(labelled, -scale * c["hard"], 0.0)[:, None])
    return {"loss": (scale * loss.double().sum()).float()[None], **_gradients(s, du)}


def _policy(s):
    labels, scale = s["labels"], s["scale"]
    live = labels >= 0
    u = _logits(s)
    e, total, top = _softmax(u)
    nothing = torch.zeros_like(total[:, 0])
    lp = torch.where(live, _at(u, labels) - top[:, 0] - torch.log(total[:, 0]), nothing)
    ratio, a, off = torch.exp(lp - s["old"]), s["advantage"], s["ref"] - lp
    loss = -torch.minimum(ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a) + KL * (torch.exp(off) - off - 1)
    cut = ((a > 0) & (ratio > 1 + CLIP_HIGH)) | ((a < 0) & (ratio < 1 - CLIP_LOW))
    g = torch.where(cut, nothing, -ratio * a) + KL * (1 - torch.exp(off))
    g = torch.where(live, scale * g, nothing)
    du = e * (-g[:, None] / total)
    du.scatter_add_(1, labels.clamp(min=0).long()[:, None], g[:, None])
    return {"loss": (scale * torch.where(live, loss, nothing).double().sum()).float()[None], "logp": lp, **_gradients(s, du)}


# ---- the definitions in 64 bits, some rows at a time -----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    W, b, z = s["W"].double(), s["b"].double(), s["z"].double()
    M, V = z.shape[0], W.shape[0]
    if _frames(case) * V * _width(case) * 6 > 6e12:
        return None
    call, out = case["call"], {}
    dW, db, loss, rows = torch.zeros_like(W), torch.zeros_like(b), 0.0, {"logp": [], "values": [], "dz": []}
    for m in range(0, M, 2048):
        part = slice(m, min(M, m + 2048))
        u = z[part] @ W.t() + b
        n = u.shape[0]
        at = torch.arange(n, device=u.device)
        if call == "topk":
            rows["values"].append(torch.sort(u, dim=1, descending=True).values[:, :case["K"]])
            continue
        lab = s["labels"][part].long() if s["labels"] is not None else torch.full((n,), -1, device=u.device)
        live = lab >= 0
        hot = torch.zeros_like(u)
        hot[at[live], lab[live]] = 1.0
        logp_all = u - torch.logsumexp(u, 1, keepdim=True)
        lp = (hot * logp_all).sum(1)
        if call in ("logprob", "policy"):
            rows["logp"].append(lp)
        if call == "logprob":
            continue
        if call == "policy":
            A, old, ref = (s[k][part].double() for k in ("advantage", "old", "ref"))
            r = torch.exp(lp - old)
            lo, hi = 1 - CLIP_LOW, 1 + CLIP_HIGH
            inner, outer = r * A, torch.clamp(r, lo, hi) * A
            kl = torch.exp(ref - lp) - (ref - lp) - 1
            loss = loss + (torch.where(live, KL * kl - torch.minimum(inner, outer), 0.0)).sum()
            slope = torch.where(inner <= outer, -r * A, 0.0) + KL * (1 - torch.exp(ref - lp))
            du = (slope * live)[:, None] * (hot - torch.exp(logp_all))
        else:
            soft = u / TEMPERATURE - torch.logsumexp(u / TEMPERATURE, 1, keepdim=True)
            target = torch.zeros_like(u)
            idx, val = s["indices"][part].long(), s["values"][part].double() / TEMPERATURE
            ok = idx >= 0
            any_ = ok.any(1)
            val = torch.where(ok, val, -math.inf)
            q = torch.where(any_[:, None], torch.exp(val - torch.logsumexp(val, 1, keepdim=True)), 0.0)
            target[at[:, None].expand_as(idx)[ok], idx[ok]] = q[ok]
            loss = loss + SOFT * TEMPERATURE ** 2 * (torch.special.xlogy(target, target) - target * soft).sum() - case["hard"] * lp.sum()
            du = SOFT * TEMPERATURE * (torch.exp(soft) * any_[:, None] - target) + case["hard"] * (torch.exp(logp_all) * live[:, None] - hot)
        du = du * s["scale"]
        rows["dz"].append(du @ W)
        dW += du.t() @ z[part]
        db += du.sum(0)
    for k, v in rows.items():
        if v:
            out[k] = torch.cat(v)
    if call == "topk":
        return {"values": out["values"], "indices": None}
    if call in ("distill", "policy"):
        out.update(loss=(loss * s["scale"]).reshape(1), dW=dW, db=db)
    return out


def work(case):
    M, V, Z, e = _frames(case), case["V"], _width(case), 2 if case["mode"] == 1 else 4
    products, read, written = 1, (V * Z + V + M * Z) * e, 0
    if case["call"] != "topk":
        read += 4 * M
    if case["call"] == "logprob":
        written = 4 * M
    if case["call"] == "topk":
        written = 8 * M * case["K"]
    if case["call"] in ("distill", "policy"):
        products, written = 3, M * Z * e + 4 * V * (Z + 1) + 4
    if case["call"] == "distill":
        read += 8 * M * case["K"]
    if case["call"] == "policy":
        read, written = read + 12 * M, written + 4 * M
    return {"bytes": read + written, "flops": 2 * products * M * V * Z}
