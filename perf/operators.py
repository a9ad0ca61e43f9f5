"""The operators at the two ends of the Actor's backward pass, as cases that can be timed and compared.

  policy  rlhf_op_policy_loss: clipped policy loss with a KL term over logits; log-probs, loss, gradient
  embed   rlhf_op_embed: embedding lookup with scaling
  egrad   rlhf_op_embed_grad: the table's gradient, rows summed by token
  clip    rlhf_op_grad_norm and rlhf_op_clip_grads: global 2-norm of many gradients, and their scaling

With `own` false a pass computes the same in elementary torch operations.  Widths, vocabularies and batch sizes
are those of the repository's model shapes, or generic.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one token of each sample of the smallest configuration: latency alone
        dict(name="policy_8x4096_fp32", kind="policy", rows=8, vocab=4096, dtype="fp32", grad=True, kl=0.05, masked=0.0, pad=0),
        # a short micro-batch, logits as the float GEMM leaves them
        dict(name="policy_64x32000_fp32", kind="policy", rows=64, vocab=32000, dtype="fp32", grad=True, kl=0.05, masked=0.0, pad=0),
        # the mini-batch of an update: as many rows as a scoring pass holds, a tenth of them prompt or padding
        dict(name="policy_8192x32000_bf16", kind="policy", rows=8192, vocab=32000, dtype="bf16", grad=True, kl=0.05, masked=0.1, pad=0),
        # evaluation of a batch without an update: loss, KL and clipped share only
        dict(name="policy_4096x32000_fp32_eval", kind="policy", rows=4096, vocab=32000, dtype="fp32", grad=False, kl=0.05, masked=0.1, pad=0),
        # a wide odd vocabulary, half logits with a loss scale, padded rows of the logits, no KL
        dict(name="policy_1500x100003_fp16", kind="policy", rows=1500, vocab=100003, dtype="fp16", grad=True, kl=0.0, masked=0.3, pad=61),
        # a decode step of the widest batch: rows of bf16 weights into the float residual stream
        dict(name="embed_256x4096", kind="embed", rows=256, d=4096, vocab=32000, dtype="bf16", out="fp32", scale=1.0),
        # a training pass of the same model, scaled lookup
        dict(name="embed_8192x4096", kind="embed", rows=8192, d=4096, vocab=32000, dtype="bf16", out="bf16", scale=64.0),
        # a short micro-batch added to a gradient that is there already
        dict(name="egrad_61x768_acc", kind="egrad", rows=61, d=768, vocab=32000, dtype="fp32", out="fp32", scale=1.0, accumulate=True, hot=0.0),
        # a training pass: the whole table's gradient, most of it zero
        dict(name="egrad_8192x4096", kind="egrad", rows=8192, d=4096, vocab=32000, dtype="bf16", out="fp32", scale=64.0, accumulate=False, hot=0.0),
        # a padded batch: half the rows carry one token
        dict(name="egrad_32768x768_hot", kind="egrad", rows=32768, d=768, vocab=32000, dtype="fp16", out="fp16", scale=1.0, accumulate=False, hot=0.5),
        # the smallest configuration, every layer's matrices on their own
        dict(name="clip_tiny_fp32", kind="clip", layers=2, d=256, qkv=768, ffn=688, vocab=4096, dtype="fp32", max_norm=1.0, odd=False),
        # four layers of a wide model, bf16 gradients
        dict(name="clip_4_layers_4096_bf16", kind="clip", layers=4, d=4096, qkv=12288, ffn=11008, vocab=32000, dtype="bf16", max_norm=1.0, odd=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(("policy", "policy", "embed", "egrad", "egrad", "clip"))
        dt, odt = rng.choice(tuple(DTYPES)), rng.choice(tuple(DTYPES))
        if kind == "policy":
            c = dict(kind=kind, rows=_log_int(rng, 1, 16384), vocab=_log_int(rng, 1000, 160000), dtype=dt, grad=rng.random() < 0.7,
                     kl=rng.choice((0.0, 0.02, 0.1)), masked=rng.choice((0.0, 0.1, 0.5)), pad=rng.choice((0, 0, 13)))
        elif kind == "clip":
            d = _log_int(rng, 8, 256) * 32
            c = dict(kind=kind, layers=_log_int(rng, 1, 24), d=d, qkv=3 * d, ffn=_log_int(rng, 2 * d, 4 * d), vocab=_log_int(rng, 1000, 64000),
                     dtype=dt, max_norm=rng.choice((0.5, 1.0)), odd=rng.random() < 0.5)
        else:
            c = dict(kind=kind, rows=_log_int(rng, 1, 65536), d=_log_int(rng, 48, 8192), vocab=_log_int(rng, 1000, 160000), dtype=dt, out=odt,
                     scale=rng.choice((1.0, 0.5, 27.5)))
            if kind == "egrad":
                c.update(accumulate=rng.random() < 0.4, hot=rng.choice((0.0, 0.0, 0.3, 0.9)))
        size = c["vocab"] * c.get("d", 1) if kind != "policy" else c["rows"] * (c["vocab"] + c["pad"])
        if work(c)["bytes"] <= most and size < 5e8:
            return c


# ------------------------------------------------------------------------------------------------ work

def _es(dt):
    return 4 if dt == "fp32" else 2


def _distinct(c):
    """Expected number of distinct tokens among the rows (see _tokens)."""
    v = np.arange(c["vocab"], dtype=np.float64)
    p = np.log((v + 2) / (v + 1)) / math.log(c["vocab"] + 1)
    n = c["rows"] * (1.0 - c.get("hot", 0.0))
    return min(float(c["rows"]), float((1.0 - (1.0 - p) ** n).sum()))


def _shapes(c):
    """The gradients of one role, every layer's tensors on their own.  odd: sizes that no vector width divides."""
    d, f, o = c["d"], c["ffn"], int(c["odd"])
    layer = [(c["qkv"] + o, d + o), (d, d + o), (2 * f + o, d), (d + o, f + o), (d + o,), (d + o,)]
    return [(c["vocab"] + o, d)] + layer * c["layers"] + [(d + o,), (c["vocab"], d + o)]


def work(case):
    c = case
    if c["kind"] == "policy":
        kept = c["rows"] * (1.0 - c["masked"])
        b = kept * c["vocab"] * _es(c["dtype"]) + 24.0 * c["rows"]
        if c["grad"]:
            b += float(c["rows"]) * c["vocab"] * _es(c["dtype"])
        return {"bytes": b, "flops": kept * c["vocab"] * (6.0 if c["grad"] else 3.0)}
    if c["kind"] == "clip":
        n = float(sum(math.prod(s) for s in _shapes(c)))
        return {"bytes": 2 * n * _es(c["dtype"]), "flops": 3 * n}
    rows, d = float(c["rows"]), float(c["d"])
    if c["kind"] == "embed":
        return {"bytes": _distinct(c) * d * _es(c["dtype"]) + rows * d * _es(c["out"]) + 4 * rows, "flops": rows * d}
    written = 2 * _distinct(c) if c["accumulate"] else c["vocab"]
    return {"bytes": rows * d * _es(c["dtype"]) + written * d * _es(c["out"]) + 4 * rows, "flops": rows * d}


# ---------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, dt="fp32", std=1.0):
    return torch.empty(shape, device="cuda", dtype=DTYPES[dt]).normal_(0.0, std, generator=g)


def _tokens(g, c):
    """Token ids as a vocabulary sorted by frequency gives them: id v in proportion to log(1 + 1/(v + 1)).  A share
    `hot` of the rows, at the batch's end, carries one token, as padding does."""
    u = torch.rand(c["rows"], device="cuda", dtype=torch.float64, generator=g)
    t = (torch.exp(u * math.log(c["vocab"] + 1)) - 1.0).long().clamp_(0, c["vocab"] - 1)
    hot = int(c["rows"] * c.get("hot", 0.0))
    if hot:
        t[c["rows"] - hot:] = 3
    return t.to(torch.int32)


def _policy_inputs(c, g):
    R, V = c["rows"], c["vocab"]
    logits = _normal(g, R, V + c["pad"], dt=c["dtype"], std=2.0)[:, :V]
    tokens = torch.randint(0, V, (R,), device="cuda", generator=g, dtype=torch.int32)
    at = tokens.long()[:, None]
    logits.scatter_(1, at, (logits.gather(1, at).float() + 9.0).to(logits.dtype))    # the chosen token is a likely one
    lp = torch.cat([z.gather(1, a).float()[:, 0] - torch.logsumexp(z.float(), 1) for z, a in zip(logits.split(1024), at.split(1024))])
    # how far the Actor has moved since the rollout.  A ratio at the very edge of the clipped range would be cut or
    # not by the rounding of its log-prob: such rows are set a little apart from the edge.
    moved = 0.15 * torch.randn(R, device="cuda", generator=g)
    for edge in (math.log(0.8), math.log(1.2)):
        moved = torch.where((moved - edge).abs() < 1e-3, moved + 4e-3, moved)
    masked = torch.rand(R, device="cuda", generator=g) < c["masked"]
    weight = torch.where(masked, 0.0, 1.0)
    weight = weight / weight.sum().clamp_(min=1.0)
    s = {"logits": logits, "tokens": tokens, "lp_old": lp - moved, "adv": _normal(g, R), "weight": weight,
         "lp_ref": lp + 0.3 * torch.randn(R, device="cuda", generator=g) if c["kl"] else None,
         "kl": c["kl"], "scale": 65536.0 if c["dtype"] == "fp16" else 1.0, "lp": torch.empty(R, device="cuda"),
         "stats": torch.empty(4, device="cuda"), "dlogits": torch.empty(R, V, device="cuda", dtype=logits.dtype) if c["grad"] else None}
    return s


def _clip_inputs(c, g):
    shapes = _shapes(c)
    std = 2.7 / math.sqrt(sum(math.prod(s) for s in shapes))       # a norm of about 2.7: gradients to be clipped
    grads = [_normal(g, *s, dt=c["dtype"], std=std) for s in shapes]
    flat = torch.empty(sum(t.numel() for t in grads), device="cuda", dtype=DTYPES[c["dtype"]])
    clipped = [p.view(t.shape) for p, t in zip(flat.split([t.numel() for t in grads]), grads)]
    return {"grads": grads, "clipped": clipped, "flat": flat, "max_norm": c["max_norm"], "norm": torch.empty(1, device="cuda")}


def _inputs(c, seed):
    g = _generator(seed)
    if c["kind"] == "policy":
        return _policy_inputs(c, g)
    if c["kind"] == "clip":
        return _clip_inputs(c, g)
    s = {"tokens": _tokens(g, c), "scale": c["scale"]}
    if c["kind"] == "embed":
        s["table"] = _normal(g, c["vocab"], c["d"], dt=c["dtype"], std=0.02)
        s["out"] = torch.empty(c["rows"], c["d"], device="cuda", dtype=DTYPES[c["out"]])
        return s
    s["dout"] = _normal(g, c["rows"], c["d"], dt=c["dtype"], std=0.5)
    s["accumulate"] = c["accumulate"]
    s["dtable"] = _normal(g, c["vocab"], c["d"], dt=c["out"], std=0.5)
    return s


def prepare(case, seed):
    return dict(_inputs(case, seed), case=case)


# ------------------------------------------------------------------------------------------------ pass

def run(state):
    if own:
        return _own(state)
    return {"policy": _plain_policy, "embed": _plain_embed, "egrad": _plain_egrad, "clip": _plain_clip}[state["case"]["kind"]](state)


def _own(s):
    import paper_2409_13221_amd as R
    kind = s["case"]["kind"]
    if kind == "policy":
        R.rlhf_op_policy_loss(s["logits"], s["tokens"], s["lp_old"], s["adv"], s["lp"], s["stats"], dlogits=s["dlogits"], lp_ref=s["lp_ref"],
                              weight=s["weight"], clip_low=0.2, clip_high=0.2, kl_coef=s["kl"], grad_scale=s["scale"])
        out = {"lp": s["lp"], "stats": s["stats"]}
        if s["dlogits"] is not None:
            out["dlogits"] = s["dlogits"]
        return out
    if kind == "embed":
        R.rlhf_op_embed(s["table"], s["tokens"], s["out"], scale=s["scale"])
        return {"out": s["out"]}
    if kind == "egrad":
        R.rlhf_op_embed_grad(s["dout"], s["tokens"], s["dtable"], scale=s["scale"], accumulate=s["accumulate"])
        return {"dtable": s["dtable"]}
    if "list" not in s:           # the addresses and sizes of a model's gradients are listed once and kept, as the model is
        s["list"] = R.rlhf_tensor_list(s["grads"], s["clipped"])
    R.rlhf_op_grad_norm(s["list"], s["norm"])
    R.rlhf_op_clip_grads(s["list"], s["norm"], s["max_norm"])
    return {"clipped": s["flat"], "norm": s["norm"]}


def _plain_policy(s):
    z, w = s["logits"].float(), s["weight"]
    at = s["tokens"].long()[:, None]
    e = torch.exp(z - z.max(1, keepdim=True).values)
    total = e.sum(1, keepdim=True)
    lp = (z.gather(1, at) - z.max(1, keepdim=True).values - torch.log(total))[:, 0]
    lp = torch.where(w != 0, lp, 0.0)
    ratio = torch.exp(lp - s["lp_old"])
    free, held = ratio * s["adv"], ratio.clamp(0.8, 1.2) * s["adv"]
    cut = held < free
    policy = -torch.where(cut, held, free)
    slope = -torch.where(cut, 0.0, free)
    if s["lp_ref"] is not None:
        x = s["lp_ref"] - lp
        kl = torch.expm1(x) - x
        slope = slope - s["kl"] * torch.expm1(x)
    else:
        kl = torch.zeros_like(lp)
    sums = [(w * v).double().sum() for v in (policy, kl, cut.float())]
    stats = torch.stack([sums[0] + s["kl"] * sums[1], sums[0], sums[1], sums[2]]).float()
    out = {"lp": lp, "stats": stats}
    if s["dlogits"] is not None:
        slope = (s["scale"] * w * slope)[:, None]
        d = e * (-slope / total)
        d.scatter_add_(1, at, slope)
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _plain_embed(s):
    return {"out": (s["table"][s["tokens"].long()].float() * s["scale"]).to(s["out"].dtype)}


def _plain_egrad(s):
    if s["accumulate"]:
        total = s["dtable"].float()
    else:
        total = torch.zeros(s["dtable"].shape, device="cuda")
    total.index_add_(0, s["tokens"].long(), s["dout"].float(), alpha=s["scale"])
    s["dtable"].copy_(total)
    return {"dtable": s["dtable"]}


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt()
    factor = (s["max_norm"] / norm).clamp(max=1.0).float()
    _ = [o.copy_(g.float() * factor) for g, o in zip(s["grads"], s["clipped"])]
    return {"clipped": s["flat"], "norm": norm.float().reshape(1)}


# ----------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    return {"policy": _exact_policy, "embed": _exact_embed, "egrad": _exact_egrad, "clip": _exact_clip}[case["kind"]](case, _inputs(case, seed))


def _exact_policy(c, s):
    """Each row by itself: log-softmax at the token, and the derivative of the loss as a function of that number."""
    lps, ds, parts = [], [], []
    for i in range(0, c["rows"], 512):
        r = slice(i, i + 512)
        logp = torch.log_softmax(s["logits"][r].double(), 1)
        w, adv, at = s["weight"][r].double(), s["adv"][r].double(), s["tokens"][r].long()
        lp = logp[torch.arange(len(at), device="cuda"), at] * (w != 0)
        rho = torch.exp(lp - s["lp_old"][r].double())
        out_of_range = ((adv > 0) & (rho > 1.2)) | ((adv < 0) & (rho < 0.8))
        bound = torch.where(adv > 0, 1.2, 0.8).double()
        pg = -adv * torch.where(out_of_range, bound, rho)
        dl = -adv * rho * ~out_of_range
        kl = torch.zeros_like(lp)
        if s["lp_ref"] is not None:
            q = torch.exp(s["lp_ref"][r].double() - lp)
            kl = q - 1.0 - torch.log(q)
            dl = dl + s["kl"] * (1.0 - q)
        lps.append(lp)
        parts.append(torch.stack([(w * pg).sum(), (w * kl).sum(), (w * out_of_range).sum()]))
        if c["grad"]:
            dz = -torch.exp(logp)
            dz[torch.arange(len(at), device="cuda"), at] += 1.0
            ds.append(dz * (s["scale"] * w * dl)[:, None])
    p = torch.stack(parts).sum(0)
    out = {"lp": torch.cat(lps), "stats": torch.stack([p[0] + s["kl"] * p[1], p[0], p[1], p[2]])}
    if c["grad"]:
        out["dlogits"] = torch.cat(ds)
    return out


def _exact_embed(c, s):
    return {"out": s["table"].double().index_select(0, s["tokens"].long()) * s["scale"]}


def _exact_egrad(c, s):
    order = torch.argsort(s["tokens"], stable=True)
    ids, counts = torch.unique_consecutive(s["tokens"][order].long(), return_counts=True)
    out = s["dtable"].double() if c["accumulate"] else torch.zeros(c["vocab"], c["d"], device="cuda", dtype=torch.float64)
    step = max(1, (1 << 28) // c["rows"])
    for j in range(0, c["d"], step):              # columns at a time: sums between two ends of each token's run
        run_sum = torch.cumsum(s["dout"][order, j:j + step].double() * s["scale"], 0)
        ends = run_sum[torch.cumsum(counts, 0) - 1]
        out[ids, j:j + step] += torch.cat([ends[:1], ends[1:] - ends[:-1]])
    return {"dtable": out}


def _exact_clip(c, s):
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["grads"]))
    f = min(1.0, c["max_norm"] / norm)
    return {"clipped": torch.cat([g.double().reshape(-1) for g in s["grads"]]) * f, "norm": torch.full((1,), norm, device="cuda", dtype=torch.float64)}
