"""One policy update on the device, operator by operator, as timed cases.

Each case is one pass through an operator at one size.  `listed` holds the
cases, `draw` makes more of the same kinds and ranges, `prepare` makes what a
program holds before the call, `run` is the pass (in elementary torch
operations, or through the package where `own` is set), `work` the bytes and
operations that the pass cannot do without and `exact` the result in 64 bits.

Operators:
  policy   the clipped policy loss with a KL term and an entropy bonus, from
           the logits of each row's choice: loss sums, the rows'
           log-probabilities and the gradient of the logits
  logprob  the log-probability of each row's choice and the entropy, forward
           only (what scores a rollout under the old and reference policies)
  pl       the clipped policy loss of ordered Plackett-Luce draws: loss sums,
           log-probabilities and the gradient of the scores
  clip     the global norm of many gradient tensors, and clipping by it
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CLIP_EPS = 1e-6


def listed():
    return [
        # Budget head of the actor over a rollout of 256 images at four blocks; the smallest call.
        dict(name="policy_budget_f32", op="policy", T=1024, V=96, dtype="f32", legal=True, masked=0.0, ref=False,
             ent=0.01, pad=0),
        # A few tokens of a large vocabulary: gradient accumulation one short sequence at a time.
        dict(name="policy_few_bf16", op="policy", T=16, V=131072, dtype="bf16", legal=False, masked=0.0, ref=True,
             ent=0.0, pad=0),
        # A packed batch in full precision.
        dict(name="policy_f32", op="policy", T=1024, V=32000, dtype="f32", legal=False, masked=0.25, ref=True, ent=0.0,
             pad=0),
        # An odd vocabulary: no row but the first starts on a 16-byte boundary; a quarter of the rows is padding.
        dict(name="policy_odd_bf16", op="policy", T=2048, V=50257, dtype="bf16", legal=False, masked=0.25, ref=True,
             ent=0.001, pad=0),
        # The largest: a training batch over a large vocabulary.
        dict(name="policy_large_bf16", op="policy", T=8192, V=131072, dtype="bf16", legal=False, masked=0.0, ref=True,
             ent=0.0, pad=0),
        # One token while serving.
        dict(name="logprob_one_bf16", op="logprob", T=1, V=131072, dtype="bf16", legal=False, masked=0.0, pad=0),
        # Scoring a rollout; the logits are a slice of a padded product.
        dict(name="logprob_rollout_bf16", op="logprob", T=4096, V=50257, dtype="bf16", legal=False, masked=0.25,
             pad=47),
        # Selector of the actor on ViT-B/384 rows, the batch of one update.
        dict(name="pl_update_384", op="pl", B=256, N=577, packed=False, ref=True),
        # Packed rows of high-resolution inputs, few and long.
        dict(name="pl_update_long", op="pl", B=48, N=2048, packed=True, ref=False),
        # Gradients of the actor itself: many tiny tensors, clipped at 0.5.
        dict(name="clip_actor_f32", op="clip", shapes="actor", dtype="f32", flat=False, max_norm=0.5),
        # A small backbone in bf16.
        dict(name="clip_small_bf16", op="clip", shapes="small", dtype="bf16", flat=False, max_norm=1.0),
        # A large backbone in fp32, the gradients views of one flat buffer.
        dict(name="clip_large_f32", op="clip", shapes="large", dtype="f32", flat=True, max_norm=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("policy", "policy", "logprob", "pl", "clip"))
    if op == "pl":
        B = _log(rng, 1, 2048)
        return dict(op=op, B=B, N=_log(rng, 2, 2048), packed=rng.random() < 0.5, ref=rng.random() < 0.5)
    if op == "clip":
        n, total = _log(rng, 1, 400), _log(rng, 1000, 1 << 28)
        return dict(op=op, shapes="random", n=n, total=total, dtype=rng.choice(("bf16", "f32")),
                    flat=rng.random() < 0.5, max_norm=rng.choice((0.5, 1.0, 1e9)))
    T = _log(rng, 1, 8192)
    V = _log(rng, 2, min(160000, (1 << 29) // T))
    case = dict(op=op, T=T, V=V, dtype=rng.choice(("bf16", "bf16", "f32")), legal=V <= 4096 and rng.random() < 0.5,
                masked=rng.choice((0.0, 0.0, 0.25, 0.5)), pad=rng.choice((0, 0, 0, 47)))
    if op == "policy":
        case.update(ref=rng.random() < 0.7, ent=rng.choice((0.0, 0.0, 0.01)))
    return case


# ---------------------------------------------------------------- inputs

CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05


def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + salt)


def _log_ratio(shape, g, dev):
    """Log of new over old probability, as a few updates leave it.  A ratio
    within rounding of the clip's border could fall on either side: moved off."""
    lr = 0.15 * torch.randn(shape, generator=g, device=dev, dtype=torch.float64)
    for border in (math.log1p(-CLIP_LOW), math.log1p(CLIP_HIGH)):
        d = lr - border
        lr = torch.where(d.abs() < 2e-3, border + torch.where(d < 0, -2e-3, 2e-3), lr)
    return lr


def _row_weights(T, masked, g, dev):
    w = torch.ones(T, device=dev)
    pad = int(T * masked)
    if pad:
        w[torch.randperm(T, generator=g, device=dev)[:pad]] = 0.0
    return w / w.sum()


def _logit_inputs(case, seed):
    dev, T, V = "cuda", case["T"], case["V"]
    g = _gen(seed, 11)
    full = torch.empty((T, V + case["pad"]), dtype=DTYPES[case["dtype"]], device=dev)
    logits = full[:, :V]
    legal = None
    if case["legal"]:  # a prefix of the choices is open to each row
        legal = torch.randint((V + 1) // 2, V + 1, (T,), generator=g, device=dev, dtype=torch.int32)
    actions = torch.empty(T, dtype=torch.int32, device=dev)
    logp = torch.empty(T, dtype=torch.float64, device=dev)
    step = max(1, (1 << 25) // V)
    for lo in range(0, T, step):
        hi = min(T, lo + step)
        full[lo:hi] = (3.0 * torch.randn((hi - lo, V + case["pad"]), generator=g, device=dev)).to(full.dtype)
        x = logits[lo:hi].float()
        if legal is not None:
            x.masked_fill_(torch.arange(V, device=dev)[None, :] >= legal[lo:hi, None], -math.inf)
        noise = torch.empty_like(x).exponential_(generator=g).log_().neg_()
        pick = (x + noise).argmax(1)
        actions[lo:hi] = pick.int()
        x = x.double()
        logp[lo:hi] = x.gather(1, pick[:, None])[:, 0] - torch.logsumexp(x, 1)
    return dict(logits=logits, actions=actions, legal=legal), logp, g


def _random_sizes(case):
    """Tensor sizes over several factors of ten, some of them tiny, odd or empty."""
    import random
    rng = random.Random(case["n"] * 7919 + case["total"])
    part = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(case["n"])]
    scale = case["total"] / sum(part)
    return [int(p * scale) for p in part]


def _sizes(case):
    if case["shapes"] == "random":
        return _random_sizes(case)
    if case["shapes"] == "actor":  # gate, encoder (width 128, one block), budget head, selector on 768-wide keys
        return [64 * 787, 64, 64, 1, 128 * 768, 128, 128 * 3, 12 * 128, 128, 128, 384 * 128, 384, 128 * 128, 128, 128,
                128, 256 * 128, 256, 128 * 256, 128, 128, 128, 128 * 128, 128, 96 * 128, 96, 128, 64 * 128, 64, 64, 1]
    d, layers = {"small": (384, 12), "large": (1024, 24)}[case["shapes"]]
    block = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, 4 * d * d, 4 * d, 4 * d * d, d]
    return [d, 197 * d, 768 * d, d] + block * layers + [d, d, 1000 * d, 1000]


def prepare(case, seed):
    dev = "cuda"
    if case["op"] in ("policy", "logprob"):
        s, logp, g = _logit_inputs(case, seed)
        T, V = case["T"], case["V"]
        s["weight"] = _row_weights(T, case["masked"], g, dev)
        if case["op"] == "policy":
            s["old"] = (logp - _log_ratio((T,), g, dev)).float()
            s["ref"] = (logp + 0.2 * torch.randn(T, generator=g, device=dev)).float() if case["ref"] else None
            s["adv"] = torch.randn(T, generator=g, device=dev)
            s["ent"] = case["ent"]
        if own:
            import paper_2609_34325_amd as dora
            s["dora"] = dora
            s["status"] = dora.new_status()
            s["logp_out"] = torch.empty(T, device=dev)
            if case["op"] == "policy":
                s["ws"] = dora.new_policy_workspace(T, V)
                s["grad"] = torch.empty((T, V), dtype=s["logits"].dtype, device=dev)
                s["stats"] = torch.empty(6, device=dev)
            else:
                s["ws"] = dora.new_policy_workspace(T, V)
                s["ent_out"] = torch.empty(T, device=dev)
    elif case["op"] == "pl":
        B, N = case["B"], case["N"]
        g = _gen(seed, 12)
        if case["packed"]:
            # The layout is the case's own: the same lengths whatever the scores.
            lens = torch.randint(max(1, N // 4), N + 1, (B,), generator=_gen(B, N), device=dev)
        else:
            lens = torch.full((B,), N, device=dev)
        cu = torch.zeros(B + 1, dtype=torch.int64, device=dev)
        cu[1:] = lens.cumsum(0)
        total = int(cu[-1])
        scores = 2.0 * torch.randn(total, generator=g, device=dev)
        k = (torch.rand(B, generator=g, device=dev) * 0.6 * (lens - 1)).long()
        # Draws by the largest score plus Gumbel noise, CLS (the first of each segment) left out.
        key = scores.double() - torch.empty_like(scores).exponential_(generator=g).double().log()
        img = torch.repeat_interleave(torch.arange(B, device=dev), lens)
        pos = torch.arange(total, device=dev) - cu[img]
        key[pos == 0] = -math.inf
        by = key.argsort(descending=True)
        by = by[img[by].argsort(stable=True)]
        rank = torch.arange(total, device=dev) - cu[img]  # by[cu[b] + r] is image b's draw r
        take = rank < k[img]
        order = pos[by][take].int()
        cuo = torch.zeros(B + 1, dtype=torch.int64, device=dev)
        cuo[1:] = k.cumsum(0)
        s = dict(scores=scores if case["packed"] else scores.view(B, N), order=order.contiguous(), cu_order=cuo.int(),
                 cu_in=cu.int() if case["packed"] else None, N=N, order_total=int(cuo[-1]))
        if s["order"].numel() == 0:
            s["order"] = torch.zeros(1, dtype=torch.int32, device=dev)
        logp = _pl_exact(s)[0]
        s["old"] = (logp - _log_ratio((B,), g, dev)).float()
        s["ref"] = (logp + 0.2 * torch.randn(B, generator=g, device=dev)).float() if case["ref"] else None
        s["adv"] = torch.randn(B, generator=g, device=dev)
        s["weight"] = torch.full((B,), 1.0 / B, device=dev)
        if own:
            import paper_2609_34325_amd as dora
            s["dora"] = dora
            s["status"] = dora.new_status()
            s["ws"] = dora.new_pl_policy_workspace(B)
            s["grad"] = torch.empty_like(s["scores"])
            s["logp_out"] = torch.empty(B, device=dev)
            s["stats"] = torch.empty(6, device=dev)
    else:
        g = _gen(seed, 13)
        sizes, dtype = _sizes(case), DTYPES[case["dtype"]]
        total = sum(sizes)
        # Gradients of a norm of a few units, their scale differing from tensor to tensor.
        scale = 3.0 / math.sqrt(max(total, 1)) * torch.exp(torch.randn(len(sizes), generator=g, device=dev))
        first = 1 if case["flat"] else 0
        if case["flat"]:  # views of one buffer, one element in, as a bucketed reduction leaves them
            grads = list(torch.empty(total + first, dtype=dtype, device=dev)[first:].split(sizes))
        else:
            grads = [torch.empty(n, dtype=dtype, device=dev) for n in sizes]
        for t, c in zip(grads, scale):
            t.copy_(torch.randn(t.numel(), generator=g, device=dev) * c)
        # The clipped gradients go to the optimizer's one flat buffer.
        flat = torch.empty(total + first, dtype=dtype, device=dev)[first:]
        s = dict(grads=grads, max_norm=case["max_norm"], flat=flat, out=list(flat.split(sizes)))
        if own:
            import paper_2609_34325_amd as dora
            s["dora"] = dora
            s["ws"] = dora.new_grad_clip_workspace(len(grads))
            s["norm"] = torch.empty(1, device=dev)
    s["op"] = case["op"]
    return s


# ---------------------------------------------------------------- the pass

def _surrogate(logp, old, ref, adv, weight):
    """Per row in 64 bits: the parts of the loss and d loss / d logp without
    the entropy's share.  Rows of weight 0 are padding."""
    on = weight != 0
    w = weight.double()
    r = torch.exp(logp - old.double())
    a = adv.double()
    free, held = r * a, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    clipped = held < free
    part = torch.where(clipped, held, free)
    G = torch.where(clipped, torch.zeros_like(r), -free)
    kl = torch.zeros_like(r)
    if ref is not None:
        d = ref.double() - logp
        kl = torch.exp(d) - d - 1
        G = G + KL * (1 - torch.exp(d))
    zero = torch.zeros_like(r)
    return (w, torch.where(on, part, zero), torch.where(on, kl, zero), torch.where(on & clipped, w, zero),
            torch.where(on, G * w, zero))


def _stats(w, part, kl, H, clipped, ent):
    loss = (w * (KL * kl - part - ent * H)).sum()
    return torch.stack([loss, (w * part).sum(), (w * kl).sum(), (w * H).sum(), clipped.sum(), w.sum()]).float()


def _plain_softmax(s):
    x = s["logits"].float()
    V = x.shape[1]
    on = s["weight"] != 0
    closed = ~on[:, None]
    if s["legal"] is not None:
        x = torch.where(torch.arange(V, device=x.device)[None, :] < s["legal"][:, None], x, -math.inf)
    x = torch.where(closed, torch.zeros_like(x), x)
    d = x - x.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, dtype=torch.float64)
    logz = torch.log(total)
    logp = torch.gather(d, 1, s["actions"].long()[:, None])[:, 0].double() - logz
    H = logz - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1, dtype=torch.float64) / total
    logp, H = (torch.where(on, t, torch.zeros_like(t)) for t in (logp, H))
    return d, e, total, logz, logp, H


def _plain_policy(s):
    d, e, total, logz, logp, H = _plain_softmax(s)
    w, part, kl, clipped, G = _surrogate(logp, s["old"], s["ref"], s["adv"], s["weight"])
    p = e / total.float()[:, None]
    grad = -G.float()[:, None] * p
    if s["ent"]:
        inner = (d - (logz - H).float()[:, None]).clamp(min=-1e30)
        grad = grad + (s["ent"] * w).float()[:, None] * p * inner
    grad.scatter_add_(1, s["actions"].long()[:, None], G.float()[:, None])
    grad = torch.where((s["weight"] != 0)[:, None], grad, torch.zeros_like(grad))
    return grad.to(s["logits"].dtype), logp.float(), _stats(w, part, kl, H, clipped, s["ent"])


def _pl_plan(s):
    """Scores by drawing order, image by image in rows of a padded matrix:
    the draws, then the tokens left, then padding."""
    scores, dev = s["scores"], s["scores"].device
    N = s["N"]
    if s["cu_in"] is None:
        B = scores.shape[0]
        lens = torch.full((B,), N, device=dev)
        start = torch.arange(B, device=dev) * N
    else:
        cu = s["cu_in"].long()
        B = cu.numel() - 1
        lens, start = cu[1:] - cu[:-1], cu[:-1]
    flat = scores.reshape(-1)
    cuo = s["cu_order"].long()
    k = cuo[1:] - cuo[:-1]
    col = torch.arange(N, device=dev)
    at = (start[:, None] + col).clamp(max=flat.numel() - 1)
    x = flat[at]
    here = (col[None, :] < lens[:, None]) & (col[None, :] > 0)
    n = s["order_total"]
    rank = torch.full((B, N), N, device=dev)  # drawing step of each position; N: not drawn
    if n:
        img = torch.repeat_interleave(torch.arange(B, device=dev), k)
        rank[img, s["order"][:n].long()] = torch.arange(n, device=dev) - cuo[img]
    return flat, start, lens, k, x, here, rank, col


def _plain_pl(s):
    flat, start, lens, k, x, here, rank, col = _pl_plan(s)
    x = torch.where(here, x, -math.inf)
    m = x.amax(1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    e = torch.exp((x - m).double())  # long sums of terms of very different size
    by = torch.where(here, rank, torch.full_like(rank, 2 * x.shape[1])).argsort(1)
    eo = e.gather(1, by)
    S = eo.flip(1).cumsum(1).flip(1)
    drawn = col[None, :] < k[:, None]
    xo = (x - m).double().gather(1, by)
    logp = torch.where(drawn, xo - torch.log(S), torch.zeros_like(S)).sum(1)
    inv = torch.where(drawn, 1.0 / S, torch.zeros_like(S)).cumsum(1)  # over the steps up to and with this one
    last = torch.minimum(rank, (k - 1)[:, None].expand_as(rank)).clamp(min=0)
    took = torch.where(k[:, None] > 0, inv.gather(1, last), torch.zeros_like(inv))
    dlp = (rank < x.shape[1]).double() - e * took
    w, part, kl, clipped, G = _surrogate(logp, s["old"], s["ref"], s["adv"], s["weight"])
    g = torch.where(here, G[:, None] * dlp, torch.zeros_like(dlp)).float()
    H = torch.zeros_like(logp)
    if s["cu_in"] is None:
        grad = g
    else:
        grad = g[col[None, :] < lens[:, None]]
    return grad, logp.float(), _stats(w, part, kl, H, clipped, 0.0)


def _plain_clip(s):
    total = torch.stack([(g.float() * g.float()).sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = torch.sqrt(total)
    c = (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0).float()
    for o, g in zip(s["out"], s["grads"]):
        o.copy_(g.float() * c)
    return s["flat"], norm.float().view(1)


def run(s):
    op = s["op"]
    if not own:
        if op == "policy":
            return _plain_policy(s)
        if op == "logprob":
            logp, H = _plain_softmax(s)[4:]
            return logp.float(), H.float()
        return _plain_pl(s) if op == "pl" else _plain_clip(s)
    dora = s["dora"]
    if op == "policy":
        grad, logp, stats, _ = dora.dora_policy_loss(
            s["logits"], s["actions"], s["old"], s["adv"], ref_logprob=s["ref"], weight=s["weight"], legal=s["legal"],
            clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL if s["ref"] is not None else 0.0, entropy_coef=s["ent"],
            dlogits=s["grad"], logprob_out=s["logp_out"], stats_out=s["stats"], workspace=s["ws"],
            dev_status=s["status"])
        return grad, logp, stats
    if op == "logprob":
        logp, H, _ = dora.dora_action_logprob(s["logits"], s["actions"], weight=s["weight"], legal=s["legal"],
                                              logprob_out=s["logp_out"], entropy_out=s["ent_out"], workspace=s["ws"],
                                              dev_status=s["status"])
        return logp, H
    if op == "pl":
        grad, logp, stats, _ = dora.dora_pl_policy_loss(
            s["scores"], s["order"], s["cu_order"], s["old"], s["adv"], ref_logprob=s["ref"], weight=s["weight"],
            cu_in=s["cu_in"], N=s["N"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
            kl_coef=KL if s["ref"] is not None else 0.0, dscores=s["grad"], logprob_out=s["logp_out"],
            stats_out=s["stats"], workspace=s["ws"], dev_status=s["status"])
        return grad, logp, stats
    _, norm = dora.dora_grad_clip(s["grads"], s["max_norm"], out=s["out"], eps=CLIP_EPS, norm_out=s["norm"],
                                  workspace=s["ws"])
    return s["flat"], norm


# ---------------------------------------------------------------- work and exact results

def work(case):
    if case["op"] == "pl":
        tokens = case["B"] * case["N"] * (0.625 if case["packed"] else 1.0)
        return dict(bytes=int(tokens * (4 + 4 + 0.3 * 4) + 24 * case["B"]), flops=int(10 * tokens))
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "clip":
        n = sum(_sizes(case))
        return dict(bytes=2 * es * n, flops=3 * n)
    T, V = case["T"], case["V"]
    live = T - int(T * case["masked"])
    read = live * V * es * (0.75 if case["legal"] else 1.0)
    if case["op"] == "logprob":
        return dict(bytes=int(read) + 16 * T, flops=6 * live * V)
    return dict(bytes=int(read) + T * V * es + 28 * T, flops=12 * live * V)


def _objective(logp, H, old, ref, adv, w, ent):
    """The loss's parts by their definition, for autograd."""
    r = torch.exp(logp - old.double())
    a = adv.double()
    gain = torch.minimum(r * a, torch.clamp(r, 1 - CLIP_LOW, 1 + CLIP_HIGH) * a)
    kl = torch.zeros_like(r) if ref is None else torch.expm1(ref.double() - logp) - (ref.double() - logp)
    parts = [(w * (KL * kl - gain - ent * H)).sum(), (w * gain).sum(), (w * kl).sum(), (w * H).sum(),
             w[(torch.clamp(r, 1 - CLIP_LOW, 1 + CLIP_HIGH) * a < r * a)].sum(), w.sum()]
    return parts


def _pl_exact(s, image_grad=None):
    """Ordered log-probabilities (and with `image_grad` the gradient of
    sum image_grad * logp) by log-sum-exp over what is left at each step."""
    flat, start, lens, k, x, here, rank, col = _pl_plan(s)
    x = x.double().requires_grad_(image_grad is not None)
    with torch.set_grad_enabled(image_grad is not None):
        # 800 below the largest score: nothing beside it in 64 bits, and finite for autograd
        masked = torch.where(here, x, (x.detach().amax(1, keepdim=True) - 800.0).expand_as(x))
        by = torch.where(here, rank, torch.full_like(rank, 4 * x.shape[1])).argsort(1)
        left = torch.logcumsumexp(masked.gather(1, by).flip(1), 1).flip(1)
        drawn = col[None, :] < k[:, None]
        lp = torch.where(drawn, masked.gather(1, by) - torch.where(drawn, left, torch.zeros_like(left)),
                         torch.zeros_like(left)).sum(1)
        if image_grad is None:
            return lp, None
        g, = torch.autograd.grad((lp * image_grad).sum(), x)
    return lp.detach(), torch.where(here, g, torch.zeros_like(g))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        grads = [g.double() for g in s["grads"]]
        norm = math.sqrt(sum(float(torch.dot(g, g)) for g in grads))
        c = min(1.0, s["max_norm"] / (norm + CLIP_EPS))
        return torch.cat(grads) * c, torch.tensor([norm], dtype=torch.float64, device="cuda")
    if op == "pl":
        lp = _pl_exact(s)[0].requires_grad_(True)
        w = s["weight"].double()
        parts = _objective(lp, torch.zeros_like(lp), s["old"], s["ref"], s["adv"], w, 0.0)
        G, = torch.autograd.grad(parts[0], lp)
        lp, g = _pl_exact(s, G)
        if s["cu_in"] is not None:
            lens = (s["cu_in"][1:] - s["cu_in"][:-1]).long()
            g = g[torch.arange(s["N"], device="cuda")[None, :] < lens[:, None]]
        return g, lp, torch.stack([p.detach() for p in parts])
    T, V = case["T"], case["V"]
    lps, Hs, grads, stats = [], [], [], torch.zeros(6, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 24) // V)
    for lo in range(0, T, step):
        rows = slice(lo, min(T, lo + step))
        w = s["weight"][rows].double()
        x = s["logits"][rows].double().requires_grad_(True)
        z = x
        if s["legal"] is not None:
            z = z.masked_fill(torch.arange(V, device="cuda")[None, :] >= s["legal"][rows, None], -math.inf)
        lsm = torch.log_softmax(z, 1)
        lp = lsm.gather(1, s["actions"][rows].long()[:, None])[:, 0]
        H = -(lsm.exp() * lsm.clamp(min=-1e300)).sum(1)
        if op == "policy":
            ref = s["ref"][rows] if s["ref"] is not None else None
            parts = _objective(lp, H, s["old"][rows], ref, s["adv"][rows], w, s["ent"])
            g, = torch.autograd.grad(parts[0], x)
            grads.append(g)
            stats += torch.stack([p.detach() for p in parts])
        zero = torch.zeros_like(w)
        lps.append(torch.where(w != 0, lp.detach(), zero))
        Hs.append(torch.where(w != 0, H.detach(), zero))
    if op == "logprob":
        return torch.cat(lps), torch.cat(Hs)
    return torch.cat(grads), torch.cat(lps), stats
