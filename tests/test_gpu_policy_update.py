"""One policy update as a training program runs it: the old policy's choices
scored (budget by its logits, selection by an ordered draw), the new policy's
losses and gradients, the weights' gradients by products, clipped together --
against the same update by automatic differentiation in 64 bits; eager, and
captured and replayed."""
import numpy as np
import pytest
import torch

from policy_ref import U32

pytestmark = pytest.mark.gpu

B, N, M, D = 48, 50, 23, 40
LOW, HIGH, KL, ENT, MAX_NORM = 0.2, 0.25, 0.1, 0.02, 0.05


def setup(dora):
    g = torch.Generator("cuda").manual_seed(11)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    p = dict(keys=r(B, N, D), wb=0.3 * r(D, M), ws=0.3 * r(D, 1), adv=r(B))
    p["legal"] = torch.randint(5, M + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    # The rollout: choices of the old policy, scored by it and by a reference.
    logits = p["keys"][:, 0] @ p["wb"]
    closed = torch.arange(M, device="cuda")[None, :] >= p["legal"][:, None]
    noise = -torch.log(-torch.log(torch.rand((B, M), generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    p["actions"] = (logits + noise).masked_fill(closed, -1e30).argmax(1).int()
    scores = (p["keys"] @ p["ws"])[:, :, 0].contiguous()
    gumbel = -torch.log(-torch.log(torch.rand((B, N), generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    p["order"], p["cu"], p["old_s"], _ = dora.dora_pl_sample(scores, gumbel, 2 * (p["actions"] + 1))
    p["old_b"], _, st = dora.dora_action_logprob(logits, p["actions"], legal=p["legal"])
    assert int(st.item()) == 0
    p["ref_b"], p["ref_s"] = p["old_b"] + 0.05 * r(B), p["old_s"] + 0.05 * r(B)
    # The policy has moved since.
    p["wb"], p["ws"] = p["wb"] + 0.02 * r(D, M), p["ws"] + 0.01 * r(D, 1)
    p["weight"] = torch.full((B,), 1.0 / B, device="cuda")
    p["weight"][5] = 0.0
    return p


def update(dora, p, buf):
    logits = torch.matmul(p["keys"][:, 0], p["wb"], out=buf["logits"])
    scores = torch.matmul(p["keys"].view(B * N, D), p["ws"], out=buf["scores"].view(B * N, 1)).view(B, N)
    dl, lp_b, st_b, _ = dora.dora_policy_loss(
        logits, p["actions"], p["old_b"], p["adv"], ref_logprob=p["ref_b"], weight=p["weight"], legal=p["legal"],
        clip_low=LOW, clip_high=HIGH, kl_coef=KL, entropy_coef=ENT, dlogits=logits, logprob_out=buf["lp_b"],
        stats_out=buf["st_b"], workspace=buf["ws_b"], dev_status=buf["flag"])
    ds, lp_s, st_s, _ = dora.dora_pl_policy_loss(
        scores, p["order"], p["cu"], p["old_s"], p["adv"], ref_logprob=p["ref_s"], weight=p["weight"], clip_low=LOW,
        clip_high=HIGH, kl_coef=KL, dscores=buf["ds"], logprob_out=buf["lp_s"], stats_out=buf["st_s"],
        workspace=buf["ws_s"], dev_status=buf["flag"])
    torch.matmul(p["keys"][:, 0].t(), dl, out=buf["gb"])
    torch.matmul(p["keys"].view(B * N, D).t(), ds.view(B * N, 1), out=buf["gs"])
    dora.dora_grad_clip([buf["gb"], buf["gs"]], MAX_NORM, norm_out=buf["norm"], workspace=buf["ws_c"])


def buffers(dora):
    e = lambda *s: torch.empty(s, device="cuda")
    return dict(logits=e(B, M), scores=e(B, N), ds=e(B, N), lp_b=e(B), lp_s=e(B), st_b=e(6), st_s=e(6), gb=e(D, M),
                gs=e(D, 1), norm=e(1), ws_b=dora.new_policy_workspace(B, M), ws_s=dora.new_pl_policy_workspace(B),
                ws_c=dora.new_grad_clip_workspace(2), flag=dora.new_status())


OUT = ("logits", "ds", "lp_b", "lp_s", "st_b", "st_s", "gb", "gs", "norm")


def by_autograd(p):
    h = {k: v.cpu() for k, v in p.items()}
    wb, ws = h["wb"].double().requires_grad_(), h["ws"].double().requires_grad_()
    keys, w, A = h["keys"].double(), h["weight"].double(), h["adv"].double()
    logits = keys[:, 0] @ wb
    closed = torch.arange(M)[None, :] >= h["legal"][:, None]
    lsm = torch.log_softmax(logits.masked_fill(closed, -np.inf), 1)
    lp = lsm.gather(1, h["actions"].long()[:, None])[:, 0]
    H = -(lsm.exp() * lsm.masked_fill(closed, 0.0)).sum(1)
    scores = (keys @ ws)[:, :, 0]
    lps = []
    for b in range(B):
        left = list(range(1, N))
        t = torch.zeros((), dtype=torch.float64)
        for i in h["order"][h["cu"][b]:h["cu"][b + 1]].tolist():
            t = t + scores[b, i] - torch.logsumexp(scores[b, left], 0)
            left.remove(i)
        lps.append(t)
    losses = []
    for x, old, ref, ent in ((lp, h["old_b"], h["ref_b"], ENT * H), (torch.stack(lps), h["old_s"], h["ref_s"], 0.0)):
        r = torch.exp(x - old.double())
        d = ref.double() - x
        losses.append((w * (KL * (torch.exp(d) - d - 1) - torch.minimum(r * A, r.clamp(1 - LOW, 1 + HIGH) * A) - ent)).sum())
    gb, gs = torch.autograd.grad(losses[0] + losses[1], (wb, ws))
    norm = torch.sqrt((gb ** 2).sum() + (gs ** 2).sum())
    c = min(1.0, MAX_NORM / (float(norm) + 1e-6))
    return [float(v) for v in losses], gb * c, gs * c, float(norm)


def test_update(gpu):
    p = setup(gpu)
    buf = buffers(gpu)
    update(gpu, p, buf)
    torch.cuda.synchronize()
    assert int(buf["flag"].item()) == 0
    (lb, ls), gb, gs, norm = by_autograd(p)
    # The heads' fp32 products (sums of D terms of a few units) put logits and scores off by about D u = 2.4e-6 a token;
    # an ordered draw sums up to 48 such terms (1.2e-4), and a gradient of the weights sums 48 images (2400 tokens).
    assert abs(float(buf["st_b"][0]) - lb) <= 1e-5 and abs(float(buf["st_s"][0]) - ls) <= 4e-4
    assert norm > MAX_NORM and abs(float(buf["norm"]) - norm) <= 1e-3 * norm
    for got, want in ((buf["gb"], gb), (buf["gs"], gs)):
        assert float((got.cpu().double() - want).abs().max()) <= 1e-3 * MAX_NORM
    total = sum(float((buf[k].double() ** 2).sum()) for k in ("gb", "gs"))
    assert abs(np.sqrt(total) - MAX_NORM) <= 4 * U32 * MAX_NORM + MAX_NORM * 1e-6 / norm


def test_captured_and_replayed(gpu):
    """Replays give the eager results, with eager work between them; two
    captured updates with workspaces of their own run side by side."""
    p = setup(gpu)
    eager, bufs = buffers(gpu), [buffers(gpu), buffers(gpu)]
    update(gpu, p, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for b in bufs:
            update(gpu, p, b)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for b in bufs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            update(gpu, p, b)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for rep in range(4):
        p["adv"].neg_()                                # new inputs in the same places
        update(gpu, p, eager)
        for b in bufs:
            for k in OUT:
                b[k].fill_(7.0)
            b["ws_b"].fill_(0xA5)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for b in bufs:
            assert int(b["flag"].item()) == 0
            for k in OUT:
                assert torch.equal(b[k], eager[k]), (rep, k)


def test_without_the_native_marshalling(gpu, monkeypatch):
    """Through ctypes and the checks in Python, to the last bit the same."""
    p = setup(gpu)
    want, got = buffers(gpu), buffers(gpu)
    update(gpu, p, want)
    for name in ("_native_call", "_native_rows", "_native_spans", "_native_vectors"):
        monkeypatch.setattr(gpu, name, gpu._leave_to_ctypes)
    update(gpu, p, got)
    lp, H, st = gpu.dora_action_logprob(p["keys"][:, 0] @ p["wb"], p["actions"], legal=p["legal"])
    torch.cuda.synchronize()
    assert int(got["flag"].item()) == 0 and int(st.item()) == 0
    for k in OUT:
        assert torch.equal(got[k], want[k]), k
    assert torch.equal(lp[p["weight"] != 0], want["lp_b"][p["weight"] != 0])
    with pytest.raises(ValueError, match="adjacent"):
        gpu.dora_action_logprob(p["keys"][:, 0].t(), p["actions"])
    with pytest.raises(ValueError, match=r"actions must be \[48\]"):
        gpu.dora_action_logprob(p["keys"][:, 0], p["actions"][:3])
    with pytest.raises(ValueError, match="tensors on devices"):
        gpu.dora_grad_clip([got["gb"]], 1.0, norm_out=torch.zeros(1))
