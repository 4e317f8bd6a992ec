"""A transformer block's attention half over packed, pruned tokens, forward and
backward, by the operators as a program uses them together: select/pack, norm,
projections (library products), rotary positions of the kept patches, attention,
residual with layer scale and dropped branches, norm.  Against automatic
differentiation in 64 bits, captured and replayed, and through ctypes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

B, SIDE, H, Hk, D = 5, 12, 4, 2, 32
N, C = SIDE * SIDE + 1, 128
U = 2.0 ** -24


def setup(gpu, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(21)

    def rnd(*shape, s=1.0, t=dtype):
        return (s * torch.randn(shape, generator=g, device="cuda")).to(t)
    keep = torch.tensor([145, 60, 1, 97, 33], dtype=torch.int32, device="cuda")
    idx, cu, packed, _ = gpu.dora_select_pack(rnd(B, N, t=torch.float32), keep, rnd(B, N, C))
    n = int(keep.sum())
    patch = (idx[:n] - 1).clamp(min=0)
    p = dict(x=packed[:n].clone(), cu=cu, n=n, max_q=int(keep.max()),
             pos=torch.stack([patch // SIDE, patch % SIDE], 1).int().contiguous(),
             freq=gpu.rope_frequencies(D // 2, base=100.0).repeat(2),
             wqkv=rnd(C, (H + 2 * Hk) * D, s=C ** -0.5), wo=rnd(H * D, C, s=(H * D) ** -0.5),
             g1=1 + rnd(C, s=0.1, t=torch.float32), b1=rnd(C, s=0.1, t=torch.float32), g2=1 + rnd(C, s=0.1, t=torch.float32),
             b2=rnd(C, s=0.1, t=torch.float32), ls=0.5 + rnd(C, s=0.1, t=torch.float32), dy=rnd(n, C), dh=rnd(n, C))
    p["gate"] = torch.repeat_interleave(torch.tensor([1.25, 0.0, 1.25, 1.25, 1.25], device="cuda"), keep.long())
    return p


def buffers(gpu, p):
    n, dev, t = p["n"], "cuda", p["x"].dtype

    def e(*s, dtype=t):
        return torch.empty(s, dtype=dtype, device=dev)
    f = torch.float32
    return dict(h0=e(n, C), y0=e(n, C), qkv=e(n, H + 2 * Hk, D), out=e(n, H, D), lse=e(n, H, dtype=f), a=e(n, C), h=e(n, C),
                y=e(n, C), dx1=e(n, C), da=e(n, C), dqkv=e(n, H + 2 * Hk, D), dout=e(n, H * D), dy0=e(n, C), dx=e(n, C),
                dwo=e(H * D, C), dwqkv=e(C, (H + 2 * Hk) * D), dg2=e(C, dtype=f), db2=e(C, dtype=f), dls=e(C, dtype=f),
                dgate=e(n, dtype=f), dg1=e(C, dtype=f), db1=e(C, dtype=f),
                ws=gpu.new_grouped_attn_workspace(B, H, Hk, D, p["max_q"], n, n, backward=True),
                ws_n=gpu.new_residual_norm_workspace(n, C), flag=gpu.new_status())


OUT = ("h", "y", "dx", "dwo", "dwqkv", "dg1", "db1", "dg2", "db2", "dls", "dgate")


def block(gpu, p, b):
    n = p["n"]
    _, y0 = gpu.dora_residual_norm(p["x"], None, p["g1"], p["b1"], y_out=b["y0"])
    torch.matmul(y0, p["wqkv"], out=b["qkv"].view(n, -1))
    q, k, v = b["qkv"][:, :H], b["qkv"][:, H:H + Hk], b["qkv"][:, H + Hk:]
    gpu.dora_rope(q, p["pos"], p["freq"], k=k, q_out=q, k_out=k)
    gpu.dora_grouped_attn(q, k, v, p["cu"], p["max_q"], out=b["out"], lse_out=b["lse"], workspace=b["ws"], dev_status=b["flag"])
    torch.matmul(b["out"].view(n, -1), p["wo"], out=b["a"])
    gpu.dora_residual_norm(p["x"], b["a"], p["g2"], p["b2"], scale=p["ls"], gate=p["gate"], h_out=b["h"], y_out=b["y"])
    # and back
    gpu.dora_residual_norm_backward(p["dy"], b["h"], b["a"], p["g2"], p["b2"], scale=p["ls"], gate=p["gate"], dh=p["dh"],
                                    dx=b["dx1"], da=b["da"], dgamma=b["dg2"], dbeta=b["db2"], dscale=b["dls"], dgate=b["dgate"],
                                    workspace=b["ws_n"])
    torch.matmul(b["out"].view(n, -1).t(), b["da"], out=b["dwo"])
    torch.matmul(b["da"], p["wo"].t(), out=b["dout"])
    dq, dk, dv = b["dqkv"][:, :H], b["dqkv"][:, H:H + Hk], b["dqkv"][:, H + Hk:]
    gpu.dora_grouped_attn_backward(b["dout"].view(n, H, D), q, k, v, b["out"], b["lse"], p["cu"], p["max_q"], dq=dq, dk=dk, dv=dv,
                                   workspace=b["ws"], dev_status=b["flag"])
    gpu.dora_rope(dq, p["pos"], p["freq"], k=dk, inverse=True, q_out=dq, k_out=dk)
    torch.matmul(y0.t(), b["dqkv"].view(n, -1), out=b["dwqkv"])
    torch.matmul(b["dqkv"].view(n, -1), p["wqkv"].t(), out=b["dy0"])
    gpu.dora_residual_norm_backward(b["dy0"], p["x"], None, p["g1"], p["b1"], dh=b["dx1"], dx=b["dx"], dgamma=b["dg1"],
                                    dbeta=b["db1"], workspace=b["ws_n"])


def by_autograd(p):
    h = {k: v.cpu().double() if v.is_floating_point() else v.cpu() for k, v in p.items() if isinstance(v, torch.Tensor)}
    leaves = ("x", "wo", "wqkv", "g1", "b1", "g2", "b2", "ls", "gate")
    for k in leaves:
        h[k].requires_grad_()
    n = p["n"]
    y0 = torch.nn.functional.layer_norm(h["x"], (C,), h["g1"], h["b1"], 1e-6)
    qkv = (y0 @ h["wqkv"]).view(n, -1, D)
    t = h["pos"].double().repeat_interleave(D // 4, 1) * h["freq"]
    z = torch.complex(qkv[:, :H + Hk, :D // 2], qkv[:, :H + Hk, D // 2:]) * torch.polar(torch.ones_like(t), t)[:, None]
    qk = torch.cat([z.real, z.imag], -1)
    outs = []
    for b in range(B):
        r = slice(int(h["cu"][b]), int(h["cu"][b + 1]))
        q = qk[r, :H].transpose(0, 1)
        k = qk[r, H:].transpose(0, 1).repeat_interleave(H // Hk, 0)
        v = qkv[r, H + Hk:].transpose(0, 1).repeat_interleave(H // Hk, 0)
        outs.append((torch.softmax(q @ k.transpose(1, 2) / math.sqrt(D), -1) @ v).transpose(0, 1))
    a = torch.cat(outs).reshape(n, -1) @ h["wo"]
    res = h["x"] + h["gate"][:, None] * h["ls"] * a
    y = torch.nn.functional.layer_norm(res, (C,), h["g2"], h["b2"], 1e-6)
    grads = torch.autograd.grad([y, res], [h[k] for k in leaves], [h["dy"], h["dh"]])
    names = dict(zip(("dx", "dwo", "dwqkv", "dg1", "db1", "dg2", "db2", "dls", "dgate"), grads))
    return dict(names, h=res.detach(), y=y.detach())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block(gpu, dtype):
    p = setup(gpu, dtype)
    b = buffers(gpu, p)
    block(gpu, p, b)
    torch.cuda.synchronize()
    assert int(b["flag"]) == 0
    want = by_autograd(p)
    # Relative to each result's size (2-norm).  fp32: about 12 stages of sums of up to 336 terms, 336 u each.  bf16: each of
    # 12 stages rounds to 2^-8 at most, their effects independent: sqrt(12) 2^-8, twice for what the norms magnify.
    limit = 12 * 336 * U if dtype == torch.float32 else 2 * math.sqrt(12) * 2.0 ** -8
    for n in OUT:
        off = float((b[n].double().cpu() - want[n]).norm() / want[n].norm())
        assert off <= limit, (n, off, limit)


def test_captured_and_replayed(gpu):
    """Replays give the eager results, with eager work between them; two captured blocks with workspaces of their own run
    side by side, beside a live autograd graph of the same inputs."""
    p = setup(gpu)
    leaf = p["x"].clone().requires_grad_()
    live = (leaf * leaf).sum()
    eager, bufs = buffers(gpu, p), [buffers(gpu, p), buffers(gpu, p)]
    block(gpu, p, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for b in bufs:
            block(gpu, p, b)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for b in bufs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            block(gpu, p, b)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for rep in range(4):
        p["dy"].neg_(), p["x"].mul_(1.0 + 0.1 * rep)
        block(gpu, p, eager)
        for b in bufs:
            for k in OUT:
                b[k].fill_(7.0)
            b["ws"].fill_(0xA5), b["ws_n"].fill_(0xA5)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for b in bufs:
            assert int(b["flag"]) == 0
            for k in OUT:
                assert torch.equal(b[k], eager[k]), (rep, k)
    live.backward()
    assert torch.equal(leaf.grad, 2 * leaf.detach())


def test_without_the_native_marshalling(gpu, monkeypatch):
    p = setup(gpu)
    want, got = buffers(gpu, p), buffers(gpu, p)
    block(gpu, p, want)
    for name in ("_native_call", "_native_vectors", "_native_describe", "_native_written"):
        monkeypatch.setattr(gpu, name, gpu._leave_to_ctypes)
    block(gpu, p, got)
    torch.cuda.synchronize()
    for k in OUT:
        assert torch.equal(got[k], want[k]), k
    q = torch.zeros((4, 2, 64), device="cuda")
    pos, freq = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(32, dtype=torch.float64, device="cuda")
    with pytest.raises(ValueError, match="adjacent"):
        gpu.dora_rope(q.transpose(1, 2), pos, freq)
    with pytest.raises(TypeError, match="int32"):
        gpu.dora_rope(q, pos.long(), freq)
    with pytest.raises(ValueError, match="tensors on devices"):
        gpu.dora_rope(q, pos.cpu(), freq)
    with pytest.raises(ValueError, match=r"gamma must be \[8\]"):
        gpu.dora_residual_norm(torch.zeros((2, 8), device="cuda"), None, torch.zeros(4, device="cuda"))


def test_arguments(gpu):
    q = torch.zeros((4, 2, 64), device="cuda")
    cu = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    for bad, error in ((dict(q=q.double()), TypeError), (dict(k=q[:, :, :32], v=q[:, :, :32]), gpu.DoraError),
                       (dict(cu_q=cu.long()), TypeError), (dict(cu_k=cu[:1]), ValueError), (dict(lse_out=q), ValueError),
                       (dict(out=q), gpu.DoraError), (dict(workspace=q[:1, :1]), gpu.DoraError),
                       (dict(q=q.bfloat16()), gpu.DoraError), (dict(v=q[:3]), gpu.DoraError)):
        args = dict(q=q, k=q, v=q, cu_q=cu, max_q=4)
        args.update(bad)
        with pytest.raises(error):
            gpu.dora_grouped_attn(**args)
    y = torch.zeros((4, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    for bad, error in ((dict(gamma=w[:32]), ValueError), (dict(scale=w), gpu.DoraError), (dict(x=y.half()), TypeError),
                       (dict(y_out=torch.zeros((4, 32), device="cuda")), gpu.DoraError), (dict(gamma=w.bfloat16()), TypeError)):
        args = dict(x=y, a=None, gamma=w)
        args.update(bad)
        with pytest.raises(error):
            gpu.dora_residual_norm(**args)
    with pytest.raises(ValueError, match="dscale without scale"):
        gpu.dora_residual_norm_backward(y, y, None, w, dscale=w.clone())
