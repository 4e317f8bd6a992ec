"""The block operators' references: against automatic differentiation, differences
and torch's own functions, in 64 bits on the CPU."""
import itertools

import pytest
import torch

import block_ref as ref


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(shape, g, dtype=torch.float64):
    return torch.randn(shape, generator=g, dtype=dtype)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_a_rotation_and_inverse_its_gradient(interleaved):
    g = gen(1)
    x = randn((5, 3, 16), g).float()
    pos = torch.randint(-50, 50, (5, 2), generator=g)
    freq = torch.rand(6, generator=g, dtype=torch.float64)
    y, _ = ref.rope(x, pos, freq, interleaved, False, 1.5)
    back, _ = ref.rope(y, pos, freq, interleaved, True, 1 / 1.5)
    assert torch.allclose(back, x.double(), atol=1e-14)
    assert torch.equal(y[..., 12:], x.double()[..., 12:])
    assert torch.allclose(y[..., :12].norm(dim=-1), 1.5 * x.double()[..., :12].norm(dim=-1))
    # pair i: its own axis, angle and places
    for i in range(6):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 6)
        t = pos[:, i // 3].double() * freq[i]
        assert torch.allclose(y[:, 1, a], 1.5 * (x[:, 1, a].double() * t.cos() - x[:, 1, b].double() * t.sin()))
    # <rope(x), w> = <x, inverse(w)>
    w = randn(x.shape, g)
    z, _ = ref.rope(w, pos, freq, interleaved, True, 1.5)
    assert torch.allclose((y * w).sum(), (x.double() * z).sum())


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients(causal):
    """Out against torch's attention, gradients against automatic differentiation and a difference."""
    g = gen(2)
    cu_q, cu_k, H, Hk, D = [0, 3, 3, 8], [0, 5, 6, 11], 4, 2, 32
    q, k, v = randn((8, H, D), g).requires_grad_(), randn((11, Hk, D), g).requires_grad_(), randn((11, Hk, D), g).requires_grad_()

    def forward(q, k, v):
        outs = []
        for b in range(3):
            qb, kb, vb = (t[c[b]:c[b + 1]].transpose(0, 1) for t, c in ((q, cu_q), (k, cu_k), (v, cu_k)))
            kb, vb = kb.repeat_interleave(H // Hk, 0), vb.repeat_interleave(H // Hk, 0)
            s = qb @ kb.transpose(1, 2) * float(torch.tensor(D ** -0.5))
            if causal:
                n, m = s.shape[1:]
                s = s.masked_fill(torch.arange(m)[None] > torch.arange(n)[:, None] + m - n, -float("inf"))
            outs.append((torch.softmax(s, -1) @ vb).transpose(0, 1))
        return torch.cat(outs)

    out = forward(q, k, v)
    w = randn(out.shape, g)
    want = torch.autograd.grad((out * w).sum(), (q, k, v))
    f, _ = ref.attention(q.detach(), k.detach(), v.detach(), cu_q, cu_k, causal)
    assert torch.allclose(f["out"], out.detach(), atol=1e-12)
    b, _ = ref.attention(q.detach(), k.detach(), v.detach(), cu_q, cu_k, causal, dout=w, out=f["out"], lse=f["lse"])
    for n, x in zip(("dq", "dk", "dv"), want):
        assert torch.allclose(b[n], x, atol=1e-12), n
    step = torch.zeros_like(k)
    step[7, 1, 5] = 1e-5
    with torch.no_grad():
        d = ((forward(q, k + step, v) - forward(q, k - step, v)) * w).sum() / 2e-5
    assert abs(float(d - b["dk"][7, 1, 5])) < 1e-7


@pytest.mark.parametrize("kind,post,gate", itertools.product(("layer", "rms"), (False, True), (False, True)))
def test_norm_gradients(kind, post, gate):
    g = gen(3)
    T, C = 6, 24
    names = ["gamma", "beta", "scale"] + (["post_gamma", "post_beta"] if post else [])
    p = {n: (1 + 0.3 * randn((C,), g)).requires_grad_() for n in names}
    if gate:
        p["gate"] = randn((T,), g)
        p["gate"][2] = 0.0
        p["gate"].requires_grad_()
    x, a = randn((T, C), g).requires_grad_(), randn((T, C), g).requires_grad_()
    eps = 1e-3

    def norm(z, w, b):
        if kind == "layer":
            return torch.nn.functional.layer_norm(z, (C,), w, b, eps)
        return z / torch.sqrt(z.pow(2).mean(1, keepdim=True) + eps) * w + b

    u = norm(a, p["post_gamma"], p["post_beta"]) if post else a
    h = x + (p["gate"][:, None] if gate else 1.0) * p["scale"] * u
    y = norm(h, p["gamma"], p["beta"])
    dp = {n: t.detach() for n, t in p.items()}
    f, _ = ref.residual_norm(x.detach(), a.detach(), dp, kind, eps)
    assert torch.allclose(f["h"], h.detach()) and torch.allclose(f["y"], y.detach())
    dy, dh = randn((T, C), g), randn((T, C), g)
    want = torch.autograd.grad([y, h], [x, a] + list(p.values()), [dy, dh])
    got, _ = ref.residual_norm_backward(dy, dh, h.detach(), a.detach(), dp, kind, eps)
    for n, w in zip(["dx", "da"] + ["d" + n for n in p], want):
        assert torch.allclose(got[n], w, atol=1e-10), n
    # the gradients that are not given count as 0
    want = torch.autograd.grad(norm(x + u, p["gamma"], p["beta"]), x, dy)[0] if post else None
    if want is not None:
        got, _ = ref.residual_norm_backward(dy, None, (x + u).detach(), a.detach(), {k: v for k, v in dp.items() if k not in ("scale", "gate")},
                                            kind, eps)
        assert torch.allclose(got["dx"], want, atol=1e-10)
