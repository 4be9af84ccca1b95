"""The gated example's private step against autograd in 64 bits: per-sample norms of all parameters together, clip factors, clipped sums, and
what the two optimizers make of them."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def reference(net, x, targets):
    """Per-sample gradients of every parameter, [B, total], in 64 bits on the CPU."""
    L, d, H, D, T = len(net.linears), net.d, net.heads, net.D, net.T
    params = [w.detach().cpu().double().requires_grad_() for w in net.weights[:2 * L]]
    params += [p.detach().cpu().double().requires_grad_() for p in net.params[2 * L:]]
    half = D // 2
    angle = torch.arange(T, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    cos, sin = angle.cos(), angle.sin()
    rows = []
    for b in range(net.B):
        def norm(n, s):
            g = params[2 * L + n]
            return (s - s.mean(-1, keepdim=True)) * (s.var(-1, unbiased=False, keepdim=True) + 1e-5) ** -0.5 * g[0] + g[1]

        def linear(i, y):
            return y @ params[2 * i] + params[2 * i + 1]

        def head(y, gain):                                   # y: [H, T, D]
            y = y * (y.square().mean(-1, keepdim=True) + 1e-6) ** -0.5 * gain
            first, second = y[..., :half], y[..., half:2 * half]
            return torch.cat((first * cos - second * sin, second * cos + first * sin, y[..., 2 * half:]), -1)
        s = x[b].cpu().double()
        for l in range(net.layers):
            gains = params[2 * L + net.n_norms + l]
            q, k, v = linear(5 * l, norm(2 * l, s)).view(T, 3, H, D).permute(1, 2, 0, 3)
            q, k = head(q, gains[0]), head(k, gains[1])
            w = (q @ k.mT / D ** 0.5).masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), float("-inf")).softmax(-1)
            s = s + linear(5 * l + 1, (w @ v).transpose(0, 1).reshape(T, d))
            y = norm(2 * l + 1, s)
            s = s + linear(5 * l + 4, torch.nn.functional.silu(linear(5 * l + 2, y)) * linear(5 * l + 3, y))
        loss = torch.nn.functional.cross_entropy(linear(L - 1, norm(net.n_norms - 1, s)), targets[b].cpu())
        rows.append(torch.cat([g.reshape(-1) for g in torch.autograd.grad(loss, params)]))
    return torch.stack(rows)


# f32: sums of some hundred products, a few layers deep.  bf16: every activation and output gradient is rounded (2^-8 at most, independent of each
# other), some sixteen roundings deep on the way to the first layer: 16^0.5 * 2^-8 = 1.6 %, doubled; norms average over many values.
@pytest.mark.parametrize("dtype,width,hidden,tokens,tol,norm_tol", [("f32", 16, 20, 9, 2e-5, 1e-5), ("bf16", 64, 136, 33, 3.2e-2, 1.3e-2)])
def test_private_gradient_of_gated_blocks(dtype, width, hidden, tokens, tol, norm_tol):
    from private_gated_block import PrivateGatedTransformer
    net = PrivateGatedTransformer(2, width, 2, hidden, 8, 3, tokens, dtype, seed=3)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((3, tokens, width), generator=gen).to(net.dtype).cuda()
    targets = torch.randint(8, (3, tokens), generator=gen).cuda()
    want = reference(net, x, targets)
    logits = net.forward(x).float()
    dlogits = torch.softmax(logits, -1) - torch.nn.functional.one_hot(targets, 8)
    net.backward(dlogits / tokens)
    net.private_gradient(1.0, 0.0, 1)
    norms = want.norm(dim=1)
    assert ((net.norm.cpu().double() - norms).abs() <= norm_tol * norms).all()
    C = 1.0 / (norms + 0.01)
    assert ((net.C.cpu().double() - C).abs() <= 2 * norm_tol * C).all()
    total = (C[:, None] * want).sum(0)
    assert (net.grad.cpu().double() - total).norm() <= tol * total.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_private_training_of_gated_blocks_runs(dtype):
    """Some steps: finite losses, copies that follow the parameters, updates of the size that the optimizers give them."""
    from private_gated_block import PrivateGatedTransformer
    net = PrivateGatedTransformer(1, 64, 2, 136, 8, 4, 24, dtype, seed=2)
    gen = torch.Generator().manual_seed(2)
    x = torch.randn((4, 24, 64), generator=gen).to(net.dtype).cuda()
    targets = torch.randint(8, (4, 24), generator=gen).cuda()
    for _ in range(6):
        before = net.param.clone()
        assert math.isfinite(net.step(x, targets, sigma=0.01, lr=3e-3).item())
        moved = [(a - b).view_as(p) for a, b, p in zip(net.param.split([p.numel() for p in net.params]), before.split([p.numel() for p in net.params]), net.params)]
        # an orthogonalised update's singular values lie within [0.6, 1.3] but for the smallest: its root mean square is near 0.2 lr
        for u in moved[:10:2]:
            assert 0.1 * 3e-3 <= u.square().mean().sqrt().item() <= 0.3 * 3e-3
    if net.copy is not net.param:
        assert torch.equal(net.copy, net.param.to(net.dtype))
