"""The example's private step against autograd in 64 bits: per-sample norms of all parameters together, clip factors and clipped sums."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def reference(net, x, targets):
    """Per-sample gradients of every parameter, [B, total], in 64 bits on the CPU."""
    L, d, H, T = len(net.linears), net.d, net.heads, net.T
    params = [w.detach().cpu().double().requires_grad_() for w in net.weights[:2 * L]]
    params += [p.detach().cpu().double().requires_grad_() for p in net.params[2 * L:]]
    rows = []
    for b in range(net.B):
        def norm(n, s):
            g = params[2 * L + n]
            return (s - s.mean(-1, keepdim=True)) * (s.var(-1, unbiased=False, keepdim=True) + 1e-5) ** -0.5 * g[0] + g[1]
        def linear(i, y):
            return y @ params[2 * i] + params[2 * i + 1]
        s = x[b].cpu().double()
        for l in range(net.layers):
            q, k, v = linear(4 * l, norm(2 * l, s)).view(T, 3, H, d // H).permute(1, 2, 0, 3)
            w = (q @ k.mT / (d // H) ** 0.5).masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), float("-inf")).softmax(-1)
            s = s + linear(4 * l + 1, (w @ v).transpose(0, 1).reshape(T, d))
            s = s + linear(4 * l + 3, torch.nn.functional.gelu(linear(4 * l + 2, norm(2 * l + 1, s))))
        logits = linear(L - 1, norm(net.n_norms - 1, s))
        loss = torch.nn.functional.cross_entropy(logits, targets[b].cpu())
        rows.append(torch.cat([g.reshape(-1) for g in torch.autograd.grad(loss, params)]))
    return torch.stack(rows)


# f32: sums of some hundred products, a few layers deep.  bf16: every activation and output gradient is rounded (2^-8 at most, independent
# of each other), some ten roundings deep on the way to the first layer: 10^0.5 * 2^-8 = 1.2 %, doubled; norms average over many values.
@pytest.mark.parametrize("dtype,width,tokens,tol,norm_tol", [("f32", 16, 9, 2e-5, 1e-5), ("bf16", 64, 33, 2.5e-2, 1e-2)])
def test_private_gradient(dtype, width, tokens, tol, norm_tol):
    from private_block import PrivateTransformer
    net = PrivateTransformer(2, width, 2, 8, 3, tokens, dtype, 32, seed=3)
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


@pytest.mark.parametrize("dtype,bits", [("bf16", 8), ("f16", 32), ("f32", 8)])
def test_private_training_learns(dtype, bits):
    """A small network fits random targets under clipping and a little noise."""
    from private_block import PrivateTransformer
    net = PrivateTransformer(1, 64, 2, 8, 4, 24, dtype, bits, seed=2)
    gen = torch.Generator().manual_seed(2)
    x = torch.randn((4, 24, 64), generator=gen).to(net.dtype).cuda()
    targets = torch.randint(8, (4, 24), generator=gen).cuda()
    losses = [net.step(x, targets, sigma=0.001, lr=3e-3).item() for _ in range(40)]
    assert losses[-1] < 0.5 * losses[0]
    if net.copy is not net.param:
        assert torch.equal(net.copy, net.param.to(net.dtype))
