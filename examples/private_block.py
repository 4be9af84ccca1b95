"""Private training of a small transformer, every step of it as the paper's section 3 has one: forward pass, output gradients,
per-sample norms of all parameters (linear weights and biases, gains and biases of the norms), clip factors, clipped sums, noise, optimizer.

    python examples/private_block.py [--layers 2 --width 256 --heads 4 --batch 8 --tokens 128 --steps 20 --state-bits 8 --dtype bf16]

The library forms norms, clipped gradients and noise, and runs layer norms, attention and AdamW; products with weights and the
activation between the two wide layers are torch's.  Parameters live in one flat fp32 buffer [W, b, ... , gain, bias, ...], the
16-bit weights of the products in another that the optimizer writes; gradients in a third, of which one rank of several would own a
contiguous shard."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2311_11822_amd import binding as dp  # noqa: E402
from paper_2311_11822_amd.block import AdamW, Attention, LayerNorm  # noqa: E402

TYPES = {"bf16": (torch.bfloat16, dp.DP_BF16), "f16": (torch.float16, dp.DP_F16), "f32": (torch.float32, dp.DP_F32)}


class PrivateTransformer:
    """`layers` pre-norm blocks of causal attention and two wide layers, a last norm and a projection to `classes`."""

    def __init__(self, layers, width, heads, classes, batch, tokens, dtype="bf16", state_bits=32, seed=0, device="cuda"):
        self.d, self.heads, self.B, self.T, self.layers, self.classes = width, heads, batch, tokens, layers, classes
        self.dtype, self.dt = TYPES[dtype]
        block = [(width, 3 * width), (width, width), (width, 4 * width), (4 * width, width)]
        self.linears = block * layers + [(width, classes)]
        self.n_norms = 2 * layers + 1
        shapes = [s for d_in, d_out in self.linears for s in ((d_in, d_out), (d_out,))] + [(2, width)] * self.n_norms
        sizes = [math.prod(s) for s in shapes]
        kw = dict(device=device)
        self.param, self.grad = torch.zeros(sum(sizes), **kw), torch.zeros(sum(sizes), **kw)
        views = lambda flat: [x.view(s) for x, s in zip(flat.split(sizes), shapes)]  # noqa: E731
        self.params, self.grads = views(self.param), views(self.grad)
        gen = torch.Generator(device=device).manual_seed(seed)
        for p in self.params[:2 * len(self.linears):2]:
            p.normal_(0, 0.5 / math.sqrt(p.shape[0]), generator=gen)
        for p in self.params[2 * len(self.linears):]:
            p[0].fill_(1.0)
        # products read 16-bit copies of the parameters, or the parameters themselves
        self.copy = self.param if self.dt == dp.DP_F32 else self.param.to(self.dtype)
        self.weights = views(self.copy)
        self.norms = [LayerNorm(p[0], p[1]) for p in self.params[2 * len(self.linears):]]
        # what is book-kept from the forward pass to the gradients
        B, T, L = batch, tokens, len(self.linears)
        empty = lambda *s: torch.empty(s, dtype=self.dtype, **kw)  # noqa: E731
        self.a = [empty(B, T, d_in) for d_in, _ in self.linears]
        self.g = [empty(B, T, d_out) for _, d_out in self.linears]
        self.stream = [empty(B, T, width) for _ in range(self.n_norms)]          # what each norm normalises
        self.stats = [(torch.empty((B, T), **kw), torch.empty((B, T), **kw)) for _ in range(self.n_norms)]
        self.kept = [torch.empty((B, 2, width), **kw) for _ in range(self.n_norms)]
        self.colsum = [torch.empty((B, d_out), **kw) for _, d_out in self.linears]
        self.o = [empty(B, T, heads, width // heads) for _ in range(layers)]
        self.lse = [torch.empty((B, heads, T), **kw) for _ in range(layers)]
        q, k, v = self.qkv(empty(B, T, 3 * width))
        self.attention = Attention(q, k, v, self.o[0], True, 1 / math.sqrt(width // heads))
        # one row of squared norms for each weight, each bias, each norm
        self.sqnorm = torch.zeros((2 * L + self.n_norms, B), **kw)
        self.C, self.norm = torch.zeros(B, **kw), torch.zeros(B, **kw)
        self.desc = dp.layer_array([(a, g, T, d_in, d_out, dp.dp_choose_path(T, d_in, d_out))
                                    for a, g, (d_in, d_out) in zip(self.a, self.g, self.linears)])
        self.ws = torch.empty(dp.dp_norms_multi_workspace_bytes(self.desc, self.dt, B), dtype=torch.uint8, **kw)
        decay = [0.1 if len(s) == 2 and s[0] > 2 else 0.0 for s in shapes]       # weights alone decay
        if state_bits == 8:
            state = torch.zeros(sum(sizes), device=device).to(torch.float8_e4m3fn), torch.zeros(sum(sizes), device=device).to(torch.float8_e4m3fn)
            blocks = [-(-n // 256) for n in sizes]
            scales = [list(torch.zeros(sum(blocks), **kw).split(blocks)) for _ in range(2)]
        else:
            state, scales = (torch.zeros(sum(sizes), **kw), torch.zeros(sum(sizes), **kw)), (None, None)
        copies = None if self.dt == dp.DP_F32 else list(self.copy.split(sizes))
        self.optimizer = AdamW(list(self.param.split(sizes)), list(self.grad.split(sizes)), *[list(s.split(sizes)) for s in state], decay,
                               copies, *scales)
        self.steps = 0

    def qkv(self, packed):
        return packed.view(self.B, self.T, 3, self.heads, self.d // self.heads).unbind(2)

    def linear(self, i, x):
        return torch.addmm(self.weights[2 * i + 1], x.view(-1, x.shape[-1]), self.weights[2 * i]).view(self.B, self.T, -1)

    def forward(self, x):
        """x: [B, T, d] in the storage type; logits [B, T, classes]."""
        add, self.packed, self.wide = None, [], []
        for n, norm in enumerate(self.norms):
            if add is None:
                self.stream[0].copy_(x)
            # the residual stream takes what the last sub-layer gave, in the norm's own pass
            norm.forward(self.stream[n - 1] if n else self.stream[0], self.a[self.linear_of(n)], *self.stats[n], add,
                         self.stream[n] if n else None)
            i, l = self.linear_of(n), n // 2
            y = self.linear(i, self.a[i])
            if n == self.n_norms - 1:
                return y
            if n % 2 == 0:
                self.packed.append(y)
                self.attention.forward(*self.qkv(y), self.o[l], self.lse[l])
                self.a[i + 1].copy_(self.o[l].view(self.B, self.T, self.d))
            else:
                self.wide.append(y)
                self.a[i + 1].copy_(torch.nn.functional.gelu(y))
            add = self.linear(i + 1, self.a[i + 1])

    def linear_of(self, n):
        """The linear layer that reads norm n."""
        return 2 * n

    def back(self, i):
        """Gradient of layer i's input from that of its output."""
        g = self.g[i].view(-1, self.g[i].shape[-1])
        return (g @ self.weights[2 * i].t()).view(self.B, self.T, -1)

    def backward(self, dlogits):
        """Output gradients of all linear layers, per-sample gradients of the norms."""
        L = len(self.linears)
        self.g[L - 1].copy_(dlogits)
        dstream = None
        for n in reversed(range(self.n_norms)):
            i, l = self.linear_of(n), n // 2
            if n < self.n_norms - 1:
                self.g[i + 1].copy_(dstream)
                da = self.back(i + 1)
                if n % 2 == 0:
                    self.attention.backward(*self.qkv(self.packed[l]), self.o[l], self.lse[l], da.view_as(self.o[l]),
                                            *self.qkv(self.g[i]))
                else:
                    self.g[i].copy_(torch.ops.aten.gelu_backward(da, self.wide[l]))
            dx = torch.empty_like(self.stream[n])
            self.norms[n].backward(self.stream[n], self.back(i), *self.stats[n], dx, self.kept[n], self.sqnorm[2 * L + n], dstream)
            dstream = dx

    def private_gradient(self, R, sigma, seed, mode=dp.DP_CLIP_AUTOMATIC, stability=0.01):
        """Clipped sum of all parameters' per-sample gradients plus noise, in self.grad."""
        B, T, L = self.B, self.T, len(self.linears)
        dp.dp_norms_multi(self.desc, self.dt, B, self.sqnorm, self.ws)
        for i, (_, d_out) in enumerate(self.linears):
            dp.dp_bias_norm(self.g[i], self.dt, B, T, d_out, self.colsum[i], self.sqnorm[L + i])
        dp.dp_clip_factors(self.sqnorm, self.sqnorm.shape[0], B, mode, R, stability, self.C, self.norm)
        dp.dp_clipped_grad_multi(self.desc, self.dt, B, self.C, self.grads[:2 * L:2])
        for i, (_, d_out) in enumerate(self.linears):
            dp.dp_clipped_bias_grad(self.colsum[i], B, d_out, self.C, self.grads[2 * i + 1])
        for n in range(self.n_norms):
            LayerNorm.clipped_gradient(self.kept[n], self.C, self.grads[2 * L + n])
        dp.dp_add_noise(self.grad, 0, self.grad.numel(), sigma, R, seed, self.steps)

    def step(self, x, targets, R=1.0, sigma=0.5, lr=1e-3, seed=1):
        """One private step; the mean loss before it."""
        logits = self.forward(x).float()
        loss = torch.nn.functional.cross_entropy(logits.view(-1, self.classes), targets.view(-1))
        dlogits = torch.softmax(logits, -1)
        dlogits.view(-1, self.classes)[torch.arange(targets.numel(), device=targets.device), targets.view(-1)] -= 1
        self.backward(dlogits / self.T)                    # a sample's loss is the mean over its tokens
        self.private_gradient(R, sigma, seed)
        self.steps += 1
        self.optimizer.step(self.steps, lr, 0.9, 0.99, 1e-8, 1.0 / self.B)
        return loss


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("layers", 2), ("width", 256), ("heads", 4), ("classes", 64), ("batch", 8), ("tokens", 128), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--dtype", default="bf16", choices=sorted(TYPES))
    ap.add_argument("--sigma", type=float, default=0.01)
    args = ap.parse_args()
    net = PrivateTransformer(args.layers, args.width, args.heads, args.classes, args.batch, args.tokens, args.dtype, args.state_bits)
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((args.batch, args.tokens, args.width), generator=gen, device="cuda").to(net.dtype)
    targets = torch.randint(args.classes, (args.batch, args.tokens), generator=gen, device="cuda")
    for step in range(args.steps):
        loss = net.step(x, targets, sigma=args.sigma)
        if step % 5 == 0 or step == args.steps - 1:
            print(f"step {step}: loss {loss.item():.4f}, clip factors {net.C.min().item():.3f} to {net.C.max().item():.3f}", flush=True)


if __name__ == "__main__":
    main()
