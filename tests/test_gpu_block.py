"""Layer norm, attention and AdamW against plain 64-bit implementations on the CPU, at the sizes, masks and layouts where they can
go wrong.

Tolerances, relative in the 2-norm unless said otherwise.  u is the rounding of the storage type, half a unit in the last place
of a number just above a power of two: 2^-8 for bf16 (8 bits of significand), 2^-11 for fp16 (11), 2^-24 for fp32 (24).
  stored results     one rounding: u
  attention          probabilities (their gradients) are rounded to the type before the second product, the result once more: the two
                     together at most 2 u; 2.5 u is asked for, and 2e-6 for fp32 (sums of up to some hundred products in fp32)
  fp32 sums          sums of n rounded products err by some sqrt(n) 2^-24, at most 2e-6 here; squares by twice that
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
FP32 = 2e-6


@pytest.fixture(scope="module")
def block():
    from paper_2311_11822_amd import block as b
    assert torch.cuda.is_available()
    return b


def rel(got, want):
    got, want = got.detach().cpu().double(), want.detach().cpu().double()
    assert got.shape == want.shape
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].nan_to_num(), want[~fine].nan_to_num())
    norm = want[fine].norm().item()
    off = (got[fine] - want[fine]).norm().item()
    return off / norm if norm else (0.0 if off == 0 else math.inf)


def rand(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(DTYPES[dtype])


# ------------------------------------------------------------------------------------------------ layer norm

NORM_SIZES = [(1, 1, 1), (4, 8, 16), (3, 5, 7), (2, 33, 64), (2, 9, 768), (1, 70, 1280), (5, 1, 2048), (2, 3, 2050), (1, 19, 2056),
              (2, 4, 12288), (1, 2, 4097), (1, 3, 16392), (1, 2, 32768), (300, 1, 40), (2, 200, 24), (1, 5, 8191)]

# Rows that begin at every place of a 16-byte piece: by waves and by workgroups, few and many rows to a sample, the last widths of a form.
NORM_SIZES += [(2, 37, 4099), (3, 50, 1021), (1, 20, 9001), (2, 70, 2041), (1, 33, 2045), (1, 3, 32767), (1, 9, 16383), (3, 9, 1017), (1, 300, 2049),
               (2, 11, 8185), (1, 130, 3), (40, 3, 2058)]


def norm_reference(x, gain, bias, eps):
    x = x.double()
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    rstd = (var + eps) ** -0.5
    return (x - mean[..., None]) * rstd[..., None] * gain.double() + bias.double(), mean, rstd


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,T,d", NORM_SIZES)
def test_layer_norm(block, dtype, B, T, d):
    gen = torch.Generator().manual_seed(B * 1000003 + T * 1009 + d)
    x, add = rand(gen, (B, T, d), dtype, 2.0), rand(gen, (B, T, d), dtype)
    gain, bias = rand(gen, (d,), "f32"), rand(gen, (d,), "f32")
    dev = [t.cuda() for t in (x, add, gain, bias)]
    for joined in (False, True):
        y, total = torch.full_like(dev[0], 9), torch.full_like(dev[0], 9)
        mean, rstd = torch.empty((B, T), device="cuda"), torch.empty((B, T), device="cuda")
        norm = block.LayerNorm(dev[2], dev[3], 1e-5)
        norm.forward(dev[0], y, mean, rstd, dev[1] if joined else None, total if joined else None)
        s = (x.double() + add.double()).to(x.dtype) if joined and dtype != "f32" else x + add if joined else x
        if joined:
            assert torch.equal(total.cpu(), s)
        want, m, r = norm_reference(s, gain, bias, 1e-5)
        # a row of one value is its bias; the mean of few values may cancel: against the values' size
        assert (mean.cpu().double() - m).abs().max() <= FP32 * s.double().abs().max()
        assert rel(rstd, r) <= FP32
        assert rel(y, want) <= U[dtype] + 4 * FP32
        again = torch.empty_like(y)
        norm.forward(dev[0], again, None, None, dev[1] if joined else None, total if joined else None)
        assert torch.equal(again, y)
    bare = torch.empty_like(dev[0])
    block.LayerNorm(None, None, 1e-5).forward(dev[0], bare)
    assert rel(bare, norm_reference(x, torch.ones(d), torch.zeros(d), 1e-5)[0]) <= U[dtype] + 4 * FP32 or d == 1


# The mean of n values comes out of fp32 sums of up to 72 values a thread, 6 steps in a wave and 8 waves: within 100 * 2^-24 of its size.  y errs by
# that times rstd, and by its own rounding; the variance, formed around that mean, by its square.
@pytest.mark.parametrize("dtype,shift", [("f32", 1e3), ("f32", -3e4), ("f16", 300.0), ("bf16", 40.0)])
@pytest.mark.parametrize("d", [64, 1000, 1021, 4096, 12289])
def test_layer_norm_of_rows_far_from_zero(block, dtype, shift, d):
    gen = torch.Generator().manual_seed(d)
    x = (torch.randn((2, 5, d), generator=gen, dtype=torch.float64) + shift).to(DTYPES[dtype])
    gain, bias = rand(gen, (d,), "f32"), rand(gen, (d,), "f32")
    y, mean, rstd = torch.empty_like(x, device="cuda"), torch.empty((2, 5), device="cuda"), torch.empty((2, 5), device="cuda")
    block.LayerNorm(gain.cuda(), bias.cuda(), 1e-5).forward(x.cuda(), y, mean, rstd)
    want, m, r = norm_reference(x, gain, bias, 1e-5)
    off = 100 * 2.0 ** -24 * abs(shift)
    assert (mean.cpu().double() - m).abs().max() <= off
    assert ((rstd.cpu().double() - r).abs() <= r * (FP32 + (off * r) ** 2)).all()
    err = (y.cpu().double() - want).norm().item()
    assert err <= U[dtype] * want.norm().item() + (off + 2.0 ** -24 * abs(shift)) * (r[..., None] * gain.double()).norm().item() + 4 * FP32 * want.norm().item()


def norm_grad_reference(x, dy, gain, mean, rstd):
    x, dy, gain, mean, rstd = (t.double() for t in (x, dy, gain, mean, rstd))
    h = (x - mean[..., None]) * rstd[..., None]
    u = dy * gain
    dx = (u - u.mean(-1, keepdim=True) - h * (u * h).mean(-1, keepdim=True)) * rstd[..., None]
    return dx, torch.stack(((dy * h).sum(1), dy.sum(1)), 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,T,d", NORM_SIZES)
def test_layer_norm_backward(block, dtype, B, T, d):
    gen = torch.Generator().manual_seed(B * 1000003 + T * 1009 + d + 1)
    x, dy, add = rand(gen, (B, T, d), dtype, 2.0), rand(gen, (B, T, d), dtype, 0.01), rand(gen, (B, T, d), dtype, 0.01)
    gain = rand(gen, (d,), "f32")
    _, mean, rstd = norm_reference(x, gain, gain, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    xd, dyd, addd, gd, md, rd = (t.cuda() for t in (x, dy, add, gain, mean, rstd))
    norm = block.LayerNorm(gd, None, 1e-5)
    dx, kept, sq = torch.full_like(xd, 9), torch.full((B, 2, d), 9.0, device="cuda"), torch.full((B,), 9.0, device="cuda")
    want, want_kept = norm_grad_reference(x, dy, gain, mean, rstd)
    size = (dy.double().norm() * gain.double().abs().max() * rstd.double().max()).item()        # what cancels in dx

    def close(got, ref):
        return (got.cpu().double() - ref).norm().item() <= 1.01 * U[dtype] * ref.norm().item() + 4 * FP32 * size

    norm.backward(xd, dyd, md, rd, dx, kept, sq)
    assert close(dx, want)
    assert rel(kept, want_kept) <= 4 * FP32
    assert rel(sq, (want_kept ** 2).sum((1, 2))) <= 8 * FP32
    with_add = torch.full_like(xd, 9)
    norm.backward(xd, dyd, md, rd, with_add, add=addd)                  # dx alone
    assert close(with_add, want + add.double())
    kept2, sq2 = torch.empty_like(kept), torch.empty_like(sq)
    norm.backward(xd, dyd, md, rd, None, kept2, sq2)                    # weights' gradients alone
    assert torch.equal(kept2, kept) and torch.equal(sq2, sq)
    norm.backward(xd, dyd, md, rd, dyd, add=addd)                       # in place of dy
    assert torch.equal(dyd, with_add)
    C = torch.linspace(0.1, 1.0, B)
    grad = torch.empty((2, d), device="cuda")
    norm.clipped_gradient(kept, C.cuda(), grad)
    want_sum = (C.double()[:, None, None] * want_kept).sum(0)
    assert (grad.cpu().double() - want_sum).norm() <= 4 * FP32 * (C.double()[:, None, None] * want_kept).norm() * math.sqrt(B)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [1021, 4100, 4099])
def test_layer_norm_in_place(block, dtype, d):
    """The sum over x or over what is added, dx over dy or over what is added: the same bits, rows beside them whole."""
    gen = torch.Generator().manual_seed(d)
    x, add, dy = (rand(gen, (2, 30, d), dtype).cuda() for _ in range(3))
    norm = block.LayerNorm(torch.randn(d, generator=gen).cuda(), None)
    new = lambda: (torch.empty((2, 30), device="cuda"), torch.empty((2, 30), device="cuda"))  # noqa: E731
    y, total, stats = torch.empty_like(x), torch.empty_like(x), new()
    norm.forward(x, y, *stats, add, total)
    for over in (0, 1):
        args, other = [x.clone(), add.clone()], torch.empty_like(x)
        norm.forward(args[0], other, *new(), args[1], args[over])
        assert torch.equal(args[over], total) and torch.equal(other, y)
    dx, kept, sq = torch.empty_like(x), torch.empty((2, 2, d), device="cuda"), torch.empty(2, device="cuda")
    norm.backward(total, dy, *stats, dx, kept, sq, add)
    for over in (0, 1):
        args, k2, s2 = [dy.clone(), add.clone()], torch.empty_like(kept), torch.empty_like(sq)
        norm.backward(total, args[0], *stats, args[over], k2, s2, args[1])
        assert torch.equal(args[over], dx) and torch.equal(k2, kept) and torch.equal(s2, sq)


def test_layer_norm_gradient_against_differences(block):
    """The gradient's formula, from the forward pass in fp32 alone: a central difference along a direction."""
    gen = torch.Generator().manual_seed(5)
    x, dy, dirn = (rand(gen, (2, 3, 96), "f32").cuda() for _ in range(3))
    gain, bias, kept, sq = rand(gen, (96,), "f32").cuda(), rand(gen, (96,), "f32").cuda(), torch.empty((2, 2, 96), device="cuda"), torch.empty(2, device="cuda")
    mean, rstd, y, dx = torch.empty((2, 3), device="cuda"), torch.empty((2, 3), device="cuda"), torch.empty_like(x), torch.empty_like(x)
    norm = block.LayerNorm(gain, bias)

    def loss(x, gain):
        block.LayerNorm(gain, bias).forward(x.contiguous(), y)
        return (y.double() * dy.double()).sum().item()

    norm.forward(x, y, mean, rstd)
    norm.backward(x, dy, mean, rstd, dx, kept, sq)
    h = 2.0 ** -6                                                       # error: h^2 of the third derivative, 2^-24 / h of rounding
    slope = (loss(x + h * dirn, gain) - loss(x - h * dirn, gain)) / (2 * h)
    assert abs(slope - (dx.double() * dirn.double()).sum().item()) <= 2e-3 * (dx.norm() * dirn.norm()).item()
    gdir = dirn[0, 0]
    slope = (loss(x, gain + h * gdir) - loss(x, gain - h * gdir)) / (2 * h)
    assert abs(slope - (kept[:, 0].sum(0).double() * gdir.double()).sum().item()) <= 1e-4 * (kept.norm() * gdir.norm()).item()


# ------------------------------------------------------------------------------------------------ attention

class Case:
    """One attention call: packed projections where Tq == Tk, reference in 64 bits."""

    def __init__(self, block, dtype, B, Tq, Tk, H, Hkv, D, causal, q_len=None, k_len=None, seed=0, scale=None):
        gen = torch.Generator().manual_seed(seed + 7919 * Tq + 104729 * Tk + D + 31 * H)
        self.block, self.dtype, self.causal = block, dtype, causal
        self.B, self.Tq, self.Tk, self.H, self.Hkv, self.D = B, Tq, Tk, H, Hkv, D
        self.scale = 1 / math.sqrt(D) if scale is None else scale
        self.q_len = None if q_len is None else torch.tensor(q_len, dtype=torch.int32)
        self.k_len = None if k_len is None else torch.tensor(k_len, dtype=torch.int32)
        self.q, self.k, self.v = self.projections(lambda shape: rand(gen, shape, dtype))
        self.do = rand(gen, (B, Tq, H, D), dtype, 0.1)

    def projections(self, make):
        if self.Tq == self.Tk:
            packed = make((self.B, self.Tq, self.H + 2 * self.Hkv, self.D))
            return packed[:, :, :self.H], packed[:, :, self.H:self.H + self.Hkv], packed[:, :, self.H + self.Hkv:]
        kv = make((self.B, self.Tk, 2 * self.Hkv, self.D))
        return make((self.B, self.Tq, self.H, self.D)), kv[:, :, :self.Hkv], kv[:, :, self.Hkv:]

    def seen(self):
        n = torch.full((self.B,), self.Tq) if self.q_len is None else self.q_len.clamp(0, self.Tq)
        m = torch.full((self.B,), self.Tk) if self.k_len is None else self.k_len.clamp(0, self.Tk)
        i, j = torch.arange(self.Tq)[None, :, None], torch.arange(self.Tk)[None, None, :]
        n, m = n[:, None, None].long(), m[:, None, None].long()
        ok = (i < n) & (j < m)
        return (ok & (j - m <= i - n) if self.causal else ok)[:, None]

    def reference(self, o=None):
        """(o, lse), and the gradients where o (as the forward pass stored it) is given."""
        G = self.H // self.Hkv
        q, do = self.q.double().transpose(1, 2), self.do.double().transpose(1, 2)
        k, v = (t.double().transpose(1, 2).repeat_interleave(G, 1) for t in (self.k, self.v))
        seen = self.seen().expand(self.B, self.H, self.Tq, self.Tk)
        # what is not seen takes no part, whatever it holds
        clean = lambda t: t.nan_to_num(0, 0, 0)  # noqa: E731
        s = (clean(q) @ clean(k).mT * self.scale).masked_fill(~seen, -math.inf)
        lse = torch.logsumexp(s, -1)
        p = torch.where(seen, torch.exp(s - lse.clamp(min=-1e300)[..., None]), 0.0)
        if o is None:
            return (p @ clean(v)).transpose(1, 2), lse
        delta = (clean(do) * o.cpu().double().transpose(1, 2)).sum(-1, keepdim=True)
        ds = torch.where(seen, p * (clean(do) @ clean(v).mT - delta), 0.0) * self.scale
        shared = lambda t: t.reshape(self.B, self.Hkv, G, self.Tk, -1).sum(2).transpose(1, 2)  # noqa: E731
        return (ds @ clean(k)).transpose(1, 2), shared(ds.mT @ clean(q)), shared(p.mT @ clean(do))

    def run(self, stream=None):
        gpu = lambda t: None if t is None else t.cuda()  # noqa: E731
        make = lambda shape: torch.full(shape, 9.0, dtype=DTYPES[self.dtype], device="cuda")  # noqa: E731
        # the packed tensor goes over whole, so that the views keep their strides
        views = self.projections(make)
        for to, t in zip(views, (self.q, self.k, self.v)):
            to.copy_(t)
        o, lse = make((self.B, self.Tq, self.H, self.D)), torch.full((self.B, self.H, self.Tq), 9.0, device="cuda")
        at = self.block.Attention(*views, o, self.causal, self.scale, gpu(self.q_len), gpu(self.k_len))
        at.forward(*views, o, lse, stream)
        grads, do = self.projections(make), self.do.cuda()
        at.backward(*views, o, lse, do, *grads, stream)
        again = self.projections(make)
        at.backward(*views, o, lse, do, *again, stream)
        assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip(grads, again))      # the same bits
        return o, lse, grads

    def check(self):
        o, lse, grads = self.run()
        want, want_lse = self.reference()
        bound = max(2.5 * U[self.dtype], FP32)
        assert rel(lse, want_lse) <= max(FP32, 4e-6 / max(1.0, want_lse[torch.isfinite(want_lse)].abs().mean().item() if torch.isfinite(want_lse).any() else 1))
        assert rel(o, want) <= bound
        for name, got, ref in zip(("dq", "dk", "dv"), grads, self.reference(o)):
            # where the parts of a sum cancel (a row that sees few keys): against the size of the parts
            size = ref.norm().item() + 0.05 * self.do.double().nan_to_num(0, 0, 0).norm().item() * (name != "dv")
            off = (got.cpu().double() - ref).norm().item()
            assert torch.isfinite(got).all() and off <= bound * size + 1e-30, (name, off / (size or 1))


SHAPES = [  # B, Tq, Tk, H, Hkv, D
    (1, 1, 1, 1, 1, 8), (2, 1, 5, 3, 1, 64), (2, 7, 1, 2, 2, 64), (3, 31, 31, 2, 2, 32), (2, 32, 32, 4, 2, 64), (2, 33, 33, 3, 3, 24),
    (1, 64, 64, 2, 1, 96), (2, 65, 65, 2, 2, 128), (1, 100, 100, 4, 4, 56), (1, 127, 129, 2, 1, 64), (1, 197, 197, 3, 3, 64),
    (1, 256, 256, 8, 1, 72), (1, 40, 300, 2, 2, 128), (1, 300, 40, 2, 2, 80), (9, 20, 20, 8, 8, 16), (1, 520, 520, 1, 1, 120), (1, 70, 650, 2, 2, 104)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention(block, dtype, shape, causal):
    Case(block, dtype, *shape, causal).check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Tq,Tk,q_len,k_len", [
    (20, 20, [20, 0, 1, 7], [20, 0, 1, 7]), (150, 150, [150, 64, 63, 129], [150, 64, 63, 129]), (70, 90, [70, 3, 70, 0], [90, 90, 2, 5]),
    (33, 200, None, [200, 128, 64, 1]), (140, 10, [140, 139, 1, 100], None), (5, 5, [9, -3, 5, 2], [5, 5, 77, -1])])
def test_attention_lengths(block, dtype, Tq, Tk, q_len, k_len, causal):
    """Rows that see nothing are zeros; lengths outside the tensor are held to it."""
    Case(block, dtype, 4, Tq, Tk, 4, 2, 64, causal, q_len, k_len).check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attention_ignores_what_is_not_seen(block, dtype):
    """NaN and infinities behind the lengths and in later tokens do not reach the rows that do not see them."""
    bad = [math.nan, math.inf, -math.inf]
    c = Case(block, dtype, 3, 100, 100, 2, 2, 64, True, [100, 40, 97], [100, 40, 97])
    plain = c.run()
    for n, t in enumerate((c.q, c.k, c.v, c.do)):
        for b, length in enumerate((100, 40, 97)):
            t[b, length:] = bad[(n + b) % 3]
    o, lse, grads = c.run()
    assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1])
    assert all(torch.equal(x, y) for x, y in zip(grads, plain[2]))
    # key and value 70 of sample 0 are seen by rows from 70 on: theirs are no numbers, the others' as before
    for t in (c.k, c.v):
        t[0, 70] = math.nan
    o, lse, (dq, dk, dv) = c.run()
    want, _, (wq, wk, wv) = plain
    assert rel(o[0, :70], want[0, :70]) <= 2.5 * U[dtype] + FP32 and torch.equal(o[1:], want[1:])
    assert torch.isnan(o[0, 70:]).all() and torch.isnan(lse[0, :, 70:]).all()
    assert rel(dq[0, :70], wq[0, :70]) <= 2.5 * U[dtype] + FP32 and torch.isnan(dq[0, 70:]).all()
    # a query that is no number: keys that it does not see keep their gradients
    c = Case(block, dtype, 1, 100, 100, 2, 1, 64, True)
    _, _, (_, wk, wv) = c.run()
    c.q[0, 20] = math.nan
    c.do[0, 33] = math.inf
    _, _, (_, dk, dv) = c.run()
    assert rel(dk[0, 34:], wk[0, 34:]) <= 2.5 * U[dtype] + FP32 and rel(dv[0, 34:], wv[0, 34:]) <= 2.5 * U[dtype] + FP32
    assert not torch.isfinite(dv[0, :34]).any() and torch.isnan(dk[0, :21]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attention_of_large_and_equal_scores(block, dtype):
    """Scores of some hundreds (no sum overflows), rows of one dominant key, and a maximum that grows tile by tile."""
    c = Case(block, dtype, 1, 200, 200, 2, 2, 64, False, scale=4.0)
    c.check()
    c = Case(block, dtype, 1, 130, 260, 1, 1, 64, False)
    c.k[0, :, 0] = (torch.arange(260)[:, None] * 0.05).to(c.k.dtype) * torch.sign(c.q[0, 0, 0].float()).to(c.k.dtype)
    c.check()
    c = Case(block, dtype, 1, 70, 70, 2, 2, 64, True)
    c.q.zero_()                                                        # equal scores: averages
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_layouts(block, dtype):
    """Heads outside tokens, tokens padded, one head's columns of a wider row."""
    base = Case(block, dtype, 2, 70, 70, 2, 2, 32, True)
    want = base.run()
    def place(t, how):
        B, T, H, D = t.shape
        if how == "heads first":
            return torch.zeros((B, H, T, D), dtype=t.dtype, device="cuda").transpose(1, 2)
        if how == "samples inside":
            return torch.zeros((T, B, H, D), dtype=t.dtype, device="cuda").transpose(0, 1)
        return torch.zeros((B, T + 3, H, D + 16), dtype=t.dtype, device="cuda")[:, :T, :, 8:8 + D]
    for how in ("heads first", "samples inside", "wider"):
        views = [place(t, how) for t in (base.q, base.k, base.v)]
        for to, t in zip(views, (base.q, base.k, base.v)):
            to.copy_(t)
        o, do, lse = place(base.do, how), place(base.do, how), torch.empty((2, 2, 70), device="cuda")
        do.copy_(base.do)
        at = block.Attention(*views, o, True, base.scale)
        at.forward(*views, o, lse)
        grads = [place(t, how) for t in (base.q, base.k, base.v)]
        at.backward(*views, o, lse, do, *grads)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        assert all(torch.equal(x, y) for x, y in zip(grads, want[2]))


# Widths and strides that are no multiples of 4, in fp32: rows are read an element at a time.  (The odd stride lies in the samples.)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1, 1), (2, 7, 7, 2, 1, 3), (2, 33, 33, 3, 3, 18), (1, 70, 45, 2, 2, 30), (1, 5, 130, 4, 1, 127),
                                   (2, 40, 40, 2, 2, 66), (1, 64, 64, 6, 2, 9)], ids=str)
def test_attention_odd_widths(block, shape, causal):
    Case(block, "f32", *shape, causal).check()


def test_attention_odd_strides(block):
    base = Case(block, "f32", 2, 70, 70, 2, 2, 32, True)
    want = base.run()
    place = lambda: torch.zeros(2 * (70 * 64 + 3), device="cuda").as_strided((2, 70, 2, 32), (70 * 64 + 3, 64, 32, 1))  # noqa: E731
    views, o, do, lse = [place() for _ in range(3)], place(), place(), torch.empty((2, 2, 70), device="cuda")
    for to, t in zip((*views, do), (base.q, base.k, base.v, base.do)):
        to.copy_(t)
    at = block.Attention(*views, o, True, base.scale)
    at.forward(*views, o, lse)
    grads = [place() for _ in range(3)]
    at.backward(*views, o, lse, do, *grads)
    for got, ref in zip((o, lse, *grads), (want[0], want[1], *want[2])):
        assert rel(got, ref) <= 2 * FP32                                    # both sides within FP32 of the same


# Few rows on one side and many on the other: waves take these in turn and are joined.  (The shapes of many tokens are for what is beside
# the rows: lengths that leave some waves nothing, a mask that ends within a turn.)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Tq,Tk,H,Hkv,D,q_len,k_len", [
    (1, 1500, 2, 1, 64, None, None), (5, 1100, 2, 2, 128, None, [1100, 37]), (40, 1999, 4, 2, 96, [40, 17], [65, 1999]),
    (1300, 6, 2, 1, 64, [1300, 1], None), (1057, 1057, 1, 1, 32, [1057, 33], [1057, 33]), (1, 1024, 1, 1, 128, None, [0, 1024]),
    (1025, 1, 2, 2, 64, None, None), (70, 1200, 2, 1, 8, [0, 70], [1200, 1000])], ids=str)
def test_attention_of_few_rows(block, dtype, Tq, Tk, H, Hkv, D, q_len, k_len, causal):
    Case(block, dtype, 2, Tq, Tk, H, Hkv, D, causal, q_len=q_len, k_len=k_len).check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_of_few_rows_ignores_what_is_not_seen(block, dtype):
    c = Case(block, dtype, 2, 9, 1300, 2, 1, 64, True, q_len=[9, 4], k_len=[1300, 800])
    c.k[1, 800:], c.v[1, 800:], c.q[1, 4:], c.do[1, 4:] = math.nan, math.inf, math.nan, math.inf
    c.v[0, 1299] = math.inf                               # the last row alone sees it
    o, lse, grads = c.run()
    want, want_lse = c.reference()
    assert rel(lse, want_lse) <= FP32 and rel(o[0, :8], want[0, :8]) <= max(2.5 * U[dtype], FP32) and rel(o[1], want[1]) <= max(2.5 * U[dtype], FP32)
    assert not torch.isfinite(o[0, 8]).any() and all(torch.isfinite(g[1]).all() for g in grads) and torch.isfinite(grads[0][0, :8]).all()


# The same with keys dealt to several workgroups, where the mask leaves some of them none; and without the workspace for it.
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,Tq,Tk,H,Hkv,D,q_len,k_len", [
    (1, 1, 4096, 2, 1, 64, None, None), (2, 3, 3001, 2, 2, 128, [3, 2], [3001, 700]), (1, 33, 2500, 4, 1, 32, None, None),
    (2, 1, 5000, 1, 1, 96, None, [0, 513]), (1, 150, 2100, 1, 1, 16, None, None)], ids=str)
def test_attention_keys_in_parts(block, dtype, B, Tq, Tk, H, Hkv, D, q_len, k_len, causal):
    c = Case(block, dtype, B, Tq, Tk, H, Hkv, D, causal, q_len=q_len, k_len=k_len)
    c.check()
    views, o, lse = [t.cuda() for t in (c.q, c.k, c.v)], torch.empty((B, Tq, H, D), dtype=DTYPES[dtype], device="cuda"), torch.empty((B, H, Tq), device="cuda")
    gpu = lambda n: None if n is None else n.cuda()  # noqa: E731
    at = block.Attention(*views, o, causal, c.scale, gpu(c.q_len), gpu(c.k_len))
    assert at._forward_need > 0
    block.dp.dp_attention(at.shape, at.dt, *views, o, lse)
    want, want_lse = c.reference()
    assert rel(o, want) <= max(2.5 * U[dtype], FP32) and rel(lse, want_lse) <= FP32


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_keys_in_parts_ignore_what_is_not_seen(block, dtype):
    c = Case(block, dtype, 1, 6, 3000, 2, 1, 64, True, k_len=[2777])
    c.k[0, 2777:], c.v[0, 2777:] = math.nan, math.inf
    c.v[0, 2776] = math.inf                               # the last row alone sees it
    o, lse, grads = c.run()
    want, want_lse = c.reference()
    assert rel(lse, want_lse) <= FP32 and rel(o[0, :5], want[0, :5]) <= max(2.5 * U[dtype], FP32)
    assert not torch.isfinite(o[0, 5]).any() and torch.isfinite(grads[0][0, :5]).all()


# Few key heads that many query heads share: the heads' sums are formed in parts and joined.
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 33, 33, 6, 1, 64), (1, 128, 128, 7, 1, 128), (1, 100, 260, 12, 2, 32), (2, 20, 20, 48, 6, 96),
                                   (1, 1, 1, 8, 2, 64), (3, 65, 65, 10, 1, 40), (1, 257, 257, 9, 3, 64)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_shared_heads_in_parts(block, dtype, shape, causal):
    Case(block, dtype, *shape, causal).check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_shared_heads_in_parts_ignore_what_is_not_seen(block, dtype):
    c = Case(block, dtype, 2, 90, 90, 8, 1, 64, True, q_len=[0, 61], k_len=[90, 77])
    for t in (c.q, c.do):
        t[0], t[1, 61:] = math.nan, math.inf
    for t in (c.k, c.v):
        t[1, 77:] = math.nan
    c.check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_of_broadcast_inputs(block, dtype):
    """One sample's keys and one head's queries for all: read where they are; gradients in such layouts are refused."""
    gen = torch.Generator().manual_seed(5)
    q = rand(gen, (2, 40, 1, 32), dtype).cuda().expand(2, 40, 4, 32)
    k, v = (rand(gen, (1, 50, 2, 32), dtype).cuda().expand(2, 50, 2, 32) for _ in range(2))
    out = []
    for views in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        o, lse = torch.empty((2, 40, 4, 32), dtype=q.dtype, device="cuda"), torch.empty((2, 4, 40), device="cuda")
        at = block.Attention(*views, o, True, 0.2)
        at.forward(*views, o, lse)
        out.append((o, lse))
        if views[0] is q:
            with pytest.raises(block.dp.DpError):
                at.backward(*views, o, lse, torch.empty_like(o), *views)
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("shape", [(1, 1, 2, 32), (1, 5, 1, 32), (2, 1, 1, 32)])
def test_attention_of_axes_of_one_entry(block, shape):
    """An axis of one entry has no stride: tensors that differ in it alone are taken, and give the same; where there are more entries, refused."""
    gen = torch.Generator().manual_seed(6)
    tensors = [rand(gen, shape, "bf16").cuda() for _ in range(5)]
    out = []
    at = block.Attention(*tensors[:4], False, 0.3)
    for other in (False, True):
        def view(t):
            strides = [4096 if other and n == 1 else st for n, st in zip(shape, t.stride())]
            return torch.empty(t.numel(), dtype=t.dtype, device="cuda").as_strided(shape, strides).copy_(t)
        q, k, v, o, do = (view(t) for t in tensors)
        assert other == (q.stride() != tensors[0].stride())
        lse, grads = torch.empty((shape[0], shape[2], shape[1]), device="cuda"), [view(t) for t in tensors[:3]]
        at.forward(q, k, v, o, lse)
        at.backward(q, k, v, o, lse, do, *grads)
        out.append([t.clone() for t in (o, lse, *grads)])
    assert all(torch.equal(a, b) for a, b in zip(*out))
    if shape[1] > 1:
        with pytest.raises(ValueError):
            at.forward(torch.zeros((1, 10, 1, 32), dtype=torch.bfloat16, device="cuda")[:, ::2], *tensors[1:4], lse)


def test_attention_gradient_against_differences(block):
    """A directional derivative of the fp32 forward pass against the gradients."""
    gen = torch.Generator().manual_seed(11)
    B, T, H, D = 2, 9, 2, 16
    q, k, v, do, dirn = (rand(gen, (B, T, H, D), "f32").cuda() for _ in range(5))
    o, lse = torch.empty_like(q), torch.empty((B, H, T), device="cuda")
    at = block.Attention(q, k, v, o, True, 0.25)
    grads = [torch.empty_like(q) for _ in range(3)]
    at.forward(q, k, v, o, lse)
    at.backward(q, k, v, o, lse, do, *grads)
    h = 2.0 ** -7
    for n, g in enumerate(grads):
        def loss(sign):
            moved = [t + sign * h * dirn if i == n else t for i, t in enumerate((q, k, v))]
            out = torch.empty_like(q)
            at.forward(*moved, out, torch.empty_like(lse))
            return (out.double() * do.double()).sum().item()
        slope = (loss(1) - loss(-1)) / (2 * h)
        assert abs(slope - (g.double() * dirn.double()).sum().item()) <= 1e-3 * (g.norm() * dirn.norm()).item()


def test_attention_offsets_past_32_bits(block):
    """Samples and tokens more than 2 GiB apart in a long buffer."""
    B, T, H, D, stride = 2, 70, 1, 64, 1 << 23
    wide = torch.zeros(B * T * stride, dtype=torch.bfloat16, device="cuda")
    base = Case(block, "bf16", B, T, T, H, H, D, True)
    want = base.run()
    views = [wide.as_strided((B, T, H, D), (T * stride, stride, D, 1), n * D) for n in range(3)]
    for to, t in zip(views, (base.q, base.k, base.v)):
        to.copy_(t)
    o, lse = torch.empty((B, T, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((B, H, T), device="cuda")
    block.Attention(*views, o, True, base.scale).forward(*views, o, lse)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


def check_fp16_gradients(block, Tq, Tk, H, Hkv, D, causal, change, seed=0):
    """fp16 gradients against the definition in 64 bits.  The bound, in the 2-norm, is what rounding costs where the type has all its bits, half as
    much again: the result's own rounding (as it is), and that of the scores' gradients or probabilities before their products, 2^-11 / sqrt(3)
    of each at most in the mean, independent of each other.  1e-5 of the same parts is for fp32 sums, lse and exponentials."""
    c = Case(block, "f16", 1, Tq, Tk, H, Hkv, D, causal, seed=seed)
    change(c)
    _, _, grads = c.run()
    G = H // Hkv
    q, do = c.q.double().transpose(1, 2), c.do.double().transpose(1, 2)
    k, v = (t.double().transpose(1, 2).repeat_interleave(G, 1) for t in (c.k, c.v))
    p = torch.softmax((q @ k.mT * c.scale).masked_fill(~c.seen(), -math.inf), -1).nan_to_num(0)
    dp = do @ v.mT
    ds = c.scale * p * (dp - (p * dp).sum(-1, keepdim=True))
    shared = lambda t: t.reshape(1, Hkv, G, Tk, -1).sum(2).transpose(1, 2)  # noqa: E731
    want = (ds @ k).transpose(1, 2), shared(ds.mT @ q), shared(p.mT @ do)
    square = lambda w, t: (w.square() @ t.square().sum(-1, keepdim=True)).sum().item()  # noqa: E731
    parts = math.sqrt(square(ds, k)), math.sqrt(square(ds.mT, q)), math.sqrt(square(p.mT, do))
    for name, got, ref, part in zip(("dq", "dk", "dv"), grads, want, parts):
        assert torch.isfinite(got).all()
        own = (ref.half().double() - ref).norm().item()
        off = (got.cpu().double() - ref).norm().item()
        assert off <= 1.5 * math.hypot(own, part * 2 ** -11 / math.sqrt(3)) + 1e-5 * part, (name, off / ref.norm().item(), own / ref.norm().item())


def times(name, factor):
    """Multiplies a tensor of a Case by a number, or its tokens by powers of two that grow or shrink evenly between two exponents."""
    def change(c):
        t = getattr(c, name)
        f = torch.tensor(float(factor)) if not isinstance(factor, tuple) else 2.0 ** torch.linspace(*factor, t.shape[1])[None, :, None, None]
        t.copy_((t.double() * f).half())
    return change


def zeros(name, tokens):
    return lambda c: getattr(c, name)[:, :tokens].zero_()


# Small output gradients (Case's are of size 0.1), of long rows; gradients and values that grow or shrink from token to token; leading zeros; score
# gradients beyond fp16's largest number; all with the forms of few rows, of shared heads and of each width.
@pytest.mark.parametrize("shape,causal,changes", [
    ((2048, 2048, 1, 1, 64), True, [times("do", 0.1)]), ((2048, 2048, 1, 1, 64), True, [times("do", 1e-2)]), ((2048, 2048, 1, 1, 64), True, [times("do", 1e-3)]),
    ((2048, 2048, 1, 1, 64), True, [times("do", 3e-5)]), ((2048, 2048, 1, 1, 64), False, [times("do", 1e-2)]), ((1100, 1500, 2, 2, 128), True, [times("do", 1e-2)]),
    ((900, 900, 2, 1, 96), False, [times("do", 1e-2)]), ((600, 600, 2, 2, 24), True, [times("do", 2e-3)]), ((3, 3000, 2, 2, 64), False, [times("do", 1e-2)]),
    ((2500, 5, 2, 2, 128), False, [times("do", 1e-2)]), ((400, 400, 8, 1, 64), True, [times("do", 1e-2)]),
    ((700, 700, 2, 2, 64), False, [times("do", (-12, 6)), times("v", (-8, 5))]), ((700, 700, 2, 2, 64), False, [times("do", (6, -12)), times("v", (5, -8))]),
    ((500, 500, 2, 2, 128), True, [times("do", (-14, 4))]), ((1024, 1024, 1, 1, 64), True, [zeros("do", 300), times("do", 1e-2)]),
    ((300, 300, 1, 1, 64), False, [zeros("v", 200), times("do", 1e-2)]), ((8, 8, 2, 2, 64), False, [times("do", 3e4), times("v", 30), times("k", 0.01), times("q", 0.01)]),
    ((8, 200, 2, 2, 128), False, [times("do", 1e5), times("v", 30), times("k", 0.01), times("q", 0.01)])])
def test_attention_fp16_gradients_of_any_size(block, shape, causal, changes):
    check_fp16_gradients(block, *shape, causal, lambda c: [change(c) for change in changes])


@pytest.mark.parametrize("Tq,Tk,D,causal", [(4, 60000, 64, False), (3, 60000, 128, True), (64, 60000, 64, False)])
def test_attention_fp16_gradients_of_small_probabilities(block, Tq, Tk, D, causal):
    """Rows so long that their probabilities are below fp16's smallest number with all its bits."""
    check_fp16_gradients(block, Tq, Tk, 2, 1, D, causal, times("do", 1e3))


class WideCase(Case):
    """The same on the GPU with tokens of q, k and v `stride` elements apart, in one buffer of NaN: only what the shape reaches may be read."""

    def projections(self, make):
        if not hasattr(self, "stride"):
            return super().projections(make)
        T, width = max(self.Tq, self.Tk), (self.H + 2 * self.Hkv) * self.D
        wide = torch.full((self.B * T * self.stride + 2 * width,), math.nan, dtype=DTYPES[self.dtype], device="cuda")
        view = lambda rows, heads, at: wide.as_strided((self.B, rows, heads, self.D), (T * self.stride, self.stride, self.D, 1), at * self.D)  # noqa: E731
        return view(self.Tq, self.H, 0), view(self.Tk, self.Hkv, self.H), view(self.Tk, self.Hkv, self.H + self.Hkv)


# Few rows against many that lie so far apart that one descriptor does not span the split forms' tiles; the strides beside that too.
@pytest.mark.parametrize("dtype,stride,Tq,Tk,D", [
    ("f32", 1 << 23, 1, 130, 24), ("f32", 1 << 23, 1, 130, 64), ("f32", 1 << 22, 3, 150, 32), ("f32", (1 << 21) + 4, 2, 300, 24), ("f32", 1 << 21, 2, 300, 24),
    ("f32", 1 << 23, 2, 100, 128), ("f32", 1 << 23, 130, 1, 24), ("f32", 1 << 22, 150, 3, 64), ("bf16", (1 << 22) + 8, 1, 1100, 24), ("f16", 1 << 23, 1, 1030, 64),
    ("bf16", (1 << 22) + 8, 1100, 2, 40), ("bf16", 1 << 23, 1, 1025, 104)])
def test_attention_of_few_rows_far_apart(block, dtype, stride, Tq, Tk, D):
    c = WideCase(block, dtype, 1, Tq, Tk, 2, 1, D, False)
    c.stride = stride
    c.check()


# ------------------------------------------------------------------------------------------------ AdamW

def fp8_reference(x, step, power):
    """Codes (as float64 values) and scales by the definition, block by block of 256; power 2: rounded between squares."""
    n = x.numel()
    codes, scales = torch.zeros(n, dtype=torch.float64), []
    e = torch.arange(n, dtype=torch.int64)
    f = (((e * 0x6A09E667 + step * 0x9E3779B1) % 2 ** 32) // 256).double() / 2 ** 24
    for b in range(0, n, 256):
        part = x[b:b + 256].double()
        scale = (part.abs().max() / 448).float().double()
        scales.append(scale)
        if scale == 0:
            continue
        a = part.abs() / scale
        unit = 2.0 ** (torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
        low = torch.floor(a / unit)
        place = ((a / unit) ** power - low ** power) / ((low + 1) ** power - low ** power)
        q = (low + (place >= 1 - f[b:b + 256])) * unit
        q = torch.where(a > 0, q.clamp(2.0 ** -9, 448), torch.zeros(()).double())
        codes[b:b + 256] = q * torch.sign(part)
    return codes, torch.stack(scales)


def adamw_reference(p, g, m, v, t, lr, b1, b2, eps, decay, scale):
    g = g.double() * scale
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    p = p.double() * (1 - lr * decay) - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
    return p, m, v


SIZES = [1, 3, 255, 256, 257, 4096, 4097, 20000]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=0.25)


@pytest.mark.parametrize("copy", [None, "bf16", "f16"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("aligned", [True, False])
def test_adamw_32_bits(block, dtype, aligned, copy):
    gen = torch.Generator().manual_seed(3)
    def cut(flat):                                                     # tensors at every fourth element, or one behind the other
        out, at = [], 0
        for n in SIZES:
            out.append(flat[at:at + n])
            at += -(-n // 8) * 8 if aligned else n
        return out
    total = sum(-(-n // 8) * 8 for n in SIZES) + 8
    p, g = rand(gen, (total,), "f32"), rand(gen, (total,), dtype)
    m, v = rand(gen, (total,), "f32", 0.1), rand(gen, (total,), "f32", 0.1).square()
    dev = [t.cuda() for t in (p, g, m, v)]
    cp = torch.full((total,), 7.0, dtype=DTYPES[copy], device="cuda") if copy else None
    before = dev[0].clone()
    decay = [0.1 * (i % 2) for i in range(len(SIZES))]
    opt = block.AdamW(*[cut(t) for t in dev], decay, cut(cp) if copy else None)
    pm, mm, vm = [t.double() for t in cut(p)], [t.double() for t in cut(m)], [t.double() for t in cut(v)]
    for step in (1, 2, 3):
        opt.step(step, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], HYPER["grad_scale"])
        for i, gi in enumerate(cut(g)):
            pm[i], mm[i], vm[i] = adamw_reference(pm[i], gi, mm[i], vm[i], step, *[HYPER[k] for k in ("lr", "beta1", "beta2", "eps")],
                                                  decay[i], HYPER["grad_scale"])
    for got, want in ((dev[0], pm), (dev[2], mm), (dev[3], vm)):
        for x, y in zip(cut(got), want):
            assert rel(x, y) <= FP32
    if copy:
        for x, y in zip(cut(cp), cut(dev[0])):
            assert torch.equal(x, y.to(x.dtype))
    covered = torch.zeros(total, dtype=torch.bool)
    for x in cut(covered):
        x |= True
    assert torch.equal(dev[0][~covered.cuda()], before[~covered.cuda()])      # what lies between the tensors is not touched


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_adamw_8_bits(block, dtype, offset):
    """Codes against the definition: a value whose rest lies within rounding of the dither may go either way, one in a thousand at most."""
    gen = torch.Generator().manual_seed(4)
    flat = lambda n, dt: torch.zeros(n + offset, dtype=dt, device="cuda")[offset:]  # noqa: E731
    lists = {k: [] for k in ("p", "g", "m", "v", "ms", "vs")}
    host = []
    for n in SIZES:
        p, g = rand(gen, (n,), "f32"), rand(gen, (n,), dtype)
        if n > 300:
            g[256:300] = 0                                             # states that stay zero
        for k, t in (("p", p), ("g", g)):
            x = flat(n, t.dtype)
            x.copy_(t)
            lists[k].append(x)
        for k in ("m", "v"):
            lists[k].append(flat(n, torch.float8_e4m3fn))
        for k in ("ms", "vs"):
            lists[k].append(flat(-(-n // 256), torch.float32))
        host.append([p, g, torch.zeros(n).double(), torch.zeros(n).double()])
    opt = block.AdamW(lists["p"], lists["g"], lists["m"], lists["v"], 0.1, None, lists["ms"], lists["vs"])
    for step in (1, 2, 3, 4):
        before = [[lists[k][i].cpu() for k in ("p", "m", "v", "ms", "vs")] for i in range(len(SIZES))]
        opt.step(step, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], HYPER["grad_scale"])
        for i, n in enumerate(SIZES):
            p, m8, v8, ms, vs = before[i]
            spread = lambda s: s.double().repeat_interleave(256)[:n]  # noqa: E731
            m, v = m8.double() * spread(ms), (v8.double() * spread(vs)) ** 2
            p, m, v = adamw_reference(p, lists["g"][i].cpu(), m, v, step, *[HYPER[k] for k in ("lr", "beta1", "beta2", "eps")], 0.1,
                                      HYPER["grad_scale"])
            assert rel(lists["p"][i], p) <= FP32
            for code, scale, x, power in ((lists["m"][i], lists["ms"][i], m, 1), (lists["v"][i], lists["vs"][i], v.sqrt(), 2)):
                want, scales = fp8_reference(x, step, power)
                assert rel(scale, scales) <= FP32
                got = code.cpu().double()
                differ = got != want
                assert differ.sum() <= 1 + n // 1000
                assert ((got - want).abs() <= want.abs() / 8 + 2.0 ** -8).all()      # the neighbouring code
                assert ((want != 0) == (got != 0)).all()


def test_adamw_8_bit_averages_move(block):
    """A slow average follows its input although a step's change is far below a code's distance: v after 2000 steps of unit noise."""
    n, steps = 4096, 2000
    p, m, v = torch.zeros(n, device="cuda"), *(torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    ms, vs, g = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda"), torch.empty(n, device="cuda")
    opt = block.AdamW([p], [g], [m], [v], 0.0, None, [ms], [vs])
    gen = torch.Generator(device="cuda").manual_seed(1)
    for step in range(1, steps + 1):
        g.normal_(generator=gen)
        opt.step(step, 0.0, 0.9, 0.999)
    second = ((v.float() * vs.repeat_interleave(256)) ** 2).mean().item() / (1 - 0.999 ** steps)
    assert abs(second - 1) < 0.03                 # the average's own noise is sqrt(2 / 2000 / 4096) = 0.05 %, the codes' a few parts in a thousand


def adamw_8_bits_once(block, g, steps=2, **kw):
    """Parameters, codes and scales of some steps from zero states."""
    n = g.numel()
    p, state = torch.ones(n, device="cuda"), [torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(-(-n // 256), device="cuda") for _ in range(2)]
    opt = block.AdamW([p], [g], [state[0]], [state[1]], 0.0, None, [scales[0]], [scales[1]])
    for step in range(1, steps + 1):
        opt.step(step, **{**dict(lr=0.25, beta1=0.875, beta2=0.9375, eps=0.0), **kw})
    return p, *[c.view(torch.uint8) for c in state], *scales


# 8-bit states have quotients and roots of two forms: short ones where nothing underflows, the compiler's elsewhere.  Both round to nearest, so that a
# change of all gradients by a power of two (betas whose products with it are exact, no eps) changes scales by it and nothing else.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_adamw_8_bits_of_either_form(block, dtype):
    gen = torch.Generator().manual_seed(21)
    g = rand(gen, (256 * 300 + 77,), dtype).cuda()
    g = torch.where(g.abs() < 2.0 ** -6, torch.full_like(g, 0.5), g)      # (nothing underflows: squares of 2^-58 / 16, rounded in 8 bits)
    p, m, v, ms, vs = adamw_8_bits_once(block, g)
    assert (ms.min() > 2.0 ** -50) and (ms.max() < 2.0 ** 50)
    for by in (-30, -52, 20, 55):                         # -52: scales below 2^-60, averages of squares below 2^-96
        p2, m2, v2, ms2, vs2 = adamw_8_bits_once(block, g * 2.0 ** by)
        assert torch.equal(p2, p) and torch.equal(m2, m) and torch.equal(v2, v), by
        assert torch.equal(ms2, ms * 2.0 ** by) and torch.equal(vs2, vs * 2.0 ** by), by
    # scales beyond 2^60, where squares are infinite: the average alone
    _, m2, _, ms2, _ = adamw_8_bits_once(block, g * 2.0 ** 76, steps=1)
    _, m, _, ms, _ = adamw_8_bits_once(block, g, steps=1)
    assert ms2.min() > 2.0 ** 60 and torch.equal(m2, m) and torch.equal(ms2, ms * 2.0 ** 76)


def adamw_8_bits_definition(g, steps, lr, beta1, beta2, eps, grad_scale):
    """The same in numpy's fp32, an operation at a time, from the header's text: parameters, code values and scales."""
    f, n = np.float32, g.size
    spread = lambda x: np.repeat(x, 256)[:n]  # noqa: E731
    p, m8, v8 = np.ones(n, f), np.zeros(n, f), np.zeros(n, f)
    ms, vs = np.zeros(-(-n // 256), f), np.zeros(-(-n // 256), f)
    b1, b2, rest1, rest2 = f(beta1), f(beta2), f(1 - beta1), f(1 - beta2)

    def coded(x, power, step):
        e = np.arange(n, dtype=np.uint64)
        dither = (((e * 0x6A09E667 + step * 0x9E3779B1) & 0xFFFFFFFF) >> 8).astype(f) * f(2.0 ** -24)
        blocks = np.zeros(-(-n // 256) * 256, f)
        blocks[:n] = np.abs(x)
        scale = blocks.reshape(-1, 256).max(1) * f(1 / 448)
        a = np.abs(x) / np.where(spread(scale) > 0, spread(scale), f(1))
        unit = np.maximum(np.frexp(a)[1] - 1, -6) - 3
        y = np.ldexp(a, -unit)
        low = np.floor(y)
        place = (y - low) * (y + low) / (f(2) * low + f(1)) if power == 2 else y - low
        c = np.clip(np.ldexp(low + np.floor(place + dither), unit), f(2.0 ** -9), f(448))
        return np.where(a > 0, np.copysign(c, x), f(0)).astype(f), scale

    for step in range(1, steps + 1):
        gs = g * f(grad_scale)
        m, v = m8 * spread(ms), v8 * spread(vs)
        m, v = b1 * m + rest1 * gs, b2 * (v * v) + rest2 * gs * gs
        fix1, fix2 = f(1) / f(1 - beta1 ** step), f(1) / f(1 - beta2 ** step)
        p = p - f(lr) * (m * fix1 / (np.sqrt(v * fix2) + f(eps)))
        (m8, ms), (v8, vs) = coded(m, 1, step), coded(np.sqrt(v), 2, step)
    return p, m8, v8, ms, vs


@pytest.mark.parametrize("hyper", [dict(lr=0.25, beta1=0.875, beta2=0.9375, eps=0.0, grad_scale=1.0), dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=0.3)])
def test_adamw_8_bits_to_the_bit(block, hyper):
    """Every operation is rounded alone, to nearest: fp32 code elsewhere gives the same bits, rare sizes of gradients among them."""
    gen = torch.Generator().manual_seed(23)
    g = torch.randn(256 * 400 + 77, generator=gen) * 2.0 ** torch.randint(-12, 12, (256 * 400 + 77,), generator=gen)
    got = adamw_8_bits_once(block, g.cuda(), steps=5, **hyper)
    want = adamw_8_bits_definition(g.numpy(), 5, **hyper)
    for name, x, y in zip(("param", "m", "v", "m_scale", "v_scale"), got, want):
        x = x.view(torch.float8_e4m3fn).float() if x.dtype == torch.uint8 else x
        assert np.array_equal(x.cpu().numpy(), y), (name, (x.cpu().numpy() != y).sum())


def test_adamw_8_bits_beside_tiny_squares(block):
    """One value whose square is below 2^-96 puts the roots of its 256 on the compiler's form: the others' bits stay."""
    gen = torch.Generator().manual_seed(22)
    g = rand(gen, (256 * 200,), "f32").cuda()
    g[::256] = 0.0
    tiny = g.clone()
    tiny[::256] = 2.0 ** -60
    want, got = adamw_8_bits_once(block, g, grad_scale=0.3), adamw_8_bits_once(block, tiny, grad_scale=0.3)
    others = torch.arange(g.numel(), device="cuda") % 256 != 0
    for a, b in zip(want[:3], got[:3]):
        assert torch.equal(a[others], b[others])
    assert torch.equal(want[3], got[3]) and torch.equal(want[4], got[4])
    assert (want[2][::256] == 0).all() and (got[2][::256] == 1).all()     # the smallest code: not rounded to zero


def test_adamw_many_tensors_and_undefined_values(block):
    """More tensors than a launch takes; NaN in a gradient stays in its own element (32 bits) or its 256 (8 bits)."""
    n = 300
    params = [torch.ones(7, device="cuda") for _ in range(n)]
    grads = [torch.full((7,), float(i + 1), device="cuda") for i in range(n)]
    grads[150][3] = math.nan
    zeros = lambda dt=torch.float32, k=7: [torch.zeros(k, device="cuda").to(dt) for _ in range(n)]  # noqa: E731
    block.AdamW(params, grads, zeros(), zeros(), 0.0).step(1, 0.5)
    for i, x in enumerate(params):                # the first step is lr * sign(g)
        want = torch.full((7,), 0.5)
        if i == 150:
            want[3] = math.nan
        assert torch.allclose(x.cpu(), want, equal_nan=True)
    p, g = torch.ones(600, device="cuda"), torch.ones(600, device="cuda")
    g[300] = math.nan
    m, v = (torch.zeros(600, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda")
    opt = block.AdamW([p], [g], [m], [v], 0.0, None, [ms], [vs])
    opt.step(1, 0.5)
    assert torch.isnan(p).sum() == 1 and torch.isnan(ms).tolist() == [False, True, False] == torch.isnan(vs).tolist()


def test_on_another_stream(block):
    """The calls run on the stream that they are given: ordered behind what it holds."""
    c = Case(block, "bf16", 2, 130, 130, 2, 2, 64, True)
    want = c.run()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = c.run()
    stream.synchronize()
    assert torch.equal(got[0], want[0]) and all(torch.equal(x, y) for x, y in zip(got[2], want[2]))


@pytest.mark.parametrize("by", ["current", "object", "handle"])
def test_calls_wait_for_their_stream(block, by):
    """Inputs that a stream fills behind a long piece of work: every call runs after them, on that stream, however it is named."""
    gen = torch.Generator().manual_seed(13)
    B, T, H, D = 2, 70, 4, 32
    new = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    x, dy, y, dx = (new(B, T, H * D) for _ in range(4))
    mean, rstd, kept, sq = new(B, T), new(B, T), new(B, 2, H * D), new(B)
    q, k, v, o, do, dq, dk, dv = (new(B, T, H, D) for _ in range(8))
    few, o1, lse, lse1 = new(B, 1, H, D), new(B, 1, H, D), new(B, H, T), new(B, H, 1)
    far_k, far_v = new(B, 2100, H, D), new(B, 2100, H, D)
    p, g, m, s = (new(5000) for _ in range(4))
    inputs = [x, dy, q, k, v, do, few, far_k, far_v, p, g]
    values = [torch.randn(t.shape, generator=gen).cuda() for t in inputs]
    norm, at, at1 = block.LayerNorm(None, None), block.Attention(q, k, v, o, True, 0.2), block.Attention(few, far_k, far_v, o1, False, 0.2)
    assert at1._forward_need > 0
    opt = block.AdamW([p], [g], [m], [s], 0.0)

    def run(stream):
        norm.forward(x, y, mean, rstd, stream=stream)
        norm.backward(x, dy, mean, rstd, dx, kept, sq, stream=stream)
        at.forward(q, k, v, o, lse, stream)
        at.backward(q, k, v, o, lse, do, dq, dk, dv, stream)
        at1.forward(few, far_k, far_v, o1, lse1, stream)
        opt.step(1, 0.1, stream=stream)

    outputs = [y, mean, rstd, dx, kept, sq, o, lse, dq, dk, dv, o1, lse1, p, m, s]
    for t, value in zip(inputs, values):
        t.copy_(value)
    run(None)
    want = [t.clone() for t in outputs]
    side, a = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for t in (*inputs, *outputs):
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(60):                               # some tens of milliseconds
            a = torch.mm(a, a).clamp_(-1, 1)
        for t, value in zip(inputs, values):
            t.copy_(value)
        assert not side.query()                           # still at it
        if by == "current":
            run(None)
    if by != "current":
        run(side if by == "object" else side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(outputs, want))


def test_replayed_in_a_graph(block):
    """Norm and attention, forward and backward, captured once and replayed on new inputs, with eager calls in between."""
    B, T, H, D = 2, 150, 6, 32
    d = H * D
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device="cuda")  # noqa: E731
    f = torch.float32
    x, add, total, y, dx = (new(B, T, d) for _ in range(5))
    mean, rstd, kept, sq = new(B, T, dt=f), new(B, T, dt=f), new(B, 2, d, dt=f), new(B, dt=f)
    kv, dkv, o, do, dq, lse = new(B, T, 2, 1, D), new(B, T, 2, 1, D), new(B, T, H, D), new(B, T, H, D), new(B, T, H, D), new(B, H, T, dt=f)
    norm = block.LayerNorm(torch.ones(d, device="cuda"), torch.zeros(d, device="cuda"))
    q, (k, v), (dk, dv) = y.view(B, T, H, D), kv.unbind(2), dkv.unbind(2)
    at = block.Attention(q, k, v, o, True, D ** -0.5)

    def run():
        norm.forward(x, y, mean, rstd, add, total)
        at.forward(q, k, v, o, lse)
        at.backward(q, k, v, o, lse, do, dq, dk, dv)
        norm.backward(total, dq.view(B, T, d), mean, rstd, dx, kept, sq, add)

    def fill():
        for t in (x, add, kv, do):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))

    outputs = (total, y, mean, rstd, o, lse, dq, dkv, dx, kept, sq)
    fill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()                                             # workspaces are there before the capture
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for _ in range(4):
        fill()
        for t in outputs:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outputs]
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outputs))


def test_workspaces_grow_and_follow_streams(block):
    """One object on calls of growing and shrinking sizes, on its own stream, another one, and one given by its handle."""
    gen = torch.Generator().manual_seed(4)
    norm = block.LayerNorm(None, None)
    streams = [None, torch.cuda.Stream(), torch.cuda.Stream().cuda_stream]
    for T in (40, 400, 7, 1000):
        x, dy = (rand(gen, (3, T, 96), "f32").cuda() for _ in range(2))
        mean, rstd = torch.empty((3, T), device="cuda"), torch.empty((3, T), device="cuda")
        norm.forward(x, torch.empty_like(x), mean, rstd)
        torch.cuda.synchronize()
        out = []
        for stream in streams:
            dx, kept, sq = torch.empty_like(x), torch.empty((3, 2, 96), device="cuda"), torch.empty(3, device="cuda")
            torch.cuda.synchronize()
            norm.backward(x, dy, mean, rstd, dx, kept, sq, stream=stream)
            torch.cuda.synchronize()
            out.append((dx, kept, sq))
        assert all(torch.equal(a, b) for other in out[1:] for a, b in zip(other, out[0]))


def segment_of(t):
    """The allocator's segment that a tensor lies in."""
    return next(s for s in torch.cuda.memory_snapshot() if s["address"] <= t.data_ptr() < s["address"] + s["total_size"])


def test_workspaces_are_memory_of_the_stream_that_uses_them(block):
    """The default stream by its handle, 0, and another one, while a third is current."""
    device, side, other = torch.device("cuda", torch.cuda.current_device()), torch.cuda.Stream(), torch.cuda.Stream()
    ws = block._Workspaces()
    with torch.cuda.stream(side):
        for stream in (0, other.cuda_stream, side.cuda_stream):
            assert segment_of(ws(3 << 20, device, device.index, stream))["stream"] == stream


def test_graphs_do_not_share_workspaces(block):
    """Two graphs of one object, captured on one stream, and calls on that stream that are not captured: each has scratch of its own, so
    that all of them may run at once."""
    gen = torch.Generator().manual_seed(10)
    norm, used, capture = block.LayerNorm(None, None), [], torch.cuda.Stream()
    inner = norm._ws
    norm._ws = lambda *args: used.append(inner(*args)) or used[-1]

    def case():
        x, dy = (rand(gen, (4, 900, 768), "f32").cuda() for _ in range(2))
        stats = torch.empty((4, 900), device="cuda"), torch.empty((4, 900), device="cuda")
        norm.forward(x, torch.empty_like(x), *stats)
        dx, kept, sq = torch.empty_like(x), torch.empty((4, 2, 768), device="cuda"), torch.empty(4, device="cuda")
        return (lambda: norm.backward(x, dy, *stats, dx, kept, sq)), (dx, kept, sq)

    cases, graphs, want = [case() for _ in range(3)], [], []
    torch.cuda.synchronize()
    with torch.cuda.stream(capture):
        for call, outputs in cases:
            call()
            want.append([t.clone() for t in outputs])
    torch.cuda.synchronize()
    for call, _ in cases[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=capture):
            call()
    eager, first, second = used[0], used[-2], used[-1]
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel()) for t in (eager, first, second))
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    del used[:], eager, first, second
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for _, outputs in cases:
            for t in outputs:
                t.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(4):
            for graph, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
            with torch.cuda.stream(capture):
                cases[2][0]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for (_, outputs), w in zip(cases, want) for a, b in zip(outputs, w))


def test_a_captured_workspace_stays(block):
    """A graph that holds a workspace's address is replayed after the object has needed a larger one."""
    gen = torch.Generator().manual_seed(9)
    norm = block.LayerNorm(None, None)

    def case(T):
        x, dy = (rand(gen, (2, T, 512), "f32").cuda() for _ in range(2))
        stats = torch.empty((2, T), device="cuda"), torch.empty((2, T), device="cuda")
        norm.forward(x, torch.empty_like(x), *stats)
        dx, kept, sq = torch.empty_like(x), torch.empty((2, 2, 512), device="cuda"), torch.empty(2, device="cuda")
        return (lambda: norm.backward(x, dy, *stats, dx, kept, sq)), (dx, kept, sq)

    side = torch.cuda.Stream()
    small, outputs = case(200)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        small()
    side.synchronize()
    want = [t.clone() for t in outputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        small()
    large, _ = case(4000)
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            large()
            guard = [torch.full((1 << 14,), 5.0, device="cuda") for _ in range(64)]       # would take freed memory
        side.synchronize()
        for t in outputs:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want)) and all((g == 5.0).all() for g in guard)
