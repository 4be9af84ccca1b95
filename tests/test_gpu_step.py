"""Rotation and norms of heads, gated feed-forward layers and the orthogonalising optimizer against plain 64-bit implementations on the
CPU, at the sizes, layouts, positions and lengths where they can go wrong.

Tolerances, relative in the 2-norm unless said otherwise.  U is half a unit in the last place of the storage type, relative to the
value: what one rounding may err by.
  stored results     one rounding: U, and what the fp32 arithmetic before it errs by
  FP32               2e-6: some ten fp32 operations in a row (each 2^-24 = 6e-8 at most), or a sum of up to 1000 products in fp32 (sqrt(1000) 2^-24;
                     longer ones are sums of such sums);
                     an angle, a fraction of a turn rounded to fp32, is within 2 pi 2^-26 = 9.4e-8
"""
import math

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
    norm = want[fine].norm().item()
    off = (got[fine] - want[fine]).norm().item()
    return off / norm if norm else (0.0 if off == 0 else math.inf)


def rand(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(DTYPES[dtype])


# ------------------------------------------------------------------------------------------------ heads

def turn(x, turns, interleaved, amplitude, position, back=False):
    """x [B, T, h, D] in 64 bits; position [B, T]."""
    n = 2 * len(turns)
    angle = 2 * math.pi * (position.double()[..., None, None] * turns)
    cos, sin = amplitude * angle.cos(), amplitude * angle.sin() * (-1 if back else 1)
    y = x.clone()
    a, b = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y


class Heads:
    """Inputs of one layout on the CPU and on the device, as views of a packed projection."""

    def __init__(self, dtype, B, T, H, Hkv, D, rotary, interleaved, start=None, ragged=False, amplitude=1.0, seed=0):
        gen = torch.Generator().manual_seed(seed + B * 7919 + T * 31 + D)
        self.B, self.T, self.H, self.Hkv, self.D, self.dtype, self.ragged = B, T, H, Hkv, D, dtype, ragged
        self.x = rand(gen, (B, T, H + 2 * Hkv, D), dtype, 1.5)
        self.dy = [rand(gen, (B, T, h, D), dtype) for h in (H, Hkv)]
        self.gains = [1 + 0.3 * rand(gen, (D,), "f32") for _ in range(2)]
        self.kw = dict(interleaved=interleaved, amplitude=amplitude)
        self.position = torch.arange(T, dtype=torch.int32).repeat(B, 1)
        if start is not None:
            self.position += torch.randint(start, start + 1000, (B, 1), generator=gen, dtype=torch.int32)
            self.kw["position"] = self.position.cuda()
        self.len = torch.full((B,), T)
        if ragged:
            self.len = torch.randint(0, T + 1, (B,), generator=gen)
            self.len[0] = T
            self.kw["length"] = self.len.to(torch.int32).cuda()
        self.there = (torch.arange(T) < self.len[:, None])[..., None, None]
        self.rotary = rotary

    def views(self, packed):
        return packed[:, :, :self.H], (packed[:, :, self.H:self.H + self.Hkv] if self.Hkv else None)

    def make(self, block, kind):
        turns = block.rotary_turns(self.rotary) if self.rotary else None
        self.turns = turns if turns is not None else torch.zeros(0, dtype=torch.float64)
        if turns is not None:
            self.kw["turns"] = turns.cuda()
        self.q, self.k = self.views(self.x.cuda())
        fresh = lambda h: torch.full((self.B, self.T, h, self.D), 7.0, dtype=DTYPES[self.dtype], device="cuda") if h else None  # noqa: E731
        self.out = [fresh(self.H), fresh(self.Hkv)]
        gains = [g.cuda() for g in self.gains] if kind == "HeadNorm" else []
        if not self.Hkv and gains:
            gains[1] = None
        return getattr(block, kind)(self.q, self.k, *self.out, *gains, **self.kw)

    def turned(self, x, back=False):
        return turn(x, self.turns, self.kw["interleaved"], self.kw["amplitude"], self.position, back) if self.rotary else x

    def check(self, got, want, tol):
        """Rows that are there to `tol`, the others untouched."""
        there = self.there.expand(want.shape)
        assert rel(got.cpu()[there], want[there]) <= tol
        assert (got.cpu()[~there] == 7).all()

    @property
    def sides(self):
        return range(2 if self.Hkv else 1)


HEADS = [  # B, T, H, Hkv, D, rotary, interleaved
    (1, 1, 1, 1, 8, 8, False), (2, 5, 3, 0, 16, 16, True), (8, 1, 12, 12, 64, 64, False), (3, 33, 4, 2, 64, 64, False),
    (2, 70, 6, 2, 128, 128, False), (2, 17, 5, 1, 128, 64, True), (3, 9, 7, 7, 56, 56, False), (2, 40, 2, 2, 24, 20, False),
    (2, 21, 3, 1, 40, 6, False), (1, 300, 2, 1, 256, 256, False), (1, 19, 9, 3, 256, 130, True), (2, 11, 20, 20, 72, 2, False),
    (5, 130, 1, 1, 8, 4, True), (1, 2, 70, 70, 64, 64, False), (1, 1100, 3, 3, 32, 32, False), (2, 3, 300, 1, 8, 6, False)]
HEADS_F32 = HEADS + [(2, 13, 3, 2, 1, 0, False), (2, 9, 2, 1, 3, 2, True), (1, 37, 5, 5, 255, 254, False), (3, 8, 2, 2, 130, 66, True),
                     (2, 6, 4, 4, 6, 6, False), (1, 5, 2, 2, 2, 2, False), (2, 12, 3, 3, 129, 126, False)]
LAYOUTS = [(d, s) for d in DTYPES for s in (HEADS_F32 if d == "f32" else HEADS)]


@pytest.mark.parametrize("dtype,size", LAYOUTS, ids=str)
def test_rotary(block, dtype, size):
    if size[5] == 0:
        return
    for start, ragged, amplitude in ((None, False, 1.0), (100000, True, 1.3)):
        h = Heads(dtype, *size, start, ragged, amplitude)
        plan = h.make(block, "Rotary")
        plan.forward(h.q, h.k, *h.out)
        for w in h.sides:
            x = (h.q, h.k)[w].cpu().double()
            h.check(h.out[w], h.turned(x), U[dtype] + FP32)
        # the gradient, in the projection's layout; values behind queries and keys stay
        packed = torch.full(h.x.shape, 7.0, dtype=DTYPES[dtype], device="cuda")
        dq, dk = h.views(packed)
        dy = [t.cuda() if w in h.sides else None for w, t in enumerate(h.dy)]
        plan.backward(*dy, dq, dk)
        for w in h.sides:
            h.check((dq, dk)[w], h.turned(h.dy[w].double(), True), U[dtype] + FP32)
        assert (packed[:, :, h.H + h.Hkv:] == 7).all()
        # in place
        q, k = (None if t is None else t.clone() for t in (h.q, h.k))
        if h.H + 2 * h.Hkv == h.H:
            continue
        same = block.Rotary(q, k, q, k, **h.kw)
        same.forward(q, k, q, k)
        for w in h.sides:
            there = h.there.expand(h.out[w].shape).cuda()
            assert torch.equal((q, k)[w][there], h.out[w][there])


@pytest.mark.parametrize("dtype,size", LAYOUTS, ids=str)
def test_head_norm(block, dtype, size):
    for start, ragged, rotary in ((None, False, size[5]), (5000, True, size[5]), (None, True, 0)):
        h = Heads(dtype, *size[:5], rotary, size[6], start, ragged)
        plan = h.make(block, "HeadNorm")
        plan.forward(h.q, h.k, *h.out)
        packed = torch.full(h.x.shape, 7.0, dtype=DTYPES[dtype], device="cuda")
        grads = h.views(packed)
        dy = [t.cuda() if w in h.sides else None for w, t in enumerate(h.dy)]
        kept = torch.empty((h.B, len(h.sides), h.D), device="cuda")
        sqnorm = torch.empty(h.B, device="cuda")
        plan.backward(h.q, h.k, *dy, *grads, kept, sqnorm)
        want = []
        for w in h.sides:
            x, gain = (h.q, h.k)[w].cpu().double(), h.gains[w].double()
            r = (x.square().mean(-1, keepdim=True) + 1e-6) ** -0.5
            h.check(h.out[w], h.turned(x * r * gain), U[dtype] + 4 * FP32)
            g = h.turned(h.dy[w].double(), True)
            u = g * gain
            dx = r * (u - x * r * (u * x * r).mean(-1, keepdim=True))
            if h.D > 1:                                  # (of one column all of dx cancels)
                h.check(grads[w], dx, U[dtype] + 8 * FP32)
            want.append((g * x * r * h.there).sum((1, 2)))
        want = torch.stack(want, 1)
        # sums of up to 1100 tokens' heads, each term's own error 4 FP32 of it at most, independent of the others'
        scale = (h.dy[0].double().square().sum((1, 2)).sqrt().max() * 4).item()
        assert (kept.cpu().double() - want).abs().max() <= 4 * FP32 * max(scale, want.abs().max().item())
        assert rel(sqnorm, kept.double().square().sum((1, 2))) <= FP32
        # without the gains' gradients, and in place of dy: the same bits
        if h.Hkv:
            again = [t.clone() for t in dy]
            inplace = block.HeadNorm(*again, *h.out, *[g.cuda() for g in h.gains], **h.kw)
            xs = [t.contiguous() for t in (h.q, h.k)]
            inplace.backward(*xs, *again, *again)
            for w in h.sides:
                there = h.there.expand(again[w].shape).cuda()
                assert torch.equal(again[w][there], grads[w][there])
                assert torch.equal(again[w][~there], dy[w][~there])


def test_rotary_far_positions(block):
    """Negative and largest positions: the angle is the fraction of a turn in 64 bits."""
    at = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789, -99999999]], dtype=torch.int32)
    gen = torch.Generator().manual_seed(5)
    x = rand(gen, (1, 7, 2, 32), "f32")
    turns = block.rotary_turns(32, 500000.0)
    q = x.cuda()
    out = torch.empty_like(q)
    block.Rotary(q, None, out, None, turns.cuda(), position=at.cuda()).forward(q, None, out, None)
    # 2^31 positions in 64 bits: 2^-53 2^31 of a turn and its own angle's rounding in the reference as well
    assert rel(out, turn(x.double(), turns, False, 1.0, at)) <= FP32


def test_rotary_rows_behind_and_empty(block):
    """Lengths of zero, below it and beyond T; what lies behind a length may be anything."""
    x = torch.full((4, 6, 2, 16), math.nan)
    lens = torch.tensor([0, -3, 99, 2], dtype=torch.int32)
    x[2], x[3, :2] = 1.0, 1.0
    q, out = x.cuda(), torch.full(x.shape, 7.0).cuda()
    gain, kept, sqnorm = torch.ones(16, device="cuda"), torch.empty((4, 1, 16), device="cuda"), torch.empty(4, device="cuda")
    norm = block.HeadNorm(q, None, out, None, gain, None, turns=block.rotary_turns(16).cuda(), length=lens.cuda())
    norm.forward(q, None, out, None)
    assert (out[:2] == 7).all() and (out[3, 2:] == 7).all() and torch.isfinite(out).all()
    dq = torch.full(x.shape, 7.0).cuda()
    norm.backward(q, None, q, None, dq, None, kept, sqnorm)
    assert (dq[:2] == 7).all() and (dq[3, 2:] == 7).all() and torch.isfinite(dq).all()
    assert (kept[:2] == 0).all() and (sqnorm[:2] == 0).all() and torch.isfinite(kept).all()


def along(f, x, direction, step):
    return (f(x + step * direction) - f(x - step * direction)) / (2 * step)


def test_head_norm_gradient_by_differences(block):
    """Central differences along the gradient itself, where they are its norm.  Step 2^-5 of values of size 1.5: third derivatives leave some
    (2^-5 / 1.5)^2 / 6 = 7e-5 of it, fp32 values FP32 / 2^-5 = 6e-5 of |y| |dy| over |dx|, which is some 10 here."""
    h = Heads("f32", 2, 5, 3, 2, 16, 12, False, 50)
    plan = h.make(block, "HeadNorm")
    x, dy = [t.contiguous() for t in (h.q, h.k)], [t.cuda() for t in h.dy]
    plan = block.HeadNorm(*x, *h.out, *[g.cuda() for g in h.gains], **h.kw)
    dx, kept, sqnorm = [torch.empty_like(t) for t in x], torch.empty((2, 2, 16), device="cuda"), torch.empty(2, device="cuda")
    plan.backward(*x, *dy, *dx, kept, sqnorm)

    def loss(w, value, gains=None):
        now = plan if gains is None else block.HeadNorm(*x, *h.out, *gains, **h.kw)
        at = list(x)
        if w is not None:
            at[w] = value.float()
        now.forward(*at, *h.out)
        return sum((a.double() * b.double()).sum() for a, b in zip(h.out, dy)).item()

    for w in range(2):
        n = dx[w].double().norm()
        v = dx[w].double() / n
        assert abs(along(lambda t: loss(w, t), x[w].double(), v, 2.0 ** -5) - n.item()) <= 2e-3 * n.item()
        total = kept.double().sum(0)[w]
        v = total / total.norm()
        gains = [g.cuda() for g in h.gains]

        def of_gain(t):
            return loss(None, None, [t.float() if i == w else g for i, g in enumerate(gains)])
        # y is linear in the gains
        assert abs(along(of_gain, gains[w].double(), v, 2.0 ** -3) - total.norm().item()) <= 1e-3 * total.norm().item()


# ------------------------------------------------------------------------------------------------ gated feed-forward layers

def act_reference(x, act):
    x = x.clone().requires_grad_()
    y = {"silu": lambda: x * torch.sigmoid(x), "gelu": lambda: 0.5 * x * torch.special.erfc(-x * 0.5 ** 0.5),
         "gelu_tanh": lambda: x * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (x + 0.044715 * x ** 3)),
         "relu": lambda: torch.where(x > 0, x, 0.0), "sigmoid": lambda: torch.sigmoid(x)}[act]()
    return y.detach(), torch.autograd.grad(y.sum(), x)[0]


ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]
GATED = [  # rows, d, f, d_out
    (1, 8, 8, 8), (1, 1280, 24, 8), (3, 64, 136, 64), (16, 40, 520, 40), (17, 264, 64, 128), (33, 48, 200, 48), (64, 128, 256, 128), (65, 72, 72, 72),
    (111, 60, 168, 60), (128, 512, 128, 512), (200, 96, 1032, 96), (257, 88, 264, 40), (300, 776, 512, 776), (520, 256, 512, 264), (1030, 40, 40, 40),
    (4, 2056, 1000, 24), (31, 16, 4104, 16), (700, 1032, 264, 512),
    (2100, 72, 4104, 40), (2100, 4104, 136, 48), (1800, 520, 2600, 136),
    # whole rounds of large tiles and some more: forward, hidden and input
    (4400, 328, 2184, 16), (4400, 40, 4360, 776), (4400, 4360, 520, 24),
    # long contractions of few tiles
    (200, 4104, 40, 3080), (1000, 7416, 216, 7416), (70, 520, 72, 4104), (40, 5000, 72, 5000), (2300, 2056, 776, 2056),
    # of what whole rounds leave: forward, hidden
    (2200, 2056, 4488, 24), (4200, 16, 3976, 2056),
    # large tiles in parts, forward and input
    (136, 6152, 5896, 16)]
GATED_F32 = GATED + [(5, 1027, 33, 517), (300, 2001, 65, 1999), (1, 1, 1, 1), (5, 3, 7, 2), (111, 60, 161, 61), (130, 257, 65, 33), (64, 17, 129, 130)]
GATED_CASES = [(d, *s) for d in DTYPES for s in (GATED_F32 if d == "f32" else [(r, 8 * -(-a // 8), b, 8 * -(-c // 8)) for r, a, b, c in GATED])]


def same(x, want, tol, dtype):
    """To a stored result's rounding and `tol` of what came before it."""
    assert rel(x, want) <= U[dtype] + tol, (rel(x, want), U[dtype] + tol)


@pytest.mark.parametrize("dtype,rows,d,f,d_out", GATED_CASES)
def test_gated_forward(block, dtype, rows, d, f, d_out):
    gen = torch.Generator().manual_seed(rows * 1009 + d)
    x, wg, wu = rand(gen, (rows, d), dtype), rand(gen, (d, f), dtype, d ** -0.5), rand(gen, (d, f), dtype, d ** -0.5)
    bg, bu = rand(gen, (f,), dtype), rand(gen, (f,), dtype)
    act = ACTS[(rows + d) % 5]
    for biases in (False, True):
        layer = block.GatedFeedForward(wg.cuda(), wu.cuda(), None, *((bg.cuda(), bu.cuda()) if biases else (None, None)), activation=act)
        guard = torch.full((3, rows + 1, f), 7.0, dtype=DTYPES[dtype], device="cuda")           # a row behind each result stays
        gate, up, h = (t[:rows] for t in guard)
        layer.forward(x.cuda(), h, gate, up)
        want_gate = x.double() @ wg.double() + (bg.double() if biases else 0)
        want_up = x.double() @ wu.double() + (bu.double() if biases else 0)
        same(gate, want_gate, FP32, dtype)
        same(up, want_up, FP32, dtype)
        same(h, act_reference(want_gate, act)[0] * want_up, 4 * FP32 + (2e-4 if dtype == "bf16" else 1e-4 if dtype == "f16" else 0), dtype)
        assert (guard[:, rows] == 7).all()
        alone = torch.empty_like(h)
        layer.forward(x.cuda(), alone)
        assert torch.equal(alone, h)


@pytest.mark.parametrize("dtype,rows,d,f,d_out", GATED_CASES)
def test_gated_backward(block, dtype, rows, d, f, d_out):
    gen = torch.Generator().manual_seed(rows * 1013 + f)
    wg, wu, wd = rand(gen, (d, f), dtype, f ** -0.5), rand(gen, (d, f), dtype, f ** -0.5), rand(gen, (f, d_out), dtype, d_out ** -0.5)
    gate, up, dy, dh = rand(gen, (rows, f), dtype, 1.5), rand(gen, (rows, f), dtype), rand(gen, (rows, d_out), dtype), rand(gen, (rows, f), dtype)
    act = ACTS[(rows + f) % 5]
    value, slope = act_reference(gate.double(), act)
    for down in (True, False):
        layer = block.GatedFeedForward(wg.cuda(), wu.cuda(), wd.cuda() if down else None, activation=act)
        guard = torch.full((2, rows + 1, f), 7.0, dtype=DTYPES[dtype], device="cuda")
        dgate, dup = (t[:rows] for t in guard)
        below = torch.full((rows + 1, d), 7.0, dtype=DTYPES[dtype], device="cuda")
        given = (dy if down else dh).cuda()
        layer.backward(given, gate.cuda(), up.cuda(), dgate, dup, below[:rows])
        back = dy.double() @ wd.double().t() if down else dh.double()
        same(dgate, back * up.double() * slope, 4 * FP32 + (0 if dtype == "f32" else 2e-4), dtype)
        same(dup, back * value, 4 * FP32 + (0 if dtype == "f32" else 2e-4), dtype)
        # of the two as they are stored
        want = dgate.cpu().double() @ wg.double().t() + dup.cpu().double() @ wu.double().t()
        same(below[:rows], want, 4 * FP32, dtype)
        assert (guard[:, rows] == 7).all() and (below[rows] == 7).all()
        # in the place of what it reads, and without dx: the same bits
        g2, u2 = gate.cuda(), up.cuda()
        layer.backward(given, g2, u2, g2, u2)
        assert torch.equal(g2, dgate) and torch.equal(u2, dup)
        if not down:
            g2 = gate.cuda()
            layer.backward(given, g2, up.cuda(), g2, given)
            assert torch.equal(g2, dgate) and torch.equal(given, dup)


@pytest.mark.parametrize("act", ACTS)
def test_gated_extreme_gates(block, act):
    """Gates far from zero: shares of exactly 0 and 1, no NaN where the value has none."""
    gate = torch.tensor([[-300.0, -90.0, -40.0, -12.0, -1e-30, 0.0, 1e-30, 12.0, 40.0, 90.0, 300.0, -3.0, 3.0, -0.5, 0.5, 1.0]])
    layer = block.GatedFeedForward(torch.eye(16).cuda(), torch.eye(16).cuda(), activation=act)
    up, dh = torch.full((1, 16), 2.0), torch.full((1, 16), 3.0)
    dgate, dup = torch.empty((1, 16), device="cuda"), torch.empty((1, 16), device="cuda")
    layer.backward(dh.cuda(), gate.cuda(), up.cuda(), dgate, dup)
    value, slope = act_reference(gate.double(), act)
    # absolute, where a share is next to nothing; gelu's tail at -12 is some 1e-32
    assert ((dup.cpu().double() - 3 * value).abs() <= 4 * FP32 * (3 * value).abs() + 1e-30).all()
    assert ((dgate.cpu().double() - 6 * slope).abs() <= 8 * FP32 * (6 * slope).abs() + 1e-6 * (slope.abs() < 1e-3) + 1e-30).all()
    h = torch.empty((1, 16), device="cuda")
    layer.forward(gate.cuda(), h)
    assert ((h.cpu().double() - value * gate.double()).abs() <= 4 * FP32 * (value * gate.double()).abs() + 1e-30).all()


def test_gated_gradient_by_differences(block):
    """Central differences of sum(dh h) along dx, as for the norms: step 2^-5, third derivatives of a gate of size 1 leave some 2e-4 of it."""
    gen = torch.Generator().manual_seed(3)
    for act in ("silu", "gelu", "gelu_tanh", "sigmoid"):
        x, wg, wu = rand(gen, (9, 24), "f32").cuda(), rand(gen, (24, 40), "f32", 0.2).cuda(), rand(gen, (24, 40), "f32", 0.2).cuda()
        dh, layer = rand(gen, (9, 40), "f32").cuda(), None
        layer = block.GatedFeedForward(wg, wu, activation=act)
        gate, up, h, dgate, dup = (torch.empty((9, 40), device="cuda") for _ in range(5))
        dx = torch.empty_like(x)
        layer.forward(x, h, gate, up)
        layer.backward(dh, gate, up, dgate, dup, dx)

        def loss(t):
            layer.forward(t.float(), h)
            return (h.double() * dh.double()).sum().item()
        n = dx.double().norm().item()
        assert abs(along(loss, x.double(), dx.double() / n, 2.0 ** -5) - n) <= 2e-3 * n


# ------------------------------------------------------------------------------------------------ orthogonalised updates

ABC = [(3.4445, -4.7750, 2.0315)] * 5


def orthogonal(u, eps=1e-7, abc=ABC):
    x = u / (u.norm() + eps)
    turned = x.shape[0] > x.shape[1]
    x = x.t() if turned else x
    for a, b, c in abc:
        gram = x @ x.t()
        x = a * x + b * (gram @ x) + c * (gram @ (gram @ x))
    return x.t() if turned else x


def muon_tolerance(shape):
    """Of X against its norm.  Entries are kept within 2^-23 of their size, products' sums within FP32.  Five iterations multiply what a
    direction next to no singular value is off by 3.4445^5 = 485 at most (what later ones add, by less: 1.41 times as much in all), of a matrix
    that starts with norm 1 and ends with about the root of its shorter side; then fifteen products' own."""
    return 1.41 * 485 * 2.0 ** -23 / min(shape) ** 0.5 + 8 * FP32


MUON_SHAPES = [[(1, 1)], [(1, 40), (40, 1), (2, 3)], [(16, 16), (24, 72), (72, 24), (65, 24), (24, 65)], [(128, 128), (129, 127), (127, 300), (260, 140)],
               [(520, 300), (256, 1030)], [(33, 2000)] * 3 + [(2000, 33)] * 2, [(96, 100), (100, 96), (90, 113), (16, 600), (1, 1900)], [(64, 256), (250, 61)] + [(130, 70)] * 3,
               [(8, 9 + i) for i in range(131)], [(1300, 1100)], [(700, 2600)] * 14,
               [(40, 4100)], [(300, 2500), (2500, 300), (130, 1030)], [(8, 5000), (5000, 16)]]          # A's contraction in parts


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shapes", MUON_SHAPES, ids=lambda s: f"{len(s)}x{s[0]}")
def test_muon(block, dtype, shapes):
    gen = torch.Generator().manual_seed(len(shapes) + shapes[0][0])
    some = sorted({0, len(shapes) // 2, len(shapes) - 1})          # those that the reference forms
    offset = 3                                                      # of no alignment but the elements' own
    make = lambda kind, scale: [(torch.randn(math.prod(s) + offset, generator=gen) * scale).to(kind).cuda()[offset:].view(s) for s in shapes]  # noqa: E731
    param, grad, momentum = make(torch.float32, 0.02), make(DTYPES[dtype], 1.0), make(torch.float32, 0.5)
    copy = make(torch.bfloat16, 0.0)
    w0, g0, m0 = ([x[i].cpu().double() for i in some] for x in (param, grad, momentum))
    opt = block.Muon(param, grad, momentum, 0.1, copy, 0.5)
    for nesterov in (True, False):
        opt.step(0.1, 0.9, nesterov, 0.25, ABC)
        for k, i in enumerate(some):
            g = 0.25 * g0[k]
            m0[k] = 0.9 * m0[k] + g
            assert rel(momentum[i], m0[k]) <= FP32
            x = orthogonal(g + 0.9 * m0[k] if nesterov else m0[k])
            want = w0[k] * (1 - 0.1 * 0.1) - 0.1 * 0.5 * x
            off = (param[i].cpu().double() - want).norm()
            assert off <= 0.05 * muon_tolerance(shapes[i]) * x.norm() + FP32 * want.norm(), (shapes[i], off / x.norm() / 0.05, muon_tolerance(shapes[i]))
            assert torch.equal(copy[i], param[i].bfloat16())
            w0[k], m0[k] = param[i].cpu().double(), momentum[i].cpu().double()


def test_muon_wide_range_and_special_values(block):
    """Singular values over six decades; a zero update; what is not a number stays in its matrix."""
    gen = torch.Generator().manual_seed(9)
    q = torch.linalg.qr(torch.randn((96, 96), generator=gen, dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn((200, 96), generator=gen, dtype=torch.float64))[0]
    wide = (q * 10.0 ** torch.linspace(0, -6, 96, dtype=torch.float64)) @ v.t()
    grads = [wide.float(), torch.zeros(20, 30), torch.full((9, 9), math.nan), 1e15 * torch.eye(16)]
    dev = [g.cuda() for g in grads]
    param, momentum = ([torch.zeros_like(g) for g in dev] for _ in range(2))
    block.Muon(param, dev, momentum, 0.0, scale=1.0).step(1.0, 0.5, eps=1e-35)
    want = -orthogonal(grads[0].double() * 1.5, 1e-35)
    assert (param[0].cpu().double() - want).norm() <= muon_tolerance((96, 200)) * 96 ** 0.5
    assert (param[1] == 0).all()
    assert torch.isnan(param[2]).all()
    assert rel(param[3], -orthogonal(torch.eye(16, dtype=torch.float64))) <= muon_tolerance((16, 16))


def test_muon_other_polynomials(block):
    """One iteration, and different ones in turn; the cubic x (3 - x^2) / 2 alone."""
    gen = torch.Generator().manual_seed(4)
    g = torch.randn((40, 56), generator=gen)
    for abc in ([(1.5, -0.5, 0.0)], [(1.5, -0.5, 0.0)] * 12, [(4.0, -6.0, 2.5), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]):
        param, momentum = torch.zeros_like(g, device="cuda"), torch.zeros_like(g, device="cuda")
        block.Muon([param], [g.cuda()], [momentum], 0.0, scale=1.0).step(1.0, 0.0, False, coefficients=abc)
        want = -orthogonal(g.double(), abc=abc)
        # the smallest singular value's direction grows by the product of the a's at most
        grown = math.prod(a for a, _, _ in abc)
        assert (param.cpu().double() - want).norm() <= (1.5 * min(grown, 500) * 2.0 ** -23 + 3 * len(abc) * FP32) * max(1.0, want.norm().item())


# ------------------------------------------------------------------------------------------------ as programs call them

class Step:
    """Every call of this file once, with the tensors that a program keeps: rotation, head norms, gated layers of many and of few rows, whose
    contractions are dealt to several workgroups or not, and updates of matrices of both kinds."""

    def __init__(self, block, seed, T=150):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device="cuda")  # noqa: E731
        B, H, D, d, f = 2, 6, 32, 96, 520
        self.x, self.q, self.k = new(B, T, H + 2, D), new(B, T, H, D), new(B, T, 1, D)
        self.dq, self.dk, self.dx = new(B, T, H, D), new(B, T, 1, D), new(B, T, H + 2, D)
        self.kept, self.sq = new(B, 2, D, dt=torch.float32), new(B, dt=torch.float32)
        views = lambda t: (t[:, :, :H], t[:, :, H:H + 1])  # noqa: E731
        kw = dict(turns=block.rotary_turns(D).cuda(), position=torch.arange(2 * T, dtype=torch.int32, device="cuda").view(B, T))
        norm = block.HeadNorm(*views(self.x), self.q, self.k, torch.ones(D, device="cuda"), None, **kw)
        turn = block.Rotary(self.q, self.k, self.q, self.k, **kw)
        self.w = [new(d, f), new(d, f), new(f, d)]
        gated = block.GatedFeedForward(*self.w, activation="gelu")
        self.w += [new(2056, 40), new(2056, 40), new(40, 2056), *(new(*s, dt=torch.float32) for s in ((520, 96), (520, 96), (96, 520)))]
        layers = [gated] * 3 + [block.GatedFeedForward(*self.w[3:6]), block.GatedFeedForward(*self.w[6:])]
        rows = [(new(n, o.d, dt=o.dtype), [new(n, o.f, dt=o.dtype) for _ in range(5)], new(n, o.d, dt=o.dtype)) for o, n in zip(layers, (7, 90, 600, 90, 20))]
        self.p, self.g, self.m = ([torch.empty(s, device="cuda") for s in ((40, 24), (200, 136), (96, 300), (8, 8))] for _ in range(3))
        muon = block.Muon(self.p, self.g, self.m, 0.1)
        self.objects, self.inputs = (norm, gated, muon, *layers[3:]), [self.x, self.dq, self.dk, *self.w, *[r[0] for r in rows], *self.g]
        self.outputs = [self.q, self.k, self.kept, self.sq, *[t for r in rows for t in (*r[1], r[2])], *self.p, *self.m]

        def run():
            norm.forward(*views(self.x), self.q, self.k)
            turn.forward(self.q, self.k, self.q, self.k)
            norm.backward(*views(self.x), self.dq, self.dk, *views(self.dx), self.kept, self.sq)
            for layer, (x, (gate, up, h, dgate, dup), dx) in zip(layers, rows):
                layer.forward(x, h, gate, up)
                layer.backward(x, gate, up, dgate, dup, dx)
            muon.step(0.01)
        self.run = run

    def fill(self):
        for t in (*self.inputs, *self.p, *self.m):
            t.copy_(torch.randn(t.shape, generator=self.gen, device="cuda"))
        for t in self.outputs[:-2 * len(self.p)]:
            t.fill_(7.0)


def test_step_replayed_in_a_graph(block):
    """All of it captured once and replayed on new inputs, with eager calls in between."""
    s = Step(block, 3)
    s.fill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()                                           # workspaces are there before the capture
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run()
    for _ in range(4):
        s.fill()
        state = [t.clone() for t in (*s.p, *s.m)]
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in s.outputs]
        for t, before in zip((*s.p, *s.m), state):
            t.copy_(before)
        s.run()
        torch.cuda.synchronize()
        assert all(torch.isfinite(t).all() and torch.equal(a, t) for a, t in zip(got, s.outputs))


def test_steps_on_streams_at_once(block):
    """Two sets of objects and two streams, and graphs of one set beside its eager calls: none shares scratch with another."""
    steps, want = [Step(block, 5), Step(block, 6, 90)], []
    for s in steps:
        s.fill()
        s.state = [t.clone() for t in (*s.p, *s.m)]
        s.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in s.outputs])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    used = []
    for o in steps[0].objects:
        inner = o._ws
        o._ws = lambda *args, inner=inner: used.append(inner(*args)) or used[-1]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        steps[0].run()
    captured = [(t.data_ptr(), t.data_ptr() + t.numel()) for t in used]
    del used[:]
    with torch.cuda.stream(streams[0]):
        steps[0].run()
    spans = sorted(captured + [(t.data_ptr(), t.data_ptr() + t.numel()) for t in used])
    torch.cuda.synchronize()
    assert len(captured) >= 8 and all(a[1] <= b[0] for a, b in zip(spans, spans[1:]) if a != b)
    for _ in range(6):
        for s in steps:
            for t, before in zip((*s.p, *s.m), s.state):
                t.copy_(before)
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[0]):
            graph.replay()
        with torch.cuda.stream(streams[1]):
            steps[1].run()
        torch.cuda.synchronize()
        for s, outputs in zip(steps, want):
            assert all(torch.equal(a, b) for a, b in zip(s.outputs, outputs))


def test_gated_rows_and_columns_do_not_meet(block):
    """What is not a number stays in its row, or its weight's column, on every kernel: few rows, small and large tiles, fp32."""
    for dtype, rows in (("bf16", 5), ("f16", 40), ("bf16", 300), ("f16", 2600), ("f32", 70), ("f32", 2600)):
        d, f = 72, 1032 if rows < 2000 else 2120
        gen = torch.Generator(device="cuda").manual_seed(rows)
        r = lambda *s: torch.randn(s, generator=gen, device="cuda").to(DTYPES[dtype])  # noqa: E731
        x, wg, wu, wd = r(rows, d), r(d, f), r(d, f), r(f, d)
        x[rows - 2] = math.nan
        x[1, 3] = math.inf
        wg[:, f - 3] = math.nan
        wd[5] = math.nan                                  # column 5 of dh
        layer = block.GatedFeedForward(wg, wu, wd)
        gate, up, h, dgate, dup = (torch.empty((rows, f), dtype=x.dtype, device="cuda") for _ in range(5))
        dx = torch.empty_like(x)
        layer.forward(x, h, gate, up)
        bad_rows, fine = [1, rows - 2], torch.ones(rows, dtype=torch.bool)
        fine[bad_rows] = False
        columns = torch.ones(f, dtype=torch.bool)
        columns[f - 3] = False
        assert torch.isfinite(gate.cpu()[fine][:, columns]).all() and torch.isfinite(up.cpu()[fine]).all()
        assert torch.isnan(gate.cpu()[:, f - 3]).all() and torch.isnan(up.cpu()[rows - 2]).all() and not torch.isfinite(up.cpu()[1]).any()
        layer.backward(r(rows, d), up.nan_to_num(0, 0, 0), up.nan_to_num(0, 0, 0), dgate, dup)
        columns[:] = True
        columns[5] = False
        assert torch.isfinite(dgate.cpu()[:, columns]).all() and torch.isnan(dgate.cpu()[:, 5]).any()
        dgate, dup = r(rows, f), r(rows, f)
        bad = block.GatedFeedForward(r(d, f), r(d, f))
        dh = r(rows, f)
        dh[rows - 1] = math.nan
        bad.backward(dh, r(rows, f), r(rows, f), dgate, dup, dx)
        assert torch.isfinite(dx[:rows - 1]).all() and torch.isnan(dx[rows - 1]).all()


def test_muon_more_matrices_than_travel_together(block):
    """Two launches of each step, fp16 copies of matrices of both kinds, gradients that two matrices share."""
    gen = torch.Generator().manual_seed(12)
    shapes = [(100, 110)] * 66 + [(20, 30)] * 2
    param = [torch.randn(s, generator=gen).cuda() for s in shapes]
    shared = {s: torch.randn(s, generator=gen).cuda() for s in set(shapes)}
    copy, before = [torch.empty(s, dtype=torch.float16, device="cuda") for s in shapes], [p.cpu().double() for p in param]
    block.Muon(param, [shared[s] for s in shapes], [torch.zeros(s, device="cuda") for s in shapes], 0.5, copy, 2.0).step(0.25, 0.5)
    x = {s: orthogonal(1.5 * shared[s].cpu().double()) for s in set(shapes)}
    for p, c, b in zip(param, copy, before):
        want = b * (1 - 0.25 * 0.5) - 0.25 * 2.0 * x[p.shape]
        assert (p.cpu().double() - want).norm() <= 0.5 * muon_tolerance(p.shape) * x[p.shape].norm() + FP32 * want.norm()
        assert torch.equal(c, p.half())


def test_gated_one_bias(block):
    for dtype, rows in (("bf16", 3), ("f16", 90), ("f32", 5)):
        gen = torch.Generator().manual_seed(rows)
        x, wg, wu = rand(gen, (rows, 64), dtype), rand(gen, (64, 40), dtype, 0.125), rand(gen, (64, 40), dtype, 0.125)
        bias = rand(gen, (40,), dtype)
        for biases in ((bias, None), (None, bias)):
            layer = block.GatedFeedForward(wg.cuda(), wu.cuda(), None, *(None if b is None else b.cuda() for b in biases))
            gate, up, h = (torch.empty((rows, 40), dtype=x.dtype, device="cuda") for _ in range(3))
            layer.forward(x.cuda(), h, gate, up)
            for got, w, b in zip((gate, up), (wg, wu), biases):
                same(got, x.double() @ w.double() + (0 if b is None else b.double()), FP32, dtype)


def test_heads_read_what_is_broadcast(block):
    """One head of keys for all of them, one row of queries for all samples; results of their own."""
    gen = torch.Generator().manual_seed(2)
    q, k = rand(gen, (1, 5, 4, 32), "bf16").cuda().expand(3, 5, 4, 32), rand(gen, (3, 5, 1, 32), "bf16").cuda().expand(3, 5, 4, 32)
    turns = block.rotary_turns(32)
    out = [torch.empty((3, 5, 4, 32), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    block.Rotary(q, k, *out, turns.cuda()).forward(q, k, *out)
    for x, y in zip((q, k), out):
        assert rel(y, turn(x.cpu().double(), turns, False, 1.0, torch.arange(5).repeat(3, 1))) <= U["bf16"] + FP32
    norm = block.HeadNorm(q, k, *out, turns=turns.cuda())
    norm.forward(q, k, *out)
    for x, y in zip((q, k), out):
        unit = x.cpu().double() * (x.cpu().double().square().mean(-1, keepdim=True) + 1e-6) ** -0.5
        assert rel(y, turn(unit, turns, False, 1.0, torch.arange(5).repeat(3, 1))) <= U["bf16"] + 4 * FP32
    with pytest.raises(block.dp.DpError):                # gradients in the layout of what is broadcast
        norm.backward(q, k, *out, q, k)


def test_far_offsets(block):
    """Samples, rows and results more than 2^31 elements into their arrays."""
    far = 2 ** 31 + 64
    base = torch.zeros(far + 4096, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(1)
    x = rand(gen, (2, 3, 4, 16), "bf16")
    q = base.as_strided((2, 3, 4, 16), (far, 128, 16, 1))
    q.copy_(x)
    out = torch.zeros(far + 4096, dtype=torch.bfloat16, device="cuda").as_strided((2, 3, 4, 16), (far, 64, 16, 1))
    turns = block.rotary_turns(16)
    kept, sq = torch.empty((2, 1, 16), device="cuda"), torch.empty(2, device="cuda")
    norm = block.HeadNorm(q, None, out, None, turns=turns.cuda())
    norm.forward(q, None, out, None)
    unit = x.double() * (x.double().square().mean(-1, keepdim=True) + 1e-6) ** -0.5
    assert rel(out, turn(unit, turns, False, 1.0, torch.arange(3).repeat(2, 1))) <= U["bf16"] + 4 * FP32
    norm.backward(q, None, out, None, q, None, kept, sq)              # in the place of the inputs
    assert torch.isfinite(q).all() and torch.isfinite(kept).all()
    del base, q, out
    rows, d, f = 66000, 16, 32768
    x, wg, wu = rand(gen, (rows, d), "bf16"), rand(gen, (d, f), "bf16", 0.25), rand(gen, (d, f), "bf16", 0.25)
    gate, up, h = (torch.empty((rows, f), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    layer = block.GatedFeedForward(wg.cuda(), wu.cuda())
    layer.forward(x.cuda(), h, gate, up)
    some = [0, 1, 65535, 65536, rows - 1]
    want = x[some].double() @ wg.double(), x[some].double() @ wu.double()
    same(gate[some], want[0], FP32, "bf16")
    same(up[some], want[1], FP32, "bf16")
    dx = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda")
    layer.backward(h, gate, up, gate, up, dx)                         # in place of gate and up
    same(dx[some], gate[some].cpu().double() @ wg.double().t() + up[some].cpu().double() @ wu.double().t(), 4 * FP32, "bf16")


def test_repeated_calls_give_the_same_bits(block):
    s = Step(block, 11)
    s.fill()
    state = [t.clone() for t in (*s.p, *s.m)]
    s.run()
    first = [t.clone() for t in s.outputs]
    for _ in range(3):
        for t, before in zip((*s.p, *s.m), state):
            t.copy_(before)
        s.run()
        assert all(torch.equal(a, b) for a, b in zip(first, s.outputs))
