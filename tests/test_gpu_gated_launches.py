"""Every way in which a gated layer's passes are launched (dp_gated_launches), with every activation and 16-bit type, element by element against 64 bits.

What one element may err by: its rounding, U of it (subnormal fp16 numbers are 2^-24 apart), and
  SUM   of the sums before it: additions of K random terms err by c sqrt(K / 2) of their root mean square, c = 2.5e-8 (a rounding spread evenly over a
        unit in the last place); of 12000 terms 2e-6, and the largest of some millions is within six times that
  SHARE of an activation's share of its argument, in 16 bits: within 1.5e-7 of 1 (the approximation of gelu's tail) and a few roundings
"""
import math

import pytest
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
SUM, SHARE = 1.2e-5, 4e-7
ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]
# pass, how it is launched, rows, d, f, d_out
CASES = [
    (0, "few", 5, 520, 264, 16), (0, "few", 20, 520, 264, 16), (0, "few", 49, 264, 520, 16), (0, "small", 71, 72, 136, 16), (0, "large", 402, 40, 9952, 16),
    (0, "large+small", 533, 24, 11144, 16), (0, "dealt128", 70, 4312, 72, 16), (0, "small+dealt128", 646, 1080, 2744, 16),
    (0, "large+dealt128", 3101, 1032, 2464, 16), (0, "large+small+dealt128", 3412, 1176, 2872, 16), (0, "dealt256", 142, 5224, 5616, 16),
    (1, "few", 5, 16, 264, 520), (1, "few", 20, 16, 264, 520), (1, "few", 49, 16, 520, 264), (1, "small", 71, 16, 136, 72), (1, "large", 10953, 16, 1048, 24),
    (1, "large+small", 19511, 16, 792, 24), (1, "dealt128", 78, 16, 136, 1032), (1, "small+dealt128", 294, 16, 10992, 1056),
    (1, "large+dealt128", 3206, 16, 5008, 480), (1, "large+small+dealt128", 9057, 16, 2248, 1392),
    (2, "few", 5, 264, 520, 16), (2, "few", 20, 264, 520, 16), (2, "few", 49, 520, 264, 16), (2, "small", 71, 136, 72, 16), (2, "large", 18331, 416, 24, 16),
    (2, "large+small", 16875, 792, 24, 16), (2, "dealt128", 75, 136, 1064, 16), (2, "small+dealt128", 260, 10984, 496, 16),
    (2, "large+dealt128", 1547, 9328, 456, 16), (2, "large+small+dealt128", 2786, 8896, 488, 16), (2, "dealt256", 132, 4120, 5832, 16)]
CASES_F32 = [(0, "large", 4100, 37, 521, 5), (0, "small", 71, 45, 77, 5), (0, "dealt64", 41, 1001, 77, 5), (1, "large", 4100, 5, 1021, 37), (1, "small", 71, 5, 77, 45),
             (1, "dealt64", 41, 5, 77, 1001), (2, "large", 4100, 1021, 37, 5), (2, "small", 71, 77, 45, 5), (2, "dealt64", 41, 77, 1001, 5)]


def launched(dp, dt, rows, d, f, d_out, which):
    plan = dp.dp_gated_launches(dt, rows, d, f, d_out, which)
    if plan["kernel"] == 1:
        return "few"
    return "+".join(k for k in ("large", "small", "dealt") if plan[k]) + (str(plan["side"]) if plan["dealt"] else "")


def activation(x, act):
    if act == "relu":
        return x.clamp(min=0), (x > 0).double()
    if act == "gelu":
        share, rise = 0.5 * torch.special.erfc(-x * 0.5 ** 0.5), torch.exp(-0.5 * x * x) * (2 * math.pi) ** -0.5
    else:
        c = 2 * (2 / math.pi) ** 0.5
        v, dv = (x, 1.0) if act != "gelu_tanh" else (c * (x + 0.044715 * x ** 3), c * (1 + 3 * 0.044715 * x * x))
        share = torch.sigmoid(v)
        rise = share * torch.sigmoid(-v) * dv
    return (share, rise) if act == "sigmoid" else (x * share, share + x * rise)


def near(got, want, before, dtype):
    """`before`: what the value before its rounding may err by."""
    bound = U[dtype] * (want.abs() + before) + before + (2.0 ** -25 if dtype == "f16" else 0)
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= bound).all(), ((off - bound).max().item(), (off > bound).sum().item(), (off > bound).nonzero()[:4].tolist())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,case", [(d, c) for d in DTYPES for c in (CASES_F32 if d == "f32" else CASES)], ids=str)
def test_gated_launch(dtype, case):
    from paper_2311_11822_amd import binding as dp, block
    which, how, rows, d, f, d_out = case
    dt = {"f32": dp.DP_F32, "bf16": dp.DP_BF16, "f16": dp.DP_F16}[dtype]
    assert launched(dp, dt, rows, d, f, d_out, which) == how
    gen = torch.Generator(device="cuda").manual_seed(rows + d + f)
    r = lambda *s, scale=1.0: (torch.randn(s, generator=gen, device="cuda") * scale).to(DTYPES[dtype])  # noqa: E731
    guard = torch.full((3, rows + 1, f), 7.0, dtype=DTYPES[dtype], device="cuda")             # a row behind each result stays
    rms = lambda t: t.square().mean().sqrt()  # noqa: E731
    if which == 0:
        x, wg, wu, bg, bu = r(rows, d), r(d, f, scale=d ** -0.5), r(d, f, scale=d ** -0.5), r(f), r(f)
        gate, up, h = (t[:rows] for t in guard)
        want_gate, want_up = x.double() @ wg.double(), x.double() @ wu.double()
        errs = SUM * rms(want_gate), SUM * rms(want_up)
        for biases in (False, True):
            if biases:
                want_gate, want_up = want_gate + bg.double(), want_up + bu.double()
            for act in ACTS:
                guard[:, :rows] = math.nan
                layer = block.GatedFeedForward(wg, wu, None, *((bg, bu) if biases else (None, None)), activation=act)
                layer.forward(x, h, gate, up)
                near(gate, want_gate, errs[0] + U["f32"] * want_gate.abs(), dtype)
                near(up, want_up, errs[1] + U["f32"] * want_up.abs(), dtype)
                value, slope = activation(want_gate, act)
                err = (slope.abs() + 1e-3) * 1.01 * errs[0] + SHARE * want_gate.abs().clamp(min=1)
                near(h, value * want_up, err * want_up.abs() + value.abs() * errs[1] + err * errs[1], dtype)
    elif which == 1:
        dy, wd, gate, up = r(rows, d_out), r(f, d_out, scale=d_out ** -0.5), r(rows, f, scale=1.5), r(rows, f)
        dgate, dup = (t[:rows] for t in guard[:2])
        dh = dy.double() @ wd.double().t()
        err = SUM * rms(dh)
        for act in ACTS:
            guard[:2, :rows] = math.nan
            value, slope = activation(gate.double(), act)
            share = SHARE * gate.double().abs().clamp(min=1)
            w = r(d, f)
            block.GatedFeedForward(w, w, wd, activation=act).backward(dy, gate, up, dgate, dup)
            near(dgate, dh * up.double() * slope, (err * (slope.abs() + share) + dh.abs() * share) * up.double().abs(), dtype)
            near(dup, dh * value, err * (value.abs() + share) + dh.abs() * share, dtype)
    else:
        wg, wu, dh = r(d, f, scale=f ** -0.5), r(d, f, scale=f ** -0.5), r(rows, f)
        gate, up = r(rows, f), r(rows, f)
        dgate, dup, dx = guard[0, :rows], guard[1, :rows], torch.full((rows + 1, d), 7.0, dtype=DTYPES[dtype], device="cuda")
        block.GatedFeedForward(wg, wu).backward(dh, gate, up, dgate, dup, dx[:rows])
        want = dgate.double() @ wg.double().t() + dup.double() @ wu.double().t()
        near(dx[:rows], want, SUM * rms(want), dtype)
        assert (dx[rows] == 7).all()
    assert (guard[:, rows] == 7).all()


def test_every_launch_has_a_case():
    """Whatever sizes' costs choose is among the cases above, and each of them is what it says."""
    import random
    import paper_2311_11822_amd.binding as dp
    for dt, cases in ((dp.DP_BF16, CASES), (dp.DP_F16, CASES), (dp.DP_F32, CASES_F32)):
        for which, how, *sizes in cases:
            assert launched(dp, dt, *sizes, which) == how, (which, sizes)
        rng, have = random.Random(1), {(which, how) for which, how, *_ in cases}
        size = lambda: 8 * max(1, round(math.exp(rng.uniform(0, math.log(2500)))))  # noqa: E731
        for _ in range(20000):
            rows, d, f, d_out = round(math.exp(rng.uniform(0, math.log(20000)))), size(), size(), size()
            for which in range(3):
                assert (which, launched(dp, dt, rows, d, f, d_out, which)) in have, (which, rows, d, f, d_out)


def test_launches_refused():
    import paper_2311_11822_amd.binding as dp
    right = dict(dt=dp.DP_BF16, rows=4, d=16, f=24, d_out=16, which=0)
    assert dp.dp_gated_launches(**right)["kernel"] == 1
    assert dp.dp_gated_launches(**dict(right, d_out=-1))["kernel"] == 1           # (looked at by the hidden pass alone)
    for bad in (dict(dt=7), dict(rows=0), dict(d=12), dict(f=0), dict(which=3), dict(which=-1), dict(which=1, d_out=12), dict(which=1, d_out=0), dict(d=1 << 21)):
        with pytest.raises(dp.DpError):
            dp.dp_gated_launches(**{**right, **bad})
