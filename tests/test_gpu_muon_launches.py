"""Every way in which the products of an orthogonalised update are launched (dp_muon_launches), against 64 bits.

Tolerance of X against its norm, as products of values in two fp16 halves give it: entries within 2^-23 of their size, in both factors of a
product; the product of the two lower halves, 2^-24 of one, left out; and sums in fp32: 1.2e-6 for one of up to 2400 terms (c sqrt(K / 2), c = 2.5e-8).
Five iterations multiply what a direction next to no singular value is off by 3.4445^5 = 485 at most, of a matrix that starts with norm 1 and ends
with about the root of its shorter side.
"""
import math

import pytest
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ABC = [(3.4445, -4.7750, 2.0315)] * 5
# matrices; held by one workgroup each; side of tiles and workgroups that share one: A, polynomial, update
CASES = [
    ([(24, 72), (72, 24)], 2, (0, 0), (0, 0), (0, 0)),
    ([(300, 520), (24, 72)], 1, (128, 1), (128, 1), (128, 1)),
    ([(770, 2300)], 0, (128, 8), (128, 1), (128, 1)),
    ([(700, 2600)] * 14, 0, (128, 1), (128, 1), (256, 1)),
    ([(300, 20000)], 0, (128, 32), (128, 1), (128, 1)),
    ([(766, 50260)], 0, (128, 12), (128, 1), (256, 1)),
    ([(2290, 2298), (2298, 2290)] * 12, 0, (256, 1), (256, 1), (256, 1))]


def plan(dp, shapes):
    p = dp.dp_muon_launches([(None,) * 4 + (*s, 0.0, 1.0) for s in shapes])
    return p["held"], p["square"], p["polynomial"], p["update"]


def orthogonal(u):
    x = u / (u.norm() + 1e-7)
    turned = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if turned else x
    for a, b, c in ABC:
        square = x @ x.t()
        x = a * x + (b * square + c * (square @ square)) @ x
    return x.t() if turned else x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{c[0][0]}")
def test_muon_launch(dtype, case):
    from paper_2311_11822_amd import binding as dp, block
    shapes, *how = case
    assert plan(dp, shapes) == tuple(how)
    gen = torch.Generator(device="cuda").manual_seed(len(shapes))
    r = lambda s, kind=torch.float32: torch.randn(s, generator=gen, device="cuda").to(kind)  # noqa: E731
    param, grad, momentum = [r(s) for s in shapes], [r(s, DTYPES[dtype]) for s in shapes], [r(s) for s in shapes]
    copy = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    some = sorted({0, 1 % len(shapes), len(shapes) - 1})
    before = {i: (param[i].double(), 0.25 * grad[i].double(), momentum[i].double()) for i in some}
    block.Muon(param, grad, momentum, 0.1, copy, 0.5).step(0.1, 0.9, True, 0.25, ABC)
    for i in some:
        w, g, m = before[i]
        m = 0.9 * m + g
        x = orthogonal(g + 0.9 * m)
        assert (momentum[i].double() - m).abs().max() <= 4 * 2.0 ** -24 * m.abs().max()
        # lr * scale = 0.05; the parameter's own rounding beside it
        off = ((w * 0.99 - param[i].double()) / 0.05 - x).norm() / x.norm()
        tol = 485 * 2.0 ** -22 / math.sqrt(min(shapes[i])) + 15 * 1.2e-6 + 2 * 2.0 ** -24 * w.norm() / (0.05 * x.norm())
        assert off <= tol, (off.item(), tol.item())
        assert torch.equal(copy[i], param[i].bfloat16())


def test_every_launch_has_a_case():
    """Whatever sizes' costs choose is among the cases above (of A's dealt tiles: any number of workgroups)."""
    import random
    import paper_2311_11822_amd.binding as dp
    kinds = lambda held, *steps: [(k, side, parts > 1) for k, (side, parts) in enumerate(steps) if side]  # noqa: E731
    have = set()
    for shapes, *how in CASES:
        assert plan(dp, shapes) == tuple(how), shapes
        have.update(kinds(*how))
    rng = random.Random(1)
    size = lambda: round(math.exp(rng.uniform(0, math.log(20000))))  # noqa: E731
    for _ in range(5000):
        shapes = [(size(), size()) for _ in range(rng.choice((1, 1, 2, 5)))] * rng.choice((1, 1, 4, 12))
        assert set(kinds(*plan(dp, shapes))) <= have, shapes


def test_launches_refused():
    import paper_2311_11822_amd.binding as dp
    for bad in ([], [(None,) * 4 + (0, 3, 0.0, 1.0)], [(None,) * 4 + (3, (1 << 20) + 1, 0.0, 1.0)]):
        with pytest.raises(dp.DpError):
            dp.dp_muon_launches(bad)
