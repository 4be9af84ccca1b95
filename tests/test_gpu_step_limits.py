"""Rotation and norms of heads, gated feed-forward layers and the orthogonalising optimizer at the ends of their ranges and where values are
next to nothing, against 64-bit values on the CPU or values that are known.

U is half a unit in the last place of the storage type, relative to the value.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def block():
    from paper_2311_11822_amd import block as b
    assert torch.cuda.is_available()
    return b


# ------------------------------------------------------------------------------------------------ heads

def slices(x, n=1 << 27):
    return (x[:, i:i + n] for i in range(0, x.shape[1], n))


@pytest.mark.parametrize("T,H_kv", [(2146435530, 5), (2 ** 31 - 1, 0), ((1 << 30) + 1, 1)])
def test_heads_of_two_thousand_million_tokens(block, T, H_kv):
    """One sample of up to 2^31 - 1 tokens, heads of one column, in place: x / sqrt(x^2 + eps) is x's sign but for eps / 8 = 1.25e-7 and three
    roundings; where heads of keys are several their chunks are others than the queries'."""
    q = torch.full((1, T, 1, 1), 2.0, device="cuda")
    q[:, 1::2] = -2.0
    k = torch.full((1, T, H_kv, 1), 2.0, device="cuda") if H_kv else None
    norm = block.HeadNorm(q, k, q, k)
    norm.forward(q, k, q, k)
    for t in (q, k):
        for s in () if t is None else slices(t):
            assert ((s.abs() - 1).abs().max() <= 5e-7).item()
    assert (q[0, ::2] > 0).all() and (q[0, 1::2] < 0).all()


def test_head_norm_gradient_of_two_thousand_million_tokens(block):
    """dy h is 1 in each of them, whose sum is their number: partial sums are whole below 2^24, later ones round 768 times at most."""
    T = 2 ** 31 - 1
    q = torch.full((1, T, 1, 1), 2.0, device="cuda")
    dy = torch.ones_like(q)
    kept, sqnorm = torch.empty((1, 1, 1), device="cuda"), torch.empty(1, device="cuda")
    norm = block.HeadNorm(q, None, dy, None, eps=0.0)
    norm.backward(q, None, dy, None, dy, None, kept, sqnorm)
    assert abs(kept.item() - T) <= 768 * U["f32"] * T
    assert abs(sqnorm.item() - float(T) ** 2) <= 2 * 769 * U["f32"] * float(T) ** 2
    for s in slices(dy):                                 # of one column all of dx cancels
        assert (s.abs().max() <= 4 * U["f32"]).item()
