"""What the rotation and norms of heads, gated feed-forward layers and the orthogonalising optimizer refuse, and their host functions, without
a GPU: every call here ends before anything is launched."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2311_11822_amd.binding as dp
from paper_2311_11822_amd import block

FAKE = 0x1000                     # an aligned address, never dereferenced
INV, UNS, WS = dp.DP_ERR_INVALID_ARG, dp.DP_ERR_UNSUPPORTED, dp.DP_ERR_WORKSPACE


def changed(args, **kw):
    unknown = set(kw) - set(args)
    assert not unknown, unknown
    return list({**args, **kw}.values())


# ------------------------------------------------------------------------------------------------ heads

def shape(B=2, T=33, H=4, H_kv=2, D=64, rotary=64, interleaved=0, amplitude=1.0, q=None, k=None, qo=None, ko=None, turns=FAKE, position=None,
          len=None):
    q, qo = q or (T * H * D, H * D, D), qo or (T * H * D, H * D, D)
    k, ko = k or (T * H_kv * D, H_kv * D, D), ko or (T * H_kv * D, H_kv * D, D)
    return dp.heads_shape(B, T, H, H_kv, D, rotary, interleaved, amplitude, q, k, qo, ko, turns, position, len)


def calls(s, dt=dp.DP_BF16, q=FAKE, k=FAKE, q_out=FAKE, k_out=FAKE):
    """Statuses of the calls that write in the results' strides, and of those that write in the inputs'."""
    forward = (dp.lib.dp_rotary(s, dt, q, k, q_out, k_out, None), dp.lib.dp_head_norm(s, dt, q, k, None, None, 1e-6, q_out, k_out, None))
    back = (dp.lib.dp_rotary_backward(s, dt, q_out, k_out, q, k, None),
            dp.lib.dp_head_norm_backward(s, dt, q, k, q_out, k_out, None, None, 1e-6, q, k, None, None, None, 0, None))
    return forward, back


@pytest.mark.parametrize("change,status", [
    (dict(B=0), INV), (dict(T=0), INV), (dict(H=0), INV), (dict(H_kv=-1), INV), (dict(D=0), INV), (dict(D=12, rotary=12), INV), (dict(rotary=66), INV),
    (dict(rotary=-2), INV), (dict(rotary=7), INV), (dict(interleaved=2), INV), (dict(amplitude=math.nan), INV), (dict(amplitude=math.inf), INV),
    (dict(turns=None), INV), (dict(turns=FAKE + 4), INV), (dict(position=FAKE + 2), INV), (dict(len=FAKE + 1), INV), (dict(q=(8448, 256, -64)), INV),
    (dict(k=(8448, 132, 64)), INV), (dict(qo=(8448, 256, 60)), INV), (dict(D=264, rotary=64), UNS), (dict(B=1 << 16, T=1 << 16), UNS),
    (dict(H=1 << 21), UNS), (dict(B=(1 << 21) + 1, T=1), UNS)], ids=str)
def test_heads_refuse_shapes(change, status):
    s = shape(**change)
    forward, back = calls(s)
    assert forward == (status,) * 2 and back == (status,) * 2
    assert dp.dp_head_norm_workspace_bytes(s, dp.DP_BF16) == 0


def test_heads_refuse_strides_whose_span_passes_64_bits():
    far = (1 << 40, 1 << 39, 64)                          # 2^24 tokens span 2^63
    assert calls(shape(B=2, T=1 << 24, qo=far, ko=far, q=far, k=far)) == ((INV,) * 2,) * 2


def test_heads_refuse_arguments():
    s = shape()
    for dt in (3, -1):
        assert calls(s, dt=dt) == ((INV,) * 2,) * 2
    assert dp.lib.dp_rotary(None, dp.DP_F32, FAKE, FAKE, FAKE, FAKE, None) == INV
    for name in ("q", "k", "q_out", "k_out"):
        for bad in (None, FAKE + 8):
            assert calls(s, **{name: bad}) == ((INV,) * 2,) * 2
    norm = dict(s=s, dt=dp.DP_BF16, q=FAKE, k=FAKE, q_gain=None, k_gain=None, eps=1e-6, q_out=FAKE, k_out=FAKE, stream=None)
    for bad in (dict(q_gain=FAKE + 2), dict(k_gain=FAKE + 1), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf)):
        assert dp.lib.dp_head_norm(*changed(norm, **bad)) == INV
    n = dp.dp_head_norm_workspace_bytes(s, dp.DP_BF16)
    back = dict(s=s, dt=dp.DP_BF16, q=FAKE, k=FAKE, dq_out=FAKE, dk_out=FAKE, q_gain=None, k_gain=None, eps=1e-6, dq=FAKE, dk=FAKE, kept=FAKE,
                sqnorm=FAKE, ws=FAKE, ws_bytes=n, stream=None)
    assert n > 0
    for bad, status in ((dict(dq_out=None), INV), (dict(dk_out=FAKE + 2), INV), (dict(dq=None), INV), (dict(dk=FAKE + 8), INV), (dict(kept=None), INV),
                        (dict(sqnorm=None), INV), (dict(kept=FAKE + 2), INV), (dict(eps=-1.0), INV), (dict(ws=None), WS), (dict(ws_bytes=n - 1), WS),
                        (dict(ws=FAKE + 4), INV), (dict(q_gain=FAKE + 2), INV)):
        assert dp.lib.dp_head_norm_backward(*changed(back, **bad)) == status, bad
    # fp32 needs no more than its own alignment, a head's width is any; queries alone have no keys to look at
    assert dp.dp_head_norm_workspace_bytes(shape(D=7, rotary=6, H_kv=0, k=(-5, 3, 1)), dp.DP_F32) > 0


# Inputs may be broadcast or overlap, results (in the backward pass: the inputs' gradients) may not.
@pytest.mark.parametrize("name,strides", [("q", (0, 256, 64)), ("k", (33 * 128, 128, 0)), ("q", (33 * 128, 256, 64)), ("k", (33 * 64, 128, 64))])
def test_heads_results_do_not_overlap(name, strides):
    forward, back = calls(shape(**{name + "o": strides}), k_out=None)          # k_out: ends the calls that get past the strides
    assert forward == (INV,) * 2
    s = shape(**{name: strides})
    assert calls(s, k_out=None)[1] == (INV,) * 2
    assert dp.dp_head_norm_workspace_bytes(s, dp.DP_BF16) == 0


@pytest.mark.parametrize("bad", [dict(rotary=7), dict(rotary=-2), dict(base=0.0), dict(base=math.inf), dict(base=math.nan), dict(scaling=4), dict(scaling=-1),
                                 dict(scaling=1, factor=0.0), dict(scaling=2, factor=math.inf), dict(scaling=3, original=0.0), dict(scaling=3, slow=4.0, fast=4.0),
                                 dict(scaling=3, fast=math.nan)], ids=str)
def test_turns_refuse(bad):
    args = dict(rotary=8, base=1e4, scaling=0, factor=2.0, original=64.0, slow=1.0, fast=32.0)
    out = (ctypes.c_double * 8)()
    assert dp.lib.dp_rotary_turns(out, *changed(args, **bad)) == INV
    assert dp.lib.dp_rotary_turns(None, *changed(args)) == INV
    assert dp.lib.dp_rotary_turns(out, *changed(args)) == dp.DP_OK


@pytest.mark.parametrize("rotary", [0, 2, 8, 64, 130])
def test_turns(rotary):
    i = np.arange(0, rotary, 2)
    plain = 10000.0 ** (-i / max(rotary, 1)) / (2 * np.pi)
    turns = lambda **kw: block.rotary_turns(rotary, **kw).numpy()  # noqa: E731
    close = lambda a, b: np.testing.assert_allclose(a, b, rtol=1e-13)  # noqa: E731
    close(turns(), plain)
    close(turns(scaling="linear", factor=4.0), plain / 4)
    if rotary > 2:
        longer = turns(scaling="base", factor=8.0)
        close(longer[0], plain[0])                      # the fastest pair as it is, the slowest 8 times slower
        close(longer[-1], plain[-1] / 8)
    parts = turns(scaling="parts", factor=16.0, original=2048.0, slow=1.0, fast=32.0)
    often, seldom = plain * 2048 >= 32, plain * 2048 <= 1
    close(parts[often], plain[often])
    close(parts[seldom], plain[seldom] / 16)
    assert ((parts <= plain * (1 + 1e-12)) & (parts >= plain / 16 * (1 - 1e-12))).all()
    with pytest.raises(ValueError):
        turns(scaling="other")


def test_heads_objects_refuse():
    q, k, turns = torch.zeros(2, 5, 4, 16), torch.zeros(2, 5, 2, 16), block.rotary_turns(16)
    f = torch.zeros

    def make(q=q, k=k, q_out=None, k_out=None, turns=turns, kind=block.Rotary, **kw):
        return kind(q, k, q if q_out is None else q_out, k if k_out is None else k_out, *([] if kind is block.Rotary else kw.pop("gains", [None, None])),
                    turns=turns, **kw)
    wrong = [dict(turns=None), dict(turns=turns.float()), dict(turns=block.rotary_turns(18)), dict(q=q[0]), dict(k=f(2, 6, 2, 16)), dict(k=f(2, 5, 2, 8)),
             dict(q_out=f(2, 5, 2, 16)), dict(k_out=k.half()), dict(position=f(2, 5)), dict(position=f(5, dtype=torch.int32)),
             dict(length=f(3, dtype=torch.int32)), dict(q=f(2, 5, 16, 4).transpose(2, 3)), dict(amplitude=math.nan), dict(q_out=q[:, :1].expand(2, 5, 4, 16)),
             dict(kind=block.HeadNorm, gains=[f(15), None]), dict(kind=block.HeadNorm, gains=[None, f(16).half()]), dict(q=f(2, 0, 4, 16), k=f(2, 0, 2, 16)), dict()]
    for kw in wrong:                                     # the last: right, but not on a GPU
        with pytest.raises(ValueError):
            make(**kw)
    with pytest.raises(ValueError):
        block.Rotary(q, k, q, None, turns)
    with pytest.raises(TypeError):
        make(q=q.double(), k=k.double())


# ------------------------------------------------------------------------------------------------ gated feed-forward layers

GATED = dict(x=FAKE, dt=dp.DP_BF16, rows=4, d=16, f=24, w_gate=FAKE, w_up=FAKE, b_gate=None, b_up=None, act=0, gate=None, up=None, h=FAKE, ws=None,
             ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INV), (dict(x=FAKE + 8), INV), (dict(w_gate=None), INV), (dict(w_up=FAKE + 2), INV), (dict(h=None), INV), (dict(h=FAKE + 4), INV),
    (dict(gate=FAKE), INV), (dict(up=FAKE), INV), (dict(gate=FAKE, up=FAKE + 8), INV), (dict(b_gate=FAKE + 2), INV), (dict(b_up=FAKE + 8), INV),
    (dict(dt=5), INV), (dict(rows=0), INV), (dict(d=0), INV), (dict(f=-8), INV), (dict(d=12), INV), (dict(f=20), INV), (dict(act=5), INV), (dict(act=-1), INV),
    (dict(d=(1 << 20) + 8), UNS), (dict(f=(1 << 20) + 8), UNS), (dict(rows=(1 << 28) + 1), UNS), (dict(rows=1 << 28, f=1 << 20), UNS)], ids=str)
def test_gated_refuses(change, status):
    assert dp.lib.dp_gated(*changed(GATED, **change)) == status


GATED_BACK = dict(dy=FAKE, w_down=FAKE, d_out=16, gate=FAKE, up=FAKE, dt=dp.DP_F16, rows=4, d=16, f=24, w_gate=FAKE, w_up=FAKE, act=0, dgate=FAKE,
                  dup=FAKE, dx=FAKE, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), INV), (dict(dy=FAKE + 2), INV), (dict(w_down=FAKE + 8), INV), (dict(d_out=0), INV), (dict(d_out=12), INV), (dict(gate=None), INV),
    (dict(up=FAKE + 4), INV), (dict(dgate=None), INV), (dict(dup=None), INV), (dict(dx=FAKE + 8), INV), (dict(w_gate=None), INV), (dict(w_up=None), INV),
    (dict(act=7), INV), (dict(dt=-1), INV), (dict(rows=-1), INV), (dict(d=20), INV), (dict(f=0), INV), (dict(d_out=(1 << 20) + 8), UNS)], ids=str)
def test_gated_backward_refuses(change, status):
    assert dp.lib.dp_gated_backward(*changed(GATED_BACK, **change)) == status


def test_gated_workspaces():
    for size, args in ((dp.dp_gated_workspace_bytes, (4, 16, 24)), (dp.dp_gated_backward_workspace_bytes, (4, 16, 24, 16))):
        assert size(7, *args) == 0 == size(dp.DP_BF16, 0, *args[1:])
    # sums of both passes of backward fit; without w_down there is one
    both, one = (dp.dp_gated_backward_workspace_bytes(dp.DP_BF16, 1000, 64, 216, k) for k in (7416, 0))
    assert both > one
    # where a workspace is used it is asked for
    # where a workspace is used it is asked for
    for dt, rows, d, f in [(dt, *sizes) for dt in (dp.DP_F32, dp.DP_BF16) for sizes in
                           ((1, 1280, 3456), (1, 16, 1 << 20), (1, 1 << 20, 16), (64, 768, 2048), (1000, 7416, 216), (4096, 1280, 3456))]:
        n = dp.dp_gated_workspace_bytes(dt, rows, d, f)
        assert n > 0 or (rows, d, f) != (1000, 7416, 216)
        if n:
            args = dict(GATED, dt=dt, rows=rows, d=d, f=f)
            assert dp.lib.dp_gated(*changed(args, ws=FAKE, ws_bytes=n - 1)) == WS == dp.lib.dp_gated(*changed(args))
            assert dp.lib.dp_gated(*changed(args, ws=FAKE + 4, ws_bytes=n)) == INV
        n = dp.dp_gated_backward_workspace_bytes(dt, rows, d, f, d)
        if n:
            args = dict(GATED_BACK, dt=dt, rows=rows, d=d, f=f, d_out=d)
            assert dp.lib.dp_gated_backward(*changed(args, ws=FAKE, ws_bytes=n - 1)) == WS == dp.lib.dp_gated_backward(*changed(args))
            assert dp.lib.dp_gated_backward(*changed(args, ws=FAKE + 4, ws_bytes=n)) == INV


def test_gated_object_refuses():
    f = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    right = (f(16, 24), f(16, 24))
    for args, kw in [((f(16, 24), f(16, 32)), {}), ((f(16, 24), f(16, 24).half()), {}), ((f(24, 16).t(), f(16, 24)), {}), ((*right, f(16, 24)), {}),
                     ((*right, f(24)), {}), ((f(2, 16, 24), f(2, 16, 24)), {}), ((*right, None, f(16)), {}), ((*right, None, None, f(24).float()), {}),
                     (right, dict(activation="tanh")), (right, {})]:
        with pytest.raises(ValueError):
            block.GatedFeedForward(*args, **kw)


# ------------------------------------------------------------------------------------------------ orthogonalised updates

MUON = dict(lr=0.02, beta=0.95, nesterov=1, grad_scale=1.0, eps=1e-7)


def muon(change=(), abc=((3.4445, -4.7750, 2.0315),) * 5, tensors=None, n=1, grad_dt=dp.DP_BF16, copy_dt=dp.DP_F32, iterations=None, ws=FAKE,
         ws_bytes=1 << 40, **kw):
    t = dict(param=FAKE, grad=FAKE, m=FAKE, copy=FAKE, rows=8, cols=12, decay=0.1, scale=1.0)
    arr = dp.muon_tensors([changed(t, **dict(change))]) if tensors is None else tensors
    flat = (ctypes.c_double * (3 * len(abc)))(*[x for row in abc for x in row])
    return dp.lib.dp_muon_multi(arr, n, grad_dt, copy_dt, *changed(MUON, **kw), flat, len(abc) if iterations is None else iterations, ws, ws_bytes, None)


def test_muon_refuses():
    assert muon(n=0) == INV == muon(tensors=ctypes.POINTER(dp.dp_muon_tensor)())
    assert muon(grad_dt=5) == INV == muon(copy_dt=-1)
    assert muon(iterations=0) == INV == muon(iterations=33)
    for bad in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta=1.0), dict(beta=-0.1), dict(beta=math.nan), dict(nesterov=2),
                dict(grad_scale=math.inf), dict(grad_scale=math.nan), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf)):
        assert muon(**bad) == INV, bad
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(param=FAKE + 2), dict(grad=FAKE + 1), dict(m=FAKE + 1), dict(rows=0), dict(cols=-1),
                dict(decay=math.nan), dict(scale=math.inf)):
        assert muon(bad) == INV, bad
    for bad in (dict(copy=None), dict(copy=FAKE + 1)):
        assert muon(bad, copy_dt=dp.DP_F16) == INV, bad
    for bad in (dict(rows=(1 << 20) + 1), dict(cols=(1 << 20) + 1), dict(rows=1 << 17, cols=1 << 17)):
        assert muon(bad) == UNS, bad
    arr = dp.muon_tensors([(FAKE, FAKE, FAKE, None, 8, 12, 0.0, 1.0)])
    n = dp.dp_muon_workspace_bytes(arr)
    assert n > 0 and muon(ws_bytes=n - 1) == WS == muon(ws=None) and muon(ws=FAKE + 8) == INV
    assert dp.dp_muon_workspace_bytes([(None, None, None, None, 0, 12, 0.0, 1.0)]) == 0


# Polynomials under which singular values, or the polynomial of A, leave what two fp16 halves hold; NaN and infinities.
@pytest.mark.parametrize("abc", [((20.0, 0.0, 0.0),), ((4.0, 0.0, 0.0),) * 4, ((0.0, 0.0, 16.0),), ((math.nan, 0.0, 0.0),), ((1.0, math.inf, 0.0),),
                                 ((3.9, 0.0, 0.0), (0.1, 0.0, 0.0), (20.0, 0.0, 0.0))])
def test_muon_refuses_polynomials(abc):
    assert muon(abc=abc) == UNS


# Polynomials whose turning points a plain quadratic formula loses: a next to vanishing leading coefficient; squares beyond 64 bits; and
# coefficients that are finite in 64 bits alone.
@pytest.mark.parametrize("abc", [((14.0, -14.0, 1e-17), (14.0, 0.0, 0.0)), ((14.0, -14.0, -1e-17), (14.0, 0.0, 0.0)), ((14.0, -14.0, 0.0), (14.0, 0.0, 0.0)),
                                 ((1.0, 1.7e308, -1.7e308),), ((0.0, 0.0, 0.0), (1.0, 1e39, 0.0)), ((0.0, 0.0, 0.0), (1.0, 0.0, -1e39))])
def test_muon_refuses_polynomials_at_their_turning_points(abc):
    assert muon(abc=abc) == UNS


def test_muon_takes_polynomials_that_fit():
    """Up to the workspace's check: the usual ones, and such next to those that are refused."""
    for abc in (((3.4445, -4.7750, 2.0315),) * 5, ((1.5, -0.5, 0.0),) * 12, ((1.5, -0.5, 1e-17),) * 12, ((14.0, -14.0, 1e-17),), ((0.0, 0.0, 0.0), (1.0, 1e30, 0.0))):
        assert muon(abc=abc, ws=None) == WS, abc


def test_muon_workspace_is_of_one_run():
    """Matrices go in runs of up to 64: the workspace is the largest run's."""
    one = [(None, None, None, None, 128, 160, 0.0, 1.0)]
    assert dp.dp_muon_workspace_bytes(one * 64) == 64 * dp.dp_muon_workspace_bytes(one)
    assert dp.dp_muon_workspace_bytes(one * 90) == 45 * dp.dp_muon_workspace_bytes(one)
    small = [(None, None, None, None, 24, 72, 0.0, 1.0)]              # those that one workgroup holds need next to none
    assert 0 < dp.dp_muon_workspace_bytes(small * 3) <= 256 and dp.dp_muon_workspace_bytes(small * 70 + one) == dp.dp_muon_workspace_bytes(one)


def test_muon_object_refuses():
    f = torch.zeros
    right = ([f(3, 4)], [f(3, 4)], [f(3, 4)], 0.0)
    for args, kw in [(([], [], [], 0.0), {}), (([f(12)], [f(12)], [f(12)], 0.0), {}), (([f(3, 4)], [f(4, 3)], [f(3, 4)], 0.0), {}),
                     (([f(3, 4).half()], *right[1:]), {}), ((*right[:2], [f(4, 3).t()], 0.0), {}), ((*right[:3], [0.0, 1.0]), {}),
                     (right, dict(copy=[])), (right, dict(copy=[f(3, 5).half()])), (right, dict(scale=[1.0, 2.0])), (right, {})]:
        with pytest.raises(ValueError):
            block.Muon(*args, **kw)
    twice = f(3, 4)
    for args in (([twice] * 2, [f(3, 4)] * 2, [f(3, 4), f(3, 4)]), ([f(3, 4), f(3, 4)], [f(3, 4)] * 2, [twice] * 2), ([twice], [f(3, 4)], [twice])):
        with pytest.raises(ValueError, match="twice"):
            block.Muon(*args, 0.0)
    with pytest.raises(TypeError):
        block.Muon(*right, copy=[f(3, 4)])
    with pytest.raises(TypeError):
        block.Muon([f(3, 4)], [f(3, 4).double()], [f(3, 4)], 0.0)
