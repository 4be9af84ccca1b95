"""What layer norm, attention and AdamW refuse, without a GPU: every call here ends before anything is launched."""
import ctypes
import math

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


NORM = dict(x=FAKE, add=None, dt=dp.DP_BF16, B=2, T=3, d=8, gain=None, bias=None, eps=1e-5, sum=None, y=FAKE, mean=None, rstd=None,
            stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INV), (dict(y=None), INV), (dict(x=FAKE + 8), INV), (dict(y=FAKE + 2), INV), (dict(add=FAKE), INV),
    (dict(sum=FAKE), INV), (dict(add=FAKE + 4, sum=FAKE), INV), (dict(add=FAKE, sum=FAKE + 4), INV), (dict(dt=3), INV),
    (dict(dt=-1), INV), (dict(B=0), INV), (dict(T=0), INV), (dict(d=0), INV), (dict(B=-1), INV), (dict(eps=-1e-9), INV),
    (dict(eps=math.nan), INV), (dict(eps=math.inf), INV), (dict(gain=FAKE + 2), INV), (dict(bias=FAKE + 1), INV),
    (dict(mean=FAKE + 2), INV), (dict(rstd=FAKE + 2), INV), (dict(d=32769), UNS), (dict(B=1 << 20, T=1 << 12), UNS)], ids=str)
def test_layer_norm_refuses(change, status):
    assert dp.lib.dp_layer_norm(*changed(NORM, **change)) == status


NORM_BACK = dict(x=FAKE, dy=FAKE, add=None, dt=dp.DP_F32, B=2, T=3, d=8, gain=None, mean=FAKE, rstd=FAKE, dx=FAKE, kept=FAKE,
                 sqnorm=FAKE, ws=FAKE, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INV), (dict(dy=None), INV), (dict(mean=None), INV), (dict(rstd=None), INV), (dict(dx=None, kept=None, sqnorm=None), INV),
    (dict(kept=None), INV), (dict(sqnorm=None), INV), (dict(add=FAKE, dx=None), INV), (dict(add=FAKE + 8), INV), (dict(dx=FAKE + 4), INV),
    (dict(kept=FAKE + 4), INV), (dict(sqnorm=FAKE + 1), INV), (dict(dt=4), INV), (dict(T=-3), INV), (dict(d=1 << 16), UNS),
    (dict(ws=None), WS), (dict(ws_bytes=0), WS), (dict(ws=FAKE + 4), INV)], ids=str)
def test_layer_norm_backward_refuses(change, status):
    assert dp.lib.dp_layer_norm_backward(*changed(NORM_BACK, **change)) == status


def test_layer_norm_workspace():
    assert dp.dp_layer_norm_workspace_bytes(dp.DP_BF16, 0, 1, 8) == 0 == dp.dp_layer_norm_workspace_bytes(dp.DP_BF16, 1, 1, 40000)
    n = dp.dp_layer_norm_workspace_bytes(dp.DP_BF16, 2, 512, 768)
    assert n > 0 and dp.lib.dp_layer_norm_backward(*changed(NORM_BACK, dt=dp.DP_BF16, T=512, d=768, ws_bytes=n - 1)) == WS


def shape(dt=dp.DP_BF16, B=2, H=4, H_kv=2, Tq=33, Tk=33, D=64, causal=1, scale=0.125, q=None, k=None, v=None, o=None, **lens):
    q, o = q or (Tq * H * D, H * D, D), o or (Tq * H * D, H * D, D)
    k, v = k or (Tk * H_kv * D, H_kv * D, D), v or (Tk * H_kv * D, H_kv * D, D)
    return dp.attention_shape(B, H, H_kv, Tq, Tk, D, causal, scale, q, k, v, o, **lens)


def forward(s, dt=dp.DP_BF16, **kw):
    return dp.lib.dp_attention(*changed(dict(shape=s, dt=dt, q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, ws=None, ws_bytes=0, stream=None), **kw))


def backward(s, dt=dp.DP_BF16, **kw):
    return dp.lib.dp_attention_backward(*changed(dict(
        shape=s, dt=dt, q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, ws_bytes=1 << 40,
        stream=None), **kw))


SHAPES_REFUSED = [
    (dict(B=0), INV), (dict(H=0), INV), (dict(H_kv=0), INV), (dict(H=3), INV), (dict(Tq=0), INV), (dict(Tk=-1), INV), (dict(D=0), INV),
    (dict(causal=2), INV), (dict(scale=0.0), INV), (dict(scale=-1.0), INV), (dict(scale=math.inf), INV), (dict(scale=math.nan), INV),
    (dict(D=12), INV), (dict(D=136), UNS), (dict(q=(8448, 256, -64)), INV), (dict(k=(8448, 132, 64)), INV), (dict(v=(1 << 20, 32, 64)), INV),
    (dict(o=(1 << 40, 1 << 24, 64)), UNS), (dict(B=1 << 20, H=1 << 12, H_kv=1), UNS), (dict(q_len=FAKE + 2), INV), (dict(k_len=FAKE + 1), INV)]


@pytest.mark.parametrize("change,status", SHAPES_REFUSED, ids=str)
def test_attention_refuses_shapes(change, status):
    s = shape(**change)
    assert forward(s) == status == backward(s)
    assert dp.dp_attention_backward_workspace_bytes(s, dp.DP_BF16) == 0


def test_attention_refuses_arguments():
    s = shape()
    assert forward(None) == INV == backward(None)
    assert forward(s, dt=7) == INV == backward(s, dt=7)
    for name in ("q", "k", "v", "o", "lse"):
        for bad in (None, FAKE + 2):
            assert forward(s, **{name: bad}) == INV == backward(s, **{name: bad})
    for name in ("dout", "dq", "dk", "dv"):
        for bad in (None, FAKE + 8):
            assert backward(s, **{name: bad}) == INV
    n = dp.dp_attention_backward_workspace_bytes(s, dp.DP_BF16)
    assert n >= 2 * 2 * 4 * 33 * 4
    assert backward(s, ws_bytes=n - 1) == WS == backward(s, ws=None)
    assert backward(s, ws=FAKE + 4) == INV
    assert dp.dp_attention_workspace_bytes(s, dp.DP_BF16) == 0 == dp.dp_attention_workspace_bytes(shape(D=136), dp.DP_BF16)
    s = shape(B=1, Tq=1, Tk=4096)                        # few queries on many keys
    n = dp.dp_attention_workspace_bytes(s, dp.DP_BF16)
    assert n >= 4 * 2 * 64 * 4 and forward(s, ws=FAKE, ws_bytes=n - 1) == WS and forward(s, ws=FAKE + 4, ws_bytes=n) == INV


# A tile's rows, a token stride apart, lie within the byte offsets of one descriptor (2^31), in all three kernels and up to the largest stride.
@pytest.mark.parametrize("dt,size", [(dp.DP_BF16, 2), (dp.DP_F16, 2), (dp.DP_F32, 4)])
@pytest.mark.parametrize("D", [8, 24, 32, 64, 72, 96, 104, 128])
def test_attention_tiles_lie_within_offsets(dt, size, D):
    strides = [1 << 12, 1 << 20, 1 << 21, (1 << 21) + 8, 1 << 22, (1 << 22) + 8, 1 << 23]
    for Tq, Tk in ((1, 130), (1, 1100), (130, 1), (1100, 1), (1100, 1100), (33, 40000), (1 << 20, 3)):
        for wide in strides:
            # each side's stride, one at a time: keys and values bound two kernels' tiles, queries and results the third's
            for name in "qkvo":
                s = shape(H=1, H_kv=1, B=1, D=D, Tq=Tq, Tk=Tk, causal=0, **{name: (1 << 50, wide, D)})
                rows = dp.dp_attention_tile_rows(s, dt)
                assert all(r * size * (wide if name in side else D) <= 1 << 31 for r, side in zip(rows, ("kv", "kv", "qo")))
                if dp.dp_attention_workspace_bytes(s, dt):              # keys in parts: whole tiles of the split form
                    assert rows[0] > 64 or D > 64 and dt == dp.DP_F32
    # the larger tiles of few rows are there where strides allow them
    few = dp.dp_attention_tile_rows(shape(H=1, H_kv=1, B=1, D=D, Tq=1, Tk=1100), dt)
    assert few[0] == few[1] == 32 * (8 if size * max(D, 32) <= 128 else 4 if size * D <= 256 else 2)


def test_attention_tile_rows_refuses():
    assert dp.lib.dp_attention_tile_rows(shape(), dp.DP_BF16, None) == INV == dp.lib.dp_attention_tile_rows(None, dp.DP_BF16, (ctypes.c_int32 * 3)())
    assert dp.lib.dp_attention_tile_rows(shape(D=136), dp.DP_BF16, (ctypes.c_int32 * 3)()) == UNS
    assert dp.dp_attention_tile_rows(shape(D=18), dp.DP_F32) == (1, 1, 1)


# D = 18 and a sample stride that is no multiple of 4 are for fp32 alone
def test_attention_widths_by_type():
    s = shape(D=18)
    assert dp.dp_attention_backward_workspace_bytes(s, dp.DP_F32) > 0 == dp.dp_attention_backward_workspace_bytes(s, dp.DP_F16)
    s = shape(q=(33 * 256 + 1, 256, 64))
    assert dp.dp_attention_backward_workspace_bytes(s, dp.DP_F32) > 0 == dp.dp_attention_backward_workspace_bytes(s, dp.DP_F16)


# Broadcast or overlapping inputs can be read; a result or a gradient in such a layout would be written over itself.
@pytest.mark.parametrize("name,strides", [("q", (0, 256, 64)), ("k", (0, 128, 64)), ("v", (33 * 128, 128, 0)), ("k", (33 * 64, 128, 64)),
                                          ("q", (33 * 256, 256, 32)), ("v", (1 << 20, 64, 64))])
def test_attention_gradients_do_not_overlap(name, strides):
    s = shape(**{name: strides})
    assert dp.dp_attention_backward_workspace_bytes(s, dp.DP_BF16) > 0
    assert backward(s, ws_bytes=0) == INV
    assert backward(shape(), ws_bytes=0) == WS


@pytest.mark.parametrize("strides", [(0, 256, 64), (33 * 256, 256, 0), (33 * 128, 256, 64)])
def test_attention_results_do_not_overlap(strides):
    assert forward(shape(o=strides)) == INV


ADAM = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, stream=None)


def adamw(change=(), tensors=None, n=1, grad_dt=dp.DP_BF16, bits=32, copy_dt=dp.DP_F32, **kw):
    t = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=FAKE, v_scale=FAKE, copy=FAKE, n=8, decay=0.1)
    arr = dp.adamw_tensors([changed(t, **dict(change))]) if tensors is None else tensors
    return dp.lib.dp_adamw_multi(arr, n, grad_dt, bits, copy_dt, *changed(ADAM, **kw))


def test_adamw_refuses():
    assert adamw(n=0) == INV == adamw(tensors=ctypes.POINTER(dp.dp_adamw_tensor)())
    assert adamw(grad_dt=5) == INV == adamw(copy_dt=-1)
    assert adamw(bits=16) == INV == adamw(step=0)
    for bad in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=math.nan),
                dict(beta2=1.0), dict(beta2=-0.1), dict(beta2=math.nan), dict(eps=-1e-8), dict(eps=math.nan), dict(eps=math.inf),
                dict(grad_scale=math.nan), dict(grad_scale=math.inf)):
        assert adamw(**bad) == INV, bad
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=FAKE + 2), dict(grad=FAKE + 1), dict(m=FAKE + 2),
                dict(v=FAKE + 1), dict(decay=math.nan), dict(decay=math.inf)):
        assert adamw(bad) == INV, bad
    for bad in (dict(m_scale=None), dict(v_scale=None), dict(m_scale=FAKE + 2), dict(v_scale=FAKE + 1)):
        assert adamw(bad, bits=8) == INV, bad
    for bad in (dict(copy=None), dict(copy=FAKE + 1)):
        assert adamw(bad, copy_dt=dp.DP_BF16) == INV, bad
    assert adamw(dict(n=(1 << 42) + 1)) == UNS
    assert adamw(dict(n=0, param=None, grad=None)) == dp.DP_OK                      # nothing to do


# ------------------------------------------------------------------------------------------------ the objects, on CPU tensors

def test_layer_norm_object_refuses():
    x, f = torch.zeros(2, 3, 8, dtype=torch.bfloat16), torch.zeros
    norm = block.LayerNorm(f(8), f(8))
    for call in (lambda: norm.forward(x[0], x[0]), lambda: norm.forward(x.transpose(0, 1), x), lambda: norm.forward(x, x.float()),
                 lambda: norm.forward(x, x[:1]), lambda: norm.forward(x, x.clone(), f(5), f(6)), lambda: norm.forward(x, x.clone(), f(6).half()),
                 lambda: norm.forward(x, x.clone(), add=x[:, :, :4]), lambda: block.LayerNorm(f(7), f(8)).forward(x, x.clone()),
                 lambda: norm.backward(x, x[:1], f(6), f(6), x.clone()), lambda: norm.backward(x, x, f(6), f(6), x.clone(), f(2, 8), f(2)),
                 lambda: norm.backward(x, x, f(6), f(6), x.clone(), f(2, 2, 8), f(3)), lambda: norm.forward(x, x.clone()),
                 lambda: norm.clipped_gradient(f(2, 2, 8), f(2), f(2, 7))):
        with pytest.raises(ValueError):
            call()


def test_attention_object_refuses():
    def make(q=(2, 5, 4, 16), k=(2, 5, 2, 16), v=None, o=None, dtype=torch.bfloat16, **kw):
        q, k, v, o = (torch.zeros(s, dtype=dtype) if isinstance(s, tuple) else s for s in (q, k, k if v is None else v, q if o is None else o))
        return block.Attention(q, k, v, o, True, kw.pop("scale", 1.0), **kw)
    t = torch.zeros(2, 5, 4, 16, dtype=torch.bfloat16)
    wrong = [dict(q=(5, 4, 16)), dict(k=(2, 5, 2, 8)), dict(v=(2, 6, 2, 16)), dict(o=(2, 5, 2, 16)), dict(k=(3, 5, 2, 16)), dict(k=(2, 5, 3, 16)),
             dict(scale=-1.0), dict(q=(2, 5, 4, 12), k=(2, 5, 2, 12)), dict(q=(2, 5, 4, 136), k=(2, 5, 2, 136)), dict(q=(2, 0, 4, 16)),
             dict(q=torch.zeros(2, 5, 16, 4, dtype=torch.bfloat16).transpose(2, 3), o=t), dict(o=t.float()), dict(k_len=torch.zeros(2)),
             dict(q_len=torch.zeros(3, dtype=torch.int32)), dict()]                  # the last: right, but not on a GPU
    for kw in wrong:
        with pytest.raises(ValueError):
            make(**kw)
    with pytest.raises(TypeError):
        make(dtype=torch.float64)


def test_adamw_object_refuses():
    f, n = torch.zeros, 300
    e8 = lambda k=n: torch.zeros(k).to(torch.float8_e4m3fn)  # noqa: E731
    right = ([f(n)], [f(n)], [f(n)], [f(n)], 0.0)
    for args, kw in [(([], [], [], [], 0.0), {}), ((right[0], right[1] * 2, *right[2:]), {}), (right[:4] + ([0.0, 0.0],), {}),
                     (([f(n).double()], *right[1:]), {}), (([f(n - 1)], *right[1:]), {}), ((*right[:2], [e8()], [e8()], 0.0), {}),
                     ((*right[:2], [e8()], [e8()], 0.0), dict(m_scale=[f(1)], v_scale=[f(2)])), ((*right[:3], [f(2 * n)[::2]], 0.0), {}),
                     ((*right[:2], [e8()], [f(n)], 0.0), dict(m_scale=[f(2)], v_scale=[f(2)])),
                     (right, dict(copy=[f(n + 1).bfloat16()])), (right, dict(copy=[])), (right, {})]:
        with pytest.raises(ValueError):
            block.AdamW(*args, **kw)
    with pytest.raises(TypeError):
        block.AdamW(*right, copy=[f(n)])
    with pytest.raises(TypeError):
        block.AdamW([f(n)], [f(n).double()], [f(n)], [f(n)], 0.0)
