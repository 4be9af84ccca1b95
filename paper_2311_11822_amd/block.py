"""What stands around the linear layers of a transformer block in a private training step: layer norm, attention and the
optimizer.  Each object holds what a program keeps from step to step (parameters, layouts, workspaces) and checks the
tensors that it is given; all arithmetic is the library's."""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as dp

_TYPES = {torch.float32: dp.DP_F32, torch.bfloat16: dp.DP_BF16, torch.float16: dp.DP_F16}


def _dtype(x: torch.Tensor) -> int:
    if x.dtype not in _TYPES:
        raise TypeError(f"float32, bfloat16 or float16, not {x.dtype}")
    return _TYPES[x.dtype]


def _same(name: str, x: Optional[torch.Tensor], shape, dtype, device) -> None:
    if x is not None and (tuple(x.shape) != tuple(shape) or x.dtype != dtype or x.device != device or not x.is_contiguous()):
        raise ValueError(f"{name}: contiguous {tuple(shape)} of {dtype} on {device}, not {tuple(x.shape)} of {x.dtype} on {x.device}")


class _Workspaces:
    """Scratch memory, one for each device and stream (calls on different streams do not share one) that grows as calls need.  What it has
    outgrown stays as long as the object (a captured graph may have its address); by halves at least, so all of it is bounded.

    A graph that torch captures has its own, from the graph's pool: it may be replayed on any stream, beside other graphs of the same object
    and calls that are not captured.  (A capture by other means has the stream's; its replays keep that stream's order.)"""

    def __init__(self):
        self.held, self.outgrown = {}, []

    def __call__(self, nbytes: int, device: torch.device, index: int, stream: int) -> torch.Tensor:
        ws = self.held.get((index, stream))
        capturing = torch.cuda.is_current_stream_capturing()
        if ws is None or ws.numel() < nbytes or capturing:
            # of that stream's own memory: what comes from another's may still be in use there
            current = torch.cuda.current_stream(device)
            own = (current if current.cuda_stream == stream else torch.cuda.ExternalStream(stream, device) if stream
                   else torch.cuda.default_stream(device))          # (an external stream of handle 0 would be a new one)
            with torch.cuda.stream(own):
                if capturing:
                    fresh = torch.empty(nbytes, dtype=torch.uint8, device=device)
                    if _of_a_graph(fresh):
                        return fresh                      # the pool's as long as the graph
                if ws is None or ws.numel() < nbytes:
                    if ws is not None:
                        self.outgrown.append(ws)
                        nbytes = max(nbytes, ws.numel() * 3 // 2)
                    ws = self.held[index, stream] = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return ws


def _of_a_graph(x: torch.Tensor) -> bool:
    """Whether x lies in the memory pool of a graph that is captured (looked up in the allocator's whole list: for captures alone)."""
    at = x.data_ptr()
    return any(s["address"] <= at < s["address"] + s["total_size"] and tuple(s["segment_pool_id"]) != (0, 0)
               for s in torch.cuda.memory_snapshot())


class LayerNorm:
    """gain, bias: [d] float32, or None (ones, zeros)."""

    def __init__(self, gain: Optional[torch.Tensor], bias: Optional[torch.Tensor], eps: float = 1e-5):
        self.gain, self.bias, self.eps = gain, bias, eps
        self._ws, self._need = _Workspaces(), {}

    def _check(self, x, like, rows, floats):
        """Tensors of x's shape and type, [B, T] float32 ones, and others by (tensor, number of values); written out, for a call of a
        few microseconds."""
        shape, dtype, device = x.shape, x.dtype, x.get_device()
        if len(shape) != 3 or not x.is_contiguous():
            raise ValueError("x: contiguous [B, T, d]")
        B, T, d = shape
        for t in like:
            if t is not None and (t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous()):
                raise ValueError(f"contiguous {tuple(shape)} of {dtype} on {x.device}, as x, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        for t in rows:
            if t is not None and (t.numel() != B * T or t.dtype is not torch.float32 or t.get_device() != device or not t.is_contiguous()):
                raise ValueError(f"mean, rstd: {B} x {T} contiguous float32 values on {x.device}")
        for t, n in floats:
            if t is not None and (t.numel() != n or t.dtype is not torch.float32 or t.get_device() != device or not t.is_contiguous()):
                raise ValueError(f"{n} contiguous float32 values on {x.device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        if device < 0:
            raise ValueError(f"tensors on a GPU, not {x.device}")
        return _dtype(x), B, T, d

    def forward(self, x, y, mean=None, rstd=None, add=None, sum=None, stream=None) -> None:
        """x, y: [B, T, d]; mean, rstd: [B, T], kept for backward; add: joins x before the norm, the sum goes to `sum`."""
        d = x.shape[-1]
        dt, B, T, d = self._check(x, (y, add, sum), (mean, rstd), ((self.gain, d), (self.bias, d)))
        dp.dp_layer_norm(x, add, dt, B, T, d, self.gain, self.bias, self.eps, sum, y, mean, rstd, stream)

    def backward(self, x, dy, mean, rstd, dx, kept=None, sqnorm=None, add=None, stream=None) -> None:
        """dx: [B, T, d] or None; kept: [B, 2, d], per-sample gradients of gain and bias, and sqnorm: [B], their squared norms;
        add: the gradient that reaches x beside the norm."""
        B, T, d = x.shape
        dt, B, T, d = self._check(x, (dy, dx, add), (mean, rstd), ((self.gain, d), (kept, 2 * B * d), (sqnorm, B)))
        ws = None
        if kept is not None:
            stream = dp._stream(stream)
            need = self._need.get((dt, B, T, d))
            if need is None:
                need = self._need[dt, B, T, d] = dp.dp_layer_norm_workspace_bytes(dt, B, T, d)
                if need == 0:
                    raise dp.DpError(dp.DP_ERR_UNSUPPORTED, "dp_layer_norm_workspace_bytes")
            ws = self._ws(need, x.device, x.get_device(), stream)
        dp.dp_layer_norm_backward(x, dy, add, dt, B, T, d, self.gain, mean, rstd, dx, kept, sqnorm, ws, stream)

    @staticmethod
    def clipped_gradient(kept, C, grad, accumulate=0, stream=None) -> None:
        """grad: [2, d] float32, gain's and bias's, (+)= sum_i C[i] kept[i]."""
        _same("grad", grad, kept.shape[1:], torch.float32, kept.device)
        dp.dp_clipped_bias_grad(kept, kept.shape[0], kept[0].numel(), C, grad, accumulate, stream)


class Attention:
    """The layout of attention calls, from tensors as they will be given: q [B, Tq, H, D], k and v [B, Tk, H_kv, D], o [B, Tq, H, D],
    views of packed projections among them.  q_len, k_len: [B] int32 on the device, or None."""

    def __init__(self, q, k, v, o, causal: bool, scale: float, q_len=None, k_len=None):
        self.device, self.index, self.dtype, self.dt = q.device, q.get_device(), q.dtype, _dtype(q)
        if any(t.dim() != 4 for t in (q, k, v, o)) or q.shape != o.shape or k.shape != v.shape or q.shape[::3] != k.shape[::3]:
            raise ValueError("q and o: [B, Tq, H, D], k and v: [B, Tk, H_kv, D]")
        B, Tq, H, D = q.shape
        Tk, H_kv = k.shape[1:3]
        for name, n in (("q_len", q_len), ("k_len", k_len)):
            _same(name, n, (B,), torch.int32, q.device)
        self.q_len, self.k_len = q_len, k_len             # held: the shape has their addresses
        self.q_shape, self.k_shape, self.rows = q.shape, k.shape, torch.Size((B, H, Tq))
        self.strides = tuple(t.stride() for t in (q, k, v, o))
        for t in (q, k, v, o):
            if D > 1 and t.stride(3) != 1:
                raise ValueError("columns of a head are adjacent")
        # an axis of one entry has whatever stride; none is needed of it
        strides = [[st if n > 1 else 0 for n, st in zip(t.shape[:3], t.stride()[:3])] for t in (q, k, v, o)]
        self.shape = dp.attention_shape(B, H, H_kv, Tq, Tk, D, causal, scale, *strides, q_len, k_len)
        self._check((q, o), (k, v), (q, k, v, o), None)
        self._ws, self._need = _Workspaces(), dp.dp_attention_backward_workspace_bytes(self.shape, self.dt)
        self._forward_need = dp.dp_attention_workspace_bytes(self.shape, self.dt)
        if self._need == 0:
            raise ValueError("sizes, strides or scale that attention does not take")
        if self.index < 0:
            raise ValueError(f"tensors on a GPU, not {q.device}")

    def _check(self, of_queries, of_keys, four, lse):
        """of_queries, of_keys: by shape and type; four: in the strides of q, k, v and o."""
        dtype, index = self.dtype, self.index
        for shape, tensors in ((self.q_shape, of_queries), (self.k_shape, of_keys)):
            for t in tensors:
                if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
                    raise ValueError(f"{tuple(shape)} of {dtype} on {self.device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        for t, strides in zip(four, self.strides):
            if t.stride() != strides and any(n > 1 and st != want for n, st, want in zip(t.shape, t.stride(), strides)):
                raise ValueError(f"strides {strides}, not {t.stride()}")
        if lse is not None and (lse.shape != self.rows or lse.dtype is not torch.float32 or lse.get_device() != index or
                                not lse.is_contiguous()):
            raise ValueError(f"lse: contiguous {tuple(self.rows)} of float32 on {self.device}")

    def forward(self, q, k, v, o, lse, stream=None) -> None:
        """o in its strides; lse: [B, H, Tq] float32, kept for backward."""
        self._check((q, o), (k, v), (q, k, v, o), lse)
        ws = None
        if self._forward_need:
            stream = dp._stream(stream)
            ws = self._ws(self._forward_need, self.device, self.index, stream)
        dp.dp_attention(self.shape, self.dt, q, k, v, o, lse, ws, stream)

    def backward(self, q, k, v, o, lse, do, dq, dk, dv, stream=None) -> None:
        """do in o's strides; dq, dk, dv in those of q, k and v."""
        self._check((q, o, do, dq), (k, v, dk, dv), (q, k, v, o), lse)
        self._check((), (), (dq, dk, dv, do), None)
        stream = dp._stream(stream)
        ws = self._ws(self._need, self.device, self.index, stream)
        dp.dp_attention_backward(self.shape, self.dt, q, k, v, o, lse, do, dq, dk, dv, ws, stream)


class AdamW:
    """Lists of tensors that are updated together.  param: float32; grad: one type; m, v: float32, or torch.float8_e4m3fn with m_scale and
    v_scale ([ceil(n / 256)] float32; v then holds roots); copy: 16-bit tensors that take the new parameters, or None; decay: a
    factor for each tensor, or one for all.  The tensors are held: their addresses go to the library."""

    def __init__(self, param: Sequence, grad: Sequence, m: Sequence, v: Sequence, decay, copy: Optional[Sequence] = None,
                 m_scale: Optional[Sequence] = None, v_scale: Optional[Sequence] = None):
        n = len(param)
        decay = [float(decay)] * n if isinstance(decay, (int, float)) else list(decay)
        if n == 0 or any(len(x) != n for x in (grad, m, v, decay)) or any(x is not None and len(x) != n for x in (copy, m_scale, v_scale)):
            raise ValueError("lists of one length, of a tensor at least")
        self.bits = 8 if m[0].dtype == torch.float8_e4m3fn else 32
        if self.bits == 8 and (m_scale is None or v_scale is None):
            raise ValueError("8-bit states have scales")
        state = torch.float8_e4m3fn if self.bits == 8 else torch.float32
        self.grad_dt = _dtype(grad[0])
        self.copy_dt = _dtype(copy[0]) if copy is not None else dp.DP_F32
        if copy is not None and self.copy_dt == dp.DP_F32:
            raise TypeError("copy: 16-bit tensors")
        device = param[0].device
        none = [None] * n
        self.held = list(zip(param, grad, m, v, m_scale if self.bits == 8 else none, v_scale if self.bits == 8 else none,
                             copy if copy is not None else none))
        kinds = (torch.float32, grad[0].dtype, state, state, torch.float32, torch.float32, copy[0].dtype if copy is not None else None)
        for tensors in self.held:
            size = tensors[0].numel()
            for k, (name, t, kind) in enumerate(zip(("param", "grad", "m", "v", "m_scale", "v_scale", "copy"), tensors, kinds)):
                want = -(-size // 256) if k in (4, 5) else size
                if t is not None and (t.dtype != kind or t.device != device or t.numel() != want or not t.is_contiguous()):
                    raise ValueError(f"{name}: contiguous, {want} values of {kind} on {device}")
        if device.type != "cuda":
            raise ValueError(f"tensors on a GPU, not {device}")
        self.tensors = dp.adamw_tensors([(*tensors, tensors[0].numel(), d) for tensors, d in zip(self.held, decay)])

    def step(self, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, grad_scale: float = 1.0,
             stream=None) -> None:
        """step counts from 1; grad_scale: what makes the gradient's sum over samples a mean."""
        dp.dp_adamw_multi(self.tensors, self.grad_dt, self.bits, self.copy_dt, lr, beta1, beta2, eps, grad_scale, step, stream)
