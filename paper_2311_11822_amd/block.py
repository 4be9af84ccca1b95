"""What stands around the linear layers of a transformer block in a private training step: layer norm, attention, the rotation and
norms of heads, gated feed-forward layers' products and the optimizers.  Each object holds what a program keeps from step to step
(parameters, layouts, workspaces) and checks the tensors that it is given; all arithmetic is the library's."""
from __future__ import annotations

import math
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


SCALINGS = {"none": dp.DP_ROTARY_PLAIN, "linear": dp.DP_ROTARY_LINEAR, "base": dp.DP_ROTARY_BASE, "parts": dp.DP_ROTARY_PARTS}


def rotary_turns(rotary: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original: float = 1.0, slow: float = 1.0,
                 fast: float = 32.0) -> torch.Tensor:
    """Whole turns of each pair of `rotary` columns from one position to the next, [rotary / 2] float64 on the CPU.  scaling, for contexts
    longer than `original` by `factor`: "linear" (all turns slower), "base" (a larger base), "parts" (slower where a pair makes few
    turns within the original context: as they are from `fast` turns on, 1 / factor up to `slow`)."""
    if scaling not in SCALINGS:
        raise ValueError(f"scaling: {', '.join(SCALINGS)}, not {scaling}")
    return torch.from_numpy(dp.dp_rotary_turns(rotary, base, SCALINGS[scaling], factor, original, slow, fast))


class _Heads:
    """The layout of calls on heads, from tensors as they will be given: q and q_out [B, T, H, D], k and k_out [B, T, H_kv, D] or None,
    views of packed projections among them."""

    def __init__(self, q, k, q_out, k_out, turns, interleaved, amplitude, position, length):
        if (k is None) != (k_out is None):
            raise ValueError("k and k_out: both or neither")
        self.tensors = 1 if k is None else 2
        given = (q, q_out) if k is None else (q, k, q_out, k_out)
        self.device, self.index, self.dtype, self.dt = q.device, q.get_device(), q.dtype, _dtype(q)
        if any(t.dim() != 4 for t in given) or (k is not None and (q.shape[:2] != k.shape[:2] or q.shape[3] != k.shape[3])):
            raise ValueError("q: [B, T, H, D], k: [B, T, H_kv, D]")
        B, T, H, D = q.shape
        rotary = 0
        if turns is not None:
            rotary = 2 * turns.numel()
            _same("turns", turns, (turns.numel(),), torch.float64, q.device)
        _same("position", position, (B, T), torch.int32, q.device)
        _same("length", length, (B,), torch.int32, q.device)
        if rotary > D:
            raise ValueError(f"turns: of no more than {D // 2} pairs, not {turns.numel()}")
        self.held = (turns, position, length)             # the shape has their addresses
        self.shapes = (q.shape, None if k is None else k.shape)
        self.in_strides = tuple(t.stride() for t in given[:self.tensors])
        self.out_strides = tuple(t.stride() for t in given[self.tensors:])
        for t in given:
            if D > 1 and t.stride(3) != 1:
                raise ValueError("columns of a head are adjacent")
        three = lambda t: [st if n > 1 else 0 for n, st in zip(t.shape[:3], t.stride()[:3])] if t is not None else (0, 0, 0)  # noqa: E731
        self.shape = dp.heads_shape(B, T, H, 0 if k is None else k.shape[2], D, rotary, interleaved, amplitude, three(q), three(k),
                                    three(q_out), three(k_out), turns, position, length)
        self._check((q, k), self.in_strides)
        self._check((q_out, k_out), self.out_strides)
        # results as gradients would be; what is read may be broadcast (and has no gradients in its own layout then)
        written = dp.heads_shape(B, T, H, 0 if k is None else k.shape[2], D, rotary, interleaved, amplitude, three(q_out), three(k_out),
                                 three(q_out), three(k_out), turns, position, length)
        if dp.dp_head_norm_workspace_bytes(written, self.dt) == 0 or (self.dt != dp.DP_F32 and any(st % 8 for t in (q, k) for st in three(t))):
            raise ValueError("sizes or strides that heads do not have")
        if self.index < 0:
            raise ValueError(f"tensors on a GPU, not {q.device}")

    def _check(self, pair, strides):
        """Queries and keys of the layout's shapes, in these strides (an axis of one entry has whatever stride)."""
        if (pair[1] is None) != (self.tensors == 1):
            raise ValueError("queries and keys" if self.tensors == 2 else "queries alone")
        for t, shape, want in zip(pair, self.shapes, strides):
            if t.shape != shape or t.dtype is not self.dtype or t.get_device() != self.index:
                raise ValueError(f"{tuple(shape)} of {self.dtype} on {self.device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
            if t.stride() != want and any(n > 1 and st != w for n, st, w in zip(shape, t.stride(), want)):
                raise ValueError(f"strides {want}, not {t.stride()}")


class Rotary(_Heads):
    """Position rotation of queries and keys.  turns: of each pair, float64 on the device (rotary_turns); the first 2 * len(turns)
    columns of a head turn, interleaved pairs or halves.  position: [B, T] int32, None: 0, 1, 2 ...; length: [B] int32, rows behind it
    are left as they are.  Turns, positions and lengths are read by every call: a program changes them in place."""

    def __init__(self, q, k, q_out, k_out, turns, interleaved: bool = False, amplitude: float = 1.0, position=None, length=None):
        if turns is None:
            raise ValueError("turns of pairs")
        super().__init__(q, k, q_out, k_out, turns, interleaved, amplitude, position, length)

    def forward(self, q, k, q_out, k_out, stream=None) -> None:
        """q_out may be q and k_out k, where their strides are the same."""
        self._check((q, k), self.in_strides)
        self._check((q_out, k_out), self.out_strides)
        dp.dp_rotary(self.shape, self.dt, q, k, q_out, k_out, stream)

    def backward(self, dq_out, dk_out, dq, dk, stream=None) -> None:
        """dq_out, dk_out in the strides of q_out and k_out; dq, dk in those of q and k."""
        self._check((dq_out, dk_out), self.out_strides)
        self._check((dq, dk), self.in_strides)
        dp.dp_rotary_backward(self.shape, self.dt, dq_out, dk_out, dq, dk, stream)


class HeadNorm(_Heads):
    """Norm of each head, x / sqrt(mean(x^2) + eps) * gain, and the rotation behind it (turns None: none).  Gains: [D] float32, of all
    query heads and of all key heads, or None (ones)."""

    def __init__(self, q, k, q_out, k_out, q_gain=None, k_gain=None, eps: float = 1e-6, turns=None, interleaved: bool = False,
                 amplitude: float = 1.0, position=None, length=None):
        super().__init__(q, k, q_out, k_out, turns, interleaved, amplitude, position, length)
        for name, gain in (("q_gain", q_gain), ("k_gain", k_gain)):
            _same(name, gain, (q.shape[3],), torch.float32, q.device)
        self.gains, self.eps = (q_gain, k_gain), eps
        self.kept_shape = torch.Size((q.shape[0], self.tensors, q.shape[3]))
        self._ws, self._need = _Workspaces(), dp.dp_head_norm_workspace_bytes(self.shape, self.dt)

    def forward(self, q, k, q_out, k_out, stream=None) -> None:
        self._check((q, k), self.in_strides)
        self._check((q_out, k_out), self.out_strides)
        dp.dp_head_norm(self.shape, self.dt, q, k, *self.gains, self.eps, q_out, k_out, stream)

    def backward(self, q, k, dq_out, dk_out, dq, dk, kept=None, sqnorm=None, stream=None) -> None:
        """q, k: what forward was given; kept: [B, 2, D] ([B, 1, D] without keys), per-sample gradients of the gains, and sqnorm: [B], their
        squared norms (LayerNorm.clipped_gradient adds the clipped ones up)."""
        self._check((q, k), self.in_strides)
        self._check((dq_out, dk_out), self.out_strides)
        self._check((dq, dk), self.in_strides)
        _same("kept", kept, self.kept_shape, torch.float32, self.device)
        _same("sqnorm", sqnorm, self.kept_shape[:1], torch.float32, self.device)
        ws = None
        if kept is not None:
            stream = dp._stream(stream)
            ws = self._ws(self._need, self.device, self.index, stream)
        dp.dp_head_norm_backward(self.shape, self.dt, q, k, dq_out, dk_out, *self.gains, self.eps, dq, dk, kept, sqnorm, ws, stream)


ACTIVATIONS = {"silu": dp.DP_ACT_SILU, "gelu": dp.DP_ACT_GELU, "gelu_tanh": dp.DP_ACT_GELU_TANH, "relu": dp.DP_ACT_RELU,
               "sigmoid": dp.DP_ACT_SIGMOID}


class GatedFeedForward:
    """h = act(x w_gate + b_gate) (x w_up + b_up).  w_gate, w_up: [d, f]; biases: [f] or None; w_down: [f, d_out], the projection that reads
    h (its product is the program's own), or None: then the backward pass is given h's gradient.  All of the activations' type."""

    def __init__(self, w_gate, w_up, w_down=None, b_gate=None, b_up=None, activation: str = "silu"):
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation: {', '.join(ACTIVATIONS)}, not {activation}")
        if w_gate.dim() != 2 or (w_down is not None and (w_down.dim() != 2 or w_down.shape[0] != w_gate.shape[1])):
            raise ValueError("w_gate, w_up: [d, f]; w_down: [f, d_out]")
        self.device, self.index, self.dtype, self.dt = w_gate.device, w_gate.get_device(), w_gate.dtype, _dtype(w_gate)
        self.d, self.f = w_gate.shape
        for name, t, shape in (("w_gate", w_gate, w_gate.shape), ("w_up", w_up, w_gate.shape), ("b_gate", b_gate, (self.f,)),
                               ("b_up", b_up, (self.f,)), ("w_down", w_down, None if w_down is None else w_down.shape)):
            _same(name, t, shape, self.dtype, self.device)
        if self.index < 0:
            raise ValueError(f"tensors on a GPU, not {self.device}")
        self.act, self.weights, self.biases, self.w_down = ACTIVATIONS[activation], (w_gate, w_up), (b_gate, b_up), w_down
        self.d_out = self.f if w_down is None else w_down.shape[1]
        self._ws, self._need = _Workspaces(), {}

    def _check(self, *sides) -> int:
        """(width, tensors): [..., width] each, all of the same rows; their number."""
        lead = None
        for width, tensors in sides:
            for t in tensors:
                if t is None:
                    continue
                if lead is None:
                    lead = t.shape[:-1]
                if (t.dim() < 2 or t.shape[:-1] != lead or t.shape[-1] != width or t.dtype is not self.dtype or t.get_device() != self.index or
                        not t.is_contiguous()):
                    raise ValueError(f"contiguous [rows.., {width}] of {self.dtype} on {self.device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        return math.prod(lead)

    def _scratch(self, key, stream, size, *args):
        """The workspace of calls like this one, or None, and their stream."""
        need = self._need.get(key)
        if need is None:
            need = self._need[key] = size(*args)
        if need == 0:
            return None, stream
        stream = dp._stream(stream)
        return self._ws(need, self.device, self.index, stream), stream

    def forward(self, x, h, gate=None, up=None, stream=None) -> None:
        """x: [B, T, d] or [rows, d]; h, and gate and up (kept for backward, or None): [.., f]."""
        rows = self._check((self.d, (x,)), (self.f, (h, gate, up)))
        ws, stream = self._scratch((rows,), stream, dp.dp_gated_workspace_bytes, self.dt, rows, self.d, self.f)
        dp.dp_gated(x, self.dt, rows, self.d, self.f, *self.weights, *self.biases, self.act, gate, up, h, ws, stream)

    def backward(self, dy, gate, up, dgate, dup, dx=None, stream=None) -> None:
        """dy: [.., d_out], or with no w_down h's own gradient [.., f]; dgate, dup: [.., f], output gradients of the two projections (may be gate
        and up); dx: [.., d] or None."""
        rows = self._check((self.d_out, (dy,)), (self.f, (gate, up, dgate, dup)), (self.d, (dx,)))
        ws, stream = self._scratch((rows, "backward"), stream, dp.dp_gated_backward_workspace_bytes, self.dt, rows, self.d, self.f,
                                   0 if self.w_down is None else self.d_out)
        dp.dp_gated_backward(dy, self.w_down, self.d_out, gate, up, self.dt, rows, self.d, self.f, *self.weights, self.act, dgate, dup, dx, ws,
                             stream)


class Muon:
    """Matrices whose update is orthogonalised before it is taken.  param, momentum: [rows, cols] float32; grad: one type; copy: 16-bit tensors that
    take the new parameters, or None; decay: a factor for each matrix, or one for all; scale: likewise, of the update (None: 0.2 times
    the root of the longer side, an AdamW update's size).  The tensors are held: their addresses go to the library."""

    COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5

    def __init__(self, param: Sequence, grad: Sequence, momentum: Sequence, decay, copy: Optional[Sequence] = None, scale=None):
        n = len(param)
        if scale is None:
            scale = [0.2 * math.sqrt(max(p.shape)) if p.dim() == 2 else 0.0 for p in param]
        decay, scale = ([float(x)] * n if isinstance(x, (int, float)) else list(x) for x in (decay, scale))
        if n == 0 or any(len(x) != n for x in (grad, momentum, decay, scale)) or (copy is not None and len(copy) != n):
            raise ValueError("lists of one length, of a matrix at least")
        self.grad_dt = _dtype(grad[0])
        self.copy_dt = _dtype(copy[0]) if copy is not None else dp.DP_F32
        if copy is not None and self.copy_dt == dp.DP_F32:
            raise TypeError("copy: 16-bit tensors")
        self.device, self.index = param[0].device, param[0].get_device()
        self.held = list(zip(param, grad, momentum, copy if copy is not None else [None] * n))
        kinds = (torch.float32, grad[0].dtype, torch.float32, copy[0].dtype if copy is not None else None)
        for tensors in self.held:
            if tensors[0].dim() != 2:
                raise ValueError(f"param: matrices, not {tuple(tensors[0].shape)}")
            for name, t, kind in zip(("param", "grad", "momentum", "copy"), tensors, kinds):
                _same(name, t, tensors[0].shape, kind, self.device)
        written = [t.data_ptr() for tensors in self.held for t in (tensors[0], *tensors[2:]) if t is not None]
        if len(set(written)) < len(written):
            raise ValueError("param, momentum, copy: a tensor twice")
        if self.index < 0:
            raise ValueError(f"tensors on a GPU, not {self.device}")
        self.tensors = dp.muon_tensors([(*t, *t[0].shape, d, x) for t, d, x in zip(self.held, decay, scale)])
        self._ws, self._need = _Workspaces(), dp.dp_muon_workspace_bytes(self.tensors)
        if self._need == 0:
            raise ValueError("sizes that the library does not take")

    def step(self, lr: float, beta: float = 0.95, nesterov: bool = True, grad_scale: float = 1.0, coefficients=COEFFICIENTS, eps: float = 1e-7,
             stream=None) -> None:
        """grad_scale: what makes the gradient's sum over samples a mean; coefficients: (a, b, c) of each iteration X <- a X + b A X + c A^2 X."""
        stream = dp._stream(stream)
        ws = self._ws(self._need, self.device, self.index, stream)
        dp.dp_muon_multi(self.tensors, self.grad_dt, self.copy_dt, lr, beta, nesterov, grad_scale, eps, coefficients, ws, stream)
