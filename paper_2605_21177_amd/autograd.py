"""Chunk-aware layers for torch autograd (Section 3.1, gradient of the active
slices only; Algorithm 1 line 18, the chunk-aware backward).

`chunk_linear(x, W, seg)` is `x @ W^T` whose backward passes the input gradient
on as usual but never forms the dense weight gradient: it hands the layer's
`X` and `dY` to libchunkft for the active segment `[begin, end)` of `W` only,
either into a gradient buffer (summed over micro-batches, the optimizer step is
then `chunkft_adamw_chunk`) or straight into the fused gradient + AdamW call.
`W` itself does not require grad.  The forward product and the input gradient
are torch's; every step of the chunk path runs in the library's kernels.

`chunk_linear(x, W, seg, bias=..., activation=..., residual=...)` is `act(x W^T + bias) + residual`
with forward, input gradient and bias gradient in the library's kernels as well, and
`chunk_norm(x, w, b, ...)` an RMSNorm or LayerNorm layer.  Their vectors (bias, scale, shift) do not
require grad either: a segment of each says which part is active and where its gradient goes.

Capturing a backward pass into a graph: a leaf that requires grad keeps the stream of its first use, so
an `x` that an eager graph still holds must not be captured on another stream (a limit of torch's
engine); with an `x` that requires no grad nothing of an earlier call is held.
"""

from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


class ChunkSegment:
    """The active chunk's segment on one weight tensor and where its gradient goes.

    Plain mode (`g` given): backward writes the segment's fp32 gradient to `g`
    (`end - begin` elements) on the first micro-batch after `reset()` and adds to
    it on the following ones. A layer's backward that runs out of memory changes and counts
    nothing, one of whose calls is refused counts nothing that comes behind it; what earlier layers or micro-batches have
    added stays: `reset()` and repeat them all.
    Fused mode (`master`, `m`, `v`, `hp` given): backward updates the chunk state
    and the segment of `W` in place (a bf16 `W` receives the rounded master, an fp32
    `W` a copy of it; `master` may also be the segment of an fp32 `W` itself, the
    parameter then being its own master); one micro-batch per step.
    With `hp` from `muon_hparams` (and no `v`) the update is the orthogonalised one, on a segment of
    whole rows of a matrix.
    A segment with `begin == end` (tensor not in the active chunk) makes backward
    skip the weight gradient altogether.
    """

    def __init__(self, begin: int, end: int, g=None, *, master=None, m=None, v=None,
                 hp=None, split_k: int = 0):
        if not 0 <= begin <= end:
            raise ValueError("need 0 <= begin <= end")
        fused = master is not None
        if fused and isinstance(hp, B.MuonHparams):
            if m is None or v is not None:
                raise ValueError("the orthogonalised update needs master, m and hp, and has no v")
        elif fused and (m is None or v is None or hp is None):
            raise ValueError("fused mode needs master, m, v and hp")
        if fused == (g is not None) and end > begin:
            raise ValueError("give either g (plain mode) or master/m/v/hp (fused mode)")
        self.begin, self.end = int(begin), int(end)
        self.g, self.master, self.m, self.v, self.hp = g, master, m, v, hp
        self.split_k = split_k
        self.micro_batches = 0
        self._ws = None

    @property
    def fused(self) -> bool:
        return self.master is not None

    @property
    def active(self) -> bool:
        return self.end > self.begin

    def reset(self) -> None:
        """Start a new optimizer step: the next backward overwrites `g`."""
        self.micro_batches = 0

    def workspace(self, layer: B.Layer):
        need = B.chunkft_workspace_bytes(layer, self.begin, self.end)
        if need == 0:
            return None
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self._ws

    def check_open(self) -> None:
        """Fused mode takes one backward pass per optimizer step."""
        if self.active and self.fused and self.micro_batches:
            raise RuntimeError("fused mode takes one micro-batch per optimizer step")

    def one_more(self) -> None:
        """Counts a backward pass, behind the calls that it made: one that failed leaves the segment as it was, to be repeated."""
        self.micro_batches += 1


def _scratch(need: int, device):
    """Workspace of one call, from the allocator of the current stream."""
    return torch.empty(need, dtype=torch.uint8, device=device) if need else None


def _weight_gradient(seg: ChunkSegment, X, dY, W):
    """The segment's gradient of y = x W^T, to where it goes; X [T, in] and dY [T, out]. What the calls need is allocated here;
    what is returned makes them, and counts them once they are made."""
    out, n_in = W.shape
    seg.check_open()
    layer = B.make_layer(B.LINEAR, X, dY, out, n_in, split_k=seg.split_k)
    ws = seg.workspace(layer)
    muon = seg.fused and isinstance(seg.hp, B.MuonHparams)
    if muon:
        rows = (seg.end - seg.begin) // n_in
        g = torch.empty(seg.end - seg.begin, dtype=torch.float32, device=W.device)
        muon_ws = _scratch(B.chunkft_orthogonalize_workspace_bytes(seg.hp.precision, rows, n_in), W.device)

    def run():
        if muon:
            B.chunkft_chunk_wgrad(layer, seg.begin, seg.end, g, ws=ws)
            B.chunkft_muon_chunk(g, seg.master, seg.m, W.view(-1)[seg.begin:seg.end], rows, n_in, seg.hp,
                                 w_dtype=B._torch_dtype_code(W), ws=muon_ws)
        elif seg.fused:
            # W is what the next forward multiplies with: it always receives the update
            B.chunkft_wgrad_adamw_fused(layer, seg.begin, seg.end, W, seg.master, seg.m, seg.v, seg.hp, ws=ws)
        else:
            B.chunkft_chunk_wgrad(layer, seg.begin, seg.end, seg.g, accumulate=seg.micro_batches > 0, ws=ws)
        seg.one_more()

    return run


class _VectorGrads:
    """Where a layer's call writes the gradients of its vectors' active parts: `g` of a plain segment, or a buffer that the
    update reads afterwards.  A call sets or adds for all of its vectors alike, so where they differ all go through buffers."""

    def __init__(self, pairs, device):
        self.pairs = [(seg, vec) for seg, vec in pairs]
        firsts = {seg.micro_batches == 0 for seg, _ in self.pairs if seg is not None and seg.active and not seg.fused}
        self.accumulate = firsts == {False}
        direct = len(firsts) <= 1 and not (self.accumulate and any(seg is not None and seg.active and seg.fused for seg, _ in self.pairs))
        self.accumulate = self.accumulate and direct
        self.bufs, self.direct = [], direct
        for seg, _ in self.pairs:
            if seg is None or not seg.active:
                self.bufs.append(None)
            elif seg.fused or not direct:
                self.bufs.append(torch.empty(seg.end - seg.begin, dtype=torch.float32, device=device))
            else:
                self.bufs.append(seg.g)

    def span(self, i):
        seg = self.pairs[i][0]
        return None if self.bufs[i] is None else (seg.begin, seg.end)

    def finish(self):
        """Updates, which can be refused, and then what only has to be counted: until then a first micro-batch can be repeated."""
        active = [(seg, vec, buf) for (seg, vec), buf in zip(self.pairs, self.bufs) if buf is not None]
        for seg, vec, buf in active:
            if seg.fused:
                B.chunkft_adamw_chunk(buf, seg.master, seg.m, seg.v, vec[seg.begin:seg.end], seg.end - seg.begin, seg.hp,
                                      w_dtype=B._torch_dtype_code(vec))
                seg.one_more()
        for seg, _, buf in active:
            if not seg.fused:
                if not self.direct:
                    seg.g.add_(buf) if seg.micro_batches else seg.g.copy_(buf)
                seg.one_more()


class _ChunkLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, anchor, seg):
        ctx.save_for_backward(x, W)
        ctx.seg = seg
        return x.matmul(W.t())

    @staticmethod
    def backward(ctx, dy):
        x, W = ctx.saved_tensors
        seg: Optional[ChunkSegment] = ctx.seg
        # the input gradient uses W as it was in the forward pass: enqueue it before any update
        dx = dy.matmul(W) if ctx.needs_input_grad[0] else None
        if seg is not None and seg.active:
            _weight_gradient(seg, _as_rows(x, W.shape[1]), _as_rows(dy, W.shape[0]), W)()
        return dx, None, None, None


class _LinearLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, bias, residual, anchor, seg, bias_seg, activation, keep):
        out, n_in = W.shape
        x2 = _as_rows(x, n_in)
        y = torch.empty(x2.shape[0], out, dtype=W.dtype, device=W.device)
        z = torch.empty_like(y) if keep and activation != B.ACT_NONE else None
        if y.shape[0]:
            layer = B.make_linear(x2, W, bias, activation, None if residual is None else _as_rows(residual, out))
            B.chunkft_linear_forward(layer, y, Z=z, ws=_scratch(B.chunkft_linear_workspace_bytes(layer), W.device))
        ctx.save_for_backward(x2 if seg is not None and seg.active else None, W, bias, z)
        ctx.seg, ctx.bias_seg, ctx.activation, ctx.shape = seg, bias_seg, activation, x.shape
        return y.view(*x.shape[:-1], out)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x2, W, bias, z = ctx.saved_tensors
        _open([ctx.seg, ctx.bias_seg])
        out, n_in = W.shape
        dy2 = _as_rows(dy, out)
        T = dy2.shape[0]
        dx = torch.empty(T, n_in, dtype=W.dtype, device=W.device) if ctx.needs_input_grad[0] else None
        grads = _VectorGrads([(ctx.bias_seg, bias)], W.device)
        dz = torch.empty_like(z) if z is not None else dy2
        weight = _weight_gradient(ctx.seg, x2, dz, W) if T and ctx.seg is not None and ctx.seg.active else None
        if T == 0:
            _no_tokens([ctx.seg, ctx.bias_seg])
        elif z is not None or dx is not None or grads.bufs[0] is not None:
            layer = B.make_linear(None, W, activation=ctx.activation, tokens=T)
            ws = _scratch(B.chunkft_linear_workspace_bytes(layer, backward=True), W.device)
            # the input gradient uses W as it was in the forward pass: it is enqueued before any update
            B.chunkft_linear_backward(layer, dy2, Z=z, dZ=dz if z is not None else None, dX=dx, db=grads.bufs[0], b_range=grads.span(0),
                                      accumulate=grads.accumulate, ws=ws)
        if T:
            if weight is not None:
                weight()
            grads.finish()
        return (None if dx is None else dx.view(ctx.shape), None, None, dy if ctx.needs_input_grad[3] else None, None, None, None,
                None, None)


class _NormLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, anchor, kind, eps, seg, bias_seg, keep):
        x2 = _as_rows(x, x.shape[-1])
        y = torch.empty(x2.shape, dtype=x.dtype, device=x.device)
        stats = torch.empty(x2.shape[0], 2, dtype=torch.float32, device=x.device) if keep else None
        if x2.shape[0]:
            B.chunkft_norm_forward(B.make_norm(kind, x2, w, b, eps), y, stats)
        ctx.save_for_backward(x2, w, b, stats)
        ctx.kind, ctx.eps, ctx.seg, ctx.bias_seg, ctx.shape = kind, eps, seg, bias_seg, x.shape
        return y.view(x.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x2, w, b, stats = ctx.saved_tensors
        _open([ctx.seg, ctx.bias_seg])
        dy2 = _as_rows(dy, x2.shape[1])
        dx = torch.empty(x2.shape, dtype=x2.dtype, device=x2.device) if ctx.needs_input_grad[0] else None
        grads = _VectorGrads([(ctx.seg, w), (ctx.bias_seg, b)], x2.device)
        if x2.shape[0] == 0:
            _no_tokens([ctx.seg, ctx.bias_seg])
        elif dx is not None or any(g is not None for g in grads.bufs):
            layer = B.make_norm(ctx.kind, x2, w, b, ctx.eps)
            ws = _scratch(B.chunkft_norm_workspace_bytes(layer), x2.device) if any(g is not None for g in grads.bufs) else None
            B.chunkft_norm_backward(layer, stats, dy2, dx, dw=grads.bufs[0], w_range=grads.span(0), db=grads.bufs[1],
                                    b_range=grads.span(1), accumulate=grads.accumulate, ws=ws)
            grads.finish()
        return (None if dx is None else dx.view(ctx.shape),) + (None,) * 8


def _as_rows(t, width: int):
    """t as [tokens, width] with unit inner stride and rows that do not overlap (an expanded tensor's do)."""
    t2 = t if t.dim() == 2 else t.reshape(-1, width)
    row, element = t2.stride()
    return t2 if element == 1 and row >= width else t2.clone(memory_format=torch.contiguous_format)


def _open(segs) -> None:
    """Before anything is enqueued: fused segments have not been updated in this step."""
    for seg in segs:
        if seg is not None:
            seg.check_open()


def _no_tokens(segs) -> None:
    """A backward pass over no tokens: the gradients are zero.  The update of a fused segment needs a gradient."""
    for seg in segs:
        if seg is None or not seg.active:
            continue
        if seg.fused:
            raise RuntimeError("a fused segment needs at least one token")
        if seg.micro_batches == 0:
            seg.g.zero_()
        seg.one_more()


def _frozen(t, name: str, n: int, dtype) -> None:
    if t.requires_grad:
        raise ValueError(f"{name} must not require grad: give a segment for its active part")
    if t.shape != (n,) or not t.is_contiguous() or t.dtype is not dtype:
        raise ValueError(f"{name} must be a contiguous vector of {n} elements of the layer's type")


def _inside(seg: Optional[ChunkSegment], n: int) -> None:
    if seg is not None and seg.active and (seg.end > n or isinstance(seg.hp, B.MuonHparams)):
        raise ValueError("the segment must lie in the vector, and a vector has no orthogonalised update")


def _apart(a: Optional[ChunkSegment], b: Optional[ChunkSegment]) -> None:
    if a is not None and a is b and a.active:
        raise ValueError("each tensor needs a segment of its own")


def _anchor_for(x, *segs):
    """A leaf of this call alone that makes autograd run backward where only a segment wants it."""
    if x.requires_grad or not torch.is_grad_enabled() or not any(s is not None and s.active for s in segs):
        return None
    return torch.empty((), device=x.device, requires_grad=True)


_anchor = None


def chunk_linear(x: torch.Tensor, W: torch.Tensor, seg: Optional[ChunkSegment], bias: Optional[torch.Tensor] = None,
                 bias_seg: Optional[ChunkSegment] = None, activation: int = B.ACT_NONE,
                 residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """`act(x @ W^T + bias) + residual` with the chunk-restricted weight gradient in backward.  `W` is
    `[out, in]` row-major on the GPU, bf16 or fp32, and must not require grad; nor must `bias`, a vector
    of `out` elements, whose active part `bias_seg` names.  `activation`: ACT_NONE, ACT_RELU, ACT_GELU
    or ACT_SILU; `residual` has the output's shape and may require grad.  With an activation the input gradient is the product
    of the pre-activation's gradient rounded to W's type.  Without bias, activation and residual the products are torch's."""
    if W.requires_grad:
        raise ValueError("W must not require grad: the dense weight gradient is never formed")
    if not W.is_contiguous():
        raise ValueError("W must be contiguous (the chunk is a range of its flattened elements)")
    if bias is None and bias_seg is not None:
        raise ValueError("a segment of a bias needs the bias")
    if seg is not None and seg.active and isinstance(seg.hp, B.MuonHparams) and (seg.begin % W.shape[1] or seg.end % W.shape[1]):
        raise ValueError("the orthogonalised update takes whole rows")
    if bias is not None or activation != B.ACT_NONE or residual is not None:
        out, n_in = W.shape
        if x.shape[-1] != n_in or x.dtype is not W.dtype:
            raise ValueError("x must be [..., in] of W's type")
        if bias is not None:
            _frozen(bias, "bias", out, W.dtype)
        _inside(bias_seg, out)
        _apart(seg, bias_seg)
        if seg is not None and seg.active and seg.end > W.numel():
            raise ValueError("the segment must lie in W")
        if residual is not None and (residual.shape != x.shape[:-1] + (out,) or residual.dtype is not W.dtype):
            raise ValueError("residual must have the output's shape and type")
        anchor = _anchor_for(x, seg, bias_seg)
        keep = anchor is not None or (x.requires_grad and torch.is_grad_enabled())
        return _LinearLayer.apply(x, W, bias, residual, anchor, seg, bias_seg, activation, keep)
    if x.requires_grad:
        return _ChunkLinear.apply(x, W, None, seg)
    global _anchor
    if _anchor is None or _anchor.device != x.device:
        # makes autograd run backward also for a first layer whose input needs no gradient
        _anchor = torch.zeros((), device=x.device, requires_grad=True)
    return _ChunkLinear.apply(x, W, _anchor, seg)


def chunk_norm(x: torch.Tensor, w: Optional[torch.Tensor], b: Optional[torch.Tensor] = None, kind: int = B.RMSNORM,
               eps: float = 1e-5, seg: Optional[ChunkSegment] = None, bias_seg: Optional[ChunkSegment] = None) -> torch.Tensor:
    """RMSNORM or LAYERNORM over the last dimension of `x`, times `w` plus `b` (either may be None).  The vectors have `x`'s type
    and do not require grad; `seg` and `bias_seg` name their active parts."""
    n = x.shape[-1]
    for vec, vec_seg, name in ((w, seg, "w"), (b, bias_seg, "b")):
        if vec is not None:
            _frozen(vec, name, n, x.dtype)
        elif vec_seg is not None:
            raise ValueError(f"a segment of {name} needs {name}")
        _inside(vec_seg, n)
    _apart(seg, bias_seg)
    anchor = _anchor_for(x, seg, bias_seg)
    keep = anchor is not None or (x.requires_grad and torch.is_grad_enabled())
    return _NormLayer.apply(x, w, b, anchor, kind, eps, seg, bias_seg, keep)
