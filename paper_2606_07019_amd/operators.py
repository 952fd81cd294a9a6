"""The operators at the ends of a collective, on torch tensors.

Argument marshalling over the C ABI (include/pccl.h, "operators at the ends of
a collective"): shapes and types are checked here, the rest by the library,
and every step runs in its HIP kernels.  Calls are queued on the current
stream of the device; outputs and workspaces come from torch's allocator, so
calls on different streams do not share any.  Threads may share an Operators:
their calls take turns.

Of torch's automatic differentiation, route()'s weights carry the router's
gradient.  Packed values are whole numbers and have none: a training step makes
its three products itself, of operands packed along the axis that each sums
over.  moe_layer() is for serving; asked for a gradient, its result raises.

    ops = Operators()
    q = ops.quantize(x)                          # rows in 4.25 bits a value
    y = ops.matmul(q, w, torch.bfloat16)         # q w^T
    weights, ids, counts, order = ops.route(logits, 8)
    y = ops.moe_layer(x, router, up, down, 8)
"""

from __future__ import annotations

import threading
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from paper_2606_07019_amd import pccl as P

_DTYPE = {torch.float32: P.PCCL_F32, torch.bfloat16: P.PCCL_BF16, torch.float16: P.PCCL_F16}


class MX(NamedTuple):
    """Packed rows: codes [..., rows, ceil(cols / 128) * 64] and scales
    [..., rows, ceil(cols / 128) * 4] (uint8), and the rows' length."""
    codes: torch.Tensor
    scales: torch.Tensor
    cols: int


def mx_bytes(cols: int):
    """(code bytes, scale bytes) of one packed row of `cols` values."""
    steps = -(-cols // 128)
    return steps * 64, steps * 4


def _learns(*tensors):
    """Whether a derivative is recorded for one of the tensors; RuntimeError for a forward-mode one, which none has here."""
    if forward_ad._current_level >= 0 and any(forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise RuntimeError("the operators have no forward-mode derivatives")
    for t in tensors:
        if t.requires_grad:
            return torch.is_grad_enabled()
    return False


class _Route(torch.autograd.Function):
    """route() with its gradient."""

    @staticmethod
    def forward(ctx, logits, ops, topk, normalize, mask):
        weights, ids, counts, order = ops._route(logits, topk, normalize, mask)
        ctx.mark_non_differentiable(ids, counts, order)
        # normalised weights' gradient does not read the logits
        ctx.save_for_backward(None if normalize else logits, weights, ids, mask)
        ctx.rest = ops, logits.shape, logits.dtype, normalize
        return weights, ids, counts, order

    @staticmethod
    @once_differentiable
    def backward(ctx, dweights, *_):
        ops, shape, dtype, normalize = ctx.rest
        logits, weights, ids, mask = ctx.saved_tensors
        return ops._route_backward(logits, shape, dtype, weights, ids, dweights.contiguous(), normalize, mask), None, None, None, None


class _Served(torch.autograd.Function):
    """A result without a gradient, for inputs that a gradient is asked of."""

    @staticmethod
    def forward(ctx, name, call, *inputs):
        ctx.name = name
        return call(*inputs)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{ctx.name} has no gradient")


class Operators:
    """A context for the operators on one device.

    The smallest calls take a few microseconds on the GPU, so the way there is
    kept short: the library's functions are called as they are, sizes of
    workspaces are asked for once per shape, and the current stream's address
    is taken without building a torch.cuda.Stream."""

    def __init__(self, device: int = 0):
        self.device = torch.device("cuda", device)
        self._index = device
        self.h = None
        self._lock = threading.Lock()   # a context takes one call at a time, its message included
        self._lib = P.load_library()
        self._spaces = {}
        try:
            with torch.cuda.device(self.device):   # making and closing a context leave it the current one
                self.h = P.pccl_create(device, 0)
        except P.PcclError:
            raise
        except RuntimeError as e:
            raise P.PcclError(5, f"cannot create a context on HIP device {device}") from e

    # -- checks ------------------------------------------------------------

    def _matrix(self, name, x, types=_DTYPE):
        if x.dim() != 2 or x.device != self.device or x.dtype not in types:
            raise ValueError(f"{name}: a matrix of {', '.join(str(t) for t in types)} on {self.device} is needed, "
                             f"got {tuple(x.shape)} {x.dtype} on {x.device}")
        rows, cols = x.shape
        if x.is_contiguous():
            return rows, cols, cols
        if rows == 0 or cols == 0:
            return rows, cols, cols
        if cols > 1 and x.stride(1) != 1:
            raise ValueError(f"{name}: rows must be contiguous (strides {x.stride()})")
        return rows, cols, (x.stride(0) if rows > 1 else cols)

    def _same(self, name, x, shape, dtype):
        if x.shape != shape or x.dtype != dtype or x.device != self.device or not x.is_contiguous():
            raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {shape} on {self.device} is needed, got "
                             f"{tuple(x.shape)} {x.dtype} on {x.device}")
        return x.data_ptr()

    def _packed(self, name, q: MX, lead):
        cb, sb = mx_bytes(q.cols)
        return (self._same(name + " codes", q.codes, (*lead, cb), torch.uint8),
                self._same(name + " scales", q.scales, (*lead, sb), torch.uint8))

    def _mask(self, mask, tokens):
        if mask is None:
            return None
        if mask.dtype == torch.bool:
            mask = mask.view(torch.uint8)
        return self._same("mask", mask, (tokens,), torch.uint8)

    def _type(self, dtype):
        if dtype not in _DTYPE:
            raise ValueError(f"one of {', '.join(str(t) for t in _DTYPE)} is needed, got {dtype}")
        return _DTYPE[dtype]

    def _stream(self):
        return torch._C._cuda_getCurrentRawStream(self._index) or None

    def _empty(self, dtype, *shape):
        return torch.empty(*shape, dtype=dtype, device=self.device)

    def _call(self, function, *args):
        with self._lock:
            status = function(self.h, *args)
            if status:
                P._check(self.h, status)

    def _space(self, ask, *sizes):
        """(workspace, its address, its size) of the call that `ask` gives the size for."""
        nbytes = self._spaces.get((ask, sizes))
        if nbytes is None:
            if len(self._spaces) >= 4096:   # a caller whose sizes keep changing
                self._spaces.clear()
            with self._lock:
                nbytes = self._spaces[ask, sizes] = ask(self.h, *sizes)
        if not nbytes:
            return None, None, 0
        ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return ws, ws.data_ptr(), nbytes

    # -- microscaled 4-bit values --------------------------------------------

    def _pack(self, x, rows_too, cols_too):
        rows, cols, ld = self._matrix("x", x)
        r = c = rc = rs = cc = cs = None
        if rows_too:
            cb, sb = mx_bytes(cols)
            r = MX(self._empty(torch.uint8, rows, cb), self._empty(torch.uint8, rows, sb), cols)
            rc, rs = r.codes.data_ptr(), r.scales.data_ptr()
        if cols_too:
            cb, sb = mx_bytes(rows)
            c = MX(self._empty(torch.uint8, cols, cb), self._empty(torch.uint8, cols, sb), rows)
            cc, cs = c.codes.data_ptr(), c.scales.data_ptr()
        self._call(self._lib.pccl_mx_quantize, x.data_ptr(), _DTYPE[x.dtype], rows, cols, ld, rc, rs, cc, cs, self._stream())
        return r, c

    def quantize(self, x) -> MX:
        """x's rows, packed."""
        return self._pack(x, True, False)[0]

    def quantize_columns(self, x) -> MX:
        """x's columns, packed (the rows of its transpose)."""
        return self._pack(x, False, True)[1]

    def quantize_both(self, x):
        """(x's rows, x's columns), packed in one pass over x."""
        return self._pack(x, True, True)

    def dequantize(self, q: MX, dtype) -> torch.Tensor:
        """The values that q stands for."""
        kind = self._type(dtype)
        rows = q.codes.shape[0]
        codes, scales = self._packed("q", q, (rows,))
        out = self._empty(dtype, rows, q.cols)
        self._call(self._lib.pccl_mx_dequantize, codes, scales, rows, q.cols, out.data_ptr(), kind, q.cols, self._stream())
        return out

    def matmul(self, a: MX, b: MX, dtype, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """a b^T: [rows of a, rows of b]."""
        kind = self._type(dtype)
        if a.cols != b.cols:
            raise ValueError(f"a has rows of {a.cols} values, b of {b.cols}")
        m, n, k = a.codes.shape[0], b.codes.shape[0], a.cols
        ac, as_ = self._packed("a", a, (m,))
        bc, bs = self._packed("b", b, (n,))
        if out is None:
            out, ld = self._empty(dtype, m, n), n
        else:
            rows, cols, ld = self._matrix("out", out)
            if (rows, cols) != (m, n) or out.dtype != dtype:
                raise ValueError(f"out: {(m, n)} of {dtype} is needed, got {(rows, cols)} of {out.dtype}")
            if _learns(out):
                raise ValueError("out: a tensor that requires grad is not written")
            if not out.is_inference():
                torch.autograd.graph.increment_version(out)
        ws, wp, nbytes = self._space(P.pccl_mx_matmul_workspace, m, n, k)
        self._call(self._lib.pccl_mx_matmul, ac, as_, bc, bs, m, n, k, out.data_ptr(), kind, ld, wp, nbytes, self._stream())
        return out

    # -- router ----------------------------------------------------------------

    def route(self, logits, topk: int, normalize: bool = True, mask: Optional[torch.Tensor] = None):
        """(weights, ids, counts, order) of the topk largest logits of every row; the weights carry the gradient."""
        if _learns(logits):
            return _Route.apply(logits, self, topk, normalize, mask)
        return self._route(logits, topk, normalize, mask)

    def _route(self, logits, topk, normalize, mask):
        tokens, experts, ld = self._matrix("logits", logits)
        mp = None if mask is None else self._mask(mask, tokens)
        ws, wp, nbytes = self._space(P.pccl_moe_route_workspace, tokens, experts, topk)
        weights = self._empty(torch.float32, tokens, topk)
        ids = self._empty(torch.int32, tokens, topk)
        counts = self._empty(torch.int32, experts)
        order = self._empty(torch.int32, tokens * topk)
        self._call(self._lib.pccl_moe_route, logits.data_ptr(), _DTYPE[logits.dtype], tokens, experts, ld, topk, normalize, mp,
                   weights.data_ptr(), ids.data_ptr(), counts.data_ptr(), order.data_ptr(), wp, nbytes, self._stream())
        return weights, ids, counts, order

    def route_backward(self, logits, weights, ids, dweights, normalize: bool = True,
                       mask: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The gradient of route()'s weights with respect to its logits, in their type."""
        return self._route_backward(logits, logits.shape, logits.dtype, weights, ids, dweights, normalize, mask)

    def _route_backward(self, logits, shape, dtype, weights, ids, dweights, normalize, mask):
        if logits is None:
            (tokens, experts), ld, address = shape, shape[1], None
        else:
            tokens, experts, ld = self._matrix("logits", logits)
            address = logits.data_ptr()
        topk = weights.shape[1] if weights.dim() == 2 else 0
        shape = (tokens, topk)
        out = self._empty(dtype, tokens, experts)
        self._call(
            self._lib.pccl_moe_route_backward, address, _DTYPE[dtype], tokens, experts, ld, topk, normalize,
            None if mask is None else self._mask(mask, tokens), self._same("weights", weights, shape, torch.float32),
            self._same("ids", ids, shape, torch.int32), self._same("dweights", dweights, shape, torch.float32),
            out.data_ptr(), experts, self._stream())
        return out

    # -- mixture-of-experts layer ------------------------------------------------

    def moe_layer(self, x, router, up, down, topk: int, normalize: bool = True,
                  mask: Optional[torch.Tensor] = None) -> torch.Tensor:
        """y [tokens, hidden] for x [tokens, hidden], router [experts, hidden],
        up [experts, 2 inter, hidden] (gate rows first) and down [experts,
        hidden, inter], the latter two of x's type or packed (MX)."""
        tensors = (x, router) if isinstance(up, MX) or isinstance(down, MX) else (x, router, up, down)
        if _learns(*tensors):
            return _Served.apply("moe_layer", lambda x, router, up, down: self._moe_layer(x, router, up, down, topk, normalize, mask),
                                 x, router, up, down)
        return self._moe_layer(x, router, up, down, topk, normalize, mask)

    def _moe_layer(self, x, router, up, down, topk, normalize, mask):
        dtype = x.dtype
        tokens, hidden, ld = self._matrix("x", x, (torch.bfloat16, torch.float16))
        experts = router.shape[0]
        rp = self._same("router", router, (experts, hidden), dtype)
        if isinstance(up, MX) != isinstance(down, MX):
            raise ValueError("either both or neither of up and down are packed")
        if isinstance(up, MX):
            inter = down.cols
            if up.cols != hidden:
                raise ValueError(f"up: rows of {hidden} values are needed, got {up.cols}")
            upp, ups = self._packed("up", up, (experts, 2 * inter))
            dp, ds = self._packed("down", down, (experts, hidden))
        else:
            inter = down.shape[-1]
            upp, ups = self._same("up", up, (experts, 2 * inter, hidden), dtype), None
            dp, ds = self._same("down", down, (experts, hidden, inter), dtype), None
        ws, wp, nbytes = self._space(P.pccl_moe_layer_workspace, tokens, experts, topk, hidden, inter)
        y = self._empty(dtype, tokens, hidden)
        self._call(
            self._lib.pccl_moe_layer, x.data_ptr(), _DTYPE[dtype], ld, tokens, experts, topk, hidden, inter, normalize,
            None if mask is None else self._mask(mask, tokens), rp, upp, ups, dp, ds, y.data_ptr(), hidden, wp, nbytes,
            self._stream())
        return y

    def close(self):
        with self._lock:
            h, self.h = self.h, None
            if h is not None:
                with torch.cuda.device(self.device):
                    P.pccl_destroy(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
