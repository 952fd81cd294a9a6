"""The operators at the ends of a collective, on torch tensors.

Argument marshalling over the C ABI (include/pccl.h, "operators at the ends of
a collective"): shapes and types are checked here, the rest by the library,
and every step runs in its HIP kernels.  Calls are queued on the current
stream of the device; outputs and workspaces come from torch's allocator, so
calls on different streams do not share any.  Threads may share an Operators:
their calls take turns.

Of torch's automatic differentiation, route()'s weights carry the router's
gradient, and balance_loss()'s loss and probabilities theirs.  Packed values are
whole numbers and have none: a training step makes its three products itself, of
operands packed along the axis that each sums over.  moe_layer() is for serving;
asked for a gradient, its result raises, as those of route_backward() and
balance_loss_backward() do.

    ops = Operators()
    q = ops.quantize(x)                          # rows in 4.25 bits a value
    y = ops.matmul(q, w, torch.bfloat16)         # q w^T
    weights, ids, counts, order = ops.route(logits, 8)
    y = ops.moe_layer(x, router, up, down, 8)

In 8 bits, with the experts' products over rows in the router's order:

    loss, counts, probs, rows = ops.balance_loss(logits, ids)
    groups = ops.expert_groups(counts, tokens * 8)
    x_rows, x_cols = ops.quantize8_both(x[order // 8], groups)
    w_rows, w_cols = ops.quantize8_tiles(w)      # [experts, n, k]: the same values either way round
    y = ops.expert_matmul8(x_rows, w_rows, groups, torch.bfloat16)
    dx = ops.expert_matmul8(dy_rows, w_cols, groups, torch.bfloat16)
    dw = ops.expert_gradient8(dy_cols, x_cols, groups, torch.float32)
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


class F8(NamedTuple):
    """Packed rows of 8-bit values: codes [..., rows, ceil(cols / 128) * 128] and
    scales [..., rows, ceil(cols / 512) * 4] (uint8), and the rows' length."""
    codes: torch.Tensor
    scales: torch.Tensor
    cols: int


def f8_bytes(cols: int):
    """(code bytes, scale bytes) of one row of `cols` 8-bit values."""
    return -(-cols // 128) * 128, -(-cols // 512) * 4


class Groups(NamedTuple):
    """The blocks of rows in expert order (expert_groups()): the table on the
    device, the number of experts and the number of rows there is room for."""
    table: torch.Tensor
    experts: int
    rows: int


def group_blocks(experts: int, rows: int, block: int = 128):
    """The most blocks of one expert's rows that so many rows can have."""
    return rows // block + min(experts, rows)


def _group_words(experts, rows):
    return experts + 2 + 2 * group_blocks(experts, rows) + 2 * group_blocks(experts, rows, 256)


def _learns(*tensors):
    """Whether a derivative is recorded for one of the tensors (or None); RuntimeError for a forward-mode one, which none has here."""
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise RuntimeError("the operators have no forward-mode derivatives")
    for t in tensors:
        if t is not None and t.requires_grad:
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


class _Balance(torch.autograd.Function):
    """balance_loss() with its gradient."""

    @staticmethod
    def forward(ctx, logits, ops, ids, mask):
        loss, counts, probs, rows = ops._balance(logits, ids, mask)
        ctx.mark_non_differentiable(counts, rows)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, counts, rows, mask)
        ctx.ops = ops
        return loss, counts, probs, rows

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss, _, dprobs, __):
        logits, counts, rows, mask = ctx.saved_tensors
        if dloss is None and dprobs is None:
            return None, None, None, None
        if dprobs is not None:
            dprobs = dprobs.contiguous()
        return ctx.ops._balance_backward(logits, dloss, dprobs, counts, rows, mask), None, None, None


class _Served(torch.autograd.Function):
    """A result without a gradient, for inputs that one is recorded for: silence would end their graph."""

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

    def _packed8(self, name, q: F8, lead):
        cb, sb = f8_bytes(q.cols)
        return (self._same(name + " codes", q.codes, (*lead, cb), torch.uint8),
                self._same(name + " scales", q.scales, (*lead, sb), torch.uint8))

    def _blocks(self, groups: Groups):
        _, experts, rows = groups
        return self._same("groups", groups.table, (_group_words(experts, rows),), torch.int32)

    def _result(self, out, rows, cols, dtype):
        """(out, its row stride): what a product is written to, made here or given by the caller."""
        if out is None:
            return self._empty(dtype, rows, cols), cols
        m, n, ld = self._matrix("out", out)
        if (m, n) != (rows, cols) or out.dtype != dtype:
            raise ValueError(f"out: {(rows, cols)} of {dtype} is needed, got {(m, n)} of {out.dtype}")
        if _learns(out):
            raise ValueError("out: a tensor that requires grad is not written")
        if not out.is_inference():
            torch.autograd.graph.increment_version(out)
        return out, ld

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
        return torch.empty(shape, dtype=dtype, device=self.device)

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
        out, ld = self._result(out, m, n, dtype)
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
        if _learns(logits, weights, dweights):
            return _Served.apply("route_backward", lambda l, w, d: self._route_backward(l, l.shape, l.dtype, w, ids, d, normalize, mask),
                                 logits, weights, dweights)
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

    def balance_loss(self, logits, ids, mask: Optional[torch.Tensor] = None):
        """(loss, counts, probs, rows) of a router's logits and picks: the balance
        loss, the picks and the mean probability of every expert, and the number
        of rows with an expert left.  The loss and probs carry the gradient."""
        if _learns(logits):
            return _Balance.apply(logits, self, ids, mask)
        return self._balance(logits, ids, mask)

    def _balance(self, logits, ids, mask):
        tokens, experts, ld = self._matrix("logits", logits)
        topk = ids.shape[1] if ids.dim() == 2 else 0
        ip = self._same("ids", ids, (tokens, topk), torch.int32)
        mp = None if mask is None else self._mask(mask, tokens)
        ws, wp, nbytes = self._space(P.pccl_moe_balance_workspace, tokens, experts)
        loss, probs = self._empty(torch.float32), self._empty(torch.float32, experts)
        counts, rows = self._empty(torch.int32, experts), self._empty(torch.int32)
        self._call(self._lib.pccl_moe_balance, logits.data_ptr(), _DTYPE[logits.dtype], tokens, experts, ld, ip, topk, mp,
                   loss.data_ptr(), probs.data_ptr(), counts.data_ptr(), rows.data_ptr(), wp, nbytes, self._stream())
        return loss, counts, probs, rows

    def balance_loss_backward(self, logits, counts, rows, dloss: Optional[torch.Tensor], dprobs: Optional[torch.Tensor] = None,
                              mask: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The gradient of balance_loss()'s loss and probs with respect to its
        logits, in their type.  With counts and rows summed over ranks it is this
        rank's part of the gradient of the loss of their joint batch."""
        if _learns(logits, dloss, dprobs):
            return _Served.apply("balance_loss_backward", lambda *given: self._balance_backward(*given, counts, rows, mask), logits, dloss, dprobs)
        return self._balance_backward(logits, dloss, dprobs, counts, rows, mask)

    def _balance_backward(self, logits, dloss, dprobs, counts, rows, mask):
        tokens, experts, ld = self._matrix("logits", logits)
        out = self._empty(logits.dtype, tokens, experts)
        self._call(
            self._lib.pccl_moe_balance_backward, logits.data_ptr(), _DTYPE[logits.dtype], tokens, experts, ld,
            None if mask is None else self._mask(mask, tokens), self._same("counts", counts, (experts,), torch.int32),
            self._same("rows", rows, (), torch.int32), None if dloss is None else self._same("dloss", dloss, (), torch.float32),
            None if dprobs is None else self._same("dprobs", dprobs, (experts,), torch.float32), out.data_ptr(), experts,
            self._stream())
        return out

    # -- 8-bit values with a scale for 128 of them -----------------------------

    def _room8(self, *shape):
        """Packed rows [..., rows] of the last extent's values."""
        cb, sb = f8_bytes(shape[-1])
        return F8(self._empty(torch.uint8, *shape[:-1], cb), self._empty(torch.uint8, *shape[:-1], sb), shape[-1])

    def _pack8(self, x, rows_too, cols_too, tiles=False, groups=None):
        lead, batch, one = (), 1, None
        if tiles and x.dim() == 3:
            lead, batch, one = x.shape[:1], x.shape[0], x.shape[1]
            try:
                x = x.view(batch * one, x.shape[2])
            except RuntimeError:
                raise ValueError(f"x: matrices that stand one behind the other are needed (strides {x.stride()})") from None
        rows, cols, ld = self._matrix("x", x)
        rows = rows if one is None else one
        if groups is not None and groups.rows != rows:
            raise ValueError(f"x: {groups.rows} rows are grouped, got {rows}")
        r = c = rc = rs = cc = cs = None
        if rows_too:
            r = self._room8(*lead, rows, cols)
            rc, rs = r.codes.data_ptr(), r.scales.data_ptr()
        if cols_too:
            c = self._room8(*lead, cols, rows if groups is None else 128 * group_blocks(groups.experts, rows))
            cc, cs = c.codes.data_ptr(), c.scales.data_ptr()
        if groups is not None:
            self._call(self._lib.pccl_f8_quantize_experts, x.data_ptr(), _DTYPE[x.dtype], rows, cols, ld, self._blocks(groups),
                       groups.experts, rc, rs, cc, cs, self._stream())
        else:
            self._call(self._lib.pccl_f8_quantize, x.data_ptr(), _DTYPE[x.dtype], batch, rows, cols, ld, tiles, rc, rs, cc, cs,
                       self._stream())
        return r, c

    def quantize8(self, x) -> F8:
        """x's rows in 8 bits, a scale for 128 values."""
        return self._pack8(x, True, False)[0]

    def quantize8_columns(self, x, groups: Optional[Groups] = None) -> F8:
        """x's columns (the rows of its transpose); with groups, in blocks of one
        expert's rows, as expert_gradient8() takes them.  Blocks behind the last
        expert's are not written: they hold what the memory held."""
        return self._pack8(x, False, True, groups=groups)[1]

    def quantize8_both(self, x, groups: Optional[Groups] = None):
        """(x's rows, x's columns) in one pass over x.  With groups, rows that are no
        expert's and blocks of the columns behind the last expert's are not written:
        they hold what the memory held, and no expert's operator reads them."""
        return self._pack8(x, True, True, groups=groups)

    def quantize8_tiles(self, w):
        """(w's rows, w's columns) with one scale for 128 x 128 values, so that
        both stand for the same ones; w is [rows, cols] or [experts, rows, cols]."""
        return self._pack8(w, True, True, tiles=True)

    def dequantize8(self, q: F8, dtype) -> torch.Tensor:
        """The values that q stands for."""
        kind = self._type(dtype)
        lead = q.codes.shape[:-1]
        codes, scales = self._packed8("q", q, lead)
        out = self._empty(dtype, *lead, q.cols)
        self._call(self._lib.pccl_f8_dequantize, codes, scales, lead.numel(), q.cols, out.data_ptr(), kind, q.cols, self._stream())
        return out

    def matmul8(self, a: F8, b: F8, dtype, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """a b^T: [rows of a, rows of b]."""
        kind = self._type(dtype)
        if a.cols != b.cols:
            raise ValueError(f"a has rows of {a.cols} values, b of {b.cols}")
        m, n, k = a.codes.shape[0], b.codes.shape[0], a.cols
        ac, as_ = self._packed8("a", a, (m,))
        bc, bs = self._packed8("b", b, (n,))
        out, ld = self._result(out, m, n, dtype)
        ws, wp, nbytes = self._space(P.pccl_f8_matmul_workspace, m, n, k)
        self._call(self._lib.pccl_f8_matmul, ac, as_, bc, bs, m, n, k, out.data_ptr(), kind, ld, wp, nbytes, self._stream())
        return out

    def expert_groups(self, counts, rows: int) -> Groups:
        """The blocks of `rows` rows in expert order, from the experts' counts,
        which stay on the device.  Rows beyond their sum are no one's."""
        experts = counts.shape[0] if counts.dim() == 1 else 0
        cp = self._same("counts", counts, (experts,), torch.int32)
        if rows < 0:
            raise ValueError(f"{rows} rows")
        table = self._empty(torch.int32, _group_words(experts, rows))
        self._call(self._lib.pccl_moe_groups, cp, experts, rows, table.data_ptr(), self._stream())
        return Groups(table, experts, rows)

    def expert_matmul8(self, a: F8, w: F8, groups: Groups, dtype, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """[rows of a, n]: each row of a, in expert order, times its expert's w
        [experts, n, a.cols].  Rows that are no expert's are left as they were:
        without `out` they hold what the memory held."""
        kind = self._type(dtype)
        if a.cols != w.cols:
            raise ValueError(f"a has rows of {a.cols} values, w of {w.cols}")
        if w.codes.dim() != 3:
            raise ValueError(f"w: [{groups.experts}, n, {a.cols}] is needed, got codes {tuple(w.codes.shape)}")
        rows, n = groups.rows, w.codes.shape[1]
        ac, as_ = self._packed8("a", a, (rows,))
        wc, ws = self._packed8("w", w, (groups.experts, n))
        out, ld = self._result(out, rows, n, dtype)
        self._call(self._lib.pccl_f8_expert_matmul, ac, as_, wc, ws, rows, groups.experts, n, a.cols, self._blocks(groups),
                   out.data_ptr(), kind, ld, self._stream())
        return out

    def expert_gradient8(self, a: F8, b: F8, groups: Groups, dtype) -> torch.Tensor:
        """[experts, rows of a, rows of b]: for every expert the sum of a_i b_i^T
        over its rows, for columns packed with the same groups."""
        kind = self._type(dtype)
        cols = 128 * group_blocks(groups.experts, groups.rows)
        if a.cols != cols or b.cols != cols:
            raise ValueError(f"columns of {cols} grouped values are needed, a has {a.cols}, b {b.cols}")
        m, n = a.codes.shape[0], b.codes.shape[0]
        ac, as_ = self._packed8("a", a, (m,))
        bc, bs = self._packed8("b", b, (n,))
        out = self._empty(dtype, groups.experts, m, n)
        self._call(self._lib.pccl_f8_expert_gradient, ac, as_, bc, bs, groups.rows, groups.experts, m, n, self._blocks(groups),
                   out.data_ptr(), kind, self._stream())
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
