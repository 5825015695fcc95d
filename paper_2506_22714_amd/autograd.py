"""Differentiable SpMM / SDDMM / edge softmax on top of the C ABI (training use of the operators, Section 5.5 of the
paper).  Only argument marshalling and the chain rule live here; every product runs in the library's kernels:

  C = A B            dB = A^T dC                 (SpMM on the plan of the transposed pattern)
                     dA_p = <dC_i, B_j>          (SDDMM without A's values)
  out_p = A_p <X_i, Y_j>
                     dX = (A o dout) Y,  dY = (A o dout)^T X,  dA_p = dout_p <X_i, Y_j>
  alpha = softmax_row(scale * s)
                     ds_p = scale alpha_p (dalpha_p - sum_row alpha dalpha)

and at the ends of a training step, before and behind the sparse layers:

  out_i = scale W[index_i]
                     dW_v = scale sum_{index_i = v} dout_i
  log p = log softmax(scale x), H = -sum p log p
                     dx_j = scale ([j = target] d + sum_a [j = top_a] d_a - p_j (d + sum_a d_a + e (log p_j + H)))

A backward pass may be captured into a HIP graph.  Let no graph of an eager pass over the same parameters live on then: torch's nodes that
add up their gradients belong to that pass's stream, and the capture ends with an error or takes the process with it.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as lb


class SparseMatrix:
    """A sparse pattern on the device with the plan of A and of A^T (both built by the device planner).  Values are
    passed to every call (they are what training changes); the plans only hold the current ones."""

    def __init__(self, M: int, Kc: int, rowptr: torch.Tensor, col: torch.Tensor, dtype=torch.float16, **opts):
        self.M, self.Kc, self.dtype = int(M), int(Kc), dtype
        self.rowptr, self.col = rowptr, col
        self.nnz = int(col.numel())
        ones = torch.ones(self.nnz, dtype=dtype, device=col.device)
        self.plan = lb.Plan.from_device_csr(M, Kc, rowptr, col, ones, resident=True, keep_host_copy=False, **opts)
        rowptr_t, col_t, perm_t = lb.transpose_csr(M, Kc, rowptr, col)
        self._perm_t = perm_t
        self.plan_t = lb.Plan.from_device_csr(Kc, M, rowptr_t, col_t, ones, resident=True, keep_host_copy=False, **opts)
        # made here and not in the first backward pass, because it waits for the stream and sorts (2^24 nonzeros: 1.2 ms, 4.1 bytes each kept);
        # a program that only runs forward needs no SparseMatrix but a Plan.  A matrix for SDDMM alone has no SpMM arrays to put values into
        self._order_t = None if opts.get("flags", 0) & lb.FLAG_NO_SPMM else self.plan_t.value_order(perm_t)

    @property
    def perm_t(self) -> torch.Tensor:
        """CSR position in A of every nonzero of A^T."""
        return self._perm_t.long()

    def set_transposed(self, vals: torch.Tensor):
        """Values of A (CSR order) into the SpMM arrays of the plan of A^T."""
        if self._order_t is not None:
            self.plan_t.set_values_ordered(vals, self._order_t)

    def close(self):
        self.plan.close()
        self.plan_t.close()


def _feature_ok(n: int) -> bool:
    return n in (32, 64, 128)


class _SpMM(torch.autograd.Function):
    @staticmethod
    def forward(ctx, sm: SparseMatrix, vals: torch.Tensor, B: torch.Tensor):
        sm.plan.set_values(vals.detach().contiguous(), lb.OP_SPMM)
        ctx.sm = sm
        ctx.save_for_backward(vals, B)
        return sm.plan.spmm(B.detach().contiguous())

    @staticmethod
    def backward(ctx, dC):
        sm = ctx.sm
        vals, B = ctx.saved_tensors
        dC16 = dC.to(sm.dtype).contiguous()
        dvals = dB = None
        if ctx.needs_input_grad[2]:
            sm.set_transposed(vals.detach().contiguous())
            dB = sm.plan_t.spmm_rounded(dC16).to(B.dtype)
        if ctx.needs_input_grad[1]:
            if not _feature_ok(B.shape[1]):
                raise RuntimeError("gradient with respect to the sparse values needs N in {32, 64, 128}")
            dvals = sm.plan.sddmm_pattern_rounded(dC16, B.detach().contiguous()).to(vals.dtype)
        return None, dvals, dB


class _SDDMM(torch.autograd.Function):
    @staticmethod
    def forward(ctx, sm: SparseMatrix, vals: torch.Tensor, X: torch.Tensor, Y: torch.Tensor):
        sm.plan.set_values(vals.detach().contiguous(), lb.OP_SDDMM)
        ctx.sm = sm
        ctx.save_for_backward(vals, X, Y)
        return sm.plan.sddmm(X.detach().contiguous(), Y.detach().contiguous())

    @staticmethod
    def backward(ctx, dout):
        sm = ctx.sm
        vals, X, Y = ctx.saved_tensors
        Xc, Yc = X.detach().contiguous(), Y.detach().contiguous()
        g = sm.plan.value_products(vals.detach().contiguous(), dout.float().contiguous())
        dvals = dX = dY = None
        if ctx.needs_input_grad[2]:
            sm.plan.set_values(g, lb.OP_SPMM)
            dX = sm.plan.spmm_rounded(Yc).to(X.dtype)
        if ctx.needs_input_grad[3]:
            sm.set_transposed(g)
            dY = sm.plan_t.spmm_rounded(Xc).to(Y.dtype)
        if ctx.needs_input_grad[1]:
            dvals = (dout * sm.plan.sddmm(Xc, Yc, pattern_only=True)).to(vals.dtype)
        return None, dvals, dX, dY


class _EdgeSoftmax(torch.autograd.Function):
    @staticmethod
    def forward(ctx, sm: SparseMatrix, scores: torch.Tensor, scale: float):
        alpha = sm.plan.edge_softmax(scores.detach().float().contiguous(), scale,
                                     out=torch.empty(sm.nnz, dtype=sm.dtype, device=scores.device))
        ctx.sm, ctx.scale = sm, scale
        ctx.save_for_backward(alpha)
        return alpha

    @staticmethod
    def backward(ctx, dalpha):
        (alpha,) = ctx.saved_tensors
        return None, ctx.sm.plan.edge_softmax_backward_rounded(alpha, dalpha.to(alpha.dtype).contiguous(), ctx.scale), None


def spmm(sm: SparseMatrix, vals: torch.Tensor, B: torch.Tensor) -> torch.Tensor:
    """C = A B with A's values `vals` (CSR order); fp32 result."""
    return _SpMM.apply(sm, vals, B)


def sddmm(sm: SparseMatrix, vals: torch.Tensor, X: torch.Tensor, Y: torch.Tensor) -> torch.Tensor:
    """out_p = vals_p <X_i, Y_j> on A's pattern (CSR order); fp32 result."""
    return _SDDMM.apply(sm, vals, X, Y)


def edge_softmax(sm: SparseMatrix, scores: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """Row-wise softmax of `scale * scores` over A's pattern; result in the matrix's value type."""
    return _EdgeSoftmax.apply(sm, scores, scale)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """x, copied if its rows are not contiguous (what lies between them may be anything)."""
    x = x.detach()
    return x if x.dim() != 2 or (x.stride(1) == 1 and x.stride(0) >= x.shape[1]) else x.contiguous()


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table: torch.Tensor, index: torch.Tensor, scale: float):
        ctx.rows, ctx.scale = table.shape[0], scale
        ctx.save_for_backward(index)
        return lb.embedding(_rows(table), index, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        (index,) = ctx.saved_tensors
        return lb.embedding_backward(dout.reshape(-1, dout.shape[-1]).contiguous(), index, ctx.rows, ctx.scale), None, None


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits: torch.Tensor, targets, top: int, scale: float):
        r = lb.log_probs(_rows(logits), targets, top, scale)
        ctx.scale = scale
        ctx.save_for_backward(logits, targets, r.entropy, r.top_index, r.stats)
        ctx.mark_non_differentiable(r.top_index)
        ctx.set_materialize_grads(False)
        return r.target, r.entropy, r.top, r.top_index

    @staticmethod
    @once_differentiable
    def backward(ctx, d_target, d_entropy, d_top, _):
        logits, targets, entropy, top_index, stats = ctx.saved_tensors
        parts = [None if d is None else d.float().contiguous() for d in (d_target, d_entropy, d_top)]
        return lb.log_probs_backward(_rows(logits), lb.LogProbs(None, entropy, None, top_index, stats), targets, *parts, scale=ctx.scale), None, None, None


def embedding(table: torch.Tensor, index: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """`scale * table[index]` in the table's type; -1 in `index` is padding: a row of zeros that has no gradient."""
    return _Embedding.apply(table, index.contiguous(), scale)


def log_probs(logits: torch.Tensor, targets: torch.Tensor | None = None, top: int = 0, scale: float = 1.0):
    """(log probability of the given class, entropy, log probabilities of the `top` most likely classes, these classes) of every row of
    `scale * logits`; all but the classes are fp32 and have gradients.  A target of -1 is none: 0, without a gradient."""
    return _LogProbs.apply(logits, targets if targets is None else targets.contiguous(), top, scale)
