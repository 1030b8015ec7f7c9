"""Two-layer full-batch GCN whose sparse aggregations run through sd_spmm.

The paper's application study (Sec. "Evaluation", GCN paragraph) trains a
two-layer GCN on a normalised adjacency Â with four sparse aggregations per
epoch: Â·(X W1) and Â·(H1 W2) forward, Âᵀ·G at both widths backward. Only the
aggregation is replaced; the dense transforms, activation, loss and optimiser
are ordinary torch operations.

GCN2Packed is the same network with a group norm before the activation and its
node tables in 8 bits: the dense transforms multiply 8-bit operands, and what the
backward pass needs of each layer (the features, the normalisation's input, the
activation) is kept at one byte an element instead of four, through the operators
of dense.py.  The aggregations stay in fp32.

`transform4` is a layer's dense transform in 4 bits with its gradients.

Each aggregation is `spmm(B, fwd, bwd)`: C = Â·B with plan `fwd`, and in the
backward pass dB = Âᵀ·dC with the transpose plan `bwd` (A is not assumed
symmetric).  Plans are built once per (graph, width) and reused every epoch.
"""
from __future__ import annotations

import torch

from . import Plan, dense, sd_plan_device, sd_plan_ex, sd_spmm
from .autograd import anchor, first_derivatives_only


class _SpMM(torch.autograd.Function):
    @staticmethod
    def forward(ctx, B, fwd: Plan, bwd: Plan):
        info = fwd.info
        if B.dim() != 2 or B.shape[0] != info["k"] or B.shape[1] != info["n"] or B.dtype != torch.float32:
            raise ValueError(f"spmm: B must be float32 [{info['k']}, {info['n']}], got {tuple(B.shape)} {B.dtype}")
        B = B.contiguous()
        C = torch.empty((info["m"], info["n"]), dtype=torch.float32, device=B.device)
        sd_spmm(fwd, B, C, torch.cuda.current_stream(B.device))
        ctx.bwd = bwd
        return C

    @staticmethod
    def backward(ctx, dC):
        bwd = ctx.bwd
        info = bwd.info
        dC = dC.contiguous()
        dB = torch.empty((info["m"], info["n"]), dtype=torch.float32, device=dC.device)
        sd_spmm(bwd, dC, dB, torch.cuda.current_stream(dC.device))
        return dB, None, None


def spmm(B: torch.Tensor, fwd: Plan, bwd: Plan) -> torch.Tensor:
    """C = Â·B; its gradient with respect to B is Âᵀ·dC (plan `bwd`)."""
    return _SpMM.apply(B, fwd, bwd)


class AggregationPlans:
    """Forward and transpose plans of one adjacency for each width used.

    A is a host CSR (an object with m, k, rowptr, colidx, values) or a
    torch sparse CSR tensor on the GPU; the latter is planned from device
    memory (sd_plan_device), its int64 indices narrowed to int32."""

    def __init__(self, A, widths, **plan_opts):
        self.plans = {}
        if isinstance(A, torch.Tensor):
            if A.layout != torch.sparse_csr or not A.is_cuda or A.dtype != torch.float32:
                raise ValueError("adjacency tensor must be a float32 sparse CSR tensor on the GPU")
            m, k = A.shape
            rowptr = A.crow_indices().to(torch.int32).contiguous()
            colidx = A.col_indices().to(torch.int32).contiguous()
            values = A.values().contiguous()
            stream = torch.cuda.current_stream(A.device)
            nnz = int(values.numel())

            def plan(n, **kw):
                return sd_plan_device(rowptr, colidx, values, m, k, nnz, n, stream=stream, **plan_opts, **kw)
        else:
            def plan(n, **kw):
                return sd_plan_ex(A, n, **plan_opts, **kw)
        for n in widths:
            self.plans[n] = (plan(n), plan(n, transpose=True))

    def __call__(self, B: torch.Tensor) -> torch.Tensor:
        fwd, bwd = self.plans[B.shape[1]]
        return spmm(B, fwd, bwd)

    def destroy(self):
        for fwd, bwd in self.plans.values():
            fwd.destroy()
            bwd.destroy()
        self.plans = {}


class GCN2(torch.nn.Module):
    """H1 = relu(Â X W1), logits = Â H1 W2 (transform, then aggregate)."""

    def __init__(self, A, in_feats: int, hidden: int, classes: int, device, seed: int = 0, **plan_opts):
        super().__init__()
        g = torch.Generator(device="cpu").manual_seed(seed)

        def glorot(fan_in, fan_out):
            bound = (6.0 / (fan_in + fan_out)) ** 0.5
            return (torch.rand((fan_in, fan_out), generator=g, dtype=torch.float32) * 2 - 1) * bound

        self.W1 = torch.nn.Parameter(glorot(in_feats, hidden).to(device))
        self.W2 = torch.nn.Parameter(glorot(hidden, classes).to(device))
        self.agg = AggregationPlans(A, sorted({hidden, classes}), **plan_opts)

    def forward(self, X: torch.Tensor) -> torch.Tensor:
        H1 = torch.relu(self.agg(X @ self.W1))
        return self.agg(H1 @ self.W2)


class _PackedTransform(torch.autograd.Function):
    """X.W from X in 8 bits, packed here where it is a float tensor.  That one has a
    gradient too, as if the packing did not round: the output gradient, multiplied
    in 8 bits.  There are no second derivatives."""

    @staticmethod
    def forward(ctx, X, W, fmt, grad_fmt):
        X8 = X if isinstance(X, dense.Packed) else dense.pack(X, fmt)
        ctx.of_table = X8.cols, X8.format
        kept = [X8.codes, X8.scales]
        all_inputs = None
        if ctx.needs_input_grad[0]:
            ctx.dtype, ctx.grad_fmt, all_inputs = X.dtype, grad_fmt, anchor(W)
            kept += W, all_inputs
        ctx.save_for_backward(*kept)
        return dense.product(X8, dense.pack(W, X8.format, transpose=True)), all_inputs

    @staticmethod
    @first_derivatives_only
    def backward(ctx, kept, dZ):
        dX, dW, dZ = None, None, dZ.contiguous()
        codes, scales, *rest = kept
        X8 = dense.Packed(codes, scales, *ctx.of_table)
        if ctx.needs_input_grad[0]:
            dX = dense.product(dense.pack(dZ, ctx.grad_fmt), dense.pack(rest[0], X8.format), dtype=ctx.dtype)
        if ctx.needs_input_grad[1]:
            dW = dense.weight_gradient(X8, dZ)
        return dX, dW, None, None


class _Transform4(torch.autograd.Function):
    """X.W and both gradients as products of 4-bit tables, each packed along its own
    sum.  What the backward pass needs of X and W is kept packed along the other side,
    at half a byte an element.  grad: whether there will be one (torch asks for no
    gradients within forward, and names the inputs that require one all the same)."""

    @staticmethod
    def forward(ctx, X, W, grad):
        need_dX, need_dW = (grad and need for need in ctx.needs_input_grad[:2])
        X4, Xt = dense.pack4_both(X) if need_dW else (dense.pack4(X), None)
        W4, Wt = dense.pack4_both(W) if need_dX else (None, dense.pack4(W, transpose=True))
        ctx.dtypes, ctx.sizes = (X.dtype, W.dtype), (X.shape[0], *W.shape)
        all_inputs = anchor(W) if need_dX and need_dW else None  # each one's gradient depends on the other
        ctx.save_for_backward(W4 and W4.store, Xt and Xt.store, all_inputs)
        return dense.product4(X4, Wt), all_inputs

    @staticmethod
    @first_derivatives_only
    def backward(ctx, kept, dZ):
        need_dX, need_dW = ctx.needs_input_grad[:2]
        W4, Xt, _ = kept
        rows, cols, n = ctx.sizes
        dX = dW = None
        if need_dX and need_dW:
            G, Gt = dense.pack4_both(dZ)
        elif need_dX:
            G = dense.pack4(dZ)
        else:
            Gt = dense.pack4(dZ, transpose=True)
        if need_dX:
            dX = dense.product4(G, dense.Packed4.of(W4, cols, n), dtype=ctx.dtypes[0])
        if need_dW:
            dW = dense.product4(dense.Packed4.of(Xt, cols, rows), Gt, dtype=ctx.dtypes[1])
        return dX, dW, None


def transform4(X: torch.Tensor, W: torch.Tensor) -> torch.Tensor:
    """X.W in float32 on the matrix units' 4-bit form, with gradients computed in the
    same way: X and W are rounded to 4 bits along the features, the output gradient
    and W along the outputs for X's gradient, X and the output gradient along the rows
    for W's, as if the rounding were the identity.  No second derivatives.  A step that is
    captured into a graph takes leaves of its own (X.detach().requires_grad_())."""
    if X.dim() != 2 or W.dim() != 2 or X.shape[1] != W.shape[0]:
        raise ValueError(f"X and W must be matrices that fit, got {tuple(X.shape)} and {tuple(W.shape)}")
    return _Transform4.apply(X, W, torch.is_grad_enabled())[0]


class _NormTransform(torch.autograd.Function):
    """act(group norm(A)).W.  A and the activation are kept in 8 bits, and the
    output gradient is multiplied in 8 bits for dA, in full for dW.  There are no second
    derivatives."""

    @staticmethod
    def forward(ctx, A, gamma, beta, W, groups, eps, activation, fmt, grad_fmt):
        out = dense.group_norm(A, groups, gamma, beta, eps, activation, keep=fmt, pack_y=fmt, dense_y=False)
        ctx.of_table, ctx.args, ctx.grad_fmt = (out.x.cols, fmt), (groups, eps, activation), grad_fmt
        all_inputs = anchor(W)
        ctx.save_for_backward(W, gamma, beta, out.x.codes, out.x.scales, out.y_packed.codes, out.y_packed.scales,
                              out.mean, out.rstd, all_inputs)
        return dense.product(out.y_packed, dense.pack(W, fmt, transpose=True)), all_inputs

    @staticmethod
    @first_derivatives_only
    def backward(ctx, kept, dZ):
        dZ = dZ.contiguous()
        W, gamma, beta, *A8, codes, scales, mean, rstd, _ = kept
        A8, H8 = dense.Packed(*A8, *ctx.of_table), dense.Packed(codes, scales, *ctx.of_table)
        groups, eps, activation = ctx.args
        dA = dgamma = dbeta = dW = None
        if ctx.needs_input_grad[3]:
            dW = dense.weight_gradient(H8, dZ)
        if any(ctx.needs_input_grad[:3]):
            dH = dense.product(dense.pack(dZ, ctx.grad_fmt), dense.pack(W, H8.format))
            dA, dgamma, dbeta = dense.group_norm_backward(dH, A8, mean, rstd, groups, gamma, beta, eps, activation)
        return dA, dgamma, dbeta, dW, None, None, None, None, None


class GCN2Packed(torch.nn.Module):
    """H1 = act(group norm(Â X W1)), logits = Â H1 W2 with the node tables in 8 bits.

    X is given as a float tensor, which has a gradient if it requires one, or,
    since it does not change between epochs, once packed by
    `dense.pack(X, model.format)`.  format: of features,
    activations and weights; grad_format: of the output gradient where it is
    multiplied by the weights."""

    def __init__(self, A, in_feats: int, hidden: int, classes: int, device, seed: int = 0, groups: int = 8,
                 activation: str = "relu", eps: float = 1e-5, format: str = "e4m3", grad_format: str = "e4m3",
                 **plan_opts):
        super().__init__()
        plain = GCN2(A, in_feats, hidden, classes, device, seed, **plan_opts)
        self.W1, self.W2, self.agg = plain.W1, plain.W2, plain.agg
        self.gamma = torch.nn.Parameter(torch.ones(hidden, device=device))
        self.beta = torch.nn.Parameter(torch.zeros(hidden, device=device))
        self.groups, self.activation, self.eps = groups, activation, eps
        self.format, self.grad_format = format, grad_format

    def forward(self, X) -> torch.Tensor:
        A1 = self.agg(_PackedTransform.apply(X, self.W1, self.format, self.grad_format)[0])
        Z2 = _NormTransform.apply(A1, self.gamma, self.beta, self.W2, self.groups, self.eps, self.activation,
                                  self.format, self.grad_format)[0]
        return self.agg(Z2)


def train_epoch(model, X, labels, opt) -> torch.Tensor:
    """One full-batch epoch: forward, cross-entropy, backward, optimiser step."""
    opt.zero_grad(set_to_none=True)
    loss = torch.nn.functional.cross_entropy(model(X), labels)
    loss.backward()
    opt.step()
    return loss.detach()
