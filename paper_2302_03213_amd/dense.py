"""The layers between the looked-up ones of a model, as torch.autograd modules around the C ABI: linear layers that stay dense
(lutnn_dense_linear) and layer norms (lutnn_layer_norm), for models that replace some of their linear layers by table lookup
(arXiv 2302.03213, Sec. 6.1: the fully connected layers of BERT's last six layers).  DenseLinear's weight has the layout that
softpq.SoftPQLinear takes it over in: [D, M].

The backward passes cannot be captured into a graph, as those of softpq.py cannot: autograd adds a parameter's gradient on the
stream that the parameter was first used on, and such a step in a capture on another stream ends the process where an eager
graph of the same parameters lives.  dense_linear_backward and layer_norm_backward can.
"""
import torch

from . import binding as _b


def _not_captured():
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("the backward pass of a dense layer's module cannot be captured: capture dense_linear_backward and "
                           "layer_norm_backward")


def _differentiated(*inputs):
    """Whether a backward pass may follow, asked before autograd.Function.forward hides the grad mode."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs)


def _rows(G):
    """A gradient as the library reads it: autograd hands over expanded and transposed ones."""
    return G if (G.stride(1) == 1 or G.shape[1] == 1) and G.stride(0) >= G.shape[1] else G.contiguous()


class _DenseLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, bias, residual, activation, differentiated):
        Z = None
        if activation is not None and differentiated:
            Z = torch.empty((X.shape[0], W.shape[1]), dtype=X.dtype, device=X.device)
        Y = _b.dense_linear(X, W, bias, activation, residual, preactivation=Z)
        ctx.save_for_backward(X, W, Z)
        ctx.activation = activation
        return Y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, G):
        _not_captured()
        X, W, Z = ctx.saved_tensors
        needs = ctx.needs_input_grad
        dX = dW = db = None
        if any(needs[:3]):
            dX, dW, db = _b.dense_linear_backward(X, W, _rows(G), Z, ctx.activation, *needs[:3])
        return dX, dW, db, G if needs[3] else None, None, None


class DenseLinear(torch.nn.Module):
    """activation(X @ W + bias) + residual, with W [D, M] and bias [M] learned.  X [N, D], W and the residual have one type (fp32,
    bf16, fp16), the bias is fp32; activation None, "relu", "gelu", "gelu_tanh" or "silu".  W is copied row by row, so that a
    torch.nn.Linear's weight.t() will do."""

    def __init__(self, W, bias=None, activation=None):
        super().__init__()
        _b._activation(activation)
        self.W = torch.nn.Parameter(W.detach().clone(memory_format=torch.contiguous_format))
        self.bias = None if bias is None else torch.nn.Parameter(bias.detach().clone(memory_format=torch.contiguous_format))
        self.activation = activation

    def forward(self, X, residual=None):
        return _DenseLinearFn.apply(X, self.W, self.bias, residual, self.activation, _differentiated(X, self.W, self.bias))


class _LayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, weight, bias, residual, eps, with_total, needed):
        ctx.set_materialize_grads(False)
        statistics = torch.empty((X.shape[0], 2), dtype=torch.float32, device=X.device) if needed else None
        total = torch.empty(X.shape, dtype=X.dtype, device=X.device) if residual is not None and (needed or with_total) else None
        Y = _b.layer_norm(X, weight, bias, eps, residual, total=total, statistics=statistics)
        ctx.save_for_backward(X if residual is None else total, weight, statistics)
        return (Y, total) if with_total else Y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, G, G_total=None):
        _not_captured()
        X, weight, statistics = ctx.saved_tensors
        needs = ctx.needs_input_grad
        if G is None:  # the total alone was used
            return (G_total if needs[0] else None, None, None, G_total if needs[3] else None, None, None, None)
        dX, dw, db = _b.layer_norm_backward(_rows(G), X, statistics, weight, None if G_total is None else _rows(G_total),
                                            needs[0] or needs[3], needs[1], needs[2])
        return dX if needs[0] else None, dw, db, dX if needs[3] else None, None, None, None


class LayerNorm(torch.nn.Module):
    """The norm of X + residual over rows of D values, with weight and bias [D] learned (fp32).  forward(X, residual) gives Y;
    forward(X, residual, with_total=True) gives (Y, X + residual).  With a residual the backward pass goes by the sum as it was kept,
    rounded to X's type: lutnn_layer_norm_backward says what that is off by."""

    def __init__(self, D, eps=1e-5, device="cuda"):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(D, dtype=torch.float32, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(D, dtype=torch.float32, device=device))
        self.eps = eps

    def forward(self, X, residual=None, with_total=False):
        if with_total and residual is None:
            raise ValueError("without a residual the total is X itself")
        return _LayerNormFn.apply(X, self.weight, self.bias, residual, self.eps, with_total,
                                  _differentiated(X, self.weight, self.bias, residual))
