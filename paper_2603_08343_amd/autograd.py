"""torch.autograd plumbing over the C-ABI entry points: a Function and a Module for the
Walsh-Hadamard output layer (paper Sec. 4.1, Eq. 1), so that it drops into a PyTorch attention block
where the dense output projection W_O used to be.  Nothing is computed here: forward calls
wht_affine_forward (or wht_affine_forward_residual), backward calls wht_affine_backward, which
recomputes H x from the saved input instead of storing it.

The paper does not say how alpha and beta start; this module starts them at 1 and 0, which makes
the layer the orthogonal transform itself at initialisation.
"""
import torch

from . import attention4, binding, rotary


class WhtAffineFunction(torch.autograd.Function):
    """y = [resid +] alpha (.) (H x) + beta over the last dimension of x."""

    @staticmethod
    def forward(ctx, x, alpha, beta, resid=None):
        d = x.shape[-1]
        x2 = x.reshape(-1, d)
        if not x2.is_contiguous():
            x2 = x2.contiguous()
        if resid is None:
            y = binding.wht_affine_forward(x2, alpha, beta)
        else:
            r2 = resid.reshape(-1, d)
            y = binding.wht_affine_forward_residual(x2, alpha, beta, r2 if r2.is_contiguous() else r2.contiguous())
        ctx.save_for_backward(x2, alpha)
        ctx.has_resid = resid is not None
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        x2, alpha = ctx.saved_tensors
        d = x2.shape[-1]
        dy2 = dy.reshape(-1, d)
        if not dy2.is_contiguous():
            dy2 = dy2.contiguous()
        want_dx = ctx.needs_input_grad[0]
        want_pg = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx = dalpha = dbeta = None
        if want_dx or want_pg:
            dx, dalpha, dbeta = binding.wht_affine_backward(dy2, x2, alpha, want_dx=want_dx,
                                                            want_param_grads=want_pg)
        # the residual stream's gradient is dy itself
        return (dx.view(dy.shape) if dx is not None else None, dalpha, dbeta,
                dy if ctx.has_resid and ctx.needs_input_grad[3] else None)


def wht_affine(x, alpha, beta, resid=None):
    """Differentiable y = [resid +] alpha (.) (H x) + beta; x: [..., d] bfloat16|float32 on the GPU.
    Plain calls go to the extension module's node of torch's C++ autograd (csrc/torch_marshal.cpp), which does what
    WhtAffineFunction does; the others, and everything under a compiler's trace, to WhtAffineFunction.  The node's grad_fn has
    a name, next_functions and hooks; saved_tensors and needs_input_grad are the Python Function's alone (WhtAffineFunction.apply)."""
    if not torch.compiler.is_compiling():
        y = binding._native().layer(x, alpha, beta, resid)
        if y is not None:
            return y
    return WhtAffineFunction.apply(x, alpha, beta, resid)


class WhtAffine(torch.nn.Module):
    """The parameter-free transform plus its 2d learnable parameters (Eq. 1; Table 1 counts 2d).
    alpha and beta are float32 whatever the activations' dtype is."""

    def __init__(self, d: int, device=None):
        super().__init__()
        self.d = d
        self.alpha = torch.nn.Parameter(torch.ones(d, dtype=torch.float32, device=device))
        self.beta = torch.nn.Parameter(torch.zeros(d, dtype=torch.float32, device=device))

    def forward(self, x, resid=None):
        return wht_affine(x, self.alpha, self.beta, resid)

    def extra_repr(self):
        return f"d={self.d}"


class WhtRotaryFunction(torch.autograd.Function):
    """Heads turned by positions of several axes; the gradient is turned back by the same angles."""

    @staticmethod
    def forward(ctx, x, rope, positions, axes, interleaved, inverse):
        axes = rotary._axis_bytes(axes)                     # as they are now: the backward pass needs the same
        heads = _heads(x)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)        # whole: a view made here could not be changed in place
        rotary.wht_rotary_rotate(heads, rope, positions, axes, interleaved, inverse, out=y.view(heads.shape))
        ctx.save_for_backward(rope, positions)              # their versions are checked: angles that have changed since raise
        ctx.how = axes, interleaved, not inverse
        return y

    @staticmethod
    def backward(ctx, dy):
        return WhtRotaryFunction.apply(dy, *ctx.saved_tensors, *ctx.how), None, None, None, None, None


def _heads(x):
    """x [..., heads, head_dim] as [T, heads, head_dim] with steps of 16 bytes: a copy where its strides or its place are others."""
    x = x.reshape(-1, *x.shape[-2:])
    step = 16 // x.element_size()
    plain = x.stride(2) == 1 and x.stride(1) % step == 0 and x.stride(0) % step == 0 and x.stride(1) >= x.shape[2] and x.data_ptr() % 16 == 0
    return x if plain else x.clone(memory_format=torch.contiguous_format)


def wht_rotary(x, rope, positions=None, axes=None, interleaved=False):
    """Differentiable rotary.wht_rotary_rotate; x: [..., heads, head_dim] bfloat16|float32 on the GPU, positions int32 [...] or [..., axes]
    (None: token s of x [..., tokens, heads, head_dim] has position s, in each batch of tokens from 0 on).
    Neither the table nor the positions have a gradient.  Plain calls go to the extension module's node of torch's C++ autograd
    (csrc/attention_marshal.cpp), the others, and everything under a compiler's trace, to WhtRotaryFunction.

    A capture into a graph that records a gradient is refused for a leaf whose gradient a living graph from outside the capture gathers: the backward pass would wait for that
    graph's stream, which is not captured, and torch ends the process over it."""
    if positions is None and x.dim() > 3 and x.shape[:-3].numel() != 1:
        positions = torch.arange(x.shape[-3], dtype=torch.int32, device=x.device).expand(x.shape[:-2])
    if positions is not None and x.dim() != 3:
        lead = positions.shape[:x.dim() - 2]
        if lead != x.shape[:-2]:
            raise ValueError(f"positions must be those of the tokens, {list(x.shape[:-2])}, got {list(positions.shape)}")
        positions = positions.reshape(-1, *positions.shape[x.dim() - 2:]).contiguous()
    if not torch.compiler.is_compiling():
        native = attention4._native()
        if torch.cuda.is_current_stream_capturing() and native.leaf_elsewhere(x):
            raise RuntimeError("x is a leaf whose gradient a graph from outside the capture gathers on another stream: let go of that graph first "
                               "(its outputs and losses), or capture with a detached x")
        y = native.rotary(x, rope, positions, axes, interleaved)
        if y is not None:
            return y
    return WhtRotaryFunction.apply(x, rope, positions, axes, interleaved, False)
