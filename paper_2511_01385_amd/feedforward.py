"""The feed-forward half of a fine-tuned encoder layer, with everything its backward needs kept in 8 bits.

    h = act(W1 x + b1),   o = W2 h + b2 + A h,   y = layer_norm(o + x)

W1 and W2 are frozen dense weights, A is a block-circulant adapter (Sec. 3.3) of W2; what is trained is
the adapter's first columns and the norm's weight and bias.  One autograd function runs the whole half
through the library's calls: the products with bias and activation in their epilogue, the adapter's output as
the second one's residual (written over it), the sum with x inside the norm.

Memory: between forward and backward a token keeps the pre-activation and h (d_ff values each) and the norm's
input (d_model values), all as 8-bit checkpoints: 33/32 bytes a value, instead of x, the pre-activation, h and the
norm's input in the storage type.  Gradients are taken at the checkpointed values, in float32 too (with "relu" that
costs accuracy: see ``api.linear_backward``).  Where no gradient can be asked for (``torch.no_grad()``, or nothing that
requires one) no checkpoint is made.
"""

from __future__ import annotations

import math

import torch
from torch.autograd.function import once_differentiable

from . import api


class _FeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, c, weight, bias, activation, eps, keep):
        # keep: whether there may be a backward, whose checkpoints are made only then
        tokens, d_model = x.shape
        d_ff = w1.shape[0]
        h = torch.empty((tokens, d_ff), dtype=x.dtype, device=x.device)
        z8 = api.checkpoint_like(h) if keep and activation != "none" else None
        api.linear_forward(x, w1, h, bias=b1, activation=activation, checkpoint=z8)
        q, kb, p = c.shape
        spectra = c.detach().to(x.dtype).contiguous()
        if spectra.data_ptr() == c.data_ptr():  # float32: do not transform the parameter itself
            spectra = spectra.clone()
        api.rdfft_forward(spectra.view(q * kb, p))
        o = torch.empty_like(x)
        api.bca_forward(h, spectra, o)
        api.linear_forward(h, w2, o, bias=b2, residual=o)
        y = torch.empty_like(x)
        if not keep:
            return api.layer_norm_forward(o, weight.detach(), bias.detach(), y, residual=x, eps=eps)
        mean, rstd = (torch.empty(tokens, dtype=torch.float32, device=x.device) for _ in range(2))
        u8 = api.checkpoint_like(x)
        api.layer_norm_forward(o, weight.detach(), bias.detach(), y, residual=x, mean=mean, rstd=rstd, checkpoint=u8,
                               eps=eps)
        h8 = api.act8_quantize(h, *api.checkpoint_like(h))
        ctx.activation = activation
        ctx.save_for_backward(w1, w2, spectra, weight, mean, rstd, *u8, *h8, *(z8 or ()))
        return y

    @staticmethod
    @once_differentiable  # (the library's calls are not recorded: second derivatives are refused, not left out)
    def backward(ctx, dy):
        w1, w2, spectra, weight, mean, rstd, u_codes, u_scales, h_codes, h_scales, *z8 = ctx.saved_tensors
        dy = dy.contiguous()
        du = torch.empty_like(dy)
        dweight, dbias = torch.empty_like(weight), torch.empty_like(weight)
        api.layer_norm_backward(dy, (u_codes, u_scales), weight.detach(), mean, rstd, du, dweight, dbias)
        h = api.act8_dequantize(h_codes, h_scales, torch.empty(h_codes.shape, dtype=dy.dtype, device=dy.device))
        dc = torch.empty(spectra.shape, dtype=torch.float32, device=dy.device)
        dh = torch.empty_like(h)
        api.bca_backward_keep(h, spectra, du, dh, dc)
        del h
        api.linear_backward(du, None, w2, dx=dh, add=dh)
        dx = None
        if ctx.needs_input_grad[0]:
            # x also reached the norm directly
            dx = torch.empty_like(du)
            api.linear_backward(dh, None, w1, dx=dx, activation=ctx.activation, checkpoint=tuple(z8) or None, add=du)
        return dx, None, None, None, None, dc, dweight, dbias, None, None, None


class AdaptedFeedForward(torch.nn.Module):
    """layer_norm(W2 h + b2 + A h + x), h = act(W1 x + b1): frozen W1, W2, a block-circulant adapter A, a trained norm.

    ``w1`` (d_ff, d_model), ``w2`` (d_model, d_ff) and their biases are buffers of the storage type ``dtype`` (random
    unless loaded); ``c`` (d_model/p, d_ff/p, p), ``weight`` and ``bias`` are float32 parameters.  p: a power of two up
    to 8192 that divides both widths.  ``activation``: "gelu", "relu", "silu" or "none".  The adapter starts at zero.
    """

    def __init__(self, d_model: int, d_ff: int, p: int, dtype: torch.dtype = torch.bfloat16, activation: str = "gelu",
                 device: str | torch.device = "cuda", eps: float = 1e-5):
        super().__init__()
        if p < 2 or p & (p - 1) or p > 8192:
            raise ValueError(f"p must be a power of two from 2 to 8192, got {p}")
        if d_model % p or d_ff % p:
            raise ValueError(f"p = {p} must divide d_model = {d_model} and d_ff = {d_ff}")
        if dtype not in (torch.bfloat16, torch.float16, torch.float32):
            raise TypeError(f"storage type must be bfloat16, float16 or float32, got {dtype}")
        if activation not in api.ACTIVATIONS:
            raise ValueError(f"activation must be one of {', '.join(api.ACTIVATIONS)}, got {activation!r}")
        self.d_model, self.d_ff, self.p = d_model, d_ff, p
        self.dtype, self.activation, self.eps = dtype, activation, eps

        def frozen(*shape, scale):
            return (torch.randn(shape, dtype=torch.float32, device=device) * scale).to(dtype)

        self.register_buffer("w1", frozen(d_ff, d_model, scale=1 / math.sqrt(d_model)))
        self.register_buffer("b1", frozen(d_ff, scale=0.0))
        self.register_buffer("w2", frozen(d_model, d_ff, scale=1 / math.sqrt(d_ff)))
        self.register_buffer("b2", frozen(d_model, scale=0.0))
        new = lambda fill, *shape: torch.nn.Parameter(torch.full(shape, fill, dtype=torch.float32, device=device))  # noqa: E731
        self.c = new(0.0, d_model // p, d_ff // p, p)
        self.weight, self.bias = new(1.0, d_model), new(0.0, d_model)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if x.shape[-1] != self.d_model:
            raise ValueError(f"last dimension {x.shape[-1]} != d_model = {self.d_model}")
        if x.dtype != self.dtype:
            raise TypeError(f"input is {x.dtype}, the layer stores {self.dtype}")
        x2d = x.reshape(-1, self.d_model).contiguous()
        trained = (x2d, self.c, self.weight, self.bias)
        keep = torch.is_grad_enabled() and any(t.requires_grad for t in trained)
        y = _FeedForward.apply(x2d, self.w1, self.b1, self.w2, self.b2, self.c, self.weight, self.bias, self.activation,
                               self.eps, keep)
        return y.reshape(x.shape)

    def extra_repr(self) -> str:
        return f"d_model={self.d_model}, d_ff={self.d_ff}, p={self.p}, activation={self.activation}, dtype={self.dtype}"
