"""The operators between a transformer block's products, and the product in 8-bit
integers (include/fewbit_residual.h has the formulas, layouts and roundings).

dropout_fwd / dropout_bwd, residual_norm_fwd / residual_norm_bwd,
residual_norm_int8, quantize_rows and int8_linear are the raw calls, in the
library's HIP kernels on the current stream; they check every tensor (device,
dtype, shape, layout) and raise TypeError or ValueError before anything is
launched.  dropout and residual_norm are the same as differentiable functions:
they take any layout, copying tensors that the kernels cannot read; dropout
keeps nothing, residual_norm its sum, which the next addition reads anyway.

Wherever elements are dropped, `seed` is a whole number of 64 bits (with or
without a sign) or an int64 tensor of one element on the data's device, read when the kernels run: a
captured graph draws anew where the program changes it between replays.  `site`
(32 bits) tells apart places that share a seed.  The backward needs the same p,
seed and site.  p is taken in steps of 2^-16; what is dropped becomes 0 whatever
it was.
"""
from __future__ import annotations

import torch

from ._lib import BF16, F16, F32, GELU, SILU, FewbitError, _native
from .block import _result, _rows

_TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_ACTS = {None: -1, "none": -1, "gelu": GELU, "silu": SILU}


def _drops(p) -> bool:
    return round(p * 65536) > 0


# ---------------------------------------------------------------- dropout
def dropout_fwd(x, p, seed, site=0):
    """x with elements dropped with probability p and the others divided by 1 - p.
    x: fp32, fp16 or bf16, contiguous, 16-byte aligned."""
    return _result(_native.dropout(x, p, seed, site), "fewbit_dropout")


def dropout_bwd(dy, p, seed, site=0):
    """The gradient of x from that of dropout_fwd's result; the mask is formed again."""
    return _result(_native.dropout(dy, p, seed, site), "fewbit_dropout")


def _flat(t):
    """t, or a contiguous copy of it."""
    if t.is_contiguous() and t.data_ptr() % 16 == 0:
        return t
    return t.clone(memory_format=torch.contiguous_format)


def _keep_seed(ctx, seed, *tensors):
    """Saves tensors and, if it is one, the seed."""
    ctx.on_device = torch.is_tensor(seed)
    ctx.seed = None if ctx.on_device else seed
    ctx.save_for_backward(*tensors, *((seed,) if ctx.on_device else ()))


def _kept_seed(ctx):
    return (ctx.saved_tensors[-1] if ctx.on_device else ctx.seed)


class Dropping(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, site):
        _keep_seed(ctx, seed)
        ctx.rest = p, site
        return dropout_fwd(_flat(x), p, seed, site)

    @staticmethod
    def backward(ctx, dy):
        p, site = ctx.rest
        return dropout(dy, p, _kept_seed(ctx), site), None, None, None


def dropout(x, p, seed, site=0):
    """dropout_fwd, differentiable with respect to x, to any order; keeps no mask."""
    # ordinary device tensors: the same function in C++ (None: not one of those)
    y = _native.dropout_layer(x, p, seed, site)
    return Dropping.apply(x, p, seed, site) if y is None else y


class Dropout(torch.nn.Module):
    """Dropout that keeps no mask.  Without a seed each call in training draws one
    from torch's generator of the host (and a captured graph repeats it: give it
    one on the device)."""

    def __init__(self, p: float = 0.5, site: int = 0):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must be between 0 and 1")
        self.p, self.site = p, site

    def forward(self, x, seed=None):
        if not self.training or not _drops(self.p):
            return x
        return dropout(x, self.p, draw_seed() if seed is None else seed, self.site)

    def extra_repr(self) -> str:
        return f"p={self.p}, site={self.site}"


def draw_seed() -> int:
    """A seed from torch's generator of the host."""
    return int(torch.randint(-2 ** 63, 2 ** 63 - 1, (), dtype=torch.int64))


# ---------------------------------------------------------------- residual and norm
def residual_norm_fwd(x, residual, weight, eps=1e-6, p=0.0, seed=0, site=0):
    """h = residual + dropout(x), rounded, and the RMS norm of h times weight, in one
    pass: (h, y), dense.

    x [..., width], residual alike or None (nothing is added; without dropout
    either h is x itself), weight [width], all fp32, all fp16 or all bf16; width a multiple
    of 8 up to 32768; rows contiguous, from multiples of 16 bytes on, the axes
    before the last two one step apart (x[:, a:b] and views of a projection
    are)."""
    return _result(_native.rnorm_fwd(x, residual, weight, eps, p, seed, site), "fewbit_rnorm_fwd")


def residual_norm_bwd(dh, dy, h, weight, eps=1e-6, p=0.0, seed=0, site=0, residual=True):
    """(dx, dresidual, dweight) from the gradients of h (None: none) and y; h as
    residual_norm_fwd gave it; dweight is fp32.  Without dropout dresidual is dx;
    residual=False with dropout: it is not formed (None)."""
    return _result(_native.rnorm_bwd(dh, dy, h, weight, eps, p, seed, site, residual, False), "fewbit_rnorm_bwd")


class ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps, p, seed, site):
        ctx.set_materialize_grads(False)
        x, weight = _rows2(x), _flat(weight)
        residual = None if residual is None else _rows2(residual)
        h, y = residual_norm_fwd(x, residual, weight, eps, p, seed, site)
        _keep_seed(ctx, seed, _flat(h), weight)
        ctx.rest = eps, p, site
        return h, y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dy):
        h, weight = ctx.saved_tensors[:2]
        if dy is None and dh is None:
            return (None,) * 7
        dy = torch.zeros_like(h) if dy is None else _rows2(dy)
        dh = None if dh is None else _rows2(dh)
        eps, p, site = ctx.rest
        need = ctx.needs_input_grad[1]
        dx, dresidual, dweight = _result(_native.rnorm_bwd(dh, dy, h, weight, eps, p, _kept_seed(ctx), site, need, True),
                                         "fewbit_rnorm_bwd")
        return dx, dresidual if need else None, dweight, None, None, None, None


def _rows2(t):
    """t, or a contiguous copy of it where its rows are not contiguous, do not start at multiples of 16
    bytes, or their first axes are not one step apart."""
    if t.is_contiguous() and t.data_ptr() % 16 == 0:
        return t
    t = _rows(t)
    ahead = [(n, s) for n, s in zip(t.shape[:-2], t.stride()[:-2]) if n > 1]
    if all(s == n2 * s2 for (_, s), (n2, s2) in zip(ahead, ahead[1:])):
        return t
    return t.clone(memory_format=torch.contiguous_format)


def residual_norm(x, residual, weight, eps=1e-6, p=0.0, seed=0, site=0):
    """residual_norm_fwd, differentiable with respect to x, residual and weight."""
    r = _native.residual_norm_layer(x, residual, weight, eps, p, seed, site)
    return ResidualNorm.apply(x, residual, weight, eps, p, seed, site) if r is None else r


# ---------------------------------------------------------------- 8-bit integers
def residual_norm_int8(x, residual, weight, eps=1e-6):
    """residual_norm_fwd without dropout, y in 8-bit integers with a scale per row:
    (h, codes, scale); codes * scale[..., None] stands for y.  For serving: not
    differentiable."""
    return _result(_native.rnorm_int8(x, residual, weight, eps), "fewbit_rnorm_int8")


def quantize_rows(x):
    """Rows of x [..., width] in 8-bit integers with a scale per row, their largest
    magnitude over 127: (codes, scale).  x as in residual_norm_fwd.  A row that
    holds a NaN or an infinity has scale NaN."""
    return _result(_native.rows8(x), "fewbit_rows8")


def int8_linear(x, x_scale, weight, weight_scale, bias=None, act=None, dtype=torch.bfloat16):
    """act(x_scale weight_scale sum_k x weight + bias), rounded once to dtype.

    x [..., width] and weight [out, width] int8 (as quantize_rows gives them),
    x_scale [...] and weight_scale [out] fp32, bias [out] of dtype or None; act
    None, "gelu" or "silu".  width a multiple of 16 up to 131056; rows contiguous,
    even steps of a multiple of 16 bytes and of at most 2^23 apart; scales dense, from
    multiples of 16 bytes on, x_scale between 2^-126 and 2^96; sums are exact.  Not
    differentiable."""
    if act not in _ACTS:
        raise ValueError(f"act must be None, 'gelu' or 'silu', not {act!r}")
    if dtype not in _TYPES:
        raise TypeError("dtype must be float32, float16 or bfloat16")
    return _result(_native.mm8(x, x_scale, weight, weight_scale, bias, _ACTS[act], _TYPES[dtype]), "fewbit_mm8_fwd")


class Int8Linear(torch.nn.Module):
    """A torch.nn.Linear on a device for serving, its weight in 8-bit integers with a
    scale per channel; what comes in is laid out in 8 bits too, with a scale per
    row, unless it comes as (codes, scale).  in_features a multiple of 16 up to 32768,
    the longest rows that quantize_rows takes.  act: "gelu" or "silu" after the bias.
    Converted to another type (.half(), .to(dtype)) its results have that type, its
    scales stay fp32."""

    def __init__(self, linear: torch.nn.Linear, act: str | None = None):
        super().__init__()
        if act not in _ACTS:
            raise ValueError(f"act must be None, 'gelu' or 'silu', not {act!r}")
        if linear.in_features % 16 != 0 or not 0 < linear.in_features <= 32768:
            raise ValueError("in_features must be a multiple of 16 up to 32768")
        codes, scale = quantize_rows(_rows(linear.weight.detach()))
        self.register_buffer("weight", codes)
        self.register_buffer("weight_scale", scale)
        self.register_buffer("bias", None if linear.bias is None else linear.bias.detach().clone())
        self.act, self.dtype = act, linear.weight.dtype

    def _apply(self, fn, recurse=True):
        scale = self.weight_scale
        super()._apply(fn, recurse)
        if self.weight_scale.dtype != scale.dtype:
            self.weight_scale = scale.to(self.weight_scale.device)
        self.dtype = fn(torch.empty(0, dtype=self.dtype, device=scale.device)).dtype
        return self

    def forward(self, x, scale=None):
        if scale is None:
            x, scale = quantize_rows(_rows2(x.detach()))
        return int8_linear(x, scale, self.weight, self.weight_scale, self.bias, self.act, self.dtype)

    def extra_repr(self) -> str:
        return f"in_features={self.weight.shape[1]}, out_features={self.weight.shape[0]}, bias={self.bias is not None}, act={self.act}"
