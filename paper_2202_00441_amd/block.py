"""The operators around the activation in a transformer block: attention, the
norm and rotary position of query and key heads, and the AdamW step
(include/fewbit_block.h has the formulas, layouts and roundings).

attention_fwd / attention_bwd, qk_norm_rope_fwd / qk_norm_rope_bwd and
adamw_step are the raw calls, in the library's HIP kernels on the current
stream; they check every tensor (device, dtype, shape, layout) and raise
TypeError or ValueError before anything is launched.  attention and
qk_norm_rope are the same as differentiable functions: they keep their inputs
(attention also its output and one number per row), take any layout, copying
tensors whose rows the kernels cannot read, and form the gradients of all of them.
"""
from __future__ import annotations

import torch

from ._lib import FewbitError, _native


def _result(r, where: str):
    if type(r) is int:
        raise FewbitError(r, where)
    return r


# ---------------------------------------------------------------- attention
def attention_fwd(q, k, v, causal=False, window=0, scale=None, k_len=None, cu_q=None, cu_k=None):
    """out_i = sum_j softmax_j(scale <q_i, k_j>) v_j over the keys the mask lets
    through, and the logarithm of each row's sum of exponentials.

    q [batch, rows, heads, d], k and v [batch, keys, kv_heads, d], or, packed,
    [rows, heads, d] with cu_q and cu_k (int32, one entry more than sequences)
    telling where sequences begin (one below one before it counts as that one);
    fp16 or bf16, d a multiple of 8 up to 128.  Heads of q share heads of k and v
    in runs.  Any strides; rows contiguous, from multiples of 16 bytes on.

    causal: the last query sees the last key, each earlier one a key less.
    window (with causal): a query sees that many keys at most.  k_len (int32,
    an entry per sequence): how many keys are there; the others are not read.
    scale: 1 / sqrt(d) unless given.

    Returns (out, lse): out like q, dense; lse fp32 [batch, heads, rows] or
    [heads, rows].  A row that sees no key has out 0 and lse -inf."""
    return _result(_native.attention_fwd(q, k, v, causal, window, scale, k_len, cu_q, cu_k), "fewbit_attn_fwd")


def attention_bwd(dout, q, k, v, out, lse, causal=False, window=0, scale=None, k_len=None, cu_q=None, cu_k=None):
    """(dq, dk, dv) from the gradient of out; out and lse as attention_fwd gave
    them, the other arguments as they were there.  The probabilities are formed
    again; equal inputs give equal bits."""
    return _result(_native.attention_bwd(dout, q, k, v, out, lse, causal, window, scale, k_len, cu_q, cu_k),
                   "fewbit_attn_bwd")


def _rows(t, per: int = 16):
    """t, or a contiguous copy of it where its rows are not contiguous or do
    not start at multiples of 16 bytes."""
    size = t.element_size()
    strides = [s * size for s, n in zip(t.stride()[:-1], t.shape[:-1]) if n > 1]
    if (t.stride(-1) == 1 or t.shape[-1] <= 1) and t.data_ptr() % per == 0 and all(s % per == 0 for s in strides):
        return t
    return t.clone(memory_format=torch.contiguous_format)


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, window, scale, k_len, cu_q, cu_k):
        q, k, v = _rows(q), _rows(k), _rows(v)
        out, lse = attention_fwd(q, k, v, causal, window, scale, k_len, cu_q, cu_k)
        ctx.save_for_backward(q, k, v, out, lse, k_len, cu_q, cu_k)
        ctx.mask = causal, window, scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, k_len, cu_q, cu_k = ctx.saved_tensors
        dq, dk, dv = attention_bwd(_rows(dout), q, k, v, out, lse, *ctx.mask, k_len, cu_q, cu_k)
        return dq, dk, dv, None, None, None, None, None, None


def attention(q, k, v, causal=False, window=0, scale=None, k_len=None, cu_q=None, cu_k=None):
    """attention_fwd's out, differentiable with respect to q, k and v."""
    return Attention.apply(q, k, v, causal, window, scale, k_len, cu_q, cu_k)


# ---------------------------------------------------------------- norm and rotation
def rope_tables(positions: int, rot: int, base: float = 10000.0, device="cuda"):
    """cos and sin [positions, rot / 2] of the angles position * base^(-2t / rot)."""
    t = torch.arange(0, rot, 2, device=device, dtype=torch.float64) / rot
    angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * base ** -t
    return torch.cos(angle).float(), torch.sin(angle).float()


def qk_norm_rope_fwd(q, k, q_weight, k_weight, cos, sin, positions=None, eps=1e-6, interleaved=False):
    """RMS norm of every head of q and k over its elements, times the weight of
    its kind, and the rotary position, in one pass: (q, k), dense.

    q [batch, tokens, heads, d], k [batch, tokens, kv_heads, d] (or without the
    batch), fp32, fp16 or bf16 with weights [d] of the same type; d and the
    rotated part multiples of 16, d up to 256; any strides, rows contiguous,
    from multiples of 16 bytes on.
    cos, sin: fp32 [positions, rotated elements / 2].  positions: int64
    [batch, tokens] or [tokens]; without, a token's place in its sequence.  A
    position that the tables do not hold gives NaN.  interleaved: the pairs are
    neighbours, else element t goes with t + rotated / 2."""
    return _result(_native.qk_fwd(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved), "fewbit_qk_fwd")


def qk_norm_rope_bwd(dq, dk, q, k, q_weight, k_weight, cos, sin, positions=None, eps=1e-6, interleaved=False):
    """The gradients of q, k and (fp32) of their weights from those of
    qk_norm_rope_fwd's results."""
    return _result(_native.qk_bwd(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved),
                   "fewbit_qk_bwd")


class QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved):
        q, k, q_weight, k_weight = (_rows(t) for t in (q, k, q_weight, k_weight))
        out = qk_norm_rope_fwd(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
        ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
        ctx.rest = eps, interleaved
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        saved = ctx.saved_tensors
        dq, dk, dq_weight, dk_weight = qk_norm_rope_bwd(_rows(dq), _rows(dk), *saved, *ctx.rest)
        return (dq, dk, dq_weight.to(saved[2].dtype), dk_weight.to(saved[3].dtype), None, None, None, None, None)


def qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions=None, eps=1e-6, interleaved=False):
    """qk_norm_rope_fwd, differentiable with respect to q, k and the weights."""
    return QkNormRope.apply(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)


# ---------------------------------------------------------------- optimizer step
ADAMW_BLOCK = 256       # elements that share a scale; tensors start at whole blocks


def adamw_blocks(n: int) -> int:
    """Blocks of the flat buffers that a tensor of n elements takes."""
    return -(-n // ADAMW_BLOCK)


def adamw_step(params, grads, exp_avg, exp_avg_sq, exp_avg_scale=None, exp_avg_sq_scale=None, master=None, *,
               lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step, seed=None):
    """One AdamW step over all tensors, in place, one launch for 256 of them.

    params: tensors of one type (fp32, fp16 or bf16); grads: of that type or
    fp32, in the parameters' layout (None: that tensor is left as it is).
    exp_avg, exp_avg_sq: flat, tensor i's moments at 256 * the blocks
    (adamw_blocks) of the tensors before it; fp32, or torch.float8_e4m3fn with a
    power of two per block in exp_avg_scale and exp_avg_sq_scale.  master: fp32
    weights laid out alike, of which the parameters are the rounded copies.
    step counts from 1.  seed (step unless given): what the rounding of 8-bit
    moments draws on; equal inputs give equal bits."""
    rc = _native.adamw_step(params, grads, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale, master, lr, beta1, beta2,
                            eps, weight_decay, step, step if seed is None else seed)
    if rc != 0:
        raise FewbitError(rc, "fewbit_adamw_step")
