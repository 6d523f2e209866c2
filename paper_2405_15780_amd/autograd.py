"""torch.autograd wrapper: attention as a differentiable op whose forward and
backward are the library's kernels (argument marshalling only).

attention(q, k, v) takes bf16 [B, H, Nq, d] queries and [B, H, Nk, d] keys
and values (any strides with d contiguous) and returns O in fp32. In the
backward, the upstream gradient is rounded to bf16 (the kernels' dO operand)
and dQ, dK, dV, computed in fp32, are returned in the inputs' dtype. For an
fp32 gradient with unit stride along d the kernels do both conversions
(binding.bwd_train); others are converted around binding.bwd, to the same bits.
"""
from __future__ import annotations

from . import binding as _b


_torch = _b._torch


class _Attention:
    _fn = None

    @classmethod
    def get(cls):
        if cls._fn is None:
            torch = _torch()

            class Attention(torch.autograd.Function):
                @staticmethod
                def forward(ctx, q, k, v, scale, store_ds):
                    o, lse = _b.fwd(q, k, v, scale)
                    ctx.save_for_backward(q, k, v, o, lse)
                    ctx.scale, ctx.store_ds = scale, store_ds
                    return o

                @staticmethod
                def backward(ctx, grad_o):
                    q, k, v, o, lse = ctx.saved_tensors
                    if not ctx.store_ds:
                        grads = _b.bwd_train(q, k, v, o, lse, grad_o, ctx.scale)
                        if grads is not None:
                            return *grads, None, None
                    dout = grad_o.to(torch.bfloat16)
                    if dout.stride(-1) != 1:
                        dout = dout.contiguous()
                    dq, dk, dv = _b.bwd(q, k, v, o, lse, dout, ctx.scale, store_ds=ctx.store_ds)
                    return dq.to(q.dtype), dk.to(k.dtype), dv.to(v.dtype), None, None

            cls._fn = Attention
        return cls._fn


def attention(q, k, v, scale=None, store_ds=False):
    """softmax(scale Q K^T) V (scale defaults to 1/sqrt(d)) with a backward
    pass; store_ds selects the dS mode of the backward."""
    return _Attention.get().apply(q, k, v, scale, store_ds)


class _LayerNorm:
    _fn = None

    @classmethod
    def get(cls):
        if cls._fn is None:
            torch = _torch()

            class LayerNorm(torch.autograd.Function):
                @staticmethod
                def forward(ctx, x, weight, bias, eps):
                    y, mean, rstd = _b.layer_norm_fwd(x, weight, bias, eps)
                    ctx.save_for_backward(x, weight, mean, rstd)
                    ctx.bias_dtype = None if bias is None else bias.dtype
                    return y

                @staticmethod
                @torch.autograd.function.once_differentiable
                def backward(ctx, dy):
                    x, weight, mean, rstd = ctx.saved_tensors
                    dx, dw, db = _b.layer_norm_bwd(x, weight, mean, rstd, _b.plain_memory(dy),
                                                   want_dweight=ctx.needs_input_grad[1],
                                                   want_dbias=ctx.needs_input_grad[2], bias_dtype=ctx.bias_dtype)
                    return dx, dw, db, None

            cls._fn = LayerNorm
        return cls._fn


def _wants_grad(*ts):
    """Whether a call goes through its autograd function: if any of its tensors
    wants a gradient, and wherever one could carry a forward-mode tangent (that
    does not set requires_grad, nor does no_grad end it), which the function
    refuses like `attention` does."""
    torch = _torch()
    if torch.autograd.forward_ad._current_level >= 0:
        return True
    if not torch.is_grad_enabled():
        return False
    for t in ts:
        if t is not None and t.requires_grad:
            return True
    return False


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dim of x (bf16, fp16 or fp32, any strides with
    that dim contiguous) with a backward pass; weight and bias are [D], of x's
    type or fp32."""
    if not _wants_grad(x, weight, bias):
        return _b.layer_norm_fwd(x, weight, bias, eps, stats=False)[0]
    return _LayerNorm.get().apply(x, weight, bias, eps)


class _Rotary:
    _fn = None

    @classmethod
    def get(cls):
        if cls._fn is None:
            torch = _torch()

            class Rotary(torch.autograd.Function):
                @staticmethod
                def forward(ctx, q, k, positions, sections, base, interleaved, joint, inverse):
                    ctx.save_for_backward(positions)
                    ctx.args = (sections, base, interleaved, joint)
                    ctx.inverse = inverse
                    return _b.rotary_fwd(q, k, positions, sections, base, interleaved, joint, inverse)

                @staticmethod
                def backward(ctx, dq, dk=None):
                    # the turn by the opposite angles, itself differentiable, of
                    # those that are asked for
                    grads = [_b.plain_memory(g) if need else None for g, need in zip((dq, dk), ctx.needs_input_grad)]
                    if not any(ctx.needs_input_grad[:2]):  # (for positions that want a gradient: they get none)
                        return (None,) * 8
                    first, *second = [g for g in grads if g is not None]
                    r = Rotary.apply(first, second[0] if second else None, ctx.saved_tensors[0], *ctx.args, not ctx.inverse)
                    turned = iter(r if second else (r,))
                    dq, dk = (None if g is None else next(turned) for g in grads)
                    return dq, dk, None, None, None, None, None, None

            cls._fn = Rotary
        return cls._fn


def rotary(q, k, positions, sections, base=10000.0, interleaved=False, joint=False):
    """q [B,Hq,N,d] and k [B,Hk,N,d] (or None) turned by their positions on several
    axes, with a backward pass (see binding.rotary_fwd); positions get no gradient."""
    sections = tuple(sections)
    if not _wants_grad(q, k):
        return _b.rotary_fwd(q, k, positions, sections, base, interleaved, joint)
    return _Rotary.get().apply(q, k, positions, sections, base, interleaved, joint, False)


class _DiffAttention:
    _fn = None

    @classmethod
    def get(cls):
        if cls._fn is None:
            torch = _torch()

            class DiffAttention(torch.autograd.Function):
                @staticmethod
                def forward(ctx, q, k, v, lam, scale, key_lens):
                    o, o2, lse = _b.diff_fwd(q, k, v, lam, scale, key_lens)
                    ctx.save_for_backward(q, k, v, lam, o2, lse, key_lens)
                    ctx.scale = scale
                    return o

                @staticmethod
                @torch.autograd.function.once_differentiable
                def backward(ctx, grad_o):
                    q, k, v, lam, o2, lse, key_lens = ctx.saved_tensors
                    g = _b.plain_memory(grad_o)
                    s = _b._diff_strides(g)
                    # shared or misaligned rows are laid out anew
                    if s.row < g.shape[3] or s.row % 8 or s.head % 8 or s.batch % 8 or g.data_ptr() % 16 \
                            or (g.shape[2] + 512) * s.row * 2 > 0x7fffffff:
                        g = torch.empty(g.shape, dtype=g.dtype, device=g.device).copy_(g)
                    dq, dk, dv, dlam = _b.diff_bwd(q, k, v, lam, None, o2, lse, g, ctx.scale, key_lens,
                                                   want_dlam=ctx.needs_input_grad[3])
                    return dq, dk, dv, dlam, None, None

            cls._fn = DiffAttention
        return cls._fn


def diff_attention(q, k, v, lam, scale=None, key_lens=None):
    """Differential attention, softmax(scale Q1 K1^T) V - lam softmax(scale Q2
    K2^T) V, with a backward pass: q [B,2H,Nq,d] and k [B,2H,Nk,d] bf16 (heads 2h
    and 2h + 1 are the two maps of head h), v [B,H,Nk,e], lam [H] or one value for
    all heads (fp32 or bf16); scale defaults to 1/sqrt(d). key_lens (int32 [B]):
    sample b attends to its first key_lens[b] keys. Returns o, bf16 [B,H,Nq,e]."""
    if not isinstance(lam, _torch().Tensor):
        raise TypeError("lam must be a tensor: [H], or one value for all heads")
    if lam.numel() == 1 and lam.shape != v.shape[1:2]:
        lam = lam.reshape(1).expand(v.shape[1])
    lam = lam.contiguous()
    if not _wants_grad(q, k, v, lam):
        return _b.diff_fwd(q, k, v, lam, scale, key_lens, save=False)[0]
    return _DiffAttention.get().apply(q, k, v, lam, scale, key_lens)
