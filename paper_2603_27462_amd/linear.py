"""Torch modules around handles (the role the paper gives its RSRLinear layer in System Overview, "Integration": a
drop-in for a linear layer whose weight is fixed after preprocessing): RsrLinear for binary and ternary weights, RsrInt4Linear
for 4-bit weights with group scales, and RsrGatedMlp, the feed-forward block of three of those.  The latter two pass gradients on
to their inputs, so that what lies before and beside them can be trained (in reverse mode, once; forward mode is refused).  Argument marshalling only: the products run
in librsr."""
from __future__ import annotations

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding as _b


class RsrLinear(torch.nn.Module):
    """y = scale * W x for a fixed int8 weight W [out_features][in_features] in {-1,0,+1}
    ({0,1} for the binary kind).  k = 0 lets the library choose the block height.  All tokens of a call
    are one batch, and the order of the sums depends on its size: a token's outputs may differ in their
    last bits between a call for it alone, a small batch and a prompt (see rsr_matvec_ex)."""

    def __init__(self, weight: torch.Tensor, scale: float = 1.0, k: int = 0,
                 kind: int = _b.RSR_TERNARY_FUSED):
        super().__init__()
        self.out_features, self.in_features = weight.shape
        self.scale = float(scale)
        self.handle = _b.rsr_preprocess(weight, k, kind)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if x.shape[-1] != self.in_features:
            raise ValueError("last dimension of x must be %d" % self.in_features)
        lead = x.shape[:-1]
        flat = x.reshape(-1, self.in_features)
        if flat.stride(-1) != 1:
            flat = flat.contiguous()
        if flat.shape[0] == 1:
            y = _b.rsr_matvec_ex(self.handle, flat[0], scale=self.scale).unsqueeze(0)
        else:
            y = _b.rsr_matvec_ex(self.handle, flat, scale=self.scale)
        return y.reshape(*lead, self.out_features)

    def extra_repr(self) -> str:
        return "in_features=%d, out_features=%d, k=%d, kind=%d" % (
            self.in_features, self.out_features, self.handle.k, self.handle.kind)


def _rows(x: torch.Tensor, length: int) -> torch.Tensor:
    """x as [tokens][length] with unit inner stride, one token behind the other (an expanded x has them all in one place)"""
    if x.shape[-1] != length:
        raise ValueError("last dimension of x must be %d" % length)
    tokens = 1
    for n in x.shape[:-1]:
        tokens *= n
    flat = x.reshape(tokens, length)
    whole = (length == 1 or flat.stride(-1) == 1) and (tokens <= 1 or flat.stride(0) >= length)
    return flat if whole else flat.contiguous()


def _differentiated(x: torch.Tensor) -> bool:
    """whether a derivative of x is asked for, in reverse mode or (refused below) in forward mode"""
    return (torch.is_grad_enabled() and x.requires_grad) or forward_ad.unpack_dual(x).tangent is not None


class _ReverseMode(torch.autograd.Function):
    @staticmethod
    def jvp(ctx, *tangents):
        raise NotImplementedError("layers of 4-bit weights pass gradients on in reverse mode only")


class _Int4Product(_ReverseMode):
    @staticmethod
    def forward(ctx, x, handle, dtype):
        ctx.handle, ctx.dtype = handle, x.dtype
        return _b.rsr_int4_matvec(handle, x, dtype=dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        dx = _b.rsr_int4_matvec(ctx.handle, _rows(dy, ctx.handle.rows), transposed=True, dtype=ctx.dtype)
        return dx, None, None


class _Gated(_ReverseMode):
    @staticmethod
    def forward(ctx, x, gate, up, act):
        pre = torch.empty((x.shape[0], 2, gate.rows), dtype=torch.float32, device=x.device)
        h = _b.rsr_gated(gate, up, x, act, dtype=x.dtype, pre=pre)
        ctx.save_for_backward(pre)
        ctx.rest = gate, up, act, x.dtype
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        gate, up, act, dtype = ctx.rest
        dx, _ = _b.rsr_gated_backward(gate, up, ctx.saved_tensors[0], _rows(dh, gate.rows), act, dtype=dtype)
        return dx, None, None, None


class RsrInt4Linear(torch.nn.Module):
    """y = W x for fixed 4-bit weights, W[r][c] = scales[r][c // group] * (codes[r][c] - zeros[r][c // group]) (see
    rsr_preprocess_int4); y is of type `dtype`.  x is float32 or bfloat16, of any leading dimensions; its gradient has its type.
    To train on bfloat16, take `dtype=torch.bfloat16` here too: the gradient of a float32 y is multiplied with all of its bits, which
    takes up to 1.7 times as long (4096 x 14336, 512 tokens 293 us against 171)."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, group: int, zeros=None, dtype=torch.float32):
        super().__init__()
        self.out_features, self.in_features = codes.shape
        self.group, self.dtype = int(group), dtype
        self.handle = _b.rsr_preprocess_int4(codes, scales, group, zeros=zeros)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        flat = _rows(x, self.in_features)
        if _differentiated(x):
            y = _Int4Product.apply(flat, self.handle, self.dtype)
        else:
            y = _b.rsr_int4_matvec(self.handle, flat.detach(), dtype=self.dtype)
        return y.reshape(*x.shape[:-1], self.out_features)

    def kept_group(self) -> int:
        """columns of a group as the handle keeps them"""
        if self.group >= self.in_features:
            return 128
        return next(n for n in (128, 64, 32) if self.group % n == 0)

    def extra_repr(self) -> str:
        return "in_features=%d, out_features=%d, group=%d" % (self.in_features, self.out_features, self.group)


class RsrGatedMlp(torch.nn.Module):
    """y = down(act(gate x) * (up x)) of three RsrInt4Linear layers: gate, up, the activation ("silu", "gelu" in its tanh form or
    "relu2") and their product in one launch, the result between the two launches in the type of x."""

    def __init__(self, gate: RsrInt4Linear, up: RsrInt4Linear, down: RsrInt4Linear, act: str = "silu"):
        super().__init__()
        if (gate.in_features, gate.out_features) != (up.in_features, up.out_features) or down.in_features != gate.out_features:
            raise ValueError("gate and up must have one shape, and down the inputs that they have outputs")
        if gate.kept_group() != up.kept_group():
            raise ValueError("the groups of gate and up must be multiples of the same of 32, 64 and 128 (%d and %d are kept as %d and %d)"
                             % (gate.group, up.group, gate.kept_group(), up.kept_group()))
        if not gate.handle.device == up.handle.device == down.handle.device:
            raise ValueError("gate, up and down must be on one device")
        _b._act_code(act)
        self.gate, self.up, self.down, self.act = gate, up, down, act

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        flat = _rows(x, self.gate.in_features)
        if _differentiated(x):
            h = _Gated.apply(flat, self.gate.handle, self.up.handle, self.act)
        else:
            h = _b.rsr_gated(self.gate.handle, self.up.handle, flat.detach(), self.act, dtype=flat.dtype)
        return self.down(h).reshape(*x.shape[:-1], self.down.out_features)

    def extra_repr(self) -> str:
        return "act=%s" % self.act
